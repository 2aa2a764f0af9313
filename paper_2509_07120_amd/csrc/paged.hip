// Attention of one new token for each sequence over a cache of pages.
//
// The query of sequence b stands at position lengths[b] - 1, its own key is in the cache.  It sees the keys that window.h describes, in
// the cache rows page_table[b][j / page], j % page.  HBM-bound: every visible key and value is read once for up to 16 of the query heads
// that share it (more of them: once for each 16), at 16 flop to the byte at most (fp32 8).  A workgroup takes a stretch of one sequence's visible keys and one key head; its four waves take
// pieces of it in turn and wait for nobody: a wave moves its pieces straight into LDS of its own, two ahead (16 KB on their way for each
// wave, 128 KB for each CU, where 8 TB/s at 2 us of latency ask for 64).  Up to 16 query heads are the columns of 16x16 products
// S^T = K Q^T and O^T = V^T P^T, in which the weights are operands as they lie in the results.
// The waves' sums are joined through LDS; stretches of one sequence by a second kernel.
// Two sequences of 412,200 and 312,300 keys of 16 heads, 2.97 GB: 480 us, 6.2 TB/s; 96 of 1 to 12,000, window of 4096, 16 query heads to 4 key heads: 66 us, 5.0 TB/s.
#include "window.h"

#include <math.h>

namespace bsga {
namespace {

constexpr int kTable = 2048;   // page numbers of a stretch
constexpr int kHeads = 16;     // query heads of a workgroup
constexpr int kWaves = 4;

template <typename T>
struct Ops16;

template <>
struct Ops16<__bf16> {
  typedef bf16x8 A;
  static constexpr int kKeys = 32;   // of a piece
  static constexpr int kBlocks = 2;  // of 16 keys
  static constexpr int kSteps = 2;   // products over the 64 numbers of a row
  static __device__ __forceinline__ f32x4 product(A a, A b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ int swizzle_k(int r) { return swz_k(r); }
  static __device__ __forceinline__ int swizzle_v(int r) { return swz_v(r); }
  static __device__ __forceinline__ void row(const unsigned char* p, int q, A (&a)[kSteps]) {
#pragma unroll
    for (int c = 0; c < 2; ++c) a[c] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(p + (4 * c + q) * 16));
  }
  static __device__ __forceinline__ void rows(const unsigned char* tile, int r, int q, A (&a)[kSteps]) {
#pragma unroll
    for (int c = 0; c < 2; ++c) a[c] = *LDS_PTR(bf16x8, tile + r * 128 + (((4 * c + q) ^ swz_k(r)) << 4));
  }
  // o += V^T P^T: the weights' products in w[block][r], of keys 16 block + 4 q + r
  static __device__ __forceinline__ void update(const unsigned char* tile, int lane, const f32x4 (&w)[kBlocks], f32x4 (&o)[4]) {
    const int m = (lane & 15) >> 2, j = lane & 3, q = lane >> 4;
    const bf16x8 b = __builtin_bit_cast(
        bf16x8, u32x4{pack_bf16(w[0][0], w[0][1]), pack_bf16(w[0][2], w[0][3]), pack_bf16(w[1][0], w[1][1]), pack_bf16(w[1][2], w[1][3])});
#pragma unroll
    for (int db = 0; db < 4; ++db) {
      u32x2 x[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = 16 * e + 4 * q + m;
        const unsigned char* p = tile + r * 128 + (((2 * db + (j >> 1)) ^ swz_v(r)) << 4) + (j & 1) * 8;
        x[e] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(p)));
      }
      o[db] = product(__builtin_bit_cast(bf16x8, u32x4{x[0][0], x[0][1], x[1][0], x[1][1]}), b, o[db]);
    }
  }
};

template <>
struct Ops16<float> {
  typedef float A;
  static constexpr int kKeys = 16;
  static constexpr int kBlocks = 1;
  static constexpr int kSteps = 16;
  static __device__ __forceinline__ f32x4 product(A a, A b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ int swizzle_k(int r) { return r & 15; }
  static __device__ __forceinline__ int swizzle_v(int r) { return r & 15; }
  static __device__ __forceinline__ void row(const unsigned char* p, int q, A (&a)[kSteps]) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(p + (4 * c + q) * 16);
#pragma unroll
      for (int e = 0; e < 4; ++e) a[4 * c + e] = x[e];
    }
  }
  static __device__ __forceinline__ void rows(const unsigned char* tile, int r, int q, A (&a)[kSteps]) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const f32x4 x = *LDS_PTR(f32x4, tile + r * 256 + (((4 * c + q) ^ swizzle_k(r)) << 4));
#pragma unroll
      for (int e = 0; e < 4; ++e) a[4 * c + e] = x[e];
    }
  }
  static __device__ __forceinline__ void update(const unsigned char* tile, int lane, const f32x4 (&w)[kBlocks], f32x4 (&o)[4]) {
    const int q = lane >> 4;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = 4 * q + e, d = 16 * db + (lane & 15);
        o[db] = product(*LDS_PTR(float, tile + r * 256 + (((d >> 2) ^ swizzle_v(r)) << 4) + (d & 3) * 4), w[0][e], o[db]);
      }
  }
};

struct PagedArgs {
  View q;                             // [batch, heads, 64]: token is the sequence's stride
  const unsigned char *k, *v;         // [n_pages, kv_heads, page, 64]
  const int32_t *page_table, *lengths;
  unsigned char* out;                 // [batch, heads, 64]
  float* lse;                         // [batch, heads] or null
  float *part, *part_lse;             // with stretches: [splits][batch, heads, 64] and [splits][batch, heads]
  int batch, heads, kv_heads, group, head_blocks, table_width, n_pages, page, frame, window, sinks, splits, stretch;
  unsigned magic;                     // j / page = umulhi(2 j, magic) >> shift, for j < 2^31
  int shift;
  float scale_log2;
};

__device__ __forceinline__ int page_of(const PagedArgs& a, int j) {
  return static_cast<int>(__umulhi(static_cast<unsigned>(j) << 1, a.magic) >> a.shift);
}

// 16 bytes per lane from memory straight into LDS, as dma16, from a 64-bit address for each lane.
__device__ __forceinline__ void dma16_at(const unsigned char* p, unsigned lds) {
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 0\n\t"  // one wait state between a scalar write of M0 and an LDS-DMA instruction that reads it
      "global_load_lds_dwordx4 %1, off"
      :
      : "s"(lds), "v"(p)
      : "memory", "m0");
}

__device__ __forceinline__ float across(float x, bool maximum) {  // over the four lanes of a column
#pragma unroll
  for (int o = 16; o < 64; o <<= 1) {
    const float y = __shfl_xor(x, o);
    x = maximum ? fmaxf(x, y) : x + y;
  }
  return x;
}

template <typename T>
__global__ __launch_bounds__(64 * kWaves, 2) void paged_kernel(const PagedArgs a) {
  typedef Ops16<T> P;
  constexpr int kRow = 64 * sizeof(T), kChunks = kRow / 16, kRowsOfLoad = 64 / kChunks, kLoads = P::kKeys / kRowsOfLoad;
  constexpr int kPiece = P::kKeys * kRow, kBuf = 2 * kPiece, kWaveLds = 2 * kBuf;
  static_assert(kLoads == 4, "eight loads of a piece");
  __shared__ __align__(16) unsigned char smem[kWaves * kWaveLds];
  __shared__ int table[kTable];
  __shared__ float sums[kWaves][2][kHeads];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, q = lane >> 4;
  const int b = blockIdx.z, split = blockIdx.x;
  const int hk = blockIdx.y / a.head_blocks, hb = blockIdx.y - hk * a.head_blocks;
  const int heads = min(kHeads, a.group - hb * kHeads);       // query heads of this workgroup,
  const int h0 = hk * a.group + hb * kHeads;                  // the first of them
  const int64_t rows = int64_t(a.batch) * a.heads, row0 = int64_t(b) * a.heads + h0;

  // the visible keys, numbered through: x < s is key x, the others lo + x - s
  const int length = min(max(a.lengths[b], 0), a.table_width * a.page);
  int s = 0, lo = 0;
  if (a.window > 0 && length > 0) {
    const int f = (length - 1) / a.frame;
    lo = f < a.window ? 0 : (f + 1 - a.window) * a.frame;
    s = min(a.sinks, lo);
  }
  const int count = s + length - lo;
  const int x0 = split * a.stretch, x1 = min(x0 + a.stretch, count);
  if (x0 >= x1 && a.splits > 1) {  // the whole workgroup: the sequence has no keys here
    if (threadIdx.x < heads) a.part_lse[split * rows + row0 + threadIdx.x] = -INFINITY;
    return;
  }
  // the page numbers of the stretch: those of its first tokens, then those of the window
  const int a0 = page_of(a, x0), a_pages = x0 < min(x1, s) ? page_of(a, min(x1, s) - 1) - a0 + 1 : 0;
  const int b0 = page_of(a, lo + max(x0, s) - s), b_pages = max(x0, s) < x1 ? page_of(a, lo + x1 - 1 - s) - b0 + 1 : 0;
  const int32_t* const pages = a.page_table + int64_t(b) * a.table_width;
  for (int i = threadIdx.x; i < min(a_pages + b_pages, kTable); i += 64 * kWaves)
    table[i] = min(max(pages[i < a_pages ? a0 + i : b0 + i - a_pages], 0), a.n_pages - 1);  // a bad entry cannot read out of bounds
  typename P::A qf[P::kSteps];
  P::row(a.q.p + b * a.q.token + (h0 + min(c, heads - 1)) * a.q.head, q, qf);
  __syncthreads();

  const unsigned lds = lds_address(smem) + wave * kWaveLds;
  unsigned char* const mine = smem + wave * kWaveLds;
  const int pieces = (x1 - x0 + P::kKeys - 1) / P::kKeys;
  const int r_in = lane / kChunks, pos = lane % kChunks;
  auto issue = [&](int p, int buf) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int r = i * kRowsOfLoad + r_in;
      const int x = min(x0 + p * P::kKeys + r, x1 - 1);  // rows past the end are the last one again, with no weight
      const int j = x < s ? x : lo + x - s;
      const int page = page_of(a, j);
      const int at = table[min(x < s ? page - a0 : a_pages + page - b0, kTable - 1)];
      const int64_t row = (int64_t(at) * a.kv_heads + hk) * a.page + (j - page * a.page);
      dma16_at(a.k + row * kRow + ((pos ^ P::swizzle_k(r)) << 4), lds + buf * kBuf + i * 1024);
      dma16_at(a.v + row * kRow + ((pos ^ P::swizzle_v(r)) << 4), lds + buf * kBuf + kPiece + i * 1024);
    }
  };
  if (wave < pieces) issue(wave, 0);
  if (wave + kWaves < pieces) issue(wave + kWaves, 1);

  f32x4 o[4];
  float m = -INFINITY, l = 0.f;
#pragma unroll
  for (int db = 0; db < 4; ++db) o[db] = f32x4{0.f, 0.f, 0.f, 0.f};
  int buf = 0;
  for (int p = wave; p < pieces; p += kWaves, buf ^= 1) {
    if (p + kWaves < pieces) asm volatile("s_waitcnt vmcnt(8)" ::: "memory");  // the next piece's eight loads may be on their way
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    unsigned char* const kt = mine + buf * kBuf;
    const int left = x1 - x0 - p * P::kKeys;
    if (left < P::kKeys) {  // the repeated values have weights of zero, which is not nothing if the last one is infinite
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int r = i * kRowsOfLoad + r_in;
        if (r >= left) *reinterpret_cast<u32x4*>(kt + kPiece + r * kRow + pos * 16) = u32x4{0u, 0u, 0u, 0u};
      }
    }
    f32x4 w[P::kBlocks];
#pragma unroll
    for (int blk = 0; blk < P::kBlocks; ++blk) {
      typename P::A ka[P::kSteps];
      P::rows(kt, 16 * blk + c, q, ka);
      w[blk] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < P::kSteps; ++e) w[blk] = P::product(ka[e], qf[e], w[blk]);
    }
    float top = -INFINITY;
#pragma unroll
    for (int blk = 0; blk < P::kBlocks; ++blk)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if (16 * blk + 4 * q + r >= left) w[blk][r] = -INFINITY;
        top = fmaxf(top, w[blk][r]);
      }
    top = across(top, true) * a.scale_log2;
    if (__any(top > m)) {
      const float to = fmaxf(m, top);
      const float keep = to == -INFINITY ? 1.f : exp2f(m - to);
      m = to;
      l *= keep;
#pragma unroll
      for (int db = 0; db < 4; ++db) o[db] *= keep;
    }
    const float from = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int blk = 0; blk < P::kBlocks; ++blk)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        w[blk][r] = __builtin_amdgcn_exp2f(fmaf(w[blk][r], a.scale_log2, -from));
        l += w[blk][r];
      }
    P::update(kt + kPiece, lane, w, o);
    if (p + 2 * kWaves < pieces) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the operands are in registers: the buffer is free
      issue(p + 2 * kWaves, buf);
    }
  }

  // the waves together: each leaves its sums in its own LDS (none of its loads are on their way any more)
  l = across(l, false);
#pragma unroll
  for (int db = 0; db < 4; ++db) *reinterpret_cast<f32x4*>(mine + (c * 64 + 16 * db + 4 * q) * 4) = o[db];
  if (q == 0) {
    sums[wave][0][c] = m;
    sums[wave][1][c] = l;
  }
  __syncthreads();
  const int head = threadIdx.x >> 4, d = (threadIdx.x & 15) * 4;
  if (head >= heads) return;
  float top = -INFINITY;
  bool nan = false;
#pragma unroll
  for (int x = 0; x < kWaves; ++x) {
    top = fmaxf(top, sums[x][0][head]);
    nan = nan || sums[x][1][head] != sums[x][1][head];
  }
  float sum = 0.f;
  f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int x = 0; x < kWaves; ++x) {
    const float weight = sums[x][0][head] == -INFINITY ? 0.f : exp2f(sums[x][0][head] - top);
    sum += sums[x][1][head] * weight;
    y += *reinterpret_cast<const f32x4*>(smem + x * kWaveLds + (head * 64 + d) * 4) * weight;
  }
  if (nan) sum = NAN;
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  const int64_t row = row0 + head;
  const float total = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
  if (a.splits > 1) {
    *reinterpret_cast<f32x4*>(a.part + (split * rows + row) * 64 + d) = y * inv;
    if (d == 0) a.part_lse[split * rows + row] = total;
  } else {
    Ops<T>::store4(a.out + row * kRow, d, y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
    if (a.lse != nullptr && d == 0) a.lse[row] = total;
  }
}

// Keys of a workgroup.  The chip holds 512, and 300 with 64 KB on their way each draw what the memory gives; a sequence's stretches cost a second
// kernel, and each wave should have a few pieces.  Measured, us, for at least 512 / 1024 / 2048 / 4096 workgroups: one sequence of 10,992 keys and 16
// key heads 14.6 / 15.2 / 15.3 / 15.2; two of 412,200 and 312,300 508 / 482 / 487 / 495; 96 of up to 4,100 keys and 4 key heads 60 (no
// stretches) / 70 / 64 / 67.  The host knows the most that a sequence can see, not its length: one long sequence among short ones must not be left to one
// workgroup (4,608 keys take one about 30 us), and the workgroups that find nothing to do have to stay few.
// Up to 8 pieces for each wave are one workgroup's whatever the launch: 1,024 bf16 keys 9.9 us a call and 27.2 alone, in stretches of 256 with
// their second kernel 13.8 and 26.7; 512 fp32 keys 13.0 and 30.3, 14.2 and 29.7.
void shape_of(PagedArgs& a, int keys_of_piece) {
  int64_t most = int64_t(a.table_width) * a.page;
  if (a.window > 0) most = smaller(most, int64_t(a.window) * a.frame + a.sinks);
  most = larger(most, int64_t(1));
  const int64_t units = int64_t(a.batch) * a.kv_heads * a.head_blocks;
  const int64_t step = kWaves * keys_of_piece;
  if (most <= 8 * step) {
    a.stretch = static_cast<int>(ceil_div(most, step) * step);
    a.splits = 1;
    return;
  }
  int64_t splits = larger(int64_t(units > 256 || most * units < 512 * 1024 ? 512 : 1024) / units, int64_t(1));
  if (units > 256) splits = larger(splits, smaller(ceil_div(most, 4608), int64_t(4096) / units));
  const int64_t stretch = ceil_div(larger(ceil_div(most, splits), 2 * step), step) * step;
  const int64_t fits = int64_t(kTable - 4) * a.page / step * step;
  a.stretch = static_cast<int>(smaller(smaller(stretch, fits), ceil_div(most, step) * step));
  a.splits = static_cast<int>(ceil_div(most, a.stretch));
}

size_t part_bytes(const PagedArgs& a) { return a.splits > 1 ? static_cast<size_t>(a.splits) * a.batch * a.heads * 65 * sizeof(float) : 0; }

int check_sizes(const char* fn, int dtype, int64_t batch, int heads, int kv_heads, int64_t table_width, int64_t n_pages, int page, int64_t frame,
                int64_t window, int64_t sinks, PagedArgs& a) {
  if (dtype != BSGA_BF16 && dtype != BSGA_FP32) return fail(BSGA_ERR_INVALID_ARG, "%s: unknown dtype %d", fn, dtype);
  if (batch < 0 || batch > 65535) return fail(BSGA_ERR_INVALID_ARG, "%s: batch must be in [0, 65535], got %lld", fn, (long long)batch);
  if (heads < 1 || heads > 65535 || kv_heads < 1 || heads % kv_heads != 0)
    return fail(BSGA_ERR_INVALID_ARG, "%s: heads must be in [1, 65535] and a multiple of kv_heads, got %d and %d", fn, heads, kv_heads);
  if (page < 1 || page > 65536) return fail(BSGA_ERR_INVALID_ARG, "%s: page must be in [1, 65536] tokens, got %d", fn, page);
  const int64_t most = int64_t(1) << 30;
  if (n_pages < 0 || n_pages > most) return fail(BSGA_ERR_INVALID_ARG, "%s: n_pages must be in [0, 2^30], got %lld", fn, (long long)n_pages);
  if (table_width < 0 || table_width > most / page)
    return fail(BSGA_ERR_INVALID_ARG, "%s: a sequence's pages must hold up to 2^30 tokens, got %lld pages", fn, (long long)table_width);
  if (frame < 1 || frame > (1 << 24)) return fail(BSGA_ERR_INVALID_ARG, "%s: frame must be in [1, 2^24] tokens, got %lld", fn, (long long)frame);
  if (window < 0) return fail(BSGA_ERR_INVALID_ARG, "%s: window must be >= 0 frames (0: no limit), got %lld", fn, (long long)window);
  if (sinks < 0) return fail(BSGA_ERR_INVALID_ARG, "%s: sinks must be >= 0, got %lld", fn, (long long)sinks);
  a.batch = static_cast<int>(batch);
  a.heads = heads;
  a.kv_heads = kv_heads;
  a.group = heads / kv_heads;
  a.head_blocks = static_cast<int>(ceil_div(a.group, kHeads));
  a.table_width = n_pages > 0 ? static_cast<int>(table_width) : 0;  // without pages there are no keys
  a.n_pages = static_cast<int>(n_pages);
  a.page = page;
  a.frame = static_cast<int>(frame);
  a.window = static_cast<int>(smaller(window, most));
  a.sinks = static_cast<int>(smaller(sinks, most));
  while ((int64_t(1) << a.shift) < page) ++a.shift;
  a.magic = static_cast<unsigned>(((uint64_t(1) << (31 + a.shift)) + page - 1) / page);
  return BSGA_OK;
}

}  // namespace
}  // namespace bsga

using namespace bsga;

extern "C" {

size_t bsga_paged_attn_workspace_bytes(int dtype, int64_t batch, int heads, int kv_heads, int64_t table_width, int64_t n_pages, int page,
                                       int64_t frame, int64_t window, int64_t sinks) {
  PagedArgs a = {};
  if (check_sizes("", dtype, batch, heads, kv_heads, table_width, n_pages, page, frame, window, sinks, a) || batch == 0) return 0;
  shape_of(a, dtype == BSGA_BF16 ? Ops16<__bf16>::kKeys : Ops16<float>::kKeys);
  return part_bytes(a);
}

int bsga_paged_attn(const void* q, int64_t q_batch, int64_t q_head, const void* k_cache, const void* v_cache, int dtype, int64_t batch, int heads,
                    int kv_heads, int head_dim, const int32_t* page_table, int64_t table_width, const int32_t* lengths, int64_t n_pages, int page,
                    float softmax_scale, int64_t frame, int64_t window, int64_t sinks, void* out, float* lse, void* workspace, size_t workspace_bytes,
                    void* stream) {
  const char* fn = "bsga_paged_attn";
  clear_error();
  PagedArgs a = {};
  if (head_dim != 64) return fail(BSGA_ERR_UNSUPPORTED, "%s: head_dim must be 64, got %d", fn, head_dim);
  if (int rc = check_sizes(fn, dtype, batch, heads, kv_heads, table_width, n_pages, page, frame, window, sinks, a)) return rc;
  if (!(softmax_scale > 0.0f) || !isfinite(softmax_scale)) return fail(BSGA_ERR_INVALID_ARG, "%s: softmax_scale must be finite and > 0", fn);
  if (int64_t(kv_heads) * a.head_blocks > 65535) return fail(BSGA_ERR_UNSUPPORTED, "%s: too many heads", fn);
  if (batch == 0) return BSGA_OK;
  if (int rc = check_view(fn, "q", q, q_batch, q_head, dtype == BSGA_BF16 ? 2 : 4, a.q)) return rc;
  if (!lengths || (a.table_width > 0 && (!page_table || !k_cache || !v_cache)))
    return fail(BSGA_ERR_INVALID_ARG, "%s: k_cache, v_cache, page_table and lengths must be non-null", fn);
  if (!out || !aligned16(out) || !aligned16(k_cache) || !aligned16(v_cache))
    return fail(BSGA_ERR_INVALID_ARG, "%s: out must be non-null, it and the caches 16-byte aligned", fn);
  a.k = static_cast<const unsigned char*>(k_cache);
  a.v = static_cast<const unsigned char*>(v_cache);
  a.page_table = page_table;
  a.lengths = lengths;
  a.out = static_cast<unsigned char*>(out);
  a.lse = lse;
  a.scale_log2 = softmax_scale * kLog2e;
  shape_of(a, dtype == BSGA_BF16 ? Ops16<__bf16>::kKeys : Ops16<float>::kKeys);
  const size_t need = part_bytes(a);
  if (need > 0 && (!workspace || workspace_bytes < need))
    return fail(BSGA_ERR_WORKSPACE, "%s: workspace has %zu bytes, %zu needed", fn, workspace ? workspace_bytes : 0, need);
  if (!aligned16(workspace)) return fail(BSGA_ERR_INVALID_ARG, "%s: workspace must be 16-byte aligned", fn);
  const int64_t rows = batch * heads;
  a.part = static_cast<float*>(workspace);
  a.part_lse = a.part + int64_t(a.splits) * rows * 64;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const dim3 grid(static_cast<unsigned>(a.splits), static_cast<unsigned>(kv_heads * a.head_blocks), static_cast<unsigned>(batch));
  if (dtype == BSGA_BF16) hipLaunchKernelGGL(paged_kernel<__bf16>, grid, dim3(64 * kWaves), 0, s, a);
  else hipLaunchKernelGGL(paged_kernel<float>, grid, dim3(64 * kWaves), 0, s, a);
  if (int rc = check_hip(hipGetLastError(), "bsga_paged_attn launch")) return rc;
  if (a.splits == 1) return BSGA_OK;
  return dtype == BSGA_BF16 ? launch_join<__bf16>(a.part, a.part_lse, rows, a.splits, a.out, a.lse, s)
                            : launch_join<float>(a.part, a.part_lse, rows, a.splits, a.out, a.lse, s);
}

}  // extern "C"
