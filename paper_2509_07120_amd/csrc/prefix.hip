// Attention of one new token for each sequence, over pages, where sequences begin with tokens that they share: a prefix, which is read once for all of them.
//
// Sequence b of prefix g sees the P_g tokens of the prefix and then its own; its query stands at position P_g + lengths[b] - 1.  The queries of all sequences of a
// prefix that share a key head are the columns of the products over the prefix; the sequences' own keys go by a workgroup each.  Both leave, for each
// stretch of keys, sums and their logarithms, which a last kernel joins.
#include "paged.h"

#include <math.h>

namespace bsga {
namespace {

struct PrefixArgs {
  View q;                             // [batch, heads, 64]: token is the sequence's stride
  Pages pages;
  const int32_t *page_table, *lengths;                     // of the own tokens
  const int32_t *prefix_table, *prefix_lengths, *starts;   // sequences starts[g] .. starts[g + 1] - 1 have prefix g
  float *part, *part_lse;             // [splits + own_splits][batch, heads, 64] and [..][batch, heads]
  int batch, heads, group, head_blocks, table_width, prefixes, prefix_width, frame, window, sinks;
  int splits, stretch, own_splits, own_stretch;
  float scale_log2;

  __device__ __forceinline__ int start(int g) const { return min(max(starts[g], 0), batch); }
  __device__ __forceinline__ int prefix_length(int g) const { return min(max(prefix_lengths[g], 0), prefix_width * pages.page); }
  __device__ __forceinline__ int length(int b) const { return min(max(lengths[b], 0), table_width * pages.page); }
  // of a query with n tokens up to itself: the first key of its window, and the first tokens in front of that it sees
  __device__ __forceinline__ void seen(int n, int& lo, int& s) const {
    lo = s = 0;
    if (window > 0 && n > 0) {
      const int f = (n - 1) / frame;
      lo = f < window ? 0 : (f + 1 - window) * frame;
      s = min(sinks, lo);
    }
  }
};

// The prefix of sequence b, or -1: whole waves.
__device__ __forceinline__ int prefix_of(const PrefixArgs& a, int b, int lane) {
  int g = 0;
  for (int i = 0; i < a.prefixes; i += 64) g += __popcll(__ballot(i + lane < a.prefixes && a.start(min(i + lane, a.prefixes - 1) + 1) <= b));
  return g < a.prefixes && a.start(g) <= b ? g : -1;
}

// Unit u of a grid over tiles of `tile` queries of every prefix, one prefix after the other: the prefix g, or -1, and the tile; whole waves.
__device__ __forceinline__ int unit_of(const PrefixArgs& a, int u, int tile, int lane, int& at) {
  int base = 0;
  for (int i = 0; i < a.prefixes; i += 64) {
    const int g = min(i + lane, a.prefixes - 1);
    const int n = i + lane < a.prefixes ? max(a.start(g + 1) - a.start(g), 0) : 0;
    const int tiles = (n * a.group + tile - 1) / tile;
    int end = tiles;
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) {
      const int other = __shfl_up(end, x);
      end += lane >= x ? other : 0;
    }
    const unsigned long long behind = __ballot(base + end > u);
    if (behind != 0) {
      const int of = __builtin_ctzll(behind);
      at = u - base - __shfl(end - tiles, of);
      return __builtin_amdgcn_readfirstlane(i + of);
    }
    base += __shfl(end, 63);
  }
  return -1;
}

__device__ __forceinline__ void leave(const PrefixArgs& a, int part, int64_t row, int d, const f32x4& y, float top, float sum) {
  const int64_t rows = int64_t(a.batch) * a.heads;
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  *reinterpret_cast<f32x4*>(a.part + (part * rows + row) * 64 + d) = y * inv;
  if (d == 0) a.part_lse[part * rows + row] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
}

// The keys of a prefix, for 16 of the queries of its sequences at one key head.
template <typename T, typename C>
__global__ __launch_bounds__(64 * kWaves, 2) void prefix_kernel(const PrefixArgs a) {
  typedef Ops16<T, C> P;
  __shared__ __align__(16) unsigned char smem[kWaves * kWaveLds<P>];
  __shared__ int table[kTable];
  __shared__ float sums[kWaves][2][kHeads];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, q = lane >> 4;
  const int split = blockIdx.x, hk = blockIdx.y;
  int tile;
  const int g = unit_of(a, blockIdx.z, kHeads, lane, tile);
  if (g < 0) return;
  const int b0 = a.start(g), first = tile * kHeads, queries = min((a.start(g + 1) - b0) * a.group - first, kHeads);
  auto row_of = [&](int i, int& b) {  // query i of the tile: its sequence, and its row of the result
    const int x = first + i;
    b = b0 + x / a.group;
    return int64_t(b) * a.heads + hk * a.group + x % a.group;
  };
  const int length = a.prefix_length(g);
  int b;
  const int64_t row = row_of(min(c, queries - 1), b);
  int lo, s;
  a.seen(length + a.length(b), lo, s);
  lo = min(lo, length);
  Stretch st = {};
  st.lo = lo;
  int most = lo;
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) {
    st.lo = min(st.lo, __shfl_xor(st.lo, o));
    most = max(most, __shfl_xor(most, o));
  }
  st.lo = __builtin_amdgcn_readfirstlane(st.lo);
  most = __builtin_amdgcn_readfirstlane(most);
  st.s = min(a.sinks, st.lo);
  const int count = st.s + length - st.lo;
  st.x0 = split * a.stretch, st.x1 = min(st.x0 + a.stretch, count);
  if (st.x0 >= st.x1) {  // the whole workgroup
    int of;
    if (threadIdx.x < queries) {
      const int64_t at = row_of(threadIdx.x, of);
      a.part_lse[int64_t(split) * a.batch * a.heads + at] = -INFINITY;
    }
    return;
  }
  st.fill(a.pages, a.prefix_table + int64_t(g) * a.prefix_width, table);
  typename P::A qf[P::kSteps];
  P::row(a.q.p + b * a.q.token + (row - int64_t(b) * a.heads) * a.q.head, q, qf);
  __syncthreads();
  f32x4 o[4];
  float m, l;
  unsigned char* const mine = smem + wave * kWaveLds<P>;
  if (most > st.lo)
    go_over<P, true>(a.pages, st, table, hk, wave, lane, mine, a.scale_log2, qf, [&](int j) { return j >= lo || j < a.sinks; }, o, m, l);
  else
    go_over<P, false>(a.pages, st, table, hk, wave, lane, mine, a.scale_log2, qf, [](int) { return true; }, o, m, l);
  f32x4 y;
  float top, sum;
  join_waves<P>(smem, sums, wave, lane, o, m, l, y, top, sum);
  const int i = threadIdx.x >> 4, d = (threadIdx.x & 15) * 4;
  if (i >= queries) return;
  leave(a, split, row_of(i, b), d, y, top, sum);
}

// The own keys of a sequence.
template <typename T, typename C>
__global__ __launch_bounds__(64 * kWaves, 2) void own_kernel(const PrefixArgs a) {
  typedef Ops16<T, C> P;
  __shared__ __align__(16) unsigned char smem[kWaves * kWaveLds<P>];
  __shared__ int table[kTable];
  __shared__ float sums[kWaves][2][kHeads];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, q = lane >> 4;
  const int b = blockIdx.z, split = blockIdx.x;
  const int hk = blockIdx.y / a.head_blocks, hb = blockIdx.y - hk * a.head_blocks;
  const int heads = min(kHeads, a.group - hb * kHeads), h0 = hk * a.group + hb * kHeads;
  const int64_t rows = int64_t(a.batch) * a.heads, row0 = int64_t(b) * a.heads + h0;
  const int g = prefix_of(a, b, lane);
  if (g < 0 && split == 0 && threadIdx.x < heads)  // nobody else writes the prefix's parts of this sequence
    for (int x = 0; x < a.splits; ++x) a.part_lse[x * rows + row0 + threadIdx.x] = -INFINITY;
  const int behind = g < 0 ? 0 : a.prefix_length(g), length = a.length(b);
  Stretch st = {};
  a.seen(behind + length, st.lo, st.s);
  st.s = max(st.s - behind, 0);
  st.lo = min(max(st.lo - behind, 0), length);
  const int count = st.s + length - st.lo;
  st.x0 = split * a.own_stretch, st.x1 = min(st.x0 + a.own_stretch, count);
  if (st.x0 >= st.x1) {  // the whole workgroup
    if (threadIdx.x < heads) a.part_lse[(a.splits + split) * rows + row0 + threadIdx.x] = -INFINITY;
    return;
  }
  st.fill(a.pages, a.page_table + int64_t(b) * a.table_width, table);
  typename P::A qf[P::kSteps];
  P::row(a.q.p + b * a.q.token + (h0 + min(c, heads - 1)) * a.q.head, q, qf);
  __syncthreads();
  f32x4 o[4];
  float m, l;
  go_over<P, false>(a.pages, st, table, hk, wave, lane, smem + wave * kWaveLds<P>, a.scale_log2, qf, [](int) { return true; }, o, m, l);
  f32x4 y;
  float top, sum;
  join_waves<P>(smem, sums, wave, lane, o, m, l, y, top, sum);
  const int head = threadIdx.x >> 4;
  if (head >= heads) return;
  leave(a, a.splits + split, row0 + head, (threadIdx.x & 15) * 4, y, top, sum);
}

int keys_of_piece(int dtype, int cache_dtype) {
  return cache_dtype == BSGA_E4M3 ? Ops16E4m3::kKeys : dtype == BSGA_BF16 ? Ops16<__bf16, __bf16>::kKeys : Ops16<float, float>::kKeys;
}

// Tiles of the prefixes' queries, whichever sequences have which prefix: at most one that is not full for each.
int64_t tiles_of(const PrefixArgs& a, int tile) {
  const int64_t queries = int64_t(a.batch) * a.group;
  return smaller(queries / tile + smaller(int64_t(a.prefixes), int64_t(a.batch)), queries);
}

void shape_of(PrefixArgs& a, int keys) {
  int64_t most = int64_t(a.prefix_width) * a.pages.page, own = int64_t(a.table_width) * a.pages.page;
  if (a.window > 0) {
    const int64_t seen = int64_t(a.window) * a.frame + a.sinks;
    most = smaller(most, seen);
    own = smaller(own, seen);
  }
  const int64_t units = larger(ceil_div(int64_t(a.batch) * a.group, kHeads), int64_t(1)) * a.pages.kv_heads;
  cut(most, units, keys, a.pages.page, a.stretch, a.splits);
  cut(own, int64_t(a.batch) * a.pages.kv_heads * a.head_blocks, keys, a.pages.page, a.own_stretch, a.own_splits);
}

size_t part_bytes(const PrefixArgs& a) { return (static_cast<size_t>(a.splits) + a.own_splits) * a.batch * a.heads * 65 * sizeof(float); }

int check_sizes(const char* fn, int dtype, int cache_dtype, int64_t batch, int heads, int kv_heads, int64_t table_width, int64_t prefixes,
                int64_t prefix_width, int64_t n_pages, int page, int64_t frame, int64_t window, int64_t sinks, PrefixArgs& a) {
  if (dtype != BSGA_BF16 && dtype != BSGA_FP32) return fail(BSGA_ERR_INVALID_ARG, "%s: unknown dtype %d", fn, dtype);
  if (cache_dtype != BSGA_E4M3 && cache_dtype != dtype)
    return fail(BSGA_ERR_INVALID_ARG, "%s: a cache must be in 8 bits or of the queries' type, got %d and %d", fn, cache_dtype, dtype);
  if (batch < 0 || batch > 65535) return fail(BSGA_ERR_INVALID_ARG, "%s: batch must be in [0, 65535], got %lld", fn, (long long)batch);
  if (heads < 1 || heads > 65535 || kv_heads < 1 || heads % kv_heads != 0)
    return fail(BSGA_ERR_INVALID_ARG, "%s: heads must be in [1, 65535] and a multiple of kv_heads, got %d and %d", fn, heads, kv_heads);
  if (int rc = check_pages(fn, kv_heads, n_pages, page, a.pages)) return rc;
  const int64_t most = int64_t(1) << 30;
  if (prefixes < 0 || prefixes > 65535) return fail(BSGA_ERR_INVALID_ARG, "%s: prefixes must be in [0, 65535], got %lld", fn, (long long)prefixes);
  if (table_width < 0 || table_width > most / page || prefix_width < 0 || prefix_width > most / page - table_width)
    return fail(BSGA_ERR_INVALID_ARG, "%s: the pages of a sequence and its prefix must hold up to 2^30 tokens, got %lld and %lld pages", fn,
                (long long)table_width, (long long)prefix_width);
  if (frame < 1 || frame > (1 << 24)) return fail(BSGA_ERR_INVALID_ARG, "%s: frame must be in [1, 2^24] tokens, got %lld", fn, (long long)frame);
  if (window < 0) return fail(BSGA_ERR_INVALID_ARG, "%s: window must be >= 0 frames (0: no limit), got %lld", fn, (long long)window);
  if (sinks < 0) return fail(BSGA_ERR_INVALID_ARG, "%s: sinks must be >= 0, got %lld", fn, (long long)sinks);
  a.batch = static_cast<int>(batch);
  a.heads = heads;
  a.group = heads / kv_heads;
  a.head_blocks = static_cast<int>(ceil_div(a.group, kHeads));
  a.table_width = n_pages > 0 ? static_cast<int>(table_width) : 0;  // without pages there are no keys
  a.prefix_width = n_pages > 0 ? static_cast<int>(prefix_width) : 0;
  a.prefixes = a.prefix_width > 0 ? static_cast<int>(prefixes) : 0;  // (prefixes of nothing)
  if (a.prefixes == 0) a.prefix_width = 0;
  a.frame = static_cast<int>(frame);
  a.window = static_cast<int>(smaller(window, most));
  a.sinks = static_cast<int>(smaller(sinks, most));
  if (batch * a.group > (int64_t(1) << 30) || tiles_of(a, kHeads) > 65535 || int64_t(kv_heads) * a.head_blocks > 65535)
    return fail(BSGA_ERR_UNSUPPORTED, "%s: too many queries (%lld sequences of %d heads)", fn, (long long)batch, heads);
  return BSGA_OK;
}

template <typename T, typename C>
int launch(const PrefixArgs& a, unsigned char* out, float* lse, hipStream_t s) {
  if (a.prefixes > 0) {
    const dim3 grid(static_cast<unsigned>(a.splits), static_cast<unsigned>(a.pages.kv_heads), static_cast<unsigned>(tiles_of(a, kHeads)));
    hipLaunchKernelGGL((prefix_kernel<T, C>), grid, dim3(64 * kWaves), 0, s, a);
  }
  const dim3 grid(static_cast<unsigned>(a.own_splits), static_cast<unsigned>(a.pages.kv_heads * a.head_blocks), static_cast<unsigned>(a.batch));
  hipLaunchKernelGGL((own_kernel<T, C>), grid, dim3(64 * kWaves), 0, s, a);
  if (int rc = check_hip(hipGetLastError(), "bsga_prefix_attn")) return rc;
  return launch_join<T>(a.part, a.part_lse, int64_t(a.batch) * a.heads, a.splits + a.own_splits, out, lse, s);
}

}  // namespace
}  // namespace bsga

using namespace bsga;

extern "C" {

size_t bsga_prefix_attn_workspace_bytes(int dtype, int cache_dtype, int64_t batch, int heads, int kv_heads, int64_t table_width, int64_t prefixes,
                                        int64_t prefix_width, int64_t n_pages, int page, int64_t frame, int64_t window, int64_t sinks) {
  PrefixArgs a = {};
  if (check_sizes("", dtype, cache_dtype, batch, heads, kv_heads, table_width, prefixes, prefix_width, n_pages, page, frame, window, sinks, a) || batch == 0)
    return 0;
  shape_of(a, keys_of_piece(dtype, cache_dtype));
  return part_bytes(a);
}

int bsga_prefix_attn(const void* q, int64_t q_batch, int64_t q_head, const void* k_cache, const void* v_cache, const uint8_t* k_scale, const uint8_t* v_scale,
                     int dtype, int cache_dtype, int64_t batch, int heads, int kv_heads, int head_dim, const int32_t* page_table, int64_t table_width,
                     const int32_t* lengths, const int32_t* prefix_table, int64_t prefix_width, const int32_t* prefix_lengths, const int32_t* starts,
                     int64_t prefixes, int64_t n_pages, int page, float softmax_scale, int64_t frame, int64_t window, int64_t sinks, void* out, float* lse,
                     void* workspace, size_t workspace_bytes, void* stream) {
  const char* fn = "bsga_prefix_attn";
  clear_error();
  PrefixArgs a = {};
  if (head_dim != 64) return fail(BSGA_ERR_UNSUPPORTED, "%s: head_dim must be 64, got %d", fn, head_dim);
  if (int rc = check_sizes(fn, dtype, cache_dtype, batch, heads, kv_heads, table_width, prefixes, prefix_width, n_pages, page, frame, window, sinks, a))
    return rc;
  if (!(softmax_scale > 0.0f) || !isfinite(softmax_scale)) return fail(BSGA_ERR_INVALID_ARG, "%s: softmax_scale must be finite and > 0", fn);
  if (batch == 0) return BSGA_OK;
  if (int rc = check_view(fn, "q", q, q_batch, q_head, dtype == BSGA_BF16 ? 2 : 4, a.q)) return rc;
  const bool any = a.table_width > 0 || a.prefixes > 0;
  if (!lengths || (a.table_width > 0 && !page_table) || (any && (!k_cache || !v_cache)))
    return fail(BSGA_ERR_INVALID_ARG, "%s: k_cache, v_cache, page_table and lengths must be non-null", fn);
  if (a.prefixes > 0 && (!prefix_table || !prefix_lengths || !starts))
    return fail(BSGA_ERR_INVALID_ARG, "%s: prefix_table, prefix_lengths and starts must be non-null", fn);
  if (any && cache_dtype == BSGA_E4M3 && (!k_scale || !v_scale)) return fail(BSGA_ERR_INVALID_ARG, "%s: k_scale and v_scale must be non-null", fn);
  if (!out || !aligned16(out) || !aligned16(k_cache) || !aligned16(v_cache))
    return fail(BSGA_ERR_INVALID_ARG, "%s: out must be non-null, it and the caches 16-byte aligned", fn);
  a.pages.k = static_cast<const unsigned char*>(k_cache);
  a.pages.v = static_cast<const unsigned char*>(v_cache);
  a.pages.k_scale = k_scale;
  a.pages.v_scale = v_scale;
  a.page_table = page_table;
  a.lengths = lengths;
  a.prefix_table = prefix_table;
  a.prefix_lengths = prefix_lengths;
  a.starts = starts;
  a.scale_log2 = softmax_scale * kLog2e;
  shape_of(a, keys_of_piece(dtype, cache_dtype));
  const size_t need = part_bytes(a);
  if (!workspace || workspace_bytes < need)
    return fail(BSGA_ERR_WORKSPACE, "%s: workspace has %zu bytes, %zu needed", fn, workspace ? workspace_bytes : 0, need);
  if (!aligned16(workspace)) return fail(BSGA_ERR_INVALID_ARG, "%s: workspace must be 16-byte aligned", fn);
  a.part = static_cast<float*>(workspace);
  a.part_lse = a.part + (int64_t(a.splits) + a.own_splits) * batch * heads * 64;
  unsigned char* const to = static_cast<unsigned char*>(out);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (dtype == BSGA_BF16) return cache_dtype == BSGA_E4M3 ? launch<__bf16, E4m3>(a, to, lse, s) : launch<__bf16, __bf16>(a, to, lse, s);
  return cache_dtype == BSGA_E4M3 ? launch<float, E4m3>(a, to, lse, s) : launch<float, float>(a, to, lse, s);
}

}  // extern "C"
