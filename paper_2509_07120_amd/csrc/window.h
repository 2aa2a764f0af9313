// What the kernels of attention with a window share, forward and backward: which keys a query sees, tiles of 64 rows in LDS, and operands of the
// matrix products for both types.
//
// Query i stands at position p = q_start + i, in frame p / F.  It sees the keys [0, min(sinks, lo)) and [lo, hi) with hi the end of its
// frame and lo the start of the frame window - 1 frames earlier; both cut to the keys that there are.  Both ends grow with p.
#pragma once

#include <type_traits>

#include "bf16_tile.h"
#include "bsga_internal.h"

namespace bsga {
namespace {

constexpr int kTile = 64;            // rows of a tile
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct Seen {
  int n_q, n_k, q_start, frame, window, sinks;
  // [lo, hi) of query i; the keys in front of lo that it sees are those below `sinks`
  __host__ __device__ void range(int i, int& lo, int& hi) const {
    const int p = q_start + i;
    if (p < 0) {
      lo = hi = 0;
      return;
    }
    const int f = p / frame;
    hi = static_cast<int>(smaller(int64_t(f + 1) * frame, int64_t(n_k)));
    lo = f < window ? 0 : static_cast<int>(smaller(int64_t(f + 1 - window) * frame, int64_t(hi)));
  }
};

// The tiles of a workgroup's rows: `first` of them from key 0 on, then those from key tile `start` on.
struct Tiles {
  int first, start, count;
  __host__ __device__ int key(int t) const { return (t < first ? t : start + t - first) * kTile; }
};

__host__ __device__ inline Tiles tiles_of(const Seen& s, int i0, int i1) {  // queries [i0, i1)
  int lo, hi, lo1, hi1;
  s.range(i0, lo, hi);
  s.range(i1 - 1, lo1, hi1);
  Tiles t;
  t.first = (min(min(s.sinks, lo1), lo) + kTile - 1) / kTile;
  t.start = max(lo / kTile, t.first);
  t.count = t.first + max((hi1 + kTile - 1) / kTile - t.start, 0);
  return t;
}

// What all lanes agree on, in scalar registers: 64-bit minima are vector instructions, and whatever is computed from them each tile would be too
// (descriptors, bounds: 45 of 250 instructions of a tile of the gradient's query rows).
__device__ __forceinline__ int scalar(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ Tiles scalar(const Tiles& t) { return {scalar(t.first), scalar(t.start), scalar(t.count)}; }

// A tensor [heads, tokens, 64] with strides in bytes.
struct View {
  const unsigned char* p;
  int64_t token, head;
};

template <typename T>
struct Ops;

template <>
struct Ops<__bf16> {
  typedef bf16x8 A;                          // what a lane holds of an operand
  static constexpr int kRow = 128;           // bytes of a row
  static constexpr int kSteps = 4;           // products over the 64 numbers of a row
  static constexpr int kCols = 2;            // products over 32 rows
  static __device__ __forceinline__ f32x16 product(A a, A b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
  // 16-byte chunk c of tile row r lies at c ^ swizzle(r).  Rows are 128 bytes, two to the 64 banks: reading one chunk of 16 rows meets every
  // bank once if the eight even rows (and the odd ones) have eight swizzles, and the transposing reads, of four chunks of four rows, if rows r and
  // r + 2 differ in the bit of 4.  Bits 1, 2, 3 of r in reverse do both, and rows 16 apart have the same.
  static __host__ __device__ constexpr int swizzle(int r) { return ((r & 2) << 1) | ((r >> 1) & 2) | ((r >> 3) & 1); }
  // row r's numbers from memory: lane half g holds 8 of each 16
  static __device__ __forceinline__ void row(const unsigned char* p, int g, A (&a)[kSteps]) {
#pragma unroll
    for (int c = 0; c < 4; ++c) a[c] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(p + (2 * c + g) * 16));
  }
  static __device__ __forceinline__ void rows(const unsigned char* tile, int r, int g, A (&a)[kSteps]) {
#pragma unroll
    for (int c = 0; c < 4; ++c) a[c] = *LDS_PTR(bf16x8, tile + r * kRow + (((2 * c + g) ^ swizzle(r)) << 4));
  }
  // columns 32 db .. + 31 of the 32 tile rows from r0 on: lane (n, g) holds column n of the rows whose products' results lie in the lane
  static __device__ __forceinline__ void columns(const unsigned char* tile, int r0, int db, int lane, A (&a)[kCols]) {
    const int m = (lane & 15) >> 2, j = lane & 3, G = lane >> 4;
    const int chunk = db * 4 + 2 * (G & 1) + (j >> 1);
#pragma unroll
    for (int cp = 0; cp < 2; ++cp) {
      u32x2 x[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = r0 + 16 * cp + 8 * e + 4 * (lane >> 5) + m;
        const unsigned char* p = tile + r * kRow + ((chunk ^ swizzle(r)) << 4) + (j & 1) * 8;
        x[e] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(p)));
      }
      a[cp] = __builtin_bit_cast(bf16x8, u32x4{x[0][0], x[0][1], x[1][0], x[1][1]});
    }
  }
  static __device__ __forceinline__ float dot(const A (&a)[kSteps], const A (&b)[kSteps]) {  // of the lane's halves of two rows
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < kSteps; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) s += static_cast<float>(a[c][e]) * static_cast<float>(b[c][e]);
    return s;
  }
  // a product's result, rounded to an operand
  static __device__ __forceinline__ void round(const f32x16& x, A (&a)[kCols]) {
#pragma unroll
    for (int cp = 0; cp < 2; ++cp) {
      u32x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = pack_bf16(x[8 * cp + 2 * e], x[8 * cp + 2 * e + 1]);
      a[cp] = __builtin_bit_cast(bf16x8, w);
    }
  }
  static __device__ __forceinline__ float number(const unsigned char* p, int i) {
    return __uint_as_float(static_cast<unsigned>(reinterpret_cast<const unsigned short*>(p)[i]) << 16);
  }
  static __device__ __forceinline__ void store4(unsigned char* p, int i, float a, float b, float c, float d) {
    *reinterpret_cast<u32x2*>(p + i * 2) = u32x2{pack_bf16(a, b), pack_bf16(c, d)};
  }
  static __device__ __forceinline__ void store1(unsigned char* p, int i, float x) {
    reinterpret_cast<unsigned short*>(p)[i] = static_cast<unsigned short>(pack_bf16(x, 0.f));
  }
};

template <>
struct Ops<float> {
  typedef float A;
  static constexpr int kRow = 256;
  static constexpr int kSteps = 32;
  static constexpr int kCols = 16;
  static __device__ __forceinline__ f32x16 product(A a, A b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0); }
  // rows are 256 bytes, all 64 banks: 16 swizzles for 16 rows, and rows 4 apart, read by the two lane halves in columns(), differ in the bit of 8
  static __host__ __device__ constexpr int swizzle(int r) { return ((r & 4) << 1) | ((r >> 1) & 4) | (r & 3); }
  // lane half g holds 4 of each 8 numbers
  static __device__ __forceinline__ void row(const unsigned char* p, int g, A (&a)[kSteps]) {
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(p + (2 * c + g) * 16);
#pragma unroll
      for (int e = 0; e < 4; ++e) a[4 * c + e] = x[e];
    }
  }
  static __device__ __forceinline__ void rows(const unsigned char* tile, int r, int g, A (&a)[kSteps]) {
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      const f32x4 x = *LDS_PTR(f32x4, tile + r * kRow + (((2 * c + g) ^ swizzle(r)) << 4));
#pragma unroll
      for (int e = 0; e < 4; ++e) a[4 * c + e] = x[e];
    }
  }
  static __device__ __forceinline__ void columns(const unsigned char* tile, int r0, int db, int lane, A (&a)[kCols]) {
    const int d = db * 32 + (lane & 31);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int r = r0 + 8 * (i >> 2) + 4 * (lane >> 5) + (i & 3);
      a[i] = *LDS_PTR(float, tile + r * kRow + (((d >> 2) ^ swizzle(r)) << 4) + (d & 3) * 4);
    }
  }
  static __device__ __forceinline__ float dot(const A (&a)[kSteps], const A (&b)[kSteps]) {
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < kSteps; ++c) s += a[c] * b[c];
    return s;
  }
  static __device__ __forceinline__ void round(const f32x16& x, A (&a)[kCols]) {
#pragma unroll
    for (int i = 0; i < 16; ++i) a[i] = x[i];
  }
  static __device__ __forceinline__ float number(const unsigned char* p, int i) { return reinterpret_cast<const float*>(p)[i]; }
  static __device__ __forceinline__ void store4(unsigned char* p, int i, float a, float b, float c, float d) {
    *reinterpret_cast<f32x4*>(p + i * 4) = f32x4{a, b, c, d};
  }
  static __device__ __forceinline__ void store1(unsigned char* p, int i, float x) { reinterpret_cast<float*>(p)[i] = x; }
};

__device__ __forceinline__ void clear(f32x16& x) {
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] = 0.f;
}

// The larger of what lanes n and n + 32 have, in both, without the way through LDS.
__device__ __forceinline__ float top_of_halves(float x) {
  const unsigned u = __float_as_uint(x);
  const auto both = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
}

// Of a lane's numbers of one product, of tile rows `at` + 8 (i / 4) + i % 4, those outside [first, last) become `hidden`: three instructions for each.
__device__ __forceinline__ void keep(f32x16& x, int at, int first, int last, float hidden) {
  const int from = first - at;
  const unsigned span = static_cast<unsigned>(max(last - first, 0));
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] = static_cast<unsigned>(8 * (i >> 2) + (i & 3) - from) < span ? x[i] : hidden;
}

// Those that a query with the range [lo, hi) does not see; `sinks` for tile rows below that.
__device__ __forceinline__ void keep_seen(f32x16& x, int at, int lo, int hi, int sinks, bool below_sinks, float hidden) {
  if (!below_sinks) {
    keep(x, at, lo, hi, hidden);
    return;
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int j = at + 8 * (i >> 2) + (i & 3);
    x[i] = j < hi && (j >= lo || j < sinks) ? x[i] : hidden;
  }
}

// Rows [r0, r0 + 64) of one head of a tensor straight into a tile (rows past the tensor's end become zeros), by `WAVES` waves.  The
// descriptor starts at the tile, so that 32-bit offsets do whatever the tensor's size is.
template <typename T, int WAVES>
struct TileLoad {
  static constexpr int kRow = Ops<T>::kRow, kChunks = kRow / 16, kRows = 64 / kChunks, kLoads = kTile / kRows / WAVES;
  int64_t token;
  unsigned offset[kLoads];  // of the lane's 16 bytes in each of the wave's loads
  unsigned wave_lds;

  __device__ __forceinline__ TileLoad(int64_t token, int wave, int lane) : token(token), wave_lds(wave * 1024u) {
    const int pos = lane % kChunks;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int r = (WAVES * i + wave) * kRows + lane / kChunks;
      offset[i] = static_cast<unsigned>(r * token) + ((pos ^ Ops<T>::swizzle(r)) << 4);
    }
  }
  // descriptor of a tile that starts at p, with `left` rows from there to the tensor's end
  __device__ __forceinline__ i32x4 rsrc_at(const unsigned char* p, int left) const {
    return make_rsrc(p, left > 0 ? static_cast<unsigned>(min(left, kTile) - 1) * static_cast<unsigned>(token) + kRow : 0u);
  }
  __device__ __forceinline__ i32x4 rsrc(const unsigned char* head, int n, int r0) const { return rsrc_at(head + r0 * token, n - r0); }
  template <int I>
  __device__ __forceinline__ void one(i32x4 rsrc, std::integral_constant<int, I>, unsigned lds) const {
    if constexpr (I < kLoads) dma16<WAVES * I * 1024>(rsrc, offset[I], 0u, __builtin_amdgcn_readfirstlane(lds + wave_lds));
  }
  // part I of four
  template <int I>
  __device__ __forceinline__ void quarter(i32x4 from, std::integral_constant<int, I>, unsigned lds) const {
    if constexpr (kLoads < 4) {
      one(from, std::integral_constant<int, I>{}, lds);
    } else {
      one(from, std::integral_constant<int, 2 * I>{}, lds);
      one(from, std::integral_constant<int, 2 * I + 1>{}, lds);
      static_assert(kLoads == 8, "two loads to a part");
    }
  }
  template <int I = 0>
  __device__ __forceinline__ void rest(i32x4 from, unsigned lds) const {
    if constexpr (I < kLoads) {
      one(from, std::integral_constant<int, I>{}, lds);
      rest<I + 1>(from, lds);
    }
  }
  __device__ __forceinline__ void all(const unsigned char* head, int n, int r0, unsigned lds) const { rest(rsrc(head, n, r0), lds); }
};

__device__ __forceinline__ unsigned lds_address(const unsigned char* p) {
  return static_cast<unsigned>(reinterpret_cast<size_t>((const __attribute__((address_space(3))) unsigned char*)p));
}

// Workgroup w of a grid runs on XCD w % 8.  The units of a grid, head after head, dealt out: an XCD gets whole heads where the number of
// heads allows (16 heads: two each), and the XCDs that share heads get eight neighbours at a time.  So neighbours share an L2, and
// every XCD gets long and short rows alike: 64 neighbours at a time gave one XCD the long rows of all heads.
__device__ __forceinline__ int64_t spread(int64_t w, int64_t all, int heads) {
  const int parts = heads % 8 == 0 ? 8 : heads % 4 == 0 ? 4 : heads % 2 == 0 ? 2 : 1, xcds = 8 / parts;  // parts of the heads, XCDs of a part
  const int64_t p = w / parts, base = p / (8 * xcds) * (8 * xcds), in_part = all / parts;
  const int r = static_cast<int>(p - base);
  return w % parts * in_part + (base + 8 * xcds <= in_part ? base + r % xcds * 8 + r / xcds : p);
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline int check_seen(const char* fn, int64_t n_q, int64_t n_k, int64_t q_start, int64_t frame, int64_t window, int64_t sinks, Seen& s) {
  const int64_t most = int64_t(1) << 24;
  if (n_q < 0 || n_q > most || n_k < 0 || n_k > most)
    return fail(BSGA_ERR_INVALID_ARG, "%s: n_q and n_k must be in [0, 2^24], got %lld and %lld", fn, (long long)n_q, (long long)n_k);
  if (q_start < -most || q_start > 2 * most)
    return fail(BSGA_ERR_INVALID_ARG, "%s: q_start must be in [-2^24, 2^25], got %lld", fn, (long long)q_start);
  if (frame < 1 || frame > most) return fail(BSGA_ERR_INVALID_ARG, "%s: frame must be in [1, 2^24] tokens, got %lld", fn, (long long)frame);
  if (window < 0) return fail(BSGA_ERR_INVALID_ARG, "%s: window must be >= 0 frames (0: no limit), got %lld", fn, (long long)window);
  if (sinks < 0) return fail(BSGA_ERR_INVALID_ARG, "%s: sinks must be >= 0, got %lld", fn, (long long)sinks);
  s.n_q = static_cast<int>(n_q);
  s.n_k = static_cast<int>(n_k);
  s.q_start = static_cast<int>(q_start);
  s.frame = static_cast<int>(frame);
  s.window = window == 0 || window > 4 * most ? static_cast<int>(4 * most) : static_cast<int>(window);  // more frames than there are
  s.sinks = static_cast<int>(sinks < n_k ? sinks : n_k);
  return BSGA_OK;
}

inline int check_view(const char* fn, const char* name, const void* p, int64_t token, int64_t head, int size, View& v) {
  if (!p || !aligned16(p) || !whole_stride(token, size) || !whole_stride(head, size) || token >= (int64_t(1) << 24) / size)
    return fail(BSGA_ERR_INVALID_ARG, "%s: %s must be non-null, it and its strides multiples of 16 bytes, a token's stride in [0, 2^24) bytes", fn, name);
  v = {static_cast<const unsigned char*>(p), token * size, head * size};
  return BSGA_OK;
}

// Parts of a row's keys together: out = sum_s exp(lse_s - lse) part_s, a part that saw nothing (lse -inf) may hold anything.  Few parts: sixteen lanes to a
// row.  Many (WIDE): a workgroup to a row, so that the loads of all parts are on their way together; 43 parts of 16 rows 6.7 -> 3.9 us.
template <typename T, bool WIDE>
__global__ __launch_bounds__(256) void join_kernel(const float* __restrict__ part, const float* __restrict__ part_lse, int64_t rows, int splits,
                                                   unsigned char* __restrict__ out, float* __restrict__ lse) {
  __shared__ f32x4 sums[16][16];
  __shared__ float total[16], tops[4];
  const int group = threadIdx.x >> 4, d = (threadIdx.x & 15) * 4;
  const int64_t row = WIDE ? blockIdx.x : int64_t(blockIdx.x) * 16 + group;
  if (!WIDE && row >= rows) return;
  // the largest lse, NaN if one is
  float top = -INFINITY;
  bool nan = false;
  for (int s = WIDE ? threadIdx.x : 0; s < splits; s += WIDE ? 256 : 1) {
    const float x = part_lse[s * rows + row];
    top = fmaxf(top, x);
    nan = nan || x != x;
  }
  if constexpr (WIDE) {
    for (int x = 32; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
    nan = __syncthreads_or(nan);
    top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
  }
  if (nan) top = NAN;
  float sum = 0.f;
  f32x4 y = {0.f, 0.f, 0.f, 0.f};
  if (top != -INFINITY)
#pragma unroll 4
    for (int s = WIDE ? group : 0; s < splits; s += WIDE ? 16 : 1) {
      const float from = part_lse[s * rows + row];
      const f32x4 x = *reinterpret_cast<const f32x4*>(part + (s * rows + row) * 64 + d);
      const float w = from == -INFINITY ? 0.f : exp2f((from - top) * kLog2e);
      sum += w;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] += from == -INFINITY ? 0.f : w * x[e];
    }
  if constexpr (WIDE) {
    sums[group][threadIdx.x & 15] = y;
    if (d == 0) total[group] = sum;
    __syncthreads();
    if (group != 0) return;
    sum = 0.f;
    y = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < 16; ++s) {
      sum += total[s];
      y += sums[s][threadIdx.x & 15];
    }
  }
  const float inv = top == -INFINITY ? 0.f : 1.f / sum;
  Ops<T>::store4(out + row * Ops<T>::kRow, d, y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
  if (lse != nullptr && d == 0) lse[row] = top == -INFINITY ? -INFINITY : top + log2f(sum) * kLn2;
}

inline int64_t workgroups_of_join(int64_t rows, int splits) { return splits > 8 ? rows : ceil_div(rows, 16); }

template <typename T>
int launch_join(const float* part, const float* part_lse, int64_t rows, int splits, unsigned char* out, float* lse, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(workgroups_of_join(rows, splits)));
  if (splits > 8) hipLaunchKernelGGL((join_kernel<T, true>), grid, dim3(256), 0, s, part, part_lse, rows, splits, out, lse);
  else hipLaunchKernelGGL((join_kernel<T, false>), grid, dim3(256), 0, s, part, part_lse, rows, splits, out, lse);
  return check_hip(hipGetLastError(), "attention launch");
}

}  // namespace
}  // namespace bsga
