// Norms of queries and keys for each head with the rotation by position in the same pass, and the gradient of that.
//
// A row is one head's 64 numbers x of one token.  rms: n = x r w with r = (mean x^2 + eps)^-1/2; layer: n = (x - mean) r w + b.  The
// rotation cuts the row into one segment for each axis of the positions; in a segment of width W the pairs (j, j + W/2) turn by
// position * base^(-2j/W).  Backwards, with g the gradient turned back and h the row before the weight: dw = sum g h, db = sum g,
// dx = r (w g - [mean w g] - h mean(w g h)).
//
// HBM-bound: 100 frames of 48 heads (1.69 GB) 338 us, 5.0 TB/s, where a copy of 1 GiB reaches 5.1.  A row is read once and written once.  Four lanes hold a row, lane c eight of its pairs (so that the rotation stays in
// the lane), and the sums over a row are two quad permutations.  A lane keeps its token over the heads that its workgroup takes: the angles are
// computed once for them.  base^(-2j/W) / 2 pi, of 64-bit arithmetic, is a 64-bit fraction of a turn, and the product with the position modulo 2^64 is the turn's fraction: an angle w is
// off by 2^-51 w, whatever its size; fp32 would be off by 0.1 at position 10^6.
//
// Into a cache in 8 bits (e4m3.h) the row goes from the 32 bits in which it was normed and turned, in one rounding: the largest magnitude is one more pair of
// quad permutations, and neighbouring lanes swap halves so that each writes 16 bytes.  A key of which the 32 bits' own error leaves a rounding open (rounded from the
// least and the largest that it may be, it differs), or whose squares 32 bits do not hold, is done again in 64 bits at the end, by a wave with a lane to a number.  100 frames,
// with the rows returned as they are read back (1.97 GB): 431 us, 4.6 TB/s; by 32 bits alone, where one key number in 200,000 went to the other side of a border, 396, all keys in 64 bits 449.
#include "bf16_tile.h"
#include "bsga_internal.h"
#include "e4m3.h"

#include <math.h>

namespace bsga {
namespace {

constexpr int kRowsPerGroup = 64;    // tokens of a workgroup of 256 threads
constexpr int kHeadsInFlight = 4;    // rows of a lane whose loads are on their way together
constexpr int kPartials = 1024;      // workgroups that a weight's gradient is summed over, about

struct NormRopeArgs {
  const unsigned char* x[3];   // q, k, v
  int64_t x_token[3], x_head[3];  // strides in bytes
  unsigned char* y[3];
  const unsigned char *weight[2], *bias[2];
  const int32_t *positions, *slots;
  int64_t n, n_slots;
  int heads[3], group_heads, axes, norm, page;
  float eps;
  double eps64;
  unsigned long long turn[32];
  unsigned char *code[2], *scale[2];  // of k and v, in a cache in 8 bits: y holds the rows as they are read back then, where it is wanted
  // the gradient
  const unsigned char* dy[3];  // [heads, n, 64]
  unsigned char* dx[3];
  int64_t dx_token[3], dx_head[3];
  float* partial[2];           // [workgroups of q or k][128]: of the weight, of the bias
};

template <typename T>
__device__ __forceinline__ void widen(const u32x4 (&raw)[sizeof(T) / 2], float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[2 * e] = __uint_as_float(raw[0][e] << 16);
      x[2 * e + 1] = __uint_as_float(raw[0][e] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(raw[e >> 2][e & 3]);
  }
}

template <typename T>
__device__ __forceinline__ void load(const unsigned char* p, u32x4 (&raw)[sizeof(T) / 2]) {
#pragma unroll
  for (unsigned i = 0; i < sizeof(T) / 2; ++i) raw[i] = reinterpret_cast<const u32x4*>(p)[i];
}

template <typename T>
__device__ __forceinline__ void store(unsigned char* p, const float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<u32x4*>(p) = u32x4{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])};
  } else {
    reinterpret_cast<f32x4*>(p)[0] = f32x4{x[0], x[1], x[2], x[3]};
    reinterpret_cast<f32x4*>(p)[1] = f32x4{x[4], x[5], x[6], x[7]};
  }
}

// sum over the four lanes of a row
__device__ __forceinline__ float row_sum(float x) {
  x += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0xb1, 0xf, 0xf, true));  // lanes 1 0 3 2
  x += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x4e, 0xf, 0xf, true));  // lanes 2 3 0 1
  return x;
}

// Where a lane's eight pairs lie in a row (elements first .. first + 7 and second .. second + 7), and their angles.
struct Lane {
  int first, second;
  float cos[8], sin[8];
};

__device__ __forceinline__ void place(const NormRopeArgs& a, int c, Lane& l) {
  l.first = a.axes == 2 ? 32 * (c >> 1) + 8 * (c & 1) : 8 * c;
  l.second = l.first + (a.axes == 2 ? 16 : 32);
}

__device__ __forceinline__ void angles(const NormRopeArgs& a, int64_t i, int c, Lane& l) {
  if (a.axes == 0) return;
  const long long at = a.positions[i * a.axes + (a.axes == 2 ? c >> 1 : 0)];
  const int j = a.axes == 2 ? 8 * (c & 1) : 8 * c;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const long long turn = static_cast<long long>(static_cast<unsigned long long>(at) * a.turn[j + e]);
    sincospif(static_cast<float>(static_cast<int>(turn >> 32)) * 0x1p-31f, &l.sin[e], &l.cos[e]);
  }
}

// Weight and bias of a lane's elements.
template <typename T>
__device__ __forceinline__ void weights(const unsigned char* p, const Lane& l, float missing, float (&lo)[8], float (&hi)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) lo[e] = hi[e] = missing;
  if (p == nullptr) return;
  u32x4 raw[sizeof(T) / 2];
  load<T>(p + l.first * sizeof(T), raw);
  widen<T>(raw, lo);
  load<T>(p + l.second * sizeof(T), raw);
  widen<T>(raw, hi);
}

constexpr float kMostShift = 0x1p16f;  // see kOff

__device__ __forceinline__ float tree_sum(const float (&x)[8]) { return ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7])); }

// (a, b) become the row before the weight; the factor that the row was multiplied with is returned.  shift: the mean that was taken off, in units of the result,
// and infinite, which leaves every rounding open, where it is large, where the sum of the squares is infinite, or so small that squares lose bits below 2^-126.
// TREE: sums by halves, which are less off.
template <bool TREE = false>
__device__ __forceinline__ float normalise(int norm, float eps, float (&a)[8], float (&b)[8], float* shift = nullptr) {
  if (norm == BSGA_NORM_NONE) return 1.f;
  float mean = 0.f;
  if (norm == BSGA_NORM_LAYER) {
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) s += a[e] * 0x1p-6f + b[e] * 0x1p-6f;  // (the mean of values that fit fits, their sum may not)
    if constexpr (TREE) {
      float t[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) t[e] = a[e] * 0x1p-6f + b[e] * 0x1p-6f;
      s = tree_sum(t);
    }
    mean = row_sum(s);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      a[e] -= mean;
      b[e] -= mean;
    }
  }
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) s += a[e] * a[e] + b[e] * b[e];
  if constexpr (TREE) {
    float t[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) t[e] = a[e] * a[e] + b[e] * b[e];
    s = tree_sum(t);
  }
  const float square = row_sum(s) * 0x1p-6f + eps, r = 1.f / sqrtf(square);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    a[e] *= r;
    b[e] *= r;
  }
  if (shift != nullptr) {
    const float by = fabsf(mean) * r;
    *shift = square >= 0x1p-100f && square <= 0x1.fffffep127f && by <= kMostShift ? by : INFINITY;
  }
  return r;
}

// The tensor (0 q, 1 k, 2 v) and the heads of group y of the grid.
__device__ __forceinline__ int kind_of(const NormRopeArgs& a, int y, int& h0, int& h1, int& group) {
  int kind = 0;
  for (; kind < 2; ++kind) {
    const int groups = (a.heads[kind] + a.group_heads - 1) / a.group_heads;
    if (y < groups) break;
    y -= groups;
  }
  group = y;
  h0 = y * a.group_heads;
  h1 = min(h0 + a.group_heads, a.heads[kind]);
  return kind;
}

__device__ __forceinline__ unsigned other_of_pair(unsigned x) {  // lanes 1 0 3 2
  return static_cast<unsigned>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), 0xb1, 0xf, 0xf, true));
}

// How far a key that was normed and turned in 32 bits may be off, relative to its pair's length, in units of 2^-24, a whole one for each rounding.  Before the turn 9: for the
// mean of the squares 2 + 3 + 2 and 1 for eps, half of which is the root's, one each for the root, its inverse, the product with that, the difference from a mean, and the
// product with the weight.  The angle 1.6, half a turn in 24 bits; sine and cosine 1.4, an ulp each; the turn 2, the sums by which it is looked for 1; a tenth for products of
// errors.  A bias is 8 of its own (what its number has before it is added), in both numbers of a pair, so times sqrt(2).  A mean is off by 1 + 3 + 2 units of the magnitudes that
// it is of, in units of the result the mean's own and at most one more, in both numbers too; what that does to the squares is less than an eighth of it as long as the
// mean is at most 2^16 of those units.  Weights up to 2^40: what a number loses below 2^-126 before them is nothing behind them.
constexpr float kOff = 15.1f * 0x1p-24f, kOffMean = 10 * 0x1p-24f, kOffBias = 12 * 0x1p-24f;
constexpr float kMostWeight = 0x1p40f;

// A row's lanes to 8 bits: the exponent, and the numbers x in code[0], y in code[1].  doubt: whether the exponent or a number may be another if the row's numbers
// are off by kOff of their pair and `terms`: the least and the largest that a number may be are rounded, and differ.
template <bool DOUBT>
__device__ __forceinline__ int to_e4m3(const float (&x)[8], const float (&y)[8], float terms, u32x2 (&code)[2], bool& doubt) {
  float most = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float u = fabsf(x[e]), v = fabsf(y[e]);
    most = fmaxf(most, fmaxf(u <= 0x1.fffffep127f ? u : 0.f, v <= 0x1.fffffep127f ? v : 0.f));
  }
  most = fmaxf(most, __uint_as_float(other_of_pair(__float_as_uint(most))));
  most = fmaxf(most, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(most), 0x4e, 0xf, 0xf, true)));
  const int byte = scale_byte(most);
  const float f = inverse_scale(byte);
  float u[8], v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    u[e] = x[e] * f;
    v[e] = y[e] * f;
    if (byte == kMostScale) {  // the only one whose numbers may be larger
      u[e] = fabsf(x[e]) <= 0x1.fffffep127f ? fminf(fmaxf(u[e], -448.f), 448.f) : NAN;
      v[e] = fabsf(y[e]) <= 0x1.fffffep127f ? fminf(fmaxf(v[e], -448.f), 448.f) : NAN;
    }
  }
  auto pack = [&](const float* t) { return u32x2{pack_e4m3(t[0], t[1], t[2], t[3]), pack_e4m3(t[4], t[5], t[6], t[7])}; };
  if constexpr (DOUBT) {
    const float off = terms * f;
    float w[8], z[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float of_pair = fmaf(fabsf(u[e]) + fabsf(v[e]), kOff, off);
      w[e] = fminf(u[e] + of_pair, 448.f);  // (NaN becomes 448, and the other one does not)
      z[e] = fminf(v[e] + of_pair, 448.f);
      u[e] = fmaxf(u[e] - of_pair, -448.f);
      v[e] = fmaxf(v[e] - of_pair, -448.f);
    }
    const u32x2 a = pack(w), b = pack(z);
    code[0] = pack(u);
    code[1] = pack(v);
    const float top = most * f;
    doubt = ((a[0] ^ code[0][0]) | (a[1] ^ code[0][1]) | (b[0] ^ code[1][0]) | (b[1] ^ code[1][1])) != 0u;
    doubt = doubt | (fabsf(top - 448.f) <= fmaf(1024.f, kOff, off)) | (fabsf(top - 224.f) <= fmaf(1024.f, kOff, off));
  } else {
    code[0] = pack(u);
    code[1] = pack(v);
  }
  return byte;
}

// To 32 bits for a rounding that follows: what is not a number of 32 bits becomes the neighbour with an odd last bit, which no later rounding takes for a tie.
__device__ __forceinline__ float to_odd(double x) {
  const float f = static_cast<float>(x);
  const double back = static_cast<double>(f);
  unsigned u = __float_as_uint(f);
  if (back != x && fabsf(f) <= 0x1.fffffep127f) u = (fabs(back) > fabs(x) ? u - 1u : u) | 1u;
  return __uint_as_float(u);
}

template <int DPP>
__device__ __forceinline__ double of_other(double x) {
  const unsigned long long u = __builtin_bit_cast(unsigned long long, x);
  const int low = __builtin_amdgcn_update_dpp(0, static_cast<int>(u), DPP, 0xf, 0xf, true);
  const int high = __builtin_amdgcn_update_dpp(0, static_cast<int>(u >> 32), DPP, 0xf, 0xf, true);
  return __builtin_bit_cast(double, static_cast<unsigned long long>(static_cast<unsigned>(high)) << 32 | static_cast<unsigned>(low));
}

// f over all lanes: pairs, quads, eights (lanes mirrored within them), sixteens, then across rows of sixteen.
template <typename F>
__device__ __forceinline__ double over_wave(double x, F f) {
  x = f(x, of_other<0xb1>(x));
  x = f(x, of_other<0x4e>(x));
  x = f(x, of_other<0x141>(x));
  x = f(x, of_other<0x140>(x));
#pragma unroll
  for (int step = 0; step < 2; ++step) {
    const unsigned long long u = __builtin_bit_cast(unsigned long long, x);
    const unsigned low = static_cast<unsigned>(u), high = static_cast<unsigned>(u >> 32);
    const auto a = step == 0 ? __builtin_amdgcn_permlane16_swap(low, low, false, false) : __builtin_amdgcn_permlane32_swap(low, low, false, false);
    const auto b = step == 0 ? __builtin_amdgcn_permlane16_swap(high, high, false, false) : __builtin_amdgcn_permlane32_swap(high, high, false, false);
    x = f(__builtin_bit_cast(double, static_cast<unsigned long long>(b[0]) << 32 | a[0]), __builtin_bit_cast(double, static_cast<unsigned long long>(b[1]) << 32 | a[1]));
  }
  return x;
}

// Keys by a wave in 64 bits, one after the other, a lane to a number: of heads h0 .. h1 - 1 of the 16 tokens from `first` on, those whose lanes have the head's bit of `open`.
template <typename T>
__device__ __forceinline__ void keys_in_64_bits(const NormRopeArgs& a, int64_t first, int h0, int h1, unsigned open, int lane) {
  if (__ballot(open != 0) == 0) return;
  const auto add = [](double x, double y) { return x + y; };
  const auto larger_of = [](double x, double y) { return fmax(x, y); };
  const auto number = [&](const unsigned char* p) { return static_cast<float>(reinterpret_cast<const T*>(p)[lane]); };
  const float weight = a.weight[1] != nullptr ? number(a.weight[1]) : 1.f, bias = a.bias[1] != nullptr ? number(a.bias[1]) : 0.f;
  const int half = a.axes == 2 ? 16 : 32;
  const unsigned long long of_position = a.turn[lane & (half - 1)];
  for (int h = h0; h < h1; ++h)
    for (unsigned long long rows = __ballot((open >> (h - h0)) & 1); rows != 0;) {
      const int r = __builtin_ctzll(rows) >> 2;
      rows &= ~(15ull << (4 * r));
      const int64_t i = first + r;
      const float of_row = number(a.x[1] + i * a.x_token[1] + h * a.x_head[1]);
      const int slot = a.slots[i];
      const long long at = a.axes > 0 ? a.positions[i * a.axes + (a.axes == 2 ? lane >> 5 : 0)] : 0;
      double x = of_row;
      if (a.norm == BSGA_NORM_LAYER) x -= over_wave(x, add) * 0x1p-6;
      if (a.norm != BSGA_NORM_NONE) x /= sqrt(over_wave(x * x, add) * 0x1p-6 + a.eps64);
      x = x * static_cast<double>(weight) + static_cast<double>(bias);
      if (a.axes > 0) {
        double sine, cosine;
        sincospi(static_cast<double>(static_cast<long long>(static_cast<unsigned long long>(at) * of_position)) * 0x1p-63, &sine, &cosine);
        const double other = __shfl_xor(x, half);
        x = x * cosine + ((lane & half) != 0 ? other : -other) * sine;
      }
      const bool finite = fabs(x) < 0x1.ffffffp127;  // as 32 bits have it
      const double most = over_wave(finite ? fabs(x) : 0.0, larger_of);
      float up = static_cast<float>(most);
      if (static_cast<double>(up) < most) up = __uint_as_float(__float_as_uint(up) + 1u);
      const int byte = scale_byte(up);
      const double t = x * static_cast<double>(inverse_scale(byte));
      const unsigned code = pack_e4m3(finite ? to_odd(fmin(fmax(t, -448.0), 448.0)) : NAN, 0.f, 0.f, 0.f) & 0xffu;
      if (slot >= 0 && slot < a.n_slots) {
        const unsigned page = static_cast<unsigned>(slot) / static_cast<unsigned>(a.page);
        const int64_t row = (int64_t(page) * a.heads[1] + h) * a.page + (static_cast<unsigned>(slot) - page * a.page);
        a.code[0][row * 64 + lane] = static_cast<unsigned char>(code);
        if (lane == 0) a.scale[0][row] = static_cast<unsigned char>(byte);
      }
      if (a.y[1] != nullptr) reinterpret_cast<T*>(a.y[1])[(int64_t(h) * a.n + i) * 64 + lane] = static_cast<T>(unpack_f32(code)[0] * scale_of(byte));
    }
}

template <typename T, bool CODED>
__global__ __launch_bounds__(256, CODED && sizeof(T) == 2 ? 3 : 1) void norm_rope_kernel(const NormRopeArgs a) {
  int h0, h1, group;
  const int kind = kind_of(a, blockIdx.y, h0, h1, group);
  const int c = threadIdx.x & 3;
  const int64_t i = int64_t(blockIdx.x) * kRowsPerGroup + (threadIdx.x >> 2);
  const bool live = i < a.n;
  const int64_t at = live ? i : a.n - 1;
  constexpr int kRow = 64 * sizeof(T);
  Lane l;
  place(a, c, l);
  const unsigned char* src = a.x[kind] + at * a.x_token[kind];
  u32x4 lo[kHeadsInFlight][sizeof(T) / 2], hi[kHeadsInFlight][sizeof(T) / 2];
  auto fetch = [&](int h) {
#pragma unroll
    for (int u = 0; u < kHeadsInFlight; ++u) {
      const unsigned char* p = src + min(h + u, h1 - 1) * a.x_head[kind];
      load<T>(p + l.first * sizeof(T), lo[u]);
      load<T>(p + l.second * sizeof(T), hi[u]);
    }
  };
  fetch(h0);
  // where the token's rows go: [heads, n, 64], or the pages of a cache
  int64_t to = at, step = a.n;
  bool write = live;
  if (kind > 0 && a.slots != nullptr) {
    const int slot = a.slots[at];
    write = live && slot >= 0 && slot < a.n_slots;
    const unsigned page = static_cast<unsigned>(slot) / static_cast<unsigned>(a.page);
    to = int64_t(page) * a.heads[kind] * a.page + (static_cast<unsigned>(slot) - page * a.page);
    step = a.page;
  }
  unsigned char* const dst = a.y[kind];
  float wa[8], wb[8], ba[8], bb[8];
  if (kind < 2) {
    angles(a, at, c, l);
    weights<T>(a.weight[kind], l, 1.f, wa, wb);
    weights<T>(a.bias[kind], l, 0.f, ba, bb);
  }
  // Keys that are rounded to 8 bits from 32: those whose rounding the 32 bits leave open are left for the end
  const bool exact = a.norm == BSGA_NORM_NONE && a.axes == 0 && a.weight[1] == nullptr && a.bias[1] == nullptr;
  float most_weight = 0.f, most_bias = 0.f;
  const float of_mean = a.norm == BSGA_NORM_LAYER ? kOffMean : 0.f;
  unsigned open = 0;
  if (CODED && kind == 1) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      most_weight = fmaxf(most_weight, fmaxf(fabsf(wa[e]), fabsf(wb[e])));
      most_bias = fmaxf(most_bias, fmaxf(fabsf(ba[e]), fabsf(bb[e])));
    }
    if (most_weight > kMostWeight) most_bias = INFINITY;  // (no row is sure)
  }
  for (int h = h0; h < h1; h += kHeadsInFlight) {
    if (h > h0) fetch(h);
#pragma unroll
    for (int u = 0; u < kHeadsInFlight; ++u) {
      if (h + u >= h1) break;
      float x[8], y[8], shift = 0.f;
      widen<T>(lo[u], x);
      widen<T>(hi[u], y);
      if (kind < 2) {
        if (CODED && kind == 1) normalise<true>(a.norm, a.eps, x, y, &shift);
        else normalise(a.norm, a.eps, x, y);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          x[e] = fmaf(x[e], wa[e], ba[e]);
          y[e] = fmaf(y[e], wb[e], bb[e]);
          if (a.axes > 0) {
            const float t = x[e] * l.cos[e] - y[e] * l.sin[e];
            y[e] = y[e] * l.cos[e] + x[e] * l.sin[e];
            x[e] = t;
          }
        }
      }
      if (CODED && kind > 0) {
        u32x2 code[2];
        bool doubt = false;
        int byte;
        if (kind == 1 && !exact) byte = to_e4m3<true>(x, y, fmaf(shift * kOffMean + of_mean, most_weight, most_bias * kOffBias), code, doubt);
        else byte = to_e4m3<false>(x, y, 0.f, code, doubt);
        const bool left = ((__ballot(doubt) >> (threadIdx.x & 60)) & 15) != 0;  // any of the row's lanes
        open |= static_cast<unsigned>(left) << (h + u - h0);
        // lanes 2j and 2j + 1 hold neighbouring eights of both halves: the first takes those of the first half, the other those of the second
        const bool odd = c & 1;
        const u32x2 mine = odd ? code[1] : code[0], gone = odd ? code[0] : code[1];
        const u32x2 got = {other_of_pair(gone[0]), other_of_pair(gone[1])};
        if (write && !left) {
          const int64_t row = to + (h + u) * step;
          *reinterpret_cast<u32x4*>(a.code[kind - 1] + row * 64 + (odd ? l.second - 8 : l.first)) =
              odd ? u32x4{got[0], got[1], mine[0], mine[1]} : u32x4{mine[0], mine[1], got[0], got[1]};
          if (c == 0) a.scale[kind - 1][row] = static_cast<unsigned char>(byte);
        }
        if (live && !left && dst != nullptr) {
          unsigned char* p = dst + ((h + u) * a.n + at) * kRow;
          const float f = scale_of(byte);
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            unsigned char* to_half = p + (half == 0 ? l.first : l.second) * sizeof(T);
            if constexpr (sizeof(T) == 2) {
              const u32x2 v0 = unpack_bf16(code[half][0], f), v1 = unpack_bf16(code[half][1], f);
              *reinterpret_cast<u32x4*>(to_half) = u32x4{v0[0], v0[1], v1[0], v1[1]};
            } else {
              reinterpret_cast<f32x4*>(to_half)[0] = unpack_f32(code[half][0]) * f;
              reinterpret_cast<f32x4*>(to_half)[1] = unpack_f32(code[half][1]) * f;
            }
          }
        }
      } else if (write) {
        unsigned char* p = dst + (to + (h + u) * step) * kRow;
        store<T>(p + l.first * sizeof(T), x);
        store<T>(p + l.second * sizeof(T), y);
      }
    }
  }
  if (CODED && kind == 1)
    keys_in_64_bits<T>(a, int64_t(blockIdx.x) * kRowsPerGroup + (threadIdx.x >> 6) * 16, h0, h1, live ? open : 0u, threadIdx.x & 63);
}

template <typename T>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 3 : 2) void norm_rope_bwd_kernel(const NormRopeArgs a) {
  __shared__ float sums[4][128];
  int h0, h1, group;
  const int kind = kind_of(a, blockIdx.y, h0, h1, group);
  const int c = threadIdx.x & 3;
  constexpr int kRow = 64 * sizeof(T);
  Lane l;
  place(a, c, l);
  float wa[8], wb[8], dwa[8], dwb[8], dba[8], dbb[8];
  if (kind < 2) weights<T>(a.weight[kind], l, 1.f, wa, wb);
#pragma unroll
  for (int e = 0; e < 8; ++e) dwa[e] = dwb[e] = dba[e] = dbb[e] = 0.f;
  for (int64_t first = int64_t(blockIdx.x) * kRowsPerGroup; first < a.n; first += int64_t(gridDim.x) * kRowsPerGroup) {
    const int64_t i = first + (threadIdx.x >> 2);
    const bool live = i < a.n;
    const int64_t at = live ? i : a.n - 1;
    if (kind < 2) angles(a, at, c, l);
    for (int h = h0; h < h1; h += 2) {
      u32x4 raw[2][4][sizeof(T) / 2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int hu = min(h + u, h1 - 1);
        const unsigned char* g = a.dy[kind] + (int64_t(hu) * a.n + at) * kRow;
        load<T>(g + l.first * sizeof(T), raw[u][0]);
        load<T>(g + l.second * sizeof(T), raw[u][1]);
        if (kind < 2) {
          const unsigned char* x = a.x[kind] + at * a.x_token[kind] + hu * a.x_head[kind];
          load<T>(x + l.first * sizeof(T), raw[u][2]);
          load<T>(x + l.second * sizeof(T), raw[u][3]);
        }
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        if (h + u >= h1) break;
        float ga[8], gb[8];
        widen<T>(raw[u][0], ga);
        widen<T>(raw[u][1], gb);
        if (kind < 2) {
          float x[8], y[8];
          widen<T>(raw[u][2], x);
          widen<T>(raw[u][3], y);
          const float r = normalise(a.norm, a.eps, x, y);
          float along = 0.f, mean = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            if (a.axes > 0) {
              const float t = ga[e] * l.cos[e] + gb[e] * l.sin[e];
              gb[e] = gb[e] * l.cos[e] - ga[e] * l.sin[e];
              ga[e] = t;
            }
            if (live) {
              dwa[e] += ga[e] * x[e];
              dwb[e] += gb[e] * y[e];
              dba[e] += ga[e];
              dbb[e] += gb[e];
            }
            ga[e] *= wa[e];
            gb[e] *= wb[e];
            along += ga[e] * x[e] + gb[e] * y[e];
            mean += ga[e] + gb[e];
          }
          along = a.norm == BSGA_NORM_NONE ? 0.f : row_sum(along) * 0x1p-6f;
          mean = a.norm == BSGA_NORM_LAYER ? row_sum(mean) * 0x1p-6f : 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            ga[e] = (ga[e] - mean - x[e] * along) * r;
            gb[e] = (gb[e] - mean - y[e] * along) * r;
          }
        }
        if (live) {
          unsigned char* p = a.dx[kind] + at * a.dx_token[kind] + (h + u) * a.dx_head[kind];
          store<T>(p + l.first * sizeof(T), ga);
          store<T>(p + l.second * sizeof(T), gb);
        }
      }
    }
  }
  if (kind == 2 || a.partial[kind] == nullptr) return;  // the whole workgroup
  // over the sixteen tokens of a wave, then the four waves: always in the same order
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int e = 0; e < 8; ++e)
    for (int o = 4; o < 64; o <<= 1) {
      dwa[e] += __shfl_xor(dwa[e], o);
      dwb[e] += __shfl_xor(dwb[e], o);
      dba[e] += __shfl_xor(dba[e], o);
      dbb[e] += __shfl_xor(dbb[e], o);
    }
  if (lane < 4)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      sums[wave][l.first + e] = dwa[e];
      sums[wave][l.second + e] = dwb[e];
      sums[wave][64 + l.first + e] = dba[e];
      sums[wave][64 + l.second + e] = dbb[e];
    }
  __syncthreads();
  if (threadIdx.x < 128) {
    const int t = threadIdx.x;
    a.partial[kind][(int64_t(group) * gridDim.x + blockIdx.x) * 128 + t] = (sums[0][t] + sums[1][t]) + (sums[2][t] + sums[3][t]);
  }
}

// Sums of the workgroups' parts, in float64: blockIdx.y is the tensor, blockIdx.x sixteen of its 128 columns.
__global__ __launch_bounds__(1024) void norm_rope_sum_kernel(const float* __restrict__ partial_q, const float* __restrict__ partial_k,
                                                             int count_q, int count_k, float* __restrict__ out) {
  __shared__ double sums[64][17];
  const float* partial = blockIdx.y == 0 ? partial_q : partial_k;
  const int count = blockIdx.y == 0 ? count_q : count_k;
  const int column = blockIdx.x * 16 + (threadIdx.x & 15), part = threadIdx.x >> 4;
  double s = 0.0;
#pragma unroll 4
  for (int p = part; p < count; p += 64) s += partial[int64_t(p) * 128 + column];
  sums[part][threadIdx.x & 15] = s;
  __syncthreads();
  if (threadIdx.x < 16) {
    s = 0.0;
    for (int p = 0; p < 64; ++p) s += sums[p][threadIdx.x];
    out[blockIdx.y * 128 + column] = static_cast<float>(s);
  }
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// What both directions have in common, checked and put into `a`.
int common(const char* fn, const void* const (&x)[3], const int64_t (&strides)[6], int dtype, int64_t n_tokens, int heads, int kv_heads,
           int head_dim, int norm, double eps, const void* const (&weight)[2], const void* const (&bias)[2], const int32_t* positions,
           int axes, double base, NormRopeArgs& a) {
  static const char* const names[3] = {"q", "k", "v"};
  if (dtype != BSGA_BF16 && dtype != BSGA_FP32) return fail(BSGA_ERR_INVALID_ARG, "%s: unknown dtype %d", fn, dtype);
  if (head_dim != 64) return fail(BSGA_ERR_UNSUPPORTED, "%s: head_dim must be 64, got %d", fn, head_dim);
  if (n_tokens < 0 || n_tokens > (int64_t(1) << 24))
    return fail(BSGA_ERR_INVALID_ARG, "%s: n_tokens must be in [0, 2^24], got %lld", fn, static_cast<long long>(n_tokens));
  if (n_tokens > 0 && !x[0] && !x[1] && !x[2])  // (tensors without elements have no address)
    return fail(BSGA_ERR_INVALID_ARG, "%s: nothing to do (q, k and v are all null)", fn);
  if (norm != BSGA_NORM_NONE && norm != BSGA_NORM_RMS && norm != BSGA_NORM_LAYER)
    return fail(BSGA_ERR_INVALID_ARG, "%s: norm must be 0 (none), 1 (rms) or 2 (layer), got %d", fn, norm);
  if (!(eps >= 0.0) || !isfinite(eps)) return fail(BSGA_ERR_INVALID_ARG, "%s: eps must be finite and >= 0", fn);
  if (axes < 0 || axes > 2) return fail(BSGA_ERR_INVALID_ARG, "%s: axes must be 0 (no rotation), 1 or 2, got %d", fn, axes);
  if (n_tokens > 0 && (axes > 0) != (positions != nullptr)) return fail(BSGA_ERR_INVALID_ARG, "%s: positions go with axes 1 or 2", fn);
  if (axes > 0 && (!(base > 0.0) || !isfinite(base))) return fail(BSGA_ERR_INVALID_ARG, "%s: base must be finite and > 0", fn);
  const int size = dtype == BSGA_BF16 ? 2 : 4;
  for (int t = 0; t < 3; ++t) {
    const int h = t == 0 ? heads : kv_heads;
    if (x[t] == nullptr) continue;
    if (h < 1 || h > 65535)
      return fail(BSGA_ERR_INVALID_ARG, "%s: heads of %s must be in [1, 65535], got %d", fn, names[t], h);
    if (!aligned16(x[t]) || !whole_stride(strides[2 * t], size) || !whole_stride(strides[2 * t + 1], size))
      return fail(BSGA_ERR_INVALID_ARG, "%s: %s and its strides must be multiples of 16 bytes, the strides not negative", fn, names[t]);
    if (t < 2) {
      if (!aligned16(weight[t]) || !aligned16(bias[t]))
        return fail(BSGA_ERR_INVALID_ARG, "%s: weights and biases must be 16-byte aligned", fn);
      if (norm != BSGA_NORM_LAYER && bias[t]) return fail(BSGA_ERR_INVALID_ARG, "%s: a bias goes with the layer norm", fn);
      if (norm == BSGA_NORM_NONE && weight[t]) return fail(BSGA_ERR_INVALID_ARG, "%s: a weight goes with a norm", fn);
      a.weight[t] = static_cast<const unsigned char*>(weight[t]);
      a.bias[t] = static_cast<const unsigned char*>(bias[t]);
    }
    a.x[t] = static_cast<const unsigned char*>(x[t]);
    a.x_token[t] = strides[2 * t] * size;
    a.x_head[t] = strides[2 * t + 1] * size;
    a.heads[t] = h;
  }
  a.n = n_tokens;
  a.norm = norm;
  a.eps = static_cast<float>(eps);
  a.eps64 = eps;
  a.positions = positions;
  a.axes = axes;
  // base^(-(8 x + y) / half) / 2 pi as a product of two powers (calls on few rows are bound by the host: 12 powers in place of 32)
  const int half = axes == 2 ? 16 : 32;
  double fine[8];
  for (int y = 0; axes > 0 && y < 8; ++y) fine[y] = pow(base, -double(y) / half);
  for (int x = 0; axes > 0 && x < half; x += 8) {
    const double coarse = pow(base, -double(x) / half) * 0.15915494309189533577;  // 1 / (2 pi)
    for (int y = 0; y < 8; ++y) {
      const double turn = coarse * fine[y], part = turn - floor(turn);
      a.turn[x + y] = static_cast<unsigned long long>((part < 1.0 ? part : 0.0) * 0x1p64);  // (a base next to 0: infinite, and no number less itself)
    }
  }
  return BSGA_OK;
}

// Heads that a workgroup takes one after the other: several, for the angles' sake, unless
// that leaves CUs without work.
int heads_of_a_group(const NormRopeArgs& a, int64_t tiles) {
  const int64_t all = int64_t(a.heads[0]) + a.heads[1] + a.heads[2];
  for (int g = 8; g > 1; g >>= 1)
    if (tiles * (all / g) >= 1024) return g;
  return 1;
}

int groups_of(const NormRopeArgs& a, int kind) { return static_cast<int>(ceil_div(a.heads[kind], a.group_heads)); }

int pages_of(const char* fn, const int32_t* slots, int64_t n_pages, int page, NormRopeArgs& a) {
  if (!slots) return BSGA_OK;
  if (page < 1 || page > 65536) return fail(BSGA_ERR_INVALID_ARG, "%s: page must be in [1, 65536] tokens, got %d", fn, page);
  if (n_pages < 1 || n_pages > ((int64_t(1) << 31) - 1) / page)
    return fail(BSGA_ERR_INVALID_ARG, "%s: the cache must hold 1 to 2^31 - 1 tokens, got %lld pages of %d", fn, static_cast<long long>(n_pages), page);
  a.slots = slots;
  a.page = page;
  a.n_slots = n_pages * page;
  return BSGA_OK;
}

int launch(const char* fn, NormRopeArgs& a, int dtype, bool coded, hipStream_t s) {
  if (a.n == 0) return BSGA_OK;
  const int64_t tiles = ceil_div(a.n, kRowsPerGroup);
  a.group_heads = heads_of_a_group(a, tiles);
  const int64_t groups = int64_t(groups_of(a, 0)) + groups_of(a, 1) + groups_of(a, 2);
  if (groups > 65535) return fail(BSGA_ERR_UNSUPPORTED, "%s: too many heads", fn);
  const dim3 grid(static_cast<unsigned>(tiles), static_cast<unsigned>(groups));
  if (dtype == BSGA_BF16) {
    if (coded) hipLaunchKernelGGL((norm_rope_kernel<__bf16, true>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((norm_rope_kernel<__bf16, false>), grid, dim3(256), 0, s, a);
  } else {
    if (coded) hipLaunchKernelGGL((norm_rope_kernel<float, true>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((norm_rope_kernel<float, false>), grid, dim3(256), 0, s, a);
  }
  return check_hip(hipGetLastError(), fn);
}

}  // namespace
}  // namespace bsga

using namespace bsga;

extern "C" {

int bsga_qk_norm_rope(const void* q, const void* k, const void* v, int64_t q_token, int64_t q_head, int64_t k_token, int64_t k_head,
                      int64_t v_token, int64_t v_head, int dtype, int64_t n_tokens, int heads, int kv_heads, int head_dim, int norm, double eps,
                      const void* q_weight, const void* q_bias, const void* k_weight, const void* k_bias, const int32_t* positions,
                      int axes, double base, const int32_t* slots, int64_t n_pages, int page, void* q_out, void* k_out, void* v_out,
                      void* stream) {
  const char* fn = "bsga_qk_norm_rope";
  clear_error();
  NormRopeArgs a = {};
  const void* const x[3] = {q, k, v};
  void* const y[3] = {q_out, k_out, v_out};
  if (int rc = common(fn, x, {q_token, q_head, k_token, k_head, v_token, v_head}, dtype, n_tokens, heads, kv_heads, head_dim, norm, eps,
                      {q_weight, k_weight}, {q_bias, k_bias}, positions, axes, base, a))
    return rc;
  for (int t = 0; t < 3; ++t) {
    if (n_tokens > 0 && !x[t] != !y[t]) return fail(BSGA_ERR_INVALID_ARG, "%s: each input must come with its output", fn);
    if (!aligned16(y[t])) return fail(BSGA_ERR_INVALID_ARG, "%s: outputs must be 16-byte aligned", fn);
    a.y[t] = static_cast<unsigned char*>(y[t]);
  }
  if (int rc = pages_of(fn, slots, n_pages, page, a)) return rc;
  return launch(fn, a, dtype, false, static_cast<hipStream_t>(stream));
}

int bsga_qk_norm_rope_e4m3(const void* q, const void* k, const void* v, int64_t q_token, int64_t q_head, int64_t k_token, int64_t k_head,
                           int64_t v_token, int64_t v_head, int dtype, int64_t n_tokens, int heads, int kv_heads, int head_dim, int norm, double eps,
                           const void* q_weight, const void* q_bias, const void* k_weight, const void* k_bias, const int32_t* positions, int axes,
                           double base, const int32_t* slots, int64_t n_pages, int page, void* q_out, void* k_rows, void* v_rows, void* k_cache,
                           void* v_cache, uint8_t* k_scale, uint8_t* v_scale, void* stream) {
  const char* fn = "bsga_qk_norm_rope_e4m3";
  clear_error();
  NormRopeArgs a = {};
  const void* const x[3] = {q, k, v};
  void* const y[3] = {q_out, k_rows, v_rows};
  void* const code[2] = {k_cache, v_cache};
  uint8_t* const scale[2] = {k_scale, v_scale};
  if (int rc = common(fn, x, {q_token, q_head, k_token, k_head, v_token, v_head}, dtype, n_tokens, heads, kv_heads, head_dim, norm, eps,
                      {q_weight, k_weight}, {q_bias, k_bias}, positions, axes, base, a))
    return rc;
  for (int t = 0; t < 3; ++t) {
    if (!aligned16(y[t])) return fail(BSGA_ERR_INVALID_ARG, "%s: outputs must be 16-byte aligned", fn);
    a.y[t] = static_cast<unsigned char*>(y[t]);
    if (n_tokens == 0) continue;  // (tensors without elements have no address)
    if (t == 0 ? !q != !q_out : !x[t] && y[t]) return fail(BSGA_ERR_INVALID_ARG, "%s: outputs go with their inputs", fn);
    if (t == 0) continue;
    if (!x[t] != !code[t - 1] || !x[t] != !scale[t - 1])
      return fail(BSGA_ERR_INVALID_ARG, "%s: k and v must each come with its cache and its scales", fn);
    if (!aligned16(code[t - 1])) return fail(BSGA_ERR_INVALID_ARG, "%s: caches must be 16-byte aligned", fn);
    a.code[t - 1] = static_cast<unsigned char*>(code[t - 1]);
    a.scale[t - 1] = scale[t - 1];
  }
  if (n_tokens > 0 && (k || v) && !slots) return fail(BSGA_ERR_INVALID_ARG, "%s: slots must be non-null", fn);
  if (int rc = pages_of(fn, slots, n_pages, page, a)) return rc;
  return launch(fn, a, dtype, true, static_cast<hipStream_t>(stream));
}

// The workgroups over which a launch's tokens are spread, and the heads of each; needs n, heads.
static int64_t bwd_shape(NormRopeArgs& a) {
  const int64_t tiles = ceil_div(a.n, kRowsPerGroup);
  a.group_heads = heads_of_a_group(a, tiles);
  const int64_t groups = int64_t(groups_of(a, 0)) + groups_of(a, 1) + groups_of(a, 2);
  const int64_t most = kPartials / groups > 0 ? kPartials / groups : 1;
  return tiles < most ? tiles : most;
}

size_t bsga_qk_norm_rope_bwd_workspace_bytes(int64_t n_tokens, int heads, int kv_heads) {
  if (n_tokens < 1 || n_tokens > (int64_t(1) << 24) || heads < 0 || heads > 65535 || kv_heads < 0 || kv_heads > 65535) return 0;
  // whichever of q, k and v a call has: at most kPartials workgroups, or one for each group of heads
  const int64_t groups = int64_t(heads) + kv_heads;
  return static_cast<size_t>(groups > kPartials ? groups : kPartials) * 128 * sizeof(float);
}

int bsga_qk_norm_rope_bwd(const void* dq, const void* dk, const void* dv, const void* q, const void* k, int64_t q_token, int64_t q_head,
                          int64_t k_token, int64_t k_head, int dtype, int64_t n_tokens, int heads, int kv_heads, int head_dim,
                          int norm, double eps, const void* q_weight, const void* k_weight, const int32_t* positions, int axes, double base,
                          void* dq_in, void* dk_in, void* dv_in, int64_t dq_token, int64_t dq_head, int64_t dk_token, int64_t dk_head,
                          int64_t dv_token, int64_t dv_head, float* d_weights, void* workspace, size_t workspace_bytes, void* stream) {
  const char* fn = "bsga_qk_norm_rope_bwd";
  clear_error();
  NormRopeArgs a = {};
  // (v needs no input; its place is that of its gradient)
  const void* const x[3] = {q, k, dv};
  const void* const dy[3] = {dq, dk, dv};
  void* const dx[3] = {dq_in, dk_in, dv_in};
  const int64_t out_strides[6] = {dq_token, dq_head, dk_token, dk_head, dv_token, dv_head};
  if (int rc = common(fn, x, {q_token, q_head, k_token, k_head, 0, 0}, dtype, n_tokens, heads, kv_heads, head_dim, norm, eps,
                      {q_weight, k_weight}, {nullptr, nullptr}, positions, axes, base, a))
    return rc;
  const int size = dtype == BSGA_BF16 ? 2 : 4;
  for (int t = 0; t < 3; ++t) {
    if (n_tokens > 0 && (!x[t] != !dy[t] || !x[t] != !dx[t]))
      return fail(BSGA_ERR_INVALID_ARG, "%s: q and k come with the gradients of both sides, dv with dv_in", fn);
    if (!aligned16(dy[t]) || !aligned16(dx[t])) return fail(BSGA_ERR_INVALID_ARG, "%s: gradients must be 16-byte aligned", fn);
    if (!x[t]) continue;
    const int64_t st = out_strides[2 * t], sh = out_strides[2 * t + 1];
    if (!whole_stride(st, size) || !whole_stride(sh, size))
      return fail(BSGA_ERR_INVALID_ARG, "%s: the gradients' strides must be multiples of 16 bytes and not negative", fn);
    a.dy[t] = static_cast<const unsigned char*>(dy[t]);
    a.dx[t] = static_cast<unsigned char*>(dx[t]);
    a.dx_token[t] = st * size;
    a.dx_head[t] = sh * size;
  }
  if (d_weights && norm == BSGA_NORM_NONE) return fail(BSGA_ERR_INVALID_ARG, "%s: gradients of weights go with a norm", fn);
  if (d_weights && n_tokens > 0) {
    // (the workspace's size goes by both, an absent tensor's as well, and would be 0 for what is no number of heads)
    if (heads < 0 || heads > 65535 || kv_heads < 0 || kv_heads > 65535)
      return fail(BSGA_ERR_INVALID_ARG, "%s: heads and kv_heads must be in [0, 65535], got %d and %d", fn, heads, kv_heads);
    const size_t need = bsga_qk_norm_rope_bwd_workspace_bytes(n_tokens, heads, kv_heads);
    if (!workspace || workspace_bytes < need)
      return fail(BSGA_ERR_WORKSPACE, "%s: workspace has %zu bytes, %zu needed", fn, workspace ? workspace_bytes : 0, need);
    if (!aligned16(workspace) || !aligned16(d_weights))
      return fail(BSGA_ERR_INVALID_ARG, "%s: workspace and d_weights must be 16-byte aligned", fn);
  }
  hipStream_t s = static_cast<hipStream_t>(stream);
  int count[2] = {0, 0};
  if (n_tokens > 0) {
    const int64_t across = bwd_shape(a);
    const int64_t groups = int64_t(groups_of(a, 0)) + groups_of(a, 1) + groups_of(a, 2);
    if (groups > 65535) return fail(BSGA_ERR_UNSUPPORTED, "%s: too many heads", fn);
    if (d_weights) {
      for (int t = 0; t < 2; ++t) count[t] = static_cast<int>(groups_of(a, t) * across);
      a.partial[0] = static_cast<float*>(workspace);
      a.partial[1] = a.partial[0] + int64_t(count[0]) * 128;
    }
    const dim3 grid(static_cast<unsigned>(across), static_cast<unsigned>(groups));
    if (dtype == BSGA_BF16) hipLaunchKernelGGL(norm_rope_bwd_kernel<__bf16>, grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL(norm_rope_bwd_kernel<float>, grid, dim3(256), 0, s, a);
    if (int rc = check_hip(hipGetLastError(), "bsga_qk_norm_rope_bwd launch")) return rc;
  }
  if (d_weights) {  // (of no tokens: zeros)
    hipLaunchKernelGGL(norm_rope_sum_kernel, dim3(8, 2), dim3(1024), 0, s, a.partial[0], a.partial[1], count[0], count[1], d_weights);
    return check_hip(hipGetLastError(), "bsga_qk_norm_rope_bwd launch");
  }
  return BSGA_OK;
}

}  // extern "C"
