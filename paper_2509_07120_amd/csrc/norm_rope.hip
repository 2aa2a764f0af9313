// Norms of queries and keys for each head with the rotation by position in the same pass, and the gradient of that.
//
// A row is one head's 64 numbers x of one token.  rms: n = x r w with r = (mean x^2 + eps)^-1/2; layer: n = (x - mean) r w + b.  The
// rotation cuts the row into one segment for each axis of the positions; in a segment of width W the pairs (j, j + W/2) turn by
// position * base^(-2j/W).  Backwards, with g the gradient turned back and h the row before the weight: dw = sum g h, db = sum g,
// dx = r (w g - [mean w g] - h mean(w g h)).
//
// HBM-bound: 100 frames of 48 heads (1.69 GB) 338 us, 5.0 TB/s, where a copy of 1 GiB reaches 5.1.  A row is read once and written once.  Four lanes hold a row, lane c eight of its pairs (so that the rotation stays in
// the lane), and the sums over a row are two quad permutations.  A lane keeps its token over the heads that its workgroup takes: the angles are
// computed once for them.  Angles are exact: base^(-2j/W) / 2 pi is a 64-bit fraction of a turn, and the product with the position
// modulo 2^64 is the turn's fraction, whatever the position's size; fp32 would be off by 0.1 at position 10^6.
#include "bf16_tile.h"
#include "bsga_internal.h"

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
  unsigned long long turn[32];
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

// (a, b) become the row before the weight; the factor that the row was multiplied with is returned.
__device__ __forceinline__ float normalise(int norm, float eps, float (&a)[8], float (&b)[8]) {
  if (norm == BSGA_NORM_NONE) return 1.f;
  if (norm == BSGA_NORM_LAYER) {
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) s += a[e] * 0x1p-6f + b[e] * 0x1p-6f;  // (the mean of values that fit fits, their sum may not)
    const float mean = row_sum(s);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      a[e] -= mean;
      b[e] -= mean;
    }
  }
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) s += a[e] * a[e] + b[e] * b[e];
  const float r = 1.f / sqrtf(row_sum(s) * 0x1p-6f + eps);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    a[e] *= r;
    b[e] *= r;
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

template <typename T>
__global__ __launch_bounds__(256) void norm_rope_kernel(const NormRopeArgs a) {
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
  for (int h = h0; h < h1; h += kHeadsInFlight) {
    if (h > h0) fetch(h);
#pragma unroll
    for (int u = 0; u < kHeadsInFlight; ++u) {
      if (h + u >= h1) break;
      unsigned char* p = dst + (to + (h + u) * step) * kRow;
      float x[8], y[8];
      widen<T>(lo[u], x);
      widen<T>(hi[u], y);
      if (kind < 2) {
        normalise(a.norm, a.eps, x, y);
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
      if (write) {
        store<T>(p + l.first * sizeof(T), x);
        store<T>(p + l.second * sizeof(T), y);
      }
    }
  }
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
  if (slots) {
    if (page < 1 || page > 65536) return fail(BSGA_ERR_INVALID_ARG, "%s: page must be in [1, 65536] tokens, got %d", fn, page);
    if (n_pages < 1 || n_pages > ((int64_t(1) << 31) - 1) / page)
      return fail(BSGA_ERR_INVALID_ARG, "%s: the cache must hold 1 to 2^31 - 1 tokens, got %lld pages of %d", fn, static_cast<long long>(n_pages), page);
    a.slots = slots;
    a.page = page;
    a.n_slots = n_pages * page;
  }
  if (n_tokens == 0) return BSGA_OK;
  const int64_t tiles = ceil_div(n_tokens, kRowsPerGroup);
  a.group_heads = heads_of_a_group(a, tiles);
  const int64_t groups = int64_t(groups_of(a, 0)) + groups_of(a, 1) + groups_of(a, 2);
  if (groups > 65535) return fail(BSGA_ERR_UNSUPPORTED, "%s: too many heads", fn);
  const dim3 grid(static_cast<unsigned>(tiles), static_cast<unsigned>(groups));
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (dtype == BSGA_BF16) hipLaunchKernelGGL(norm_rope_kernel<__bf16>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(norm_rope_kernel<float>, grid, dim3(256), 0, s, a);
  return check_hip(hipGetLastError(), "bsga_qk_norm_rope launch");
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
