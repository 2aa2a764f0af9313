// Attention with a sliding window, counted in frames, and a few first tokens that stay visible.
//
// o_i = sum_j softmax_j(scale <q_i, k_j>) v_j over the keys that query i sees (window.h).  A workgroup takes 64 queries (fp32: 32) for each of its waves;
// a wave holds its queries as B operands and computes S^T = K Q^T, so that a lane has scores of one query, and their weights
// are the B operand of O^T = V^T P^T as they are.  Tiles of 64 keys go straight into LDS, two ahead, one barrier a tile.  Every wave
// sorts a tile for its own rows: seen by all (no masking), by none (skipped), by some.
// Weights are exp2(scale log2(e) s - m) with the products' s in fp32: queries are not scaled beforehand, which would round them a second time.
// The running maximum m follows when a tile exceeds it by 2^8.
//
// Bound by vector issue: 32 keys x 32 queries are 8 products (256 cycles of the matrix pipe) and 448 cycles of exponentials, scaling, sums and packing for
// a wave, two waves to a SIMD.  100 frames of 16 heads, window of 4 and the first: 3.79 TFLOP in 3.8 ms, 1.0 PFLOP/s, matrix pipe 53 % and vector pipe 75 % busy at 1.82 GHz.
#include "window.h"

#include <math.h>

#include <type_traits>

namespace bsga {
namespace {

constexpr float kRaise = 8.0f;
constexpr int kPlaces = 512;   // workgroups of four waves that the chip holds

struct WindowArgs {
  View q, k, v;
  unsigned char* out;     // [heads, n_q, 64]
  float* lse;             // [heads, n_q] or null
  float *part, *part_lse; // with splits: [splits][heads, n_q, 64] and [splits][heads, n_q]
  Seen seen;
  int heads, group, row_tiles, splits;
  float scale_log2;
};

// One query again, by a wave on its own, over the keys that it sees and no others: rows whose result is not finite.  A key that a row does not
// see is multiplied by a weight of zero in the products, which is not nothing if the value is infinite or not a number.
template <typename T>
__device__ void exact_row(const WindowArgs& a, const unsigned char* q, const unsigned char* k, const unsigned char* v, int i, int t0, int t1,
                          const Tiles& tiles, unsigned char* out, float* part, float* lse, int lane) {
  int lo, hi;
  a.seen.range(i, lo, hi);
  float m = -INFINITY, l = 0.f, o = 0.f;
  for (int t = t0; t < t1; ++t) {
    const int j = tiles.key(t) + lane;
    const bool sees = j < hi && (j >= lo || j < a.seen.sinks);
    float s = -INFINITY;
    if (sees) {
      s = 0.f;
      for (int d = 0; d < 64; ++d) s += Ops<T>::number(q, d) * Ops<T>::number(k + j * a.k.token, d);
      s *= a.scale_log2;
    }
    float top = s;
    for (int x = 32; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
    const float to = fmaxf(m, top);
    const float keep = m == -INFINITY ? 0.f : exp2f(m - to);
    const float w = sees ? exp2f(s - (to == -INFINITY ? 0.f : to)) : 0.f;  // (NaN stays)
    float sum = w;
    for (int x = 32; x > 0; x >>= 1) sum += __shfl_xor(sum, x);
    l = l * keep + sum;
    o *= keep;
    m = to;
    unsigned long long all = __ballot(sees);
    while (all != 0) {
      const int e = __builtin_ctzll(all);
      all &= all - 1;
      o += __shfl(w, e) * Ops<T>::number(v + (tiles.key(t) + int64_t(e)) * a.v.token, lane);
    }
  }
  const float value = l == 0.f ? 0.f : o / l;
  if (out != nullptr) Ops<T>::store1(out, lane, value);
  else part[lane] = value;
  if (lse != nullptr && lane == 0) *lse = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

template <int N>
using Int = std::integral_constant<int, N>;

template <typename T, int WAVES, int R>  // R: 32-row parts of a wave's queries
__global__ __launch_bounds__(64 * WAVES, 2) void window_kernel(const WindowArgs a) {
  typedef Ops<T> P;
  constexpr int kTileBytes = kTile * P::kRow, kBuf = 2 * kTileBytes;
  constexpr bool kRuns = sizeof(T) == 2 && R == 2;  // tiles that all rows see go through run()
  extern __shared__ __align__(16) unsigned char smem[];  // K, V of buffer 0, K, V of buffer 1
  __shared__ int flag;
  const int lane = threadIdx.x & 63;
  const int wave = WAVES == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 31, g = lane >> 5;
  // later rows see more where the window is long: they go first
  const int64_t unit = spread(blockIdx.x, gridDim.x, a.heads);
  const int split = static_cast<int>(unit % a.splits);
  const int h = static_cast<int>(unit / a.splits / a.row_tiles);
  const int rt = a.row_tiles - 1 - static_cast<int>(unit / a.splits % a.row_tiles);
  const int i0 = rt * 32 * R * WAVES, i1 = min(i0 + 32 * R * WAVES, a.seen.n_q);
  const Tiles tiles = tiles_of(a.seen, i0, i1);
  const int t0 = static_cast<int>(int64_t(tiles.count) * split / a.splits), t1 = static_cast<int>(int64_t(tiles.count) * (split + 1) / a.splits);
  const unsigned char* const qh = a.q.p + h * a.q.head;
  const unsigned char* const kh = a.k.p + h / a.group * a.k.head;
  const unsigned char* const vh = a.v.p + h / a.group * a.v.head;
  const unsigned lds = lds_address(smem);
  const TileLoad<T, WAVES> k_load(a.k.token, wave, lane), v_load(a.v.token, wave, lane);
  auto issue = [&](int t) {  // buffers by turns
    const int key = tiles.key(t), buf = (t - t0) & 1;
    k_load.all(kh, a.seen.n_k, key, lds + buf * kBuf);
    v_load.all(vh, a.seen.n_k, key, lds + buf * kBuf + kTileBytes);
  };
  auto begin = [&]() {
    if (t0 < t1) issue(t0);
    if (t0 + 1 < t1) issue(t0 + 1);
  };
  begin();

  // the wave's rows [w0, w1); rows past the end are computed as the last one and not stored
  const int w0 = i0 + wave * 32 * R, w1 = min(w0 + 32 * R, a.seen.n_q);
  const bool none = w0 >= a.seen.n_q;
  typename P::A qf[R][P::kSteps];
  int lo[R], hi[R], lo_min = 0, hi_min = 0, lo_max = 0, hi_max = 0;
#pragma unroll
  for (int b = 0; b < R; ++b) {
    const int i = min(w0 + 32 * b + n, a.seen.n_q - 1);
    P::row(qh + i * a.q.token, g, qf[b]);
    a.seen.range(i, lo[b], hi[b]);
  }
  if (!none) {
    a.seen.range(w0, lo_min, hi_min);
    a.seen.range(w1 - 1, lo_max, hi_max);
  }
  auto seen_by_none = [&](int key) { return none || key >= hi_max || (key + kTile <= lo_min && key >= a.seen.sinks); };
  auto seen_by_all = [&](int key) {
    return !none && key + kTile <= hi_min && (key >= lo_max || key + kTile <= a.seen.sinks || a.seen.sinks >= lo_max);
  };

  f32x16 o[2][R];  // [dimensions][queries]
  float m[R], l[R];

  // A tile with masks and a maximum that follows.
  auto plain = [&](int t) {
    const int lane = fresh_lane(), n = lane & 31, g = lane >> 5;  // (addresses are not kept in registers between tiles)
    const int key = tiles.key(t);
    const bool all = seen_by_all(key);
    const unsigned char* const kt = smem + ((t - t0) & 1) * kBuf;
    const unsigned char* const vt = kt + kTileBytes;
    constexpr int U = R == 1 ? 2 : 1;  // 32-key parts at a time: as many as registers allow, for fewer steps of the maximum
#pragma unroll
    for (int u0 = 0; u0 < 2; u0 += U) {
      const int part = key + 32 * u0;  // (left out where no row sees it: 32 frames 1063 -> 1048 us)
      if (U == 1 && (part >= hi_max || (part + 32 <= lo_min && part >= a.seen.sinks))) continue;
      f32x16 s[U][R];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        typename P::A ka[P::kSteps];
        P::rows(kt, 32 * (u0 + u) + n, g, ka);
#pragma unroll
        for (int b = 0; b < R; ++b) {
          clear(s[u][b]);
#pragma unroll
          for (int c = 0; c < P::kSteps; ++c) s[u][b] = P::product(ka[c], qf[b][c], s[u][b]);
          if (!all) keep_seen(s[u][b], key + 32 * (u0 + u) + 4 * g, lo[b], hi[b], a.seen.sinks, key + 32 * (u0 + u) < a.seen.sinks, -INFINITY);
        }
      }
      typename P::A w[U][R][P::kCols];
#pragma unroll
      for (int b = 0; b < R; ++b) {
        float top = s[0][b][0];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int i = 0; i < 16; ++i) top = fmaxf(top, s[u][b][i]);
        top = top_of_halves(top) * a.scale_log2;
        const bool raise = m[b] == -INFINITY ? top > -INFINITY : top > m[b] + kRaise;
        if (__any(raise)) {
          const float to = raise ? top : m[b];
          const float keep = m[b] == -INFINITY ? 1.f : exp2f(m[b] - to);  // (of nothing so far, what is kept is zero)
          m[b] = to;
          l[b] *= keep;
#pragma unroll
          for (int db = 0; db < 2; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[db][b][i] *= keep;
        }
        const float from = m[b] == -INFINITY ? 0.f : m[b];
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            s[u][b][i] = __builtin_amdgcn_exp2f(fmaf(s[u][b][i], a.scale_log2, -from));
            l[b] += s[u][b][i];
          }
          P::round(s[u][b], w[u][b]);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int db = 0; db < 2; ++db) {
          typename P::A va[P::kCols];
          P::columns(vt, 32 * (u0 + u), db, lane, va);
#pragma unroll
          for (int c = 0; c < P::kCols; ++c)
#pragma unroll
            for (int b = 0; b < R; ++b) o[db][b] = P::product(va[c], w[u][b][c], o[db][b]);
        }
    }
  };

  // Whether the wave takes a tile through run(): every row sees all of it or nothing.  from: what is subtracted from a row's scores, its maximum or
  // infinity.  (Rows of two frames share a wave, and tiles that one of them sees need no mask: through plain(), 32 frames take
  // 1235 us instead of 1137.)
  auto whole = [&](int key, bool ready, float (&from)[R]) -> bool {
    if (ready && seen_by_all(key)) {
#pragma unroll
      for (int b = 0; b < R; ++b) from[b] = m[b];
      return true;
    }
    if (seen_by_none(key)) return false;
    bool ok = true;
#pragma unroll
    for (int b = 0; b < R; ++b) {
      const bool in = key + kTile <= hi[b] && (key >= lo[b] || key + kTile <= a.seen.sinks);
      const bool out = key >= hi[b] || (key + kTile <= lo[b] && key >= a.seen.sinks);
      ok = ok && (out || (in && m[b] > -INFINITY));
      from[b] = in ? m[b] : INFINITY;
    }
    return __all(ok);
  };

  // Tiles from t on that whole() lets through; returns the first that is not one.  The vector instructions of one unit of 32 keys x 32
  // queries stand between the products of its neighbours: unit N's weights beside the scores of unit N + 1 and the update of O by
  // unit N - 1, one product and two weights to a slot.  Weights are taken from the maximum that the tiles before have left, without a look at the
  // scores: there is room for 2^100 above it, and rows that need more are found at the end.
  auto run = [&](int t, bool ready, float (&from)[R]) -> int {
    if constexpr (!kRuns) {
      return t;
    } else {
      const int lane = fresh_lane(), n = lane & 31, g = lane >> 5;
      // In LDS, of the first 32 rows of the tile's buffer: K chunks; [dimensions][rows + 8].  (As offsets from smem each read would cost an addition.)
      unsigned kaddr[4], vaddr[2][2];
      unsigned to = lds + ((t - t0) & 1) * kBuf, other = ((t - t0) & 1) ? -kBuf : kBuf;  // the tile's buffer, and from it to the other one
#pragma unroll
      for (int c = 0; c < 4; ++c) kaddr[c] = to + n * P::kRow + (((2 * c + g) ^ P::swizzle(n)) << 4);
      {
        const int mm = (lane & 15) >> 2, j = lane & 3, r = 4 * g + mm;
#pragma unroll
        for (int db = 0; db < 2; ++db)
#pragma unroll
          for (int e = 0; e < 2; ++e)
            vaddr[db][e] = to + kTileBytes + (r + 8 * e) * P::kRow + (((db * 4 + 2 * ((lane >> 4) & 1) + (j >> 1)) ^ P::swizzle(r + 8 * e)) << 4) + (j & 1) * 8;
      }
      f32x16 sc[2];        // scores
      u32x4 pw[2][2];      // weights: [queries][16 keys]
      bf16x8 ka[4];        // K operands of the unit whose scores come next
      bf16x8 va[2][2][2];  // V operands: [32 keys][dimensions][16 keys]
      float ex[2][2];      // the two weights that are packed in the next slot
      float next_from[2] = {INFINITY, INFINITY};  // of the next tile, whose first weights are made in this one's last slot
      auto read_k = [&](int u, int c) {
        ka[c] = *reinterpret_cast<const bf16x8 __attribute__((address_space(3)))*>(kaddr[c] + u * 32 * P::kRow);
      };
      auto read_v = [&](auto uc, auto ic) {  // in the order of their use
        constexpr int u = decltype(uc)::value, db = decltype(ic)::value & 1, cp = decltype(ic)::value >> 1;
        u32x2 x[2];
#pragma unroll
        for (int e = 0; e < 2; ++e)
          x[e] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<s16x4 __attribute__((address_space(3)))*>(
                                               vaddr[db][e] + (32 * u + 16 * cp) * P::kRow)));
        va[u][db][cp] = __builtin_bit_cast(bf16x8, u32x4{x[0][0], x[0][1], x[1][0], x[1][1]});
      };
      auto weight = [&](float s, float from) { return __builtin_amdgcn_exp2f(fmaf(s, a.scale_log2, -from)); };
      auto slot = [&](auto nc, auto sc_, auto&& mid) {
        constexpr int N = decltype(nc)::value, S = decltype(sc_)::value;
        constexpr int BQ = N & 1, BN = (N + 1) & 1, BP = (N + 3) & 1, UP = ((N + 3) & 3) >> 1;  // queries of this unit, the next, the last; keys of the last
        if constexpr (S < 4) {
          if constexpr (S == 0) clear(sc[BN]);
          sc[BN] = P::product(ka[S & 3], qf[BN][S & 3], sc[BN]);
        } else {
          o[S & 1][BP] = P::product(va[UP][S & 1][(S >> 1) & 1], __builtin_bit_cast(bf16x8, pw[BP][(S >> 1) & 1]), o[S & 1][BP]);
        }
        const unsigned pk = pack_bf16(ex[S & 1][0], ex[S & 1][1]);
        l[BQ] += ex[S & 1][0] + ex[S & 1][1];
        asm volatile("" : "+v"(l[BQ]));  // pinned: added up later, all of a unit's weights would stay alive
        if constexpr (S < 7) {
          ex[(S + 1) & 1][0] = weight(sc[BQ][2 * S + 2], from[BQ]);
          ex[(S + 1) & 1][1] = weight(sc[BQ][2 * S + 3], from[BQ]);
        } else {
          ex[0][0] = weight(sc[BN][0], N == 3 ? next_from[0] : from[BN]);
          ex[0][1] = weight(sc[BN][1], N == 3 ? next_from[0] : from[BN]);
        }
        __builtin_amdgcn_sched_barrier(0);
        pw[BQ][S >> 2][S & 3] = pk;
        mid(sc_);
        __builtin_amdgcn_sched_barrier(0);
      };
      auto four = [&](auto nc, auto&& mid) {
        slot(nc, Int<0>{}, mid); slot(nc, Int<1>{}, mid); slot(nc, Int<2>{}, mid); slot(nc, Int<3>{}, mid);
        slot(nc, Int<4>{}, mid); slot(nc, Int<5>{}, mid); slot(nc, Int<6>{}, mid); slot(nc, Int<7>{}, mid);
      };
      // On entry sc[0] holds the first scores, ka the K operands of the first 32 keys, pw[1] and va[1] the last unit before (zeros at the start).
      auto turn = [&]() {
#pragma unroll
        for (int c = 0; c < 4; ++c) kaddr[c] += other;
      };
      auto tile = [&]() {
        const int next = tiles.key(t + 2 < t1 ? t + 2 : t);  // past the end: a load that nobody reads, in place of a branch
        const i32x4 krsrc = k_load.rsrc(kh, a.seen.n_k, next), vrsrc = v_load.rsrc(vh, a.seen.n_k, next);
        // One or two reads of LDS a slot, eight slots ahead of their use: the waves of a workgroup are in step, and reads in one go wait for each other.
        four(Int<0>{}, [&](auto s) {
          constexpr int S = decltype(s)::value;
          if constexpr (S < 4) read_k(1, S);
          else read_v(Int<0>{}, Int<S - 4>{});
        });
        four(Int<1>{}, [&](auto s) {
          constexpr int S = decltype(s)::value;
          if constexpr (S < 4) read_v(Int<1>{}, s);
          if constexpr (S == 4) turn();
          if constexpr (S >= 4) vaddr[S & 1][(S >> 1) & 1] += other;
        });
        four(Int<2>{}, [&](auto s) {
          constexpr int S = decltype(s)::value;
          if constexpr (S == 0) {  // the next tile has landed; this one is read, in every wave
            __builtin_amdgcn_s_waitcnt(0x0f70);
            __syncthreads();
          }
          if constexpr (S < 4) read_k(0, S);
          else k_load.quarter(krsrc, Int<S - 4>{}, to);
        });
        four(Int<3>{}, [&](auto s) {
          constexpr int S = decltype(s)::value;
          if constexpr (S < 4) v_load.quarter(vrsrc, Int<S>{}, to + kTileBytes);
        });
        to += other;
        other = -other;
      };
#pragma unroll
      for (int c = 0; c < 4; ++c) read_k(0, c);
#pragma unroll
      for (int cp = 0; cp < 2; ++cp) {
        pw[1][cp] = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
        for (int db = 0; db < 2; ++db) va[1][db][cp] = __builtin_bit_cast(bf16x8, u32x4{0u, 0u, 0u, 0u});
      }
      clear(sc[0]);
#pragma unroll
      for (int c = 0; c < 4; ++c) sc[0] = P::product(ka[c], qf[0][c], sc[0]);
      ex[0][0] = weight(sc[0][0], from[0]);
      ex[0][1] = weight(sc[0][1], from[0]);
      __builtin_amdgcn_sched_barrier(0);
      for (bool more = true; more; ++t) {
        more = t + 1 < t1 && whole(tiles.key(t + 1), ready, next_from);
        tile();
        from[0] = next_from[0];
        from[1] = next_from[1];
      }
#pragma unroll
      for (int db = 0; db < 2; ++db)
#pragma unroll
        for (int cp = 0; cp < 2; ++cp) o[db][1] = P::product(va[1][db][cp], __builtin_bit_cast(bf16x8, pw[1][cp]), o[db][1]);
      return t;
    }
  };

  // All tiles.  At the top of the loop tile t has landed and the loads of the next are on their way; a tile is one barrier, after which its buffer is
  // free and the loads of the tile after next are issued.  Returns whether (to the whole workgroup) rows left the range of run().
  auto pass = [&](bool runs) -> bool {
#pragma unroll
    for (int b = 0; b < R; ++b) {
      clear(o[0][b]);
      clear(o[1][b]);
      m[b] = -INFINITY;
      l[b] = 0.f;
    }
    if (t0 + 1 < t1) {
      constexpr int kInFlight = kBuf / 1024 / WAVES;
      __builtin_amdgcn_s_waitcnt((kInFlight & 15) | (kInFlight >> 4 << 14) | 0x0f70);
    } else {
      __builtin_amdgcn_s_waitcnt(0x0f70);
    }
    if (threadIdx.x == 0) flag = 0;
    __syncthreads();
    bool ready = false;  // whether all rows have a maximum
    for (int t = t0; t < t1;) {
      if constexpr (kRuns) {
        float from[R];
        if (runs && whole(tiles.key(t), ready, from)) t = run(t, ready, from);
      }
      if (t >= t1) break;
      if (!seen_by_none(tiles.key(t))) {
        plain(t);
        ready = true;
#pragma unroll
        for (int b = 0; b < R; ++b) ready = ready && __all(m[b] > -INFINITY);
      }
      __builtin_amdgcn_s_waitcnt(0x0f70);
      __syncthreads();
      if (t + 2 < t1) issue(t + 2);
      ++t;
    }
    __builtin_amdgcn_s_waitcnt(0x0f70);  // nothing is on its way into LDS any more
    if (!kRuns || !runs) return false;
    bool bad = false;
#pragma unroll
    for (int b = 0; b < R; ++b) {
      bad = bad || !(l[b] < 0x1p100f);
#pragma unroll
      for (int i = 0; i < 16; ++i) bad = bad || !(fabsf(o[0][b][i]) < INFINITY) || !(fabsf(o[1][b][i]) < INFINITY);
    }
    if (bad && !none) flag = 1;
    __syncthreads();
    return flag != 0;
  };
  if (pass(true)) {
    __syncthreads();  // everybody has read the flag
    begin();
    pass(false);
  }

  if (none) return;  // (no barrier follows)
#pragma unroll
  for (int b = 0; b < R; ++b) {
    const float sum = l[b] + __shfl_xor(l[b], 32);
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    bool bad = !(sum < INFINITY);
#pragma unroll
    for (int db = 0; db < 2; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        bad = bad || !(fabsf(o[db][b][i]) < INFINITY);
        o[db][b][i] *= inv;
      }
    const int i = w0 + 32 * b + n;
    const int64_t at = int64_t(h) * a.seen.n_q + i;
    const int64_t in_part = int64_t(split) * a.heads * a.seen.n_q + at;
    float* const lse = a.splits > 1 ? a.part_lse + in_part : a.lse != nullptr ? a.lse + at : nullptr;
    if (i < a.seen.n_q) {
#pragma unroll
      for (int db = 0; db < 2; ++db)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const f32x16& x = o[db][b];
          const int d = db * 32 + 8 * r + 4 * g;
          if (a.splits > 1) *reinterpret_cast<f32x4*>(a.part + in_part * 64 + d) = f32x4{x[4 * r], x[4 * r + 1], x[4 * r + 2], x[4 * r + 3]};
          else P::store4(a.out + at * P::kRow, d, x[4 * r], x[4 * r + 1], x[4 * r + 2], x[4 * r + 3]);
        }
      if (lse != nullptr && g == 0) *lse = sum > 0.f ? (m[b] + log2f(sum)) * kLn2 : -INFINITY;
    }
    unsigned long long again = __ballot(bad && i < a.seen.n_q);
    again = (again | again >> 32) & 0xffffffffull;
    while (again != 0) {
      const int row = w0 + 32 * b + __builtin_ctzll(again);
      again &= again - 1;
      const int64_t to = int64_t(h) * a.seen.n_q + row, to_part = int64_t(split) * a.heads * a.seen.n_q + to;
      exact_row<T>(a, qh + row * a.q.token, kh, vh, row, t0, t1, tiles, a.splits > 1 ? nullptr : a.out + to * P::kRow,
                   a.splits > 1 ? a.part + to_part * 64 : nullptr, a.splits > 1 ? a.part_lse + to_part : a.lse != nullptr ? a.lse + to : nullptr, lane);
    }
  }
}

// How a launch is cut up: waves of a workgroup, 32-row parts of a wave's queries, splits of the keys.  Four waves share tiles; a launch of few rows
// or short windows takes one to a workgroup, and one part where that holds them.  fp32 has no registers for two parts.
struct Shape {
  int waves, parts, splits;
  int rows() const { return waves * parts * 32; }  // of a workgroup
};

// Whether a bf16 launch of more than 128 queries goes by waves of 64 queries on their own, not by four that share tiles: four go in step, and a tile
// that one of them has to mask holds all of them up.  That counts where frames are no longer than a tile, so that every row sees other keys, and
// the window is short (up to 8 tiles for 256 queries), or a CU has one such workgroup at most and few tiles to go through.  Measured, us, four / one:
// 16 heads of 42,116 queries, windows of 1, 64, 256 and 1,024 tokens 123 / 99, 145 / 140, 207 / 196, 311 / 353; 8 heads of 1,100 queries, windows of 1, 64, 256 and
// 1,024 19.7 / 10.0, 23.4 / 12.9, 22.1 / 17.6, 27.6 / 24.5; 16 heads, all keys before the query, 1,156 queries 33.9 / 27.7, 3,804 69 / 74; frames
// of 500 tokens, window of two of them, 6,000 queries 60 / 78.
bool goes_by_waves(const Seen& s, int heads) {
  if (s.frame > kTile) return false;
  const int rows = 256, row_tiles = static_cast<int>(ceil_div(s.n_q, rows)), step = row_tiles / 64 + 1;  // (64 of them or so)
  int most = 0;
  for (int rt = row_tiles - 1; rt >= 0; rt -= step) most = max(most, tiles_of(s, rt * rows, min((rt + 1) * rows, s.n_q)).count);
  return most <= 8 || (int64_t(row_tiles) * heads <= kPlaces / 2 && most <= 32);
}

// The keys are dealt out where that is worth a second kernel.  What a number of parts costs: the chip holds two workgroups of four waves to a CU (of one:
// four), a tile takes such a pair twice 1.15 us (fp32 4.9) and one that is alone 1.4 times, a workgroup begins for 1.5 us; whole rounds last as
// long as the mean workgroup, what is left over as the longest; and parts cost 528 bytes a row at 4 TB/s and 5 us.  us for 1 / 3 / 5 / 8 parts
// with their join: one new frame (1,374 queries, 16 heads) on 12 233 / 144 / 107 / 108, two frames in fp32 418 / 309 / 289 / 310.
Shape shape_of(const Seen& s, int heads, int dtype) {
  const bool bf16 = dtype == BSGA_BF16;
  const double tile = bf16 ? 1.15 : 4.9;
  Shape best = {1, 1, 1};
  if (bf16 && s.n_q > 32) best.parts = 2;
  if (s.n_q > 2 * best.rows() && !(bf16 && goes_by_waves(s, heads))) best.waves = 4;
  const int rows = best.rows();
  const int64_t units = ceil_div(s.n_q, rows) * heads, places = best.waves == 4 ? kPlaces : 2 * kPlaces;
  if (units > 4 * places) return best;  // the last round is one of many
  int most = 0;
  int64_t all = 0;
  for (int i0 = 0; i0 < s.n_q; i0 += rows) {
    const int c = tiles_of(s, i0, min(i0 + rows, s.n_q)).count;
    most = c > most ? c : most;
    all += c;
  }
  const double mean = static_cast<double>(all) / static_cast<double>(ceil_div(s.n_q, rows));
  const double full = best.waves == 4 ? 2.0 : 1.4;
  double least = 0.0;
  for (int n = 1; n == 1 || (n <= 64 && n <= most); ++n) {
    const int64_t rounds = units * n / places, left = units * n - rounds * places;
    const double us = static_cast<double>(rounds) * (full * tile * mean / n + 1.5) +
                      (left == 0 ? 0.0 : (left <= kPlaces / 2 ? 1.4 : full) * tile * static_cast<double>(ceil_div(most, n)) + 1.5) +
                      (n > 1 ? 5.0 + static_cast<double>(heads) * s.n_q * n * 528 / 4e6 : 0.0);
    if (n > 1 && us >= least) continue;
    least = us;
    best.splits = n;
  }
  return best;
}

size_t split_bytes(int heads, int64_t n_q, int splits) { return splits > 1 ? static_cast<size_t>(splits) * heads * n_q * 65 * sizeof(float) : 0; }

template <typename T, int WAVES, int R>
int launch(const WindowArgs& a, hipStream_t s) {
  const int64_t units = int64_t(a.heads) * a.row_tiles * a.splits;
  if (units > 0x7fffffff) return fail(BSGA_ERR_UNSUPPORTED, "bsga_window_attn: too many rows");
  hipLaunchKernelGGL((window_kernel<T, WAVES, R>), dim3(static_cast<unsigned>(units)), dim3(64 * WAVES), 4 * kTile * Ops<T>::kRow, s, a);
  if (int rc = check_hip(hipGetLastError(), "bsga_window_attn launch")) return rc;
  if (a.splits == 1) return BSGA_OK;
  return launch_join<T>(a.part, a.part_lse, int64_t(a.heads) * a.seen.n_q, a.splits, a.out, a.lse, s);
}

}  // namespace
}  // namespace bsga

using namespace bsga;

extern "C" {

size_t bsga_window_attn_workspace_bytes(int dtype, int heads, int64_t n_q, int64_t n_k, int64_t q_start, int64_t frame, int64_t window,
                                        int64_t sinks) {
  Seen s;
  if ((dtype != BSGA_BF16 && dtype != BSGA_FP32) || heads < 1 || heads > 65535 || n_q < 1 || n_k < 1) return 0;
  if (check_seen("", n_q, n_k, q_start, frame, window, sinks, s)) return 0;
  return split_bytes(heads, n_q, shape_of(s, heads, dtype).splits);
}

int bsga_window_attn(const void* q, const void* k, const void* v, int64_t q_token, int64_t q_head, int64_t k_token, int64_t k_head,
                     int64_t v_token, int64_t v_head, int dtype, int heads, int kv_heads, int64_t n_q, int64_t n_k, int head_dim,
                     float softmax_scale, int64_t q_start, int64_t frame, int64_t window, int64_t sinks, void* out, float* lse, void* workspace,
                     size_t workspace_bytes, void* stream) {
  const char* fn = "bsga_window_attn";
  clear_error();
  WindowArgs a = {};
  if (dtype != BSGA_BF16 && dtype != BSGA_FP32) return fail(BSGA_ERR_INVALID_ARG, "%s: unknown dtype %d", fn, dtype);
  if (head_dim != 64) return fail(BSGA_ERR_UNSUPPORTED, "%s: head_dim must be 64, got %d", fn, head_dim);
  if (heads < 1 || heads > 65535 || kv_heads < 1 || heads % kv_heads != 0)
    return fail(BSGA_ERR_INVALID_ARG, "%s: heads must be in [1, 65535] and a multiple of kv_heads, got %d and %d", fn, heads, kv_heads);
  if (int rc = check_seen(fn, n_q, n_k, q_start, frame, window, sinks, a.seen)) return rc;
  if (!(softmax_scale > 0.0f) || !isfinite(softmax_scale)) return fail(BSGA_ERR_INVALID_ARG, "%s: softmax_scale must be finite and > 0", fn);
  if (n_q == 0) return BSGA_OK;
  const int size = dtype == BSGA_BF16 ? 2 : 4;
  if (int rc = check_view(fn, "q", q, q_token, q_head, size, a.q)) return rc;
  if (n_k > 0) {
    if (int rc = check_view(fn, "k", k, k_token, k_head, size, a.k)) return rc;
    if (int rc = check_view(fn, "v", v, v_token, v_head, size, a.v)) return rc;
  }
  if (!out || !aligned16(out)) return fail(BSGA_ERR_INVALID_ARG, "%s: out must be non-null and 16-byte aligned", fn);
  a.out = static_cast<unsigned char*>(out);
  a.lse = lse;
  a.heads = heads;
  a.group = heads / kv_heads;
  a.scale_log2 = softmax_scale * kLog2e;
  const Shape shape = shape_of(a.seen, heads, dtype);
  a.splits = shape.splits;
  if (!workspace || !aligned16(workspace) || workspace_bytes < split_bytes(heads, n_q, a.splits)) a.splits = 1;  // one workgroup takes all keys of its rows
  a.row_tiles = static_cast<int>(ceil_div(n_q, shape.rows()));
  a.part = static_cast<float*>(workspace);
  if (a.splits > 1) a.part_lse = a.part + int64_t(a.splits) * heads * n_q * 64;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (dtype == BSGA_FP32) return shape.waves == 4 ? launch<float, 4, 1>(a, s) : launch<float, 1, 1>(a, s);
  if (shape.waves == 4) return launch<__bf16, 4, 2>(a, s);
  return shape.parts == 2 ? launch<__bf16, 1, 2>(a, s) : launch<__bf16, 1, 1>(a, s);
}

}  // extern "C"
