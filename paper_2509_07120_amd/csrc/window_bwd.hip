// The gradient of attention with a sliding window (window.hip).
//
// With P = exp(s - lse) for the keys j that query i sees and D_i = sum_d dO_id O_id:
//   dV_j = sum_i P_ij dO_i,  dS_ij = P_ij (<dO_i, V_j> - D_i),  dQ_i = scale sum_j dS_ij K_j,  dK_j = scale sum_i dS_ij Q_i,
// the sums of dV and dK over the query heads that share the key head as well.
// Two kinds of workgroups, so that every sum has one owner and one order (no atomics): for query rows, which go over the keys as the forward pass
// does, and for key rows, which go over the queries that see them.  Seven products in place of the five that one kind with shared
// sums of dQ would need.  Both recompute S and P from lse.  They are one launch: the key rows' workgroups, which are longer, come first, and the
// others fill up what they leave.
// Key rows that are seen from far (the first tokens) have many more queries than others: their queries are dealt out to several workgroups, whose
// sums in fp32 are added up at the end, always in the same order.
// 20,011 tokens of 16 heads to 4 key heads, window of 4096: 1.02 ms, 1.03 PFLOP/s of the seven products; matrix pipe 60 % busy, vector pipe 56 %, LDS 38 %,
// at 1.69 GHz.
#include "window.h"

#include <math.h>

#include <type_traits>

namespace bsga {
namespace {

constexpr int kPlaces = 512;
constexpr int kOwnRows = 128;     // queries or keys of a workgroup, 32 for each wave
constexpr int kEarlyKeys = 256;   // D of queries that see fewer is summed over the keys
constexpr int kStatBytes = 1024;  // of a tile's queries: 512 bytes, and as much that the load of a whole wave adds

struct BwdArgs {
  View q, k, v;
  const unsigned char *out, *dout;  // [heads, n_q, 64]
  const float* lse;
  float* stats;                     // [heads][2][stat_rows]: -lse / scale and -D, what the products' sums of a query begin with; whole tiles of rows
  unsigned char *dq, *dk, *dv;      // contiguous
  float* part_q;                    // [q_splits][heads, n_q, 64]
  float* part_kv[2];                // first tokens: [sink_splits][kv_heads, sink_rows, 128]; the others [splits][kv_heads, n_k - sink_rows, 128]
  Seen seen;
  int heads, kv_heads, group, stat_rows, row_tiles, q_splits;
  int key_tiles, sink_tiles, sink_splits, splits;  // of kOwnRows keys
  float scale, scale_log2;
};

// Queries that see key j: [first, last).
struct Queries {
  int first, last;
};

__host__ __device__ inline Queries queries_of(const Seen& s, int j) {
  const int f = j / s.frame;
  Queries r;
  r.first = static_cast<int>(larger(int64_t(f) * s.frame - s.q_start, int64_t(0)));
  r.last = j < s.sinks ? s.n_q : static_cast<int>(larger(smaller((int64_t(f) + s.window) * s.frame - s.q_start, int64_t(s.n_q)), int64_t(0)));
  return r;
}

template <typename T>
__device__ __forceinline__ float dot_rows(const unsigned char* x, const unsigned char* y) {
  float s = 0.f;
  for (int d = 0; d < 64; ++d) s += Ops<T>::number(x, d) * Ops<T>::number(y, d);
  return s;
}

// The gradient of one query again, by a wave on its own, over the keys that it sees and no others, see exact_row in window.hip.
template <typename T>
__device__ float exact_query(const BwdArgs& a, const unsigned char* q, const unsigned char* dout, const unsigned char* k, const unsigned char* v,
                             float from, float D, int i, int t0, int t1, const Tiles& tiles, int lane) {
  int lo, hi;
  a.seen.range(i, lo, hi);
  float sum = 0.f;
  for (int t = t0; t < t1; ++t) {
    const int j = tiles.key(t) + lane;
    const bool sees = j < hi && (j >= lo || j < a.seen.sinks);
    float ds = 0.f;
    if (sees) ds = exp2f((dot_rows<T>(q, k + j * a.k.token) + from) * a.scale_log2) * (dot_rows<T>(dout, v + j * a.v.token) + D);
    unsigned long long all = __ballot(sees);
    while (all != 0) {
      const int e = __builtin_ctzll(all);
      all &= all - 1;
      sum += __shfl(ds, e) * Ops<T>::number(k + (tiles.key(t) + int64_t(e)) * a.k.token, lane);
    }
  }
  return sum * a.scale;
}

template <int N>
using Int = std::integral_constant<int, N>;
template <int A, int B, typename F>
__device__ __forceinline__ void each(F&& f) {
  if constexpr (A < B) {
    f(Int<A>{});
    each<A + 1, B>(f);
  }
}

// Tiles of the streamed rows (X: those of the first product, Y: of the second) that see all of a wave's own rows, or are seen by them: from t on as
// long as more(t).  A tile is two units of 32 streamed rows.  In unit N, while the vector instructions make P and dS of it, the
// matrix pipe makes S and dP of unit N + 1 (eight products) and adds unit N - 1 to the sums (SUMS products: eight of key rows, four of query
// rows): one product to a slot, with the operand that its register gets next asked for right behind it, half a unit ahead of its use.
//   own0, own1  the wave's rows as operands of S and dP;  sums0 += columns of Y (key rows) or X (query rows) by P or dS, sums1 += columns of X by dS
//   first0, first1  what S and dP of query rows begin with; those of key rows begin with the 64 + 64 numbers behind X and Y
//   land(): all loads of the wave's next tile have landed and everybody has read the last one; load(I): load I of the tile after next
template <int SUMS, typename More, typename Land, typename Load>
__device__ __forceinline__ int run(int t, unsigned at, const unsigned char* smem, float scale_log2, const bf16x8 (&own0)[4], const bf16x8 (&own1)[4],
                                   const f32x16& first0, const f32x16& first1, f32x16 (&sums0)[2], f32x16 (&sums1)[2], More&& more, Land&& land,
                                   Load&& load) {
  typedef Ops<__bf16> P;
  constexpr bool KEYS = SUMS == 8;
  constexpr int kTileBytes = kTile * P::kRow, kBuf = 2 * kTileBytes + (KEYS ? kStatBytes : 0), kSlots = SUMS + 8;
  const int lane = fresh_lane(), n = lane & 31, g = lane >> 5;
  // In LDS, of the first 32 rows: chunks of a row; [dimensions][rows + 8] of the transposed operands; where S and dP begin.  (As offsets each read
  // would cost an addition.)
  unsigned raddr[4], caddr[2][2], saddr = lds_address(smem) + at + 2 * kTileBytes + g * 16;
#pragma unroll
  for (int c = 0; c < 4; ++c) raddr[c] = lds_address(smem) + at + n * P::kRow + (((2 * c + g) ^ P::swizzle(n)) << 4);
  {
    const int m = (lane & 15) >> 2, j = lane & 3, r = 4 * g + m;
#pragma unroll
    for (int db = 0; db < 2; ++db)
#pragma unroll
      for (int e = 0; e < 2; ++e)
        caddr[db][e] = lds_address(smem) + at + (r + 8 * e) * P::kRow + (((db * 4 + 2 * ((lane >> 4) & 1) + (j >> 1)) ^ P::swizzle(r + 8 * e)) << 4) + (j & 1) * 8;
  }
  auto step_from = [](unsigned at) { return at == 2 * kBuf ? static_cast<unsigned>(-2 * kBuf) : static_cast<unsigned>(kBuf); };
  unsigned step = step_from(at), last_step = 0;  // from this tile's buffer to the next one, from the last one's to this
  f32x16 s[2], dp[2];                                       // [unit]; P and dS take their places
  u32x4 pw[2], dw[2];                                       // packed: [16 streamed rows]
  bf16x8 op[8];
  auto row_operand = [&](auto ic, auto uc) {  // of S (0 to 3) and dP
    constexpr int I = decltype(ic)::value, U = decltype(uc)::value;
    op[I] = *reinterpret_cast<const bf16x8 __attribute__((address_space(3)))*>(raddr[I & 3] + (I >> 2) * kTileBytes + U * 32 * P::kRow);
  };
  auto sum_operand = [&](auto ic, auto uc) {  // of the sums
    constexpr int I = decltype(ic)::value, U = decltype(uc)::value;
    constexpr int kind = KEYS ? I & 1 : 1, db = KEYS ? (I >> 1) & 1 : I & 1, cp = KEYS ? I >> 2 : I >> 1;
    u32x2 x[2];
#pragma unroll
    for (int e = 0; e < 2; ++e)
      x[e] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<s16x4 __attribute__((address_space(3)))*>(
                                           caddr[db][e] + (kind == 0 ? kTileBytes : 0) + (32 * U + 16 * cp) * P::kRow)));
    op[I] = __builtin_bit_cast(bf16x8, u32x4{x[0][0], x[0][1], x[1][0], x[1][1]});
  };
  auto begin_from = [&](auto ic, auto uc) {  // quarter I of what S and dP of key rows begin with
    constexpr int I = decltype(ic)::value, U = decltype(uc)::value;
    typedef const f32x4 __attribute__((address_space(3)))* Quarter;
    const f32x4 x = *reinterpret_cast<Quarter>(saddr + (32 * U + 8 * I) * 4), y = *reinterpret_cast<Quarter>(saddr + (32 * U + 8 * I) * 4 + 256);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      s[U][4 * I + e] = x[e];
      dp[U][4 * I + e] = y[e];
    }
  };
  auto product = [&](auto jc, auto uc) {  // number J of S and dP of unit U
    constexpr int J = decltype(jc)::value, U = decltype(uc)::value;
    if constexpr (J < 4) s[U] = P::product(op[J], own0[J & 3], !KEYS && J == 0 ? first0 : s[U]);
    else dp[U] = P::product(op[J], own1[J & 3], !KEYS && J == 4 ? first1 : dp[U]);
  };
  auto add = [&](auto ic) {  // number I of the sums
    constexpr int I = decltype(ic)::value;
    if constexpr (KEYS) {
      constexpr int db = (I >> 1) & 1, cp = I >> 2;
      if constexpr ((I & 1) == 0) sums0[db] = P::product(op[I], __builtin_bit_cast(bf16x8, pw[cp]), sums0[db]);
      else sums1[db] = P::product(op[I], __builtin_bit_cast(bf16x8, dw[cp]), sums1[db]);
    } else {
      sums0[I & 1] = P::product(op[I], __builtin_bit_cast(bf16x8, dw[I >> 1]), sums0[I & 1]);
    }
  };
  auto slot = [&](auto uc, auto sc) {
    constexpr int U = decltype(uc)::value, S = decltype(sc)::value, V = U ^ 1;
    if constexpr (S < SUMS) {
      add(Int<S>{});
      row_operand(Int<S>{}, Int<V>{});
      if constexpr (SUMS == 4) row_operand(Int<4 + S>{}, Int<V>{});
      if constexpr (KEYS && S < 4) begin_from(Int<S>{}, Int<V>{});
    } else {
      product(Int<S - SUMS>{}, Int<V>{});
      if constexpr (S - SUMS < SUMS) sum_operand(Int<S - SUMS>{}, uc);
    }
    // on to the next buffer, whose rows are read from unit 1 on and whose columns from its own unit 0 on
    if constexpr (U == 0 && S < 4) caddr[S & 1][S >> 1] += last_step;
    if constexpr (U == 0 && S >= SUMS && S < SUMS + 4) raddr[S - SUMS] += step;
    if constexpr (KEYS && U == 0 && S == SUMS + 4) saddr += step;
    if constexpr (U == 1 && S >= 1 && S < 6) load(Int<S - 1>{});
    // numbers of P done before slot x, of dS (two slots later: dP is the last that the matrix pipe makes), and words packed: the sums of the last
    // unit read the first four until slot SUMS / 2 - 1, the others until SUMS - 1
    constexpr auto ps = [](int x) { return x * 16 / kSlots; };
    constexpr auto dss = [](int x) { return x >= kSlots ? 16 : x < 2 ? 0 : (x - 2) * 16 / kSlots; };
    constexpr auto words = [](int done, int x) { return x < SUMS / 2 ? 0 : x < SUMS ? (done / 2 < 4 ? done / 2 : 4) : done / 2; };
    each<ps(S), ps(S + 1)>([&](auto e) {
      constexpr int E = decltype(e)::value;
      s[U][E] = __builtin_amdgcn_exp2f(s[U][E] * scale_log2);
    });
    each<dss(S), dss(S + 1)>([&](auto e) {
      constexpr int E = decltype(e)::value;
      dp[U][E] *= s[U][E];
    });
    if constexpr (KEYS)
      each<words(ps(S), S), words(ps(S + 1), S + 1)>([&](auto w) {
        constexpr int W = decltype(w)::value;
        unsigned x = pack_bf16(s[U][2 * W], s[U][2 * W + 1]);
        asm volatile("" : "+v"(x));  // here, and not where it is used
        pw[W >> 2][W & 3] = x;
      });
    each<words(dss(S), S), words(dss(S + 1), S + 1)>([&](auto w) {
      constexpr int W = decltype(w)::value;
      unsigned x = pack_bf16(dp[U][2 * W], dp[U][2 * W + 1]);
      asm volatile("" : "+v"(x));
      dw[W >> 2][W & 3] = x;
    });
    __builtin_amdgcn_sched_barrier(0);
  };

  each<0, 8>([&](auto i) { row_operand(i, Int<0>{}); });
  if constexpr (KEYS) each<0, 4>([&](auto i) { begin_from(i, Int<0>{}); });
  each<0, 8>([&](auto j) { product(j, Int<0>{}); });
#pragma unroll
  for (int i = 0; i < 8; ++i) op[i] = __builtin_bit_cast(bf16x8, u32x4{0u, 0u, 0u, 0u});
#pragma unroll
  for (int i = 0; i < 2; ++i) pw[i] = dw[i] = u32x4{0u, 0u, 0u, 0u};
  __builtin_amdgcn_sched_barrier(0);
  do {
    each<0, kSlots>([&](auto x) { slot(Int<0>{}, x); });
    land();
    each<0, kSlots>([&](auto x) { slot(Int<1>{}, x); });
    at += step;
    last_step = step;
    step = step_from(at);
    ++t;
  } while (more(t));
  each<0, SUMS>([&](auto i) { add(i); });
  return t;
}

// Whether S and dP begin with -lse / scale and -D, or have them added at the end: in fp32, 32 sums that begin far from zero would each be rounded
// there (two frames: error of dQ 1.8e-6, 1.1e-6 as it is).
template <typename T>
constexpr bool kFromStats = sizeof(T) == 2;

// Buffers of a workgroup's tiles.  Three let a wave read the next tile while others are still at the last one, as run() does; fp32 has no
// room for three and does not run.
template <typename T>
constexpr int Buffers = sizeof(T) == 2 ? 3 : 2;

// The tiles [t0, t1) in turn, of which the first two are on their way (`loads` loads of each wave for a tile).  plain(t) takes one tile; ahead(t, land) takes
// none or more and returns the first that is left.  A tile is one barrier, behind which its successor has landed in every wave.
template <typename T, typename Issue, typename Plain, typename Ahead>
__device__ __forceinline__ void stream(int t0, int t1, int loads, Issue&& issue, Plain&& plain, Ahead&& ahead) {
  auto land = []() {
    __builtin_amdgcn_s_waitcnt(0x0f70);
    __syncthreads();
  };
  if (t0 + 1 < t1) {
    if (loads == 4) __builtin_amdgcn_s_waitcnt(0x0f74);
    else if (loads == 5) __builtin_amdgcn_s_waitcnt(0x0f75);
    else if (loads == 8) __builtin_amdgcn_s_waitcnt(0x0f78);
    else __builtin_amdgcn_s_waitcnt(0x0f70);
  } else {
    __builtin_amdgcn_s_waitcnt(0x0f70);
  }
  __syncthreads();
  for (int t = t0; t < t1; ++t) {
    t = ahead(t, land);
    if (t >= t1) break;
    if constexpr (Buffers<T> == 2) plain(t);
    land();
    if (t + 2 < t1) issue(t + 2);
    if constexpr (Buffers<T> == 3) plain(t);  // behind the barrier: the tile after next goes where the last one was
  }
  __builtin_amdgcn_s_waitcnt(0x0f70);  // nothing is on its way into LDS any more
}

// dQ of 32 queries for each of four waves.  smem: K, V of each buffer.
template <typename T>
__device__ __forceinline__ void query_rows(const BwdArgs& a, int64_t block, int64_t blocks, unsigned char* smem) {
  typedef Ops<T> P;
  constexpr int WAVES = 4, kBuffers = Buffers<T>;
  constexpr int kTileBytes = kTile * P::kRow, kBuf = 2 * kTileBytes;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 31, g = lane >> 5;
  const int64_t unit = spread(block, blocks, a.heads);
  const int split = scalar(static_cast<int>(unit % a.q_splits));
  const int h = scalar(static_cast<int>(unit / a.q_splits / a.row_tiles));
  const int rt = a.row_tiles - 1 - scalar(static_cast<int>(unit / a.q_splits % a.row_tiles));
  const int i0 = rt * kOwnRows, i1 = min(i0 + kOwnRows, a.seen.n_q);
  const Tiles tiles = scalar(tiles_of(a.seen, i0, i1));
  const int t0 = scalar(static_cast<int>(int64_t(tiles.count) * split / a.q_splits)), t1 = scalar(static_cast<int>(int64_t(tiles.count) * (split + 1) / a.q_splits));
  const unsigned char* const qh = a.q.p + h * a.q.head;
  const unsigned char* const kh = a.k.p + h / a.group * a.k.head;
  const unsigned char* const vh = a.v.p + h / a.group * a.v.head;
  const int64_t row0 = int64_t(h) * a.seen.n_q;
  const unsigned lds = lds_address(smem);
  const TileLoad<T, WAVES> k_load(a.k.token, wave, lane), v_load(a.v.token, wave, lane);
  auto place = [&](int t) { return static_cast<unsigned>(scalar((t - t0) % kBuffers)) * kBuf; };
  auto issue = [&](int t) {
    const int key = tiles.key(t);
    k_load.all(kh, a.seen.n_k, key, lds + place(t));
    v_load.all(vh, a.seen.n_k, key, lds + place(t) + kTileBytes);
  };
  if (t0 < t1) issue(t0);
  if (t0 + 1 < t1) issue(t0 + 1);

  const int w0 = i0 + wave * 32, w1 = min(w0 + 32, a.seen.n_q);
  const bool none = w0 >= a.seen.n_q;
  typename P::A qf[P::kSteps], df[P::kSteps];
  int lo, hi, lo_min = 0, hi_min = 0, lo_max = 0, hi_max = 0;
  f32x16 from, D;  // what S and dP begin with
  {
    const int i = min(w0 + n, a.seen.n_q - 1);
    P::row(qh + i * a.q.token, g, qf);
    P::row(a.dout + (row0 + i) * P::kRow, g, df);
    a.seen.range(i, lo, hi);
    const float* const st = a.stats + int64_t(h) * 2 * a.stat_rows + i;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      from[e] = st[0];
      D[e] = st[a.stat_rows];
    }
  }
  if (!none) {
    a.seen.range(w0, lo_min, hi_min);
    a.seen.range(w1 - 1, lo_max, hi_max);
  }
  lo_min = scalar(lo_min), hi_min = scalar(hi_min), lo_max = scalar(lo_max), hi_max = scalar(hi_max);
  auto seen_by_none = [&](int key) { return none || key >= hi_max || (key + kTile <= lo_min && key >= a.seen.sinks); };
  auto seen_by_all = [&](int key) {
    return !none && key + kTile <= hi_min && (key >= lo_max || key + kTile <= a.seen.sinks || a.seen.sinks >= lo_max);
  };

  f32x16 dq[2];  // [dimensions], queries in the columns
  clear(dq[0]);
  clear(dq[1]);
  auto plain = [&](int t) {
    const int lane = fresh_lane(), n = lane & 31, g = lane >> 5;  // (addresses are not kept in registers between tiles)
    const int key = tiles.key(t);
    const bool all = seen_by_all(key);
    const unsigned char* const kt = smem + place(t);
    const unsigned char* const vt = kt + kTileBytes;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if (key + 32 * u >= hi_max || (key + 32 * u + 32 <= lo_min && key + 32 * u >= a.seen.sinks)) continue;  // no query of the wave sees these
      typename P::A w[P::kCols];
      {
        typename P::A ka[P::kSteps], va[P::kSteps];
        P::rows(kt, 32 * u + n, g, ka);
        P::rows(vt, 32 * u + n, g, va);
        f32x16 s, dp;
        if constexpr (kFromStats<T>) {
          s = from;
          dp = D;
        } else {
          clear(s);
          clear(dp);
        }
#pragma unroll
        for (int c = 0; c < P::kSteps; ++c) {
          s = P::product(ka[c], qf[c], s);
          dp = P::product(va[c], df[c], dp);
        }
        if constexpr (!kFromStats<T>) {
          s += from;
          dp += D;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(s[i] * a.scale_log2) * dp[i];
        if (!all) keep_seen(s, key + 32 * u + 4 * g, lo, hi, a.seen.sinks, key + 32 * u < a.seen.sinks, 0.f);
        P::round(s, w);
      }
#pragma unroll
      for (int db = 0; db < 2; ++db) {
        typename P::A kc[P::kCols];
        P::columns(kt, 32 * u, db, lane, kc);
#pragma unroll
        for (int c = 0; c < P::kCols; ++c) dq[db] = P::product(kc[c], w[c], dq[db]);
      }
    }
  };
  stream<T>(t0, t1, 2 * TileLoad<T, WAVES>::kLoads, issue, [&](int t) {
    if (!seen_by_none(tiles.key(t))) plain(t);
  }, [&](int t, auto&& land) {
    if constexpr (sizeof(T) == 2) {
      if (!seen_by_all(tiles.key(t))) return t;
      // the keys of this tile, the next and the one after; and the places of the last in memory and in LDS.  Past the end: loads that nobody reads
      int key = tiles.key(t), key1 = tiles.key(t + 1), key2 = tiles.key(t + 2);
      const int jump = tiles.first > t + 2 ? tiles.first * kTile : -1, behind = tiles.start * kTile;  // where the window's tiles follow the first tokens'
      const unsigned char *kp = kh + key2 * a.k.token, *vp = vh + key2 * a.v.token;
      const int64_t k_step = kTile * a.k.token, v_step = kTile * a.v.token;
      unsigned to = lds + place(t + 2);
      i32x4 krsrc, vrsrc;
      f32x16 unused[2];
      t = run<4>(t, place(t), smem, a.scale_log2, qf, df, from, D, dq, unused, [&](int x) { return x < t1 && seen_by_all(key); },
                 [&]() {
                   land();
                   krsrc = k_load.rsrc_at(kp, a.seen.n_k - key2);
                   vrsrc = v_load.rsrc_at(vp, a.seen.n_k - key2);
                 },
                 [&](auto i) {
                   constexpr int I = decltype(i)::value;
                   if constexpr (I < 2) {
                     k_load.one(krsrc, i, to);
                   } else if constexpr (I < 4) {
                     v_load.one(vrsrc, Int<I - 2>{}, to + kTileBytes);
                   } else {  // on to the next
                     to = to + kBuf == lds + kBuffers * kBuf ? lds : to + kBuf;
                     key = key1;
                     key1 = key2;
                     key2 += kTile;
                     kp += k_step;
                     vp += v_step;
                     if (key2 == jump) {
                       key2 = behind;
                       kp = kh + key2 * a.k.token;
                       vp = vh + key2 * a.v.token;
                     }
                   }
                 });
    }
    return t;
  });

  if (none) return;  // (no barrier follows)
  const int i = w0 + n;
  const int64_t in_part = int64_t(split) * a.heads * a.seen.n_q + row0 + i;
  bool bad = false;
#pragma unroll
  for (int db = 0; db < 2; ++db)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      dq[db][e] *= a.scale;
      bad = bad || !(fabsf(dq[db][e]) < INFINITY);
    }
  if (i < a.seen.n_q) {
#pragma unroll
    for (int db = 0; db < 2; ++db)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const f32x16& x = dq[db];
        const int d = db * 32 + 8 * r + 4 * g;
        if (a.q_splits > 1) *reinterpret_cast<f32x4*>(a.part_q + in_part * 64 + d) = f32x4{x[4 * r], x[4 * r + 1], x[4 * r + 2], x[4 * r + 3]};
        else P::store4(a.dq + (row0 + i) * P::kRow, d, x[4 * r], x[4 * r + 1], x[4 * r + 2], x[4 * r + 3]);
      }
  }
  unsigned long long again = __ballot(bad && i < a.seen.n_q);
  again = (again | again >> 32) & 0xffffffffull;
  while (again != 0) {
    const int row = w0 + __builtin_ctzll(again);
    again &= again - 1;
    const float* const st = a.stats + int64_t(h) * 2 * a.stat_rows + row;
    const float x = exact_query<T>(a, qh + row * a.q.token, a.dout + (row0 + row) * P::kRow, kh, vh, st[0], st[a.stat_rows], row, t0, t1, tiles, lane);
    if (a.q_splits > 1) a.part_q[(int64_t(split) * a.heads * a.seen.n_q + row0 + row) * 64 + lane] = x;
    else P::store1(a.dq + (row0 + row) * P::kRow, lane, x);
  }
}

// A sequence of query tiles: those of each query head of the group in turn.
struct Sequence {
  int first, per_head, begin, end;  // first tile of a head, tiles of a head; this workgroup's part
};

// The gradients of one key again, by a wave on its own, over the queries that see it: as exact_query.  dk and dv of number `lane`.
template <typename T>
__device__ void exact_key(const BwdArgs& a, const unsigned char* k, const unsigned char* v, int j, int h0, const Sequence& seq, float& dk, float& dv,
                          int lane) {
  const Queries see = queries_of(a.seen, j);
  dk = dv = 0.f;
  for (int s = seq.begin; s < seq.end; ++s) {
    const int h = h0 + s / seq.per_head, i0 = (seq.first + s % seq.per_head) * kTile;
    const int64_t row0 = int64_t(h) * a.seen.n_q;
    const unsigned char* const qh = a.q.p + h * a.q.head;
    const int i = i0 + lane;
    const bool sees = i >= see.first && i < see.last;
    float p = 0.f, ds = 0.f;
    if (sees) {
      const float* const st = a.stats + int64_t(h) * 2 * a.stat_rows + i;
      p = exp2f((dot_rows<T>(qh + i * a.q.token, k) + st[0]) * a.scale_log2);
      ds = p * (dot_rows<T>(a.dout + (row0 + i) * Ops<T>::kRow, v) + st[a.stat_rows]);
    }
    unsigned long long all = __ballot(sees);
    while (all != 0) {
      const int e = __builtin_ctzll(all);
      all &= all - 1;
      dv += __shfl(p, e) * Ops<T>::number(a.dout + (row0 + i0 + e) * Ops<T>::kRow, lane);
      dk += __shfl(ds, e) * Ops<T>::number(qh + (i0 + e) * a.q.token, lane);
    }
  }
  dk *= a.scale;
}

// dK and dV of 32 keys for each of four waves.  smem: Q, dO and what S and dP begin with, of each buffer.
template <typename T>
__device__ __forceinline__ void key_rows(const BwdArgs& a, int64_t block, int64_t blocks, unsigned char* smem) {
  typedef Ops<T> P;
  constexpr int WAVES = 4, kBuffers = Buffers<T>;
  constexpr int kTileBytes = kTile * P::kRow, kBuf = 2 * kTileBytes + kStatBytes;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 31, g = lane >> 5;
  // the first tokens' units come first: they are the longest
  const int64_t sink_units = int64_t(a.kv_heads) * a.sink_tiles * a.sink_splits;
  const bool sink = block < sink_units;
  const int64_t unit = sink ? block : spread(block - sink_units, blocks - sink_units, a.kv_heads);
  const int splits = sink ? a.sink_splits : a.splits, of_head = sink ? a.sink_tiles : a.key_tiles - a.sink_tiles;
  const int split = static_cast<int>(unit % splits);
  const int hk = static_cast<int>(unit / splits / of_head);
  const int kt = static_cast<int>(unit / splits % of_head) + (sink ? 0 : a.sink_tiles);
  const int j0 = kt * kOwnRows, j1 = min(j0 + kOwnRows, a.seen.n_k);
  Sequence seq;
  {
    const Queries from = queries_of(a.seen, j0), to = queries_of(a.seen, j1 - 1);
    const int last = j0 < a.seen.sinks ? a.seen.n_q : to.last;
    seq.first = from.first / kTile;
    seq.per_head = last > from.first ? (last + kTile - 1) / kTile - seq.first : 0;
    const int64_t all = int64_t(seq.per_head) * a.group;
    seq.begin = static_cast<int>(all * split / splits);
    seq.end = static_cast<int>(all * (split + 1) / splits);
  }
  const int h0 = hk * a.group;
  const unsigned lds = lds_address(smem);
  const TileLoad<T, WAVES> q_load(a.q.token, wave, lane), d_load(P::kRow, wave, lane);
  auto place = [&](int s) { return static_cast<unsigned>(scalar((s - seq.begin) % kBuffers)) * kBuf; };
  auto row_of = [&](int s) { return (seq.first + s % seq.per_head) * kTile; };
  const unsigned stat_offset = lane < 16 ? lane * 16u : lane < 32 ? a.stat_rows * 4u + (lane - 16) * 16u : 1u << 30;
  auto stat_rsrc = [&](int h) { return make_rsrc(a.stats + int64_t(h) * 2 * a.stat_rows, a.stat_rows * 8u); };
  // (every wave, so that all wait for the same number of loads: the same bytes to the same place, 256 of each kind)
  auto load_stats = [&](i32x4 rsrc, int i0, unsigned to) { dma16<0>(rsrc, stat_offset, i0 * 4u, __builtin_amdgcn_readfirstlane(to + 2 * kTileBytes)); };
  auto issue = [&](int s) {
    const int h = h0 + s / seq.per_head, i0 = row_of(s);
    const unsigned to = lds + place(s);
    q_load.all(a.q.p + h * a.q.head, a.seen.n_q, i0, to);
    d_load.all(a.dout + int64_t(h) * a.seen.n_q * P::kRow, a.seen.n_q, i0, to + kTileBytes);
    load_stats(stat_rsrc(h), i0, to);
  };
  if (seq.begin < seq.end) issue(seq.begin);
  if (seq.begin + 1 < seq.end) issue(seq.begin + 1);

  // the wave's keys [w0, w1): rows past the end are computed as the last one and not stored
  const int w0 = j0 + wave * 32, w1 = min(w0 + 32, a.seen.n_k);
  const bool none = w0 >= a.seen.n_k;
  const int j = min(w0 + n, a.seen.n_k - 1);
  const unsigned char* const kh = a.k.p + hk * a.k.head;
  const unsigned char* const vh = a.v.p + hk * a.v.head;
  typename P::A kf[P::kSteps], vf[P::kSteps];
  P::row(kh + j * a.k.token, g, kf);
  P::row(vh + j * a.v.token, g, vf);
  const Queries see = queries_of(a.seen, j);
  Queries head = {0, 0}, tail = {0, 0};
  if (!none) {
    head = queries_of(a.seen, w0);
    tail = queries_of(a.seen, w1 - 1);
  }
  // queries of which all, and of which some, see all or some of the wave's keys
  const int some_last = w0 < a.seen.sinks ? a.seen.n_q : tail.last;
  const int all_last = none ? 0 : w1 <= a.seen.sinks ? a.seen.n_q : queries_of(a.seen, max(w0, a.seen.sinks)).last;

  f32x16 dk[2], dv[2];  // [dimensions], keys in the columns
#pragma unroll
  for (int db = 0; db < 2; ++db) {
    clear(dk[db]);
    clear(dv[db]);
  }
  auto seen_by_all = [&](int i0) { return i0 >= tail.first && i0 + kTile <= all_last; };
  auto plain = [&](int s) {
    const int lane = fresh_lane(), n = lane & 31, g = lane >> 5;  // (addresses are not kept in registers between tiles)
    const int i0 = row_of(s);
    const bool all = seen_by_all(i0);
    const unsigned char* const qt = smem + place(s);
    const unsigned char* const dt = qt + kTileBytes;
    const unsigned char* const st = dt + kTileBytes;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if (i0 + 32 * u >= some_last || i0 + 32 * u + 32 <= head.first) continue;  // no key of the wave is seen by these
      f32x16 p, ds;
      clear(p);
      clear(ds);
      auto begin = [&]() {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const f32x4 x = *LDS_PTR(f32x4, st + (32 * u + 8 * r + 4 * g) * 4), y = *LDS_PTR(f32x4, st + 256 + (32 * u + 8 * r + 4 * g) * 4);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            p[4 * r + e] += x[e];
            ds[4 * r + e] += y[e];
          }
        }
      };
      if constexpr (kFromStats<T>) begin();
      {
        typename P::A qa[P::kSteps], da[P::kSteps];
        P::rows(qt, 32 * u + n, g, qa);
        P::rows(dt, 32 * u + n, g, da);
#pragma unroll
        for (int c = 0; c < P::kSteps; ++c) {
          p = P::product(qa[c], kf[c], p);
          ds = P::product(da[c], vf[c], ds);
        }
      }
      if constexpr (!kFromStats<T>) begin();
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        p[e] = __builtin_amdgcn_exp2f(p[e] * a.scale_log2);
        ds[e] *= p[e];
      }
      if (!all) {
        keep(p, i0 + 32 * u + 4 * g, see.first, see.last, 0.f);
        keep(ds, i0 + 32 * u + 4 * g, see.first, see.last, 0.f);
      }
      typename P::A pw[P::kCols], dw[P::kCols];
      P::round(p, pw);
      P::round(ds, dw);
#pragma unroll
      for (int db = 0; db < 2; ++db) {
        typename P::A c0[P::kCols], c1[P::kCols];
        P::columns(dt, 32 * u, db, lane, c0);
        P::columns(qt, 32 * u, db, lane, c1);
#pragma unroll
        for (int c = 0; c < P::kCols; ++c) {
          dv[db] = P::product(c0[c], pw[c], dv[db]);
          dk[db] = P::product(c1[c], dw[c], dk[db]);
        }
      }
    }
  };
  stream<T>(seq.begin, seq.end, 2 * TileLoad<T, WAVES>::kLoads + 1, issue, [&](int s) {
    const int i0 = row_of(s);
    if (!none && i0 < some_last && i0 + kTile > head.first) plain(s);
  }, [&](int s, auto&& land) {
    if constexpr (sizeof(T) == 2) {
      if (none || !seen_by_all(row_of(s))) return s;
      // as above: the first queries of three tiles, and of the last of them its number in its head and its place
      int i0 = row_of(s), i1 = row_of(s + 1), i2 = row_of(s + 2), of_head = (s + 2) % seq.per_head;
      const int h = min(h0 + (s + 2) / seq.per_head, a.heads - 1);
      const unsigned char* qp = a.q.p + h * a.q.head + i2 * a.q.token;
      const unsigned char* dp = a.dout + (int64_t(h) * a.seen.n_q + i2) * P::kRow;
      const float* sp = a.stats + int64_t(h) * 2 * a.stat_rows;
      const int64_t q_step = kTile * a.q.token;
      const int64_t q_turn = a.q.head - (seq.per_head - 1) * q_step;  // from the last tile of a head to the first of the next
      const int64_t d_turn = (int64_t(a.seen.n_q) - (seq.per_head - 1) * kTile) * P::kRow;
      int heads_left = a.heads - 1 - h;  // past the last one: the last one again, loads that nobody reads
      unsigned to = lds + place(s + 2);
      i32x4 qrsrc, drsrc;
      const f32x16 unused = {};
      s = run<8>(s, place(s), smem, a.scale_log2, kf, vf, unused, unused, dv, dk, [&](int x) { return x < seq.end && seen_by_all(i0); },
                 [&]() {
                   land();
                   qrsrc = q_load.rsrc_at(qp, a.seen.n_q - i2);
                   drsrc = d_load.rsrc_at(dp, a.seen.n_q - i2);
                 },
                 [&](auto i) {
                   constexpr int I = decltype(i)::value;
                   if constexpr (I < 2) {
                     q_load.one(qrsrc, i, to);
                   } else if constexpr (I < 4) {
                     d_load.one(drsrc, Int<I - 2>{}, to + kTileBytes);
                   } else {
                     load_stats(make_rsrc(sp, a.stat_rows * 8u), i2, to);
                     to = to + kBuf == lds + kBuffers * kBuf ? lds : to + kBuf;
                     i0 = i1;
                     i1 = i2;
                     if (++of_head == seq.per_head) {
                       of_head = 0;
                       i2 = seq.first * kTile;
                       qp += heads_left > 0 ? q_turn : q_turn - a.q.head;
                       dp += heads_left > 0 ? d_turn : d_turn - int64_t(a.seen.n_q) * P::kRow;
                       sp += heads_left > 0 ? 2 * a.stat_rows : 0;
                       --heads_left;
                     } else {
                       i2 += kTile;
                       qp += q_step;
                       dp += kTile * P::kRow;
                     }
                   }
                 });
    }
    return s;
  });

  if (none) return;  // (no barrier follows)
  bool bad = false;
#pragma unroll
  for (int db = 0; db < 2; ++db)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      dk[db][e] *= a.scale;
      bad = bad || !(fabsf(dk[db][e]) < INFINITY) || !(fabsf(dv[db][e]) < INFINITY);
    }
  const int sink_rows = min(a.sink_tiles * kOwnRows, a.seen.n_k);
  const int64_t out0 = int64_t(hk) * a.seen.n_k;
  // the place of key jj in the partial sums
  auto part = [&](int jj) {
    const int64_t rows = sink ? sink_rows : a.seen.n_k - sink_rows;
    return a.part_kv[sink ? 0 : 1] + ((int64_t(split) * a.kv_heads + hk) * rows + jj - (sink ? 0 : sink_rows)) * 128;
  };
  if (w0 + n < a.seen.n_k) {
#pragma unroll
    for (int db = 0; db < 2; ++db)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int d = db * 32 + 8 * r + 4 * g;
        const f32x16 &x = dk[db], &y = dv[db];
        if (splits > 1) {
          float* const to = part(j);
          *reinterpret_cast<f32x4*>(to + d) = f32x4{x[4 * r], x[4 * r + 1], x[4 * r + 2], x[4 * r + 3]};
          *reinterpret_cast<f32x4*>(to + 64 + d) = f32x4{y[4 * r], y[4 * r + 1], y[4 * r + 2], y[4 * r + 3]};
        } else {
          P::store4(a.dk + (out0 + j) * P::kRow, d, x[4 * r], x[4 * r + 1], x[4 * r + 2], x[4 * r + 3]);
          P::store4(a.dv + (out0 + j) * P::kRow, d, y[4 * r], y[4 * r + 1], y[4 * r + 2], y[4 * r + 3]);
        }
      }
  }
  unsigned long long again = __ballot(bad && w0 + n < a.seen.n_k);
  again = (again | again >> 32) & 0xffffffffull;
  while (again != 0) {
    const int jj = w0 + __builtin_ctzll(again);
    again &= again - 1;
    float x, y;
    exact_key<T>(a, kh + jj * a.k.token, vh + jj * a.v.token, jj, h0, seq, x, y, lane);
    if (splits > 1) {
      part(jj)[lane] = x;
      part(jj)[64 + lane] = y;
    } else {
      P::store1(a.dk + (out0 + jj) * P::kRow, lane, x);
      P::store1(a.dv + (out0 + jj) * P::kRow, lane, y);
    }
  }
}

// Queries [first, end) that see at most 256 keys, all from key 0 on: the first ones of a sequence.
__host__ __device__ inline void early_queries(const Seen& s, int& first, int& end) {
  const int64_t positions = smaller(int64_t(kEarlyKeys / s.frame), int64_t(s.window)) * s.frame;
  first = static_cast<int>(smaller(larger(-int64_t(s.q_start), int64_t(0)), int64_t(s.n_q)));
  end = static_cast<int>(smaller(larger(positions - s.q_start, int64_t(first)), int64_t(s.n_q)));
}

// D of one of these queries by a wave, as sum_j P_j <dO, V_j>: the rounding of O to bf16 in the sum of dO O is seen in dQ where few keys share the
// weight (20,011 tokens, window of 4096: largest error of dQ 0.10 of its root mean square without this, 0.05 as it is).
// Eight lanes take a key, so that a load takes whole rows: with a lane to a key, and these queries last, the kernel below takes 68 us for
// 20,011 tokens of 16 heads instead of 30.
template <typename T>
struct alignas(16) Eight {
  unsigned char bytes[8 * sizeof(T)];
  __device__ __forceinline__ Eight(const unsigned char* row, int lane) { *this = reinterpret_cast<const Eight*>(row)[lane & 7]; }
  __device__ __forceinline__ float dot(const Eight& y) const {  // of the eight lanes' rows
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += Ops<T>::number(bytes, e) * Ops<T>::number(y.bytes, e);
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) sum += __shfl_xor(sum, o);
    return sum;
  }
};

template <typename T>
__device__ void early_query(const BwdArgs& a, int h, int i, int lane) {
  int lo, hi;
  a.seen.range(i, lo, hi);
  const int64_t row = int64_t(h) * a.seen.n_q + i;
  const Eight<T> q(a.q.p + h * a.q.head + i * a.q.token, lane), d(a.dout + row * Ops<T>::kRow, lane);
  const unsigned char *k = a.k.p + h / a.group * a.k.head, *v = a.v.p + h / a.group * a.v.head;
  const float lse = a.lse[row] * kLog2e;
  float sum = 0.f;
#pragma unroll 4
  for (int j = lane >> 3; j < hi; j += 8)
    sum += exp2f(q.dot(Eight<T>(k + j * a.k.token, lane)) * a.scale_log2 - lse) * d.dot(Eight<T>(v + j * a.v.token, lane));
  for (int o = 8; o < 64; o <<= 1) sum += __shfl_xor(sum, o);
  if (lane == 0) a.stats[int64_t(h) * 2 * a.stat_rows + a.stat_rows + i] = -sum;
}

// Eight lanes to a query: what its products' sums begin with.  A query that sees nothing has lse -inf, and -inf here: weights of zero.
// The grid's second dimension are heads; the first blocks of one take its early queries, which are chains of loads and overlap with what follows.
template <typename T>
__global__ __launch_bounds__(256) void window_stats_kernel(const BwdArgs a, unsigned early_blocks) {
  int first, end;
  early_queries(a.seen, first, end);
  if (sizeof(T) != 2) end = first;
  const int h = blockIdx.y;
  if (blockIdx.x < early_blocks) {
    const int i = first + static_cast<int>(blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (i < end) early_query<T>(a, h, i, threadIdx.x & 63);
    return;
  }
  const int i = static_cast<int>(blockIdx.x - early_blocks) * 32 + (threadIdx.x >> 3);
  if (i >= a.seen.n_q) return;
  const int64_t row = int64_t(h) * a.seen.n_q + i;
  const float sum = Eight<T>(a.out + row * Ops<T>::kRow, threadIdx.x).dot(Eight<T>(a.dout + row * Ops<T>::kRow, threadIdx.x));
  if ((threadIdx.x & 7) != 0) return;
  float* const st = a.stats + int64_t(h) * 2 * a.stat_rows + i;
  st[0] = a.lse[row] == -INFINITY ? -INFINITY : -a.lse[row] / a.scale;
  if (i < first || i >= end) st[a.stat_rows] = -sum;
}

template <typename T>
__global__ __launch_bounds__(256, 2) void window_bwd_kernel(const BwdArgs a, int64_t key_blocks) {
  extern __shared__ __align__(16) unsigned char smem[];
  if (blockIdx.x < key_blocks) key_rows<T>(a, blockIdx.x, key_blocks, smem);
  else query_rows<T>(a, blockIdx.x - key_blocks, gridDim.x - key_blocks, smem);
}

// Sums of the splits: WIDTH numbers of each row, the second 64 to a tensor of their own.  Row r of head h goes to row first + r of it.
template <typename T, int WIDTH>
__global__ __launch_bounds__(256) void window_sum_kernel(const float* __restrict__ part, int64_t rows_of_head, int heads, int splits, int64_t first,
                                                         int64_t out_rows, unsigned char* __restrict__ out0, unsigned char* __restrict__ out1) {
  constexpr int kLanes = WIDTH / 4;
  const int64_t rows = rows_of_head * heads;
  const int64_t row = (int64_t(blockIdx.x) * 256 + threadIdx.x) / kLanes;
  const int d = threadIdx.x % kLanes * 4;
  if (row >= rows) return;
  f32x4 y = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < splits; ++s) {
    const f32x4 x = *reinterpret_cast<const f32x4*>(part + (s * rows + row) * WIDTH + d);
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] += x[e];
  }
  const int64_t to = row / rows_of_head * out_rows + first + row % rows_of_head;
  Ops<T>::store4((d < 64 ? out0 : out1) + to * Ops<T>::kRow, d & 63, y[0], y[1], y[2], y[3]);
}

// How a launch is cut up.  A workgroup's rows go over at most so many tiles; longer ways are dealt out to several, whose sums are added up by one more
// kernel for each kind (query rows, first tokens, other keys).  What that costs, as fitted to 20,011 tokens (bf16) and two frames (fp32): a CU takes 0.85
// (9.5) us a tile of key rows and 0.63 (7) of query rows, a workgroup alone on its CU 1.4 times that; beside the whole work's share of a CU half of the
// longest way of query rows counts, which end last, and a tenth of key rows'; parts are written and read at 4 TB/s, a sum is 3 us, a round of workgroups begins for 1.5.  Two frames in fp32, all
// ways whole 943 us, queries in 2 parts 854, both in 3 835; forward and backward of 565 fp32 tokens of 16 heads, ways of 4 tiles 150, of 1 98.
void shape_of(BwdArgs& a, bool bf16) {
  const Seen& s = a.seen;
  a.stat_rows = static_cast<int>(ceil_div(s.n_q, kTile)) * kTile;
  a.row_tiles = static_cast<int>(ceil_div(s.n_q, kOwnRows));
  a.key_tiles = static_cast<int>(ceil_div(s.n_k, kOwnRows));
  a.sink_tiles = static_cast<int>(ceil_div(s.sinks, kOwnRows));
  a.q_splits = a.splits = a.sink_splits = 1;
  // tiles of the longest way of each kind, and of all
  int64_t q_most = 0, q_all = 0, k_most = 0, k_all = 0;
  for (int rt = 0; rt < a.row_tiles; ++rt) {
    const int64_t c = tiles_of(s, rt * kOwnRows, smaller((rt + 1) * kOwnRows, s.n_q)).count;
    q_most = larger(q_most, c);
    q_all += c;
  }
  for (int kt = a.sink_tiles; kt < a.key_tiles; ++kt) {
    const Queries from = queries_of(s, kt * kOwnRows), to = queries_of(s, smaller((kt + 1) * kOwnRows, s.n_k) - 1);
    if (to.last <= from.first) continue;
    const int64_t c = (ceil_div(to.last, kTile) - from.first / kTile) * a.group;
    k_most = larger(k_most, c);
    k_all += c;
  }
  const int64_t sink_most = a.sink_tiles > 0 ? ceil_div(s.n_q, kTile) * a.group : 0;
  const double k_tile = bf16 ? 0.85 : 9.5, q_tile = bf16 ? 0.63 : 7.0;
  const double share = (static_cast<double>(k_all + a.sink_tiles * sink_most) * a.kv_heads * k_tile + static_cast<double>(q_all) * a.heads * q_tile) / 256;
  const double q_rows = static_cast<double>(a.heads) * s.n_q, sink_rows = static_cast<double>(a.kv_heads) * smaller(a.sink_tiles * kOwnRows, s.n_k),
               k_rows = static_cast<double>(a.kv_heads) * s.n_k - sink_rows;
  auto sum_us = [](int64_t splits, double rows, int bytes) { return splits > 1 ? 3.0 + rows * static_cast<double>(splits) * bytes * 2 / 4e6 : 0.0; };
  const int64_t longest = larger(larger(q_most, k_most), sink_most);
  double least = -1.0;
  // ways of 1, 2, 3, 4, 6, 8, 12, ... tiles
  for (int64_t kp = 1;; kp += kp > 1 && (kp & (kp - 1)) == 0 ? kp / 2 : kp > 2 ? kp / 3 : 1) {
    const int64_t splits = larger(ceil_div(k_most, kp), int64_t(1)), sink_splits = larger(ceil_div(sink_most, kp), int64_t(1));
    for (int64_t qp = 1; splits <= 64 && sink_splits <= 256; qp += qp > 1 && (qp & (qp - 1)) == 0 ? qp / 2 : qp > 2 ? qp / 3 : 1) {
      const int64_t q_splits = larger(ceil_div(q_most, qp), int64_t(1));
      if (q_splits <= 64) {
        const double k_way = larger(ceil_div(k_most, splits), ceil_div(sink_most, sink_splits)) * k_tile, q_way = ceil_div(q_most, q_splits) * q_tile;
        const int64_t groups = a.kv_heads * (a.sink_tiles * sink_splits + (a.key_tiles - a.sink_tiles) * splits) + int64_t(a.heads) * a.row_tiles * q_splits;
        const double us = larger(larger(share, 1.4 * k_way), 1.4 * q_way) + 0.1 * k_way + 0.5 * q_way + 1.5 * static_cast<double>(ceil_div(groups, kPlaces)) + sum_us(splits, k_rows, 512) +
                          sum_us(sink_splits, sink_rows, 512) + sum_us(q_splits, q_rows, 256);
        if (least < 0.0 || us < least) {
          least = us;
          a.q_splits = static_cast<int>(q_splits);
          a.splits = static_cast<int>(splits);
          a.sink_splits = static_cast<int>(sink_splits);
        }
      }
      if (qp >= q_most) break;
    }
    if (kp >= longest) break;
  }
}

size_t stats_bytes(const BwdArgs& a) { return static_cast<size_t>(a.heads) * a.stat_rows * 8; }
size_t part_q_bytes(const BwdArgs& a) { return a.q_splits > 1 ? static_cast<size_t>(a.q_splits) * a.heads * a.seen.n_q * 256 : 0; }
size_t part_kv_bytes(const BwdArgs& a, bool sink) {
  const int64_t sink_rows = smaller(int64_t(a.sink_tiles) * kOwnRows, int64_t(a.seen.n_k));
  const int splits = sink ? a.sink_splits : a.splits;
  return splits > 1 ? static_cast<size_t>(splits) * a.kv_heads * (sink ? sink_rows : a.seen.n_k - sink_rows) * 512 : 0;
}

template <typename T>
int launch(const BwdArgs& a, hipStream_t s) {
  const char* what = "bsga_window_attn_bwd launch";
  const int64_t q_units = int64_t(a.heads) * a.row_tiles * a.q_splits;
  const int64_t k_units = int64_t(a.kv_heads) * (int64_t(a.sink_tiles) * a.sink_splits + int64_t(a.key_tiles - a.sink_tiles) * a.splits);
  if (q_units + k_units > 0x7fffffff) return fail(BSGA_ERR_UNSUPPORTED, "bsga_window_attn_bwd: too many rows");
  const int64_t q_rows = int64_t(a.heads) * a.seen.n_q;
  if (q_rows > 0) {
    int first, end;
    early_queries(a.seen, first, end);
    const unsigned early = sizeof(T) == 2 ? static_cast<unsigned>(ceil_div(end - first, 4)) : 0;
    hipLaunchKernelGGL(window_stats_kernel<T>, dim3(early + static_cast<unsigned>(ceil_div(a.seen.n_q, 32)), a.heads), dim3(256), 0, s, a, early);
    if (int rc = check_hip(hipGetLastError(), what)) return rc;
  }
  hipLaunchKernelGGL(window_bwd_kernel<T>, dim3(static_cast<unsigned>(q_units + k_units)), dim3(256), Buffers<T> * (2 * kTile * Ops<T>::kRow + kStatBytes), s, a,
                     k_units);
  if (int rc = check_hip(hipGetLastError(), what)) return rc;
  if (a.q_splits > 1) {
    hipLaunchKernelGGL((window_sum_kernel<T, 64>), dim3(static_cast<unsigned>(ceil_div(q_rows, 16))), dim3(256), 0, s, a.part_q, a.seen.n_q, a.heads,
                       a.q_splits, 0, a.seen.n_q, a.dq, nullptr);
    if (int rc = check_hip(hipGetLastError(), what)) return rc;
  }
  const int64_t sink_rows = smaller(int64_t(a.sink_tiles) * kOwnRows, int64_t(a.seen.n_k));
  for (int x = 0; x < 2; ++x) {
    const int splits = x == 0 ? a.sink_splits : a.splits;
    const int64_t rows = x == 0 ? sink_rows : a.seen.n_k - sink_rows;
    if (splits == 1 || rows == 0) continue;
    hipLaunchKernelGGL((window_sum_kernel<T, 128>), dim3(static_cast<unsigned>(ceil_div(rows * a.kv_heads, 8))), dim3(256), 0, s, a.part_kv[x], rows,
                       a.kv_heads, splits, x == 0 ? 0 : sink_rows, a.seen.n_k, a.dk, a.dv);
    if (int rc = check_hip(hipGetLastError(), what)) return rc;
  }
  return BSGA_OK;
}

}  // namespace
}  // namespace bsga

using namespace bsga;

extern "C" {

size_t bsga_window_attn_bwd_workspace_bytes(int dtype, int heads, int kv_heads, int64_t n_q, int64_t n_k, int64_t q_start, int64_t frame,
                                            int64_t window, int64_t sinks) {
  BwdArgs a = {};
  if ((dtype != BSGA_BF16 && dtype != BSGA_FP32) || heads < 1 || heads > 65535 || kv_heads < 1 || heads % kv_heads != 0 || n_q < 0 || n_k < 0) return 0;
  if (check_seen("", n_q, n_k, q_start, frame, window, sinks, a.seen)) return 0;
  a.heads = heads;
  a.kv_heads = kv_heads;
  a.group = heads / kv_heads;
  shape_of(a, dtype == BSGA_BF16);
  return stats_bytes(a) + part_q_bytes(a) + part_kv_bytes(a, true) + part_kv_bytes(a, false);
}

int bsga_window_attn_bwd(const void* dout, const void* q, const void* k, const void* v, int64_t q_token, int64_t q_head, int64_t k_token,
                         int64_t k_head, int64_t v_token, int64_t v_head, const void* out, const float* lse, int dtype, int heads, int kv_heads,
                         int64_t n_q, int64_t n_k, int head_dim, float softmax_scale, int64_t q_start, int64_t frame, int64_t window, int64_t sinks,
                         void* dq, void* dk, void* dv, void* workspace, size_t workspace_bytes, void* stream) {
  const char* fn = "bsga_window_attn_bwd";
  clear_error();
  BwdArgs a = {};
  if (dtype != BSGA_BF16 && dtype != BSGA_FP32) return fail(BSGA_ERR_INVALID_ARG, "%s: unknown dtype %d", fn, dtype);
  if (head_dim != 64) return fail(BSGA_ERR_UNSUPPORTED, "%s: head_dim must be 64, got %d", fn, head_dim);
  if (heads < 1 || heads > 65535 || kv_heads < 1 || heads % kv_heads != 0)
    return fail(BSGA_ERR_INVALID_ARG, "%s: heads must be in [1, 65535] and a multiple of kv_heads, got %d and %d", fn, heads, kv_heads);
  if (int rc = check_seen(fn, n_q, n_k, q_start, frame, window, sinks, a.seen)) return rc;
  // (-lse / scale is what a query's sums begin with: below about 5e-38 that of a logarithm alone would be infinite, and every weight zero)
  if (!(softmax_scale >= 0x1p-120f) || !isfinite(softmax_scale))
    return fail(BSGA_ERR_INVALID_ARG, "%s: softmax_scale must be finite and at least 2^-120", fn);
  if (n_q == 0 && n_k == 0) return BSGA_OK;
  const int size = dtype == BSGA_BF16 ? 2 : 4;
  if (n_q > 0) {
    if (int rc = check_view(fn, "q", q, q_token, q_head, size, a.q)) return rc;
    if (!dout || !out || !lse || !dq || !aligned16(dout) || !aligned16(out) || !aligned16(dq))
      return fail(BSGA_ERR_INVALID_ARG, "%s: dout, out, lse and dq must be non-null, tensors 16-byte aligned", fn);
  }
  if (n_k > 0) {
    if (int rc = check_view(fn, "k", k, k_token, k_head, size, a.k)) return rc;
    if (int rc = check_view(fn, "v", v, v_token, v_head, size, a.v)) return rc;
    if (!dk || !dv || !aligned16(dk) || !aligned16(dv))
      return fail(BSGA_ERR_INVALID_ARG, "%s: dk and dv must be non-null and 16-byte aligned", fn);
  }
  a.out = static_cast<const unsigned char*>(out);
  a.dout = static_cast<const unsigned char*>(dout);
  a.lse = lse;
  a.dq = static_cast<unsigned char*>(dq);
  a.dk = static_cast<unsigned char*>(dk);
  a.dv = static_cast<unsigned char*>(dv);
  a.heads = heads;
  a.kv_heads = kv_heads;
  a.group = heads / kv_heads;
  a.scale = softmax_scale;
  a.scale_log2 = softmax_scale * kLog2e;
  shape_of(a, dtype == BSGA_BF16);
  const size_t need = stats_bytes(a) + part_q_bytes(a) + part_kv_bytes(a, true) + part_kv_bytes(a, false);
  if (need > 0 && (!workspace || workspace_bytes < need))
    return fail(BSGA_ERR_WORKSPACE, "%s: workspace has %zu bytes, %zu needed", fn, workspace ? workspace_bytes : 0, need);
  if (!aligned16(workspace)) return fail(BSGA_ERR_INVALID_ARG, "%s: workspace must be 16-byte aligned", fn);
  unsigned char* at = static_cast<unsigned char*>(workspace);
  a.stats = reinterpret_cast<float*>(at);
  at += stats_bytes(a);
  a.part_q = reinterpret_cast<float*>(at);
  at += part_q_bytes(a);
  a.part_kv[0] = reinterpret_cast<float*>(at);
  at += part_kv_bytes(a, true);
  a.part_kv[1] = reinterpret_cast<float*>(at);
  hipStream_t s = static_cast<hipStream_t>(stream);
  return dtype == BSGA_BF16 ? launch<__bf16>(a, s) : launch<float>(a, s);
}

}  // extern "C"
