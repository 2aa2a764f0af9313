// Attention of one new token for each sequence, over pages, where sequences begin with tokens that they share: a prefix, which is read once for all of them.
//
// Sequence b of prefix g sees the P_g tokens of the prefix and then its own; its query stands at position P_g + lengths[b] - 1.  The queries of all sequences of a
// prefix that share a key head are the columns of the products over the prefix; the sequences' own keys go by a workgroup each.  Both leave, for each
// stretch of keys, sums and their logarithms, which a last kernel joins.
//
// A key and value are read once for a tile of queries of one key head, and by the tiles of a prefix one after the other from the same L2: 64 queries do 64 flop
// to the byte in bf16 and 126 in 8 bits, so few queries are bound by HBM and many by what the vector pipe does for a weight (an exponential, its share of a
// rounding, of a sum and of the conversions of the key and value) beside the two products, of which a wave does one piece's at a time. 64 sequences of 16 heads
// on 137,400 tokens, up to 2,000 of their own, bf16 (0.83 GB): 152 us, 5.5 TB/s; 128 of 16 heads to 4 on as many, up to 500 of their own, in 8 bits: 107 us,
// 670 TFLOP/s (exponentials alone 34 us); 60 on five prefixes of up to 82,440 with a window in frames: 57 us; 8 on 5,496: 13.5, of which the host's call is
// most.
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
  int queries, tiles, blocks;  // queries of a tile, tiles of all prefixes, workgroups for prefixes (own keys have those behind them)
  float scale_log2, ln2_scale;        // c = scale log2(e), 1 / c

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

// LDS of a workgroup; pieces: a wave's share follows the other's.
struct Shared {
  unsigned char* pieces;
  int* table;               // [kTable]
  float* sums;              // [kWaves][2][queries]
};

// The prefix of sequence b, or -1: whole waves.
__device__ __forceinline__ int prefix_of(const PrefixArgs& a, int b, int lane) {
  int g = 0;
  for (int i = 0; i < a.prefixes; i += 64) g += __popcll(__ballot(i + lane < a.prefixes && a.start(min(i + lane, a.prefixes - 1) + 1) <= b));
  return g < a.prefixes && a.start(g) <= b ? g : -1;
}

// What workgroup `block` of those for prefixes does: the prefix, or -1 if there is nothing left, and the key head, the stretch and the tile of its queries; whole waves.
// Workgroup w runs on XCD w % 8.  The tiles that read the same keys follow each other on one, and the first stretches, which more prefixes have, come first on
// all of them.  How many tiles there are is in `starts` alone, the host knows an upper bound: workgroups without one are the last.  (In between they took every other
// CU's place: 64 sequences of 16 heads on 100 frames had two workgroups on half of the CUs, 162 -> 151 us; the order of the stretches, five prefixes 60.6 -> 57.5.)
__device__ __forceinline__ int unit_of(const PrefixArgs& a, int block, int tile, int lane, int& hk, int& split, int& at) {
  auto tiles_of = [&](int g) {
    const int x = min(g, a.prefixes - 1);
    const int n = g < a.prefixes ? max(a.start(x + 1) - a.start(x), 0) : 0;
    return (n * a.group + tile - 1) / tile;
  };
  auto up_to = [&](int end) {  // the sum of the lanes up to this one
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) {
      const int other = __shfl_up(end, x);
      end += lane >= x ? other : 0;
    }
    return end;
  };
  int tiles = tiles_of(lane), end = up_to(tiles), total = __builtin_amdgcn_readlane(end, 63);
  for (int i = 64; i < a.prefixes; i += 64) total += __builtin_amdgcn_readlane(up_to(tiles_of(i + lane)), 63);
  if (total == 0) return -1;
  const int pair = block / 8 / total * 8 + block % 8, u = block / 8 % total;
  split = pair / a.pages.kv_heads, hk = pair % a.pages.kv_heads;
  if (split >= a.splits) return -1;
  int base = 0;
  for (int i = 0; i < a.prefixes; i += 64) {
    if (i > 0) tiles = tiles_of(i + lane), end = up_to(tiles);
    const unsigned long long behind = __ballot(base + end > u);
    if (behind != 0) {
      const int of = __builtin_ctzll(behind);
      at = u - base - __builtin_amdgcn_readlane(end - tiles, of);
      return i + of;
    }
    base += __builtin_amdgcn_readlane(end, 63);
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
__device__ __forceinline__ void over_prefix(const PrefixArgs& a, const Shared& lds, int block) {
  typedef Ops16<T, C> P;
  unsigned char* const smem = lds.pieces;
  int* const table = lds.table;
  float (&sums)[kWaves][2][kHeads] = *reinterpret_cast<float (*)[kWaves][2][kHeads]>(lds.sums);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, q = lane >> 4;
  int hk, split, tile;
  const int g = unit_of(a, block, kHeads, lane, hk, split, tile);
  if (g < 0) return;
  const int b0 = a.start(g), first = tile * kHeads, queries = min((a.start(g + 1) - b0) * a.group - first, kHeads);
  auto row_of = [&](int i, int& b) {  // query i of the tile: its sequence, and its row of the result
    const int x = first + i;
    b = b0 + x / a.group;
    return int64_t(b) * a.heads + hk * a.group + x % a.group;
  };
  Stretch st = {};
  st.x0 = split * a.stretch;
  if (a.window == 0) st.fill_ahead(a.pages, a.prefix_table + int64_t(g) * a.prefix_width, a.prefix_width, a.stretch, table);
  const int length = a.prefix_length(g);
  int b;
  const int64_t row = row_of(min(c, queries - 1), b);
  int lo, s;
  a.seen(length + a.length(b), lo, s);
  lo = min(lo, length);
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
  st.x1 = min(st.x0 + a.stretch, count);
  if (st.x0 >= st.x1) {  // the whole workgroup
    int of;
    if (threadIdx.x < queries) {
      const int64_t at = row_of(threadIdx.x, of);
      a.part_lse[int64_t(split) * a.batch * a.heads + at] = -INFINITY;
    }
    return;
  }
  if (a.window > 0) st.fill(a.pages, a.prefix_table + int64_t(g) * a.prefix_width, table);
  typename P::A qf[P::kSteps];
  P::row(a.q.p + b * a.q.token + (row - int64_t(b) * a.heads) * a.q.head, q, qf);
  have(qf);
  __syncthreads();
  f32x4 o[4];
  float m, l;
  unsigned char* const mine = smem + wave * kWaveLds<P>;
  if (most > st.lo)
    go_over<P, true, true>(a.pages, st, table, hk, wave, lane, mine, a.scale_log2, qf, [&](int j) { return j >= lo || j < a.sinks; }, o, m, l);
  else
    go_over<P, false, true>(a.pages, st, table, hk, wave, lane, mine, a.scale_log2, qf, [](int) { return true; }, o, m, l);
  f32x4 y;
  float top, sum;
  join_waves<P>(smem, sums, wave, lane, o, m, l, y, top, sum);
  const int i = threadIdx.x >> 4, d = (threadIdx.x & 15) * 4;
  if (i >= queries) return;
  leave(a, split, row_of(i, b), d, y, top, sum);
}

// Operands of 32x32x16 products, queries in bf16: S^T = K Q^T has keys as rows, O^T = V^T P^T numbers of the values.
template <typename C>
struct Wide;

template <>
struct Wide<__bf16> {
  typedef __bf16 Cache;
  static constexpr int kRow = 128, kKeys = 32;
  static constexpr bool kScaled = false;
  static __host__ __device__ constexpr int swizzle_k(int r) { return Ops<__bf16>::swizzle(r); }
  static __host__ __device__ constexpr int swizzle_v(int r) { return Ops<__bf16>::swizzle(r); }
  static __device__ __forceinline__ void query(const unsigned char* p, int g, bf16x8 (&a)[4]) { Ops<__bf16>::row(p, g, a); }
  static __device__ __forceinline__ void keys(const unsigned char* tile, float, int r0, int lane, bf16x8 (&a)[4]) {
    Ops<__bf16>::rows(tile, r0 + (lane & 31), lane >> 5, a);
  }
  typedef bf16x8 Raw;  // a value operand as it is read
  static __device__ __forceinline__ void values(const unsigned char* tile, int r0, int db, int lane, Raw (&a)[2]) { Ops<__bf16>::columns(tile, r0, db, lane, a); }
  static __device__ __forceinline__ bf16x8 operand(Raw x) { return x; }
  static __device__ __forceinline__ float number(const unsigned char* p, const unsigned char*, int64_t row, int d) {
    return Ops<__bf16>::number(p + row * kRow, d);
  }
};

// Rows of 64 bytes, four to the 64 banks: a lane half takes 32 numbers of a key, 8 for each of four steps, so the swizzle of keys keeps r, r + 4, r + 8, r + 12 apart;
// columns are read in two neighbouring chunks of the rows r and r + 8 together.
template <>
struct Wide<E4m3> {
  typedef E4m3 Cache;
  static constexpr int kRow = 64, kKeys = 64;
  static constexpr bool kScaled = true;
  static __host__ __device__ constexpr int swizzle_k(int r) { return (r >> 2) & 3; }
  static __host__ __device__ constexpr int swizzle_v(int r) { return (r >> 2) & 2; }
  static __device__ __forceinline__ void query(const unsigned char* p, int g, bf16x8 (&a)[4]) {
#pragma unroll
    for (int c = 0; c < 4; ++c) a[c] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(p + (4 * g + c) * 16));
  }
  static __device__ __forceinline__ void keys(const unsigned char* tile, float f, int r0, int lane, bf16x8 (&a)[4]) {  // f: scale of key r0 + lane % 32
    const int r = r0 + (lane & 31), g = lane >> 5;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const u32x4 x = *LDS_PTR(u32x4, tile + r * kRow + (((2 * g + i) ^ swizzle_k(r)) << 4));
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const u32x2 y0 = unpack_bf16(x[2 * e], f), y1 = unpack_bf16(x[2 * e + 1], f);
        a[2 * i + e] = __builtin_bit_cast(bf16x8, u32x4{y0[0], y0[1], y1[0], y1[1]});
      }
    }
  }
  typedef u32x2 Raw;
  static __device__ __forceinline__ bf16x8 operand(Raw x) {
    const u32x2 y0 = unpack_bf16(x[0], 1.f), y1 = unpack_bf16(x[1], 1.f);
    return __builtin_bit_cast(bf16x8, u32x4{y0[0], y0[1], y1[0], y1[1]});
  }
  static __device__ __forceinline__ void values(const unsigned char* tile, int r0, int db, int lane, Raw (&a)[2]) {
    const int m = (lane & 15) >> 1, G = lane >> 4;
#pragma unroll
    for (int cp = 0; cp < 2; ++cp) {
      const int r = r0 + 16 * cp + 4 * (G >> 1) + (m & 3) + 2 * (m & 4);
      const unsigned char* p = tile + r * kRow + (((2 * db + (G & 1)) ^ swizzle_v(r)) << 4) + (lane & 1) * 8;
      a[cp] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((s32x2 __attribute__((address_space(3)))*)(p)));
    }
  }
  static __device__ __forceinline__ float number(const unsigned char* p, const unsigned char* scale, int64_t row, int d) {
    return unpack_f32(p[row * kRow + d])[0] * scale_of(scale[row]);
  }
};

// Value scales that may be part of a weight, see over_prefix_wide.
constexpr unsigned kMostInWeight = 127 + 16;

// One query by a wave, over the keys of a stretch that it sees and no others: where values that are not finite have met weights of zero in the
// products, and where values' scales are too far apart.  For results that are right, not for speed.
template <typename C>
__device__ void one_query(const PrefixArgs& a, const Stretch& st, const int* table, int hk, int split, int64_t row, const unsigned char* q, int lo, int lane) {
  typedef Wide<C> P;
  float m = -INFINITY, l = 0.f, o = 0.f;
  for (int x0 = st.x0; x0 < st.x1; x0 += 64) {
    const int x = min(x0 + lane, st.x1 - 1), j = st.key(x);
    const bool sees = x0 + lane < st.x1 && (j >= lo || j < a.sinks);
    const int64_t at = st.row(a.pages, table, hk, x);
    float s = -INFINITY;
    if (sees) {
      s = 0.f;
      for (int d = 0; d < 64; ++d) s += Ops<__bf16>::number(q, d) * P::number(a.pages.k, a.pages.k_scale, at, d);
      s *= a.scale_log2;
    }
    float top = s;
    for (int e = 32; e > 0; e >>= 1) top = fmaxf(top, __shfl_xor(top, e));
    const float to = fmaxf(m, top), keep = m == -INFINITY ? 0.f : exp2f(m - to);
    const float w = sees ? exp2f(s - (to == -INFINITY ? 0.f : to)) : 0.f;  // (NaN stays)
    float sum = w;
    for (int e = 32; e > 0; e >>= 1) sum += __shfl_xor(sum, e);
    l = l * keep + sum;
    o *= keep;
    m = to;
    for (unsigned long long left = __ballot(sees); left != 0; left &= left - 1) {
      const int e = __builtin_ctzll(left);
      o += __shfl(w, e) * P::number(a.pages.v, a.pages.v_scale, __shfl(at, e), lane);
    }
  }
  const int64_t rows = int64_t(a.batch) * a.heads;
  a.part[(split * rows + row) * 64 + lane] = l == 0.f ? 0.f : o / l;
  if (lane == 0) a.part_lse[split * rows + row] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

template <typename C, int R>
constexpr int kWideLds = larger(2 * (2 * PieceLoad<Wide<C>>::kBytes + (Wide<C>::kScaled ? 512 : 0)), 32 * R * 64 * 4);

// The same for 32 R queries, bf16.  A wave has them all, as columns, and goes over its own pieces of the keys; what it holds of a piece serves R products.
template <typename C, int R>
__device__ __forceinline__ void over_prefix_wide(const PrefixArgs& a, const Shared& shared, int block) {
  typedef Wide<C> P;
  constexpr int kQueries = 32 * R, kBytes = PieceLoad<P>::kBytes, kBufBytes = 2 * kBytes + (P::kScaled ? 512 : 0);
  constexpr int kWaveBytes = kWideLds<C, R>;
  unsigned char* const smem = shared.pieces;
  int* const table = shared.table;
  float (&sums)[kWaves][2][kQueries] = *reinterpret_cast<float (*)[kWaves][2][kQueries]>(shared.sums);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 31, g = lane >> 5;
  int hk, split, tile;
  const int of = unit_of(a, block, kQueries, lane, hk, split, tile);
  if (of < 0) return;
  const int b0 = a.start(of), first = tile * kQueries, queries = min((a.start(of + 1) - b0) * a.group - first, kQueries);
  auto row_of = [&](int i, int& b) {  // query i of the tile: its sequence, and its row of the result
    const int x = first + i;
    b = b0 + x / a.group;
    return int64_t(b) * a.heads + hk * a.group + x % a.group;
  };
  Stretch st = {};
  st.x0 = split * a.stretch;
  if (a.window == 0) st.fill_ahead(a.pages, a.prefix_table + int64_t(of) * a.prefix_width, a.prefix_width, a.stretch, table);
  const int length = a.prefix_length(of);
  int lo[R], b[R];
  int64_t row[R];
  st.lo = length;
  int most = 0;
#pragma unroll
  for (int e = 0; e < R; ++e) {
    int s;
    row[e] = row_of(min(32 * e + n, queries - 1), b[e]);
    a.seen(length + a.length(b[e]), lo[e], s);
    lo[e] = min(lo[e], length);
    st.lo = min(st.lo, lo[e]);
    most = max(most, lo[e]);
  }
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    st.lo = min(st.lo, __shfl_xor(st.lo, o));
    most = max(most, __shfl_xor(most, o));
  }
  st.lo = scalar(st.lo);
  most = scalar(most);
  st.s = min(a.sinks, st.lo);
  const int count = st.s + length - st.lo;
  st.x1 = min(st.x0 + a.stretch, count);
  if (st.x0 >= st.x1) {  // the whole workgroup
    int to;
    if (threadIdx.x < queries) {
      const int64_t at = row_of(threadIdx.x, to);
      a.part_lse[int64_t(split) * a.batch * a.heads + at] = -INFINITY;
    }
    return;
  }
  if (a.window > 0) st.fill(a.pages, a.prefix_table + int64_t(of) * a.prefix_width, table);
  bf16x8 qf[R][4];
#pragma unroll
  for (int e = 0; e < R; ++e) P::query(a.q.p + b[e] * a.q.token + (row[e] - int64_t(b[e]) * a.heads) * a.q.head, g, qf[e]);
#pragma unroll
  for (int e = 0; e < R; ++e) have(qf[e]);
  __syncthreads();

  unsigned char* const mine = smem + wave * kWaveBytes;
  const unsigned lds = scalar(lds_address(mine));
  const int pieces = (st.x1 - st.x0 + P::kKeys - 1) / P::kKeys;
  const PieceLoad<P> load(lane);
  auto issue = [&](int p, int buf) { load.template issue<true>(a.pages, st, table, hk, st.x0 + p * P::kKeys, lds + buf * kBufBytes); };
  if (wave < pieces) issue(wave, 0);
  if (wave + kWaves < pieces) issue(wave + kWaves, 1);

  // Weights are 2^(c x - m).  The reference m is the largest logit of a column's first keys, and stays until the sum of its weights passes 2^24: then the
  // half piece is done again with an m that follows the largest logit and the sum.  That saves a maximum over every piece, a tenth of the vector instructions.
  // In 8 bits a value's scale 2^s is part of its weight, which costs nothing: products begin with s / c in place of zero, and the sum takes 2^-s of the weight.
  // A weight below 2^-126 is zero, in the sum as well, so this holds for s of -64 to 16 only: with L the logarithm of the sum, m is L + 17 at most, and a key is
  // lost if its logit is below L + 17 - 126 + 64 = L - 45: 2^30 of them are 2^-15 of the sum, less than a rounding to bf16.  And m is L - 70 at least (64 for the scales of
  // the first keys), so that a wave whose m lies 126 below another's has 2^-39 of the sum.  Stretches with values above 448 * 2^16 (or foreign bytes) go by one_query.
  f32x16 o[R][2];
  float m[R], minus[R], l[R];  // minus: what is added to logits, -m or, as long as nothing was seen, 0
#pragma unroll
  for (int e = 0; e < R; ++e) {
    m[e] = -INFINITY, minus[e] = 0.f, l[e] = 0.f;
    clear(o[e][0]);
    clear(o[e][1]);
  }
  int buf = 0;
  int bad = 0, first_half = 1;  // bad: whether a value that is not finite has met weights of zero
  unsigned apart = 0;           // the farthest value scale from the least that fits into weights
  for (int p = wave; p < pieces; p += kWaves, buf ^= 1) {
    load.wait(p + kWaves >= pieces);
    unsigned char* const kt = mine + buf * kBufBytes;
    unsigned char* const vt = kt + kBytes;
    unsigned* const extra = reinterpret_cast<unsigned*>(kt + 2 * kBytes);
    const int x = st.x0 + p * P::kKeys, left = st.x1 - x;
    if (left < P::kKeys) load.clear_from(kt, left);
    // key i of the piece is key x + i of the stretch, and no query sees less than keys `most` ..; those in front of it are looked at one by one
    const bool masked = (left < P::kKeys) | ((x + P::kKeys > st.s) & (st.key(max(x, st.s)) < most));
    if (masked & (most > st.lo)) bad |= load.bad_keys(kt) != 0;
    float k_scale = 1.f;
    if constexpr (P::kScaled) {  // a lane to a key: the exponents make room for what they stand for (as bits: stores of another type could pass the loads)
      const unsigned kb = extra[lane], vb = extra[64 + lane];
      apart = max(apart, vb - kLeastScale);
      k_scale = scale_of(kb);
      extra[lane] = __float_as_uint((static_cast<float>(vb) - 127.f) * a.ln2_scale);
      extra[64 + lane] = __float_as_uint(inverse_scale(vb));
    }
#pragma unroll 1
    for (int h = 0; h < P::kKeys / 32; ++h) {
      f32x16 w[R];
      auto products = [&]() {
        bf16x8 ka[4];
        P::keys(kt, P::kScaled ? __shfl(k_scale, 32 * h + n) : 1.f, 32 * h, lane, ka);
        f32x16 from;
        clear(from);
        if constexpr (P::kScaled)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const f32x4 y = *LDS_PTR(f32x4, extra + 32 * h + 8 * i + 4 * g);
#pragma unroll
            for (int r = 0; r < 4; ++r) from[4 * i + r] = y[r];
          }
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int e = 0; e < R; ++e) w[e] = Ops<__bf16>::product(ka[c], qf[e][c], c == 0 ? from : w[e]);
        if (masked) {
          int r0 = 32 * h + 4 * g;
          asm volatile("" : "+v"(r0));  // (most pieces are not: nothing of this is computed beforehand)
#pragma unroll
          for (int e = 0; e < R; ++e)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int r = r0 + 8 * (i >> 2) + (i & 3), j = st.key(x + r);
              w[e][i] = (r >= left) | ((j < lo[e]) & (j >= a.sinks)) ? -INFINITY : w[e][i];
            }
        }
      };
      float sum[R];
      auto weights = [&]() {
#pragma unroll
        for (int e = 0; e < R; ++e)
#pragma unroll
          for (int i = 0; i < 16; ++i) w[e][i] = __builtin_amdgcn_exp2f(fmaf(w[e][i], a.scale_log2, minus[e]));
#pragma unroll
        for (int e = 0; e < R; ++e) sum[e] = l[e];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          f32x4 y = {1.f, 1.f, 1.f, 1.f};
          if constexpr (P::kScaled) y = *LDS_PTR(f32x4, extra + 64 + 32 * h + 8 * i + 4 * g);
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int e = 0; e < R; ++e) sum[e] = P::kScaled ? fmaf(w[e][4 * i + r], y[r], sum[e]) : sum[e] + w[e][4 * i + r];
        }
      };
      products();
      typename P::Raw raw[2][2];
#pragma unroll
      for (int db = 0; db < 2; ++db) P::values(vt, 32 * h, db, lane, raw[db]);
      int again = first_half;
      if (!first_half) {
        weights();
#pragma unroll
        for (int e = 0; e < R; ++e) again |= !(sum[e] <= 0x1p24f) | (m[e] == -INFINITY);
      }
      if (__any(again)) {
        if (!first_half) products();
        first_half = 0;
#pragma unroll
        for (int e = 0; e < R; ++e) {
          float top = w[e][0];
#pragma unroll
          for (int i = 1; i < 16; ++i) top = fmaxf(top, w[e][i]);
          float to = fmaxf(m[e], top_of_halves(top) * a.scale_log2);
          const float grown = top_of_halves(l[e]);
          if (grown > 0x1p16f) to = fmaxf(to, m[e] + log2f(grown));
          const float keep = to == -INFINITY ? 1.f : exp2f(m[e] - to);
          m[e] = to;
          minus[e] = to == -INFINITY ? 0.f : -to;
          l[e] *= keep;
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            o[e][0][i] *= keep;
            o[e][1][i] *= keep;
          }
        }
        weights();
      }
      bf16x8 pw[R][2];
#pragma unroll
      for (int e = 0; e < R; ++e) {
        l[e] = sum[e];
        Ops<__bf16>::round(w[e], pw[e]);
      }
#pragma unroll
      for (int db = 0; db < 2; ++db) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const bf16x8 v = P::operand(raw[db][c]);
#pragma unroll
          for (int e = 0; e < R; ++e) o[e][db] = Ops<__bf16>::product(v, pw[e][c], o[e][db]);
        }
      }
    }
    if (p + 2 * kWaves < pieces) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the operands are in registers: the buffer is free
      issue(p + 2 * kWaves, buf);
    }
  }

  // the waves together: each leaves its sums in its own LDS (none of its loads are on their way any more)
#pragma unroll
  for (int e = 0; e < R; ++e) {
#pragma unroll
    for (int db = 0; db < 2; ++db)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<f32x4*>(mine + ((32 * e + n) * 64 + (((8 * db + 2 * i + g) ^ (n & 15)) * 4)) * 4) =
            f32x4{o[e][db][4 * i], o[e][db][4 * i + 1], o[e][db][4 * i + 2], o[e][db][4 * i + 3]};
    l[e] += __shfl_xor(l[e], 32);
    if (g == 0) {
      sums[wave][0][32 * e + n] = m[e];
      sums[wave][1][32 * e + n] = l[e];
    }
  }
  if (__syncthreads_or(bad | (apart > kMostInWeight - kLeastScale))) {
    for (int i = wave; i < queries; i += kWaves) {
      int to, low, s;
      const int64_t row = row_of(i, to);
      a.seen(length + a.length(to), low, s);
      one_query<C>(a, st, table, hk, split, row, a.q.p + to * a.q.token + (row - int64_t(to) * a.heads) * a.q.head, low, lane);
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < 2 * R; ++e) {
    const int i = 16 * e + (threadIdx.x >> 4), chunk = threadIdx.x & 15;
    float top = -INFINITY, sum = 0.f;
    bool nan = false;
#pragma unroll
    for (int x = 0; x < kWaves; ++x) {
      top = fmaxf(top, sums[x][0][i]);
      nan = nan || sums[x][1][i] != sums[x][1][i];
    }
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < kWaves; ++x) {
      const float weight = sums[x][0][i] == -INFINITY ? 0.f : exp2f(sums[x][0][i] - top);
      sum += sums[x][1][i] * weight;
      y += *reinterpret_cast<const f32x4*>(smem + x * kWaveBytes + (i * 64 + ((chunk ^ (i & 15)) * 4)) * 4) * weight;
    }
    if (nan) sum = NAN;
    int to;
    if (i < queries) leave(a, split, row_of(i, to), chunk * 4, y, top, sum);
  }
}

// The own keys of a sequence.
template <typename T, typename C>
__device__ __forceinline__ void over_own(const PrefixArgs& a, const Shared& lds, int block) {
  typedef Ops16<T, C> P;
  unsigned char* const smem = lds.pieces;
  int* const table = lds.table;
  float (&sums)[kWaves][2][kHeads] = *reinterpret_cast<float (*)[kWaves][2][kHeads]>(lds.sums);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, q = lane >> 4;
  const int split = block % a.own_splits, of = block / a.own_splits;
  const int hb = of % a.head_blocks, hk = of / a.head_blocks % a.pages.kv_heads, b = of / a.head_blocks / a.pages.kv_heads;
  const int heads = min(kHeads, a.group - hb * kHeads), h0 = hk * a.group + hb * kHeads;
  const int64_t rows = int64_t(a.batch) * a.heads, row0 = int64_t(b) * a.heads + h0;
  Stretch st = {};
  st.x0 = split * a.own_stretch;
  const int32_t* const own_pages = a.page_table + int64_t(b) * a.table_width;
  if (a.window == 0) st.fill_ahead(a.pages, own_pages, a.table_width, a.own_stretch, table);
  const int length = a.length(b);
  if (a.window > 0 || split == 0) {  // (where it is in the sequence matters to a window only)
    const int g = prefix_of(a, b, lane);
    if (g < 0 && split == 0 && threadIdx.x < heads)  // nobody else writes the prefix's parts of this sequence
      for (int x = 0; x < a.splits; ++x) a.part_lse[x * rows + row0 + threadIdx.x] = -INFINITY;
    if (a.window > 0) {
      const int behind = g < 0 ? 0 : a.prefix_length(g);
      a.seen(behind + length, st.lo, st.s);
      st.s = max(st.s - behind, 0);
      st.lo = min(max(st.lo - behind, 0), length);
    }
  }
  const int count = st.s + length - st.lo;
  st.x1 = min(st.x0 + a.own_stretch, count);
  if (st.x0 >= st.x1) {  // the whole workgroup
    if (threadIdx.x < heads) a.part_lse[(a.splits + split) * rows + row0 + threadIdx.x] = -INFINITY;
    return;
  }
  if (a.window > 0) st.fill(a.pages, own_pages, table);
  typename P::A qf[P::kSteps];
  P::row(a.q.p + b * a.q.token + (h0 + min(c, heads - 1)) * a.q.head, q, qf);
  have(qf);
  __syncthreads();
  f32x4 o[4];
  float m, l;
  go_over<P, false, true>(a.pages, st, table, hk, wave, lane, smem + wave * kWaveLds<P>, a.scale_log2, qf, [](int) { return true; }, o, m, l);
  f32x4 y;
  float top, sum;
  join_waves<P>(smem, sums, wave, lane, o, m, l, y, top, sum);
  const int head = threadIdx.x >> 4;
  if (head >= heads) return;
  leave(a, a.splits + split, row0 + head, (threadIdx.x & 15) * 4, y, top, sum);
}

template <typename T, typename C, int Q>
constexpr int lds_of_wave() {
  if constexpr (Q == kHeads) return kWaveLds<Ops16<T, C>>;
  else return larger(kWaveLds<Ops16<T, C>>, kWideLds<C, Q / 32>);
}

// Q: queries of a tile.
template <typename T, typename C, int Q>
__global__ __launch_bounds__(64 * kWaves, 2) void prefix_kernel(const PrefixArgs a) {
  __shared__ __align__(16) unsigned char pieces[kWaves * lds_of_wave<T, C, Q>()];
  __shared__ int table[kTable];
  __shared__ float sums[kWaves * 2 * Q];
  const Shared shared = {pieces, table, sums};
  const int block = blockIdx.x;
  if (block >= a.blocks) over_own<T, C>(a, shared, block - a.blocks);
  else if constexpr (Q == kHeads) over_prefix<T, C>(a, shared, block);
  else over_prefix_wide<C, Q / 32>(a, shared, block);
}

int keys_of_piece(int dtype, int cache_dtype) {
  return cache_dtype == BSGA_E4M3 ? Ops16E4m3::kKeys : dtype == BSGA_BF16 ? Ops16<__bf16, __bf16>::kKeys : Ops16<float, float>::kKeys;
}

// Tiles of the prefixes' queries, whichever sequences have which prefix: at most one that is not full for each.
int64_t tiles_of(const PrefixArgs& a, int tile) {
  const int64_t queries = int64_t(a.batch) * a.group;
  return smaller(queries / tile + smaller(int64_t(a.prefixes), int64_t(a.batch)), queries);
}

// Tiles of 32 and 64 queries take so long over a piece that a workgroup more than the chip holds is a round more, and what they leave for the join counts.  If one tile
// reads a key head's keys, one workgroup to a CU does, beside those of the own keys; otherwise all places are taken, unless that leaves less than 2,048 keys to each.
// 256 / 384 / 512 / 1024 workgroups, us: 64 sequences of 16 heads on 100 frames, 2,000 own tokens at most, 152 / 157 / 158 / 163, 8 of 16 heads to 2 24 / 27 / 27 / 33; with more
// tiles, 64 of 16 heads to 4, 84 / 81 / 70 / 82, 128 of them in 8 bits 144 / 136 / 116 / 121; 128 of 8 heads on 20, 40 and 60 frames 35 / 39 / 41, 52 / 55 / 57, 66 / 65 / 67.
// Returns the workgroups of the launch.
int64_t shape_of(PrefixArgs& a, int dtype, int cache_dtype) {
  const int keys = keys_of_piece(dtype, cache_dtype);
  const int64_t of_a_prefix = ceil_div(int64_t(a.batch) * a.group, larger(smaller(int64_t(a.prefixes), int64_t(a.batch)), int64_t(1)));  // about
  a.queries = dtype != BSGA_BF16 || of_a_prefix <= 16 ? kHeads : of_a_prefix <= 32 ? 32 : 64;
  int64_t most = int64_t(a.prefix_width) * a.pages.page, own = int64_t(a.table_width) * a.pages.page;
  if (a.window > 0) {
    const int64_t seen = int64_t(a.window) * a.frame + a.sinks;
    most = smaller(most, seen);
    own = smaller(own, seen);
  }
  const int64_t tiles = larger(ceil_div(int64_t(a.batch) * a.group, a.queries), smaller(int64_t(a.prefixes), int64_t(a.batch)));  // about
  const int64_t units = larger(tiles, int64_t(1)) * a.pages.kv_heads;
  const int64_t places = units == a.pages.kv_heads || most * units < 512 * 2048 ? 256 : 512;
  cut(most, units, keys, a.pages.page, a.stretch, a.splits, a.queries == kHeads ? 0 : places);
  cut(own, int64_t(a.batch) * a.pages.kv_heads * a.head_blocks, keys, a.pages.page, a.own_stretch, a.own_splits);
  a.tiles = a.prefixes > 0 ? static_cast<int>(tiles_of(a, a.queries)) : 0;
  const int64_t blocks = 8 * ceil_div(int64_t(a.pages.kv_heads) * a.splits, 8) * a.tiles;
  a.blocks = static_cast<int>(smaller(blocks, int64_t(INT32_MAX)));
  return blocks + int64_t(a.own_splits) * a.pages.kv_heads * a.head_blocks * a.batch;
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
int launch(const PrefixArgs& a, int64_t blocks, unsigned char* out, float* lse, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(blocks));
  if constexpr (std::is_same<T, __bf16>::value) {
    if (a.queries == 64) hipLaunchKernelGGL((prefix_kernel<T, C, 64>), grid, dim3(64 * kWaves), 0, s, a);
    else if (a.queries == 32) hipLaunchKernelGGL((prefix_kernel<T, C, 32>), grid, dim3(64 * kWaves), 0, s, a);
    else hipLaunchKernelGGL((prefix_kernel<T, C, kHeads>), grid, dim3(64 * kWaves), 0, s, a);
  } else {
    hipLaunchKernelGGL((prefix_kernel<T, C, kHeads>), grid, dim3(64 * kWaves), 0, s, a);
  }
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
  shape_of(a, dtype, cache_dtype);
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
  // (a value's exponent is divided by it, see over_prefix_wide)
  if (!(softmax_scale >= 0x1p-100f) || !isfinite(softmax_scale))
    return fail(BSGA_ERR_INVALID_ARG, "%s: softmax_scale must be finite and at least 2^-100", fn);
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
  a.ln2_scale = 1.f / a.scale_log2;
  const int64_t blocks = shape_of(a, dtype, cache_dtype);
  if (larger(blocks, workgroups_of_join(batch * heads, a.splits + a.own_splits)) >= (int64_t(1) << 32) / (64 * kWaves))  // (a grid has up to 2^32 - 1 threads)
    return fail(BSGA_ERR_UNSUPPORTED, "%s: too many keys of too many queries for one launch", fn);
  const size_t need = part_bytes(a);
  if (!workspace || workspace_bytes < need)
    return fail(BSGA_ERR_WORKSPACE, "%s: workspace has %zu bytes, %zu needed", fn, workspace ? workspace_bytes : 0, need);
  if (!aligned16(workspace)) return fail(BSGA_ERR_INVALID_ARG, "%s: workspace must be 16-byte aligned", fn);
  a.part = static_cast<float*>(workspace);
  a.part_lse = a.part + (int64_t(a.splits) + a.own_splits) * batch * heads * 64;
  unsigned char* const to = static_cast<unsigned char*>(out);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (dtype == BSGA_BF16) return cache_dtype == BSGA_E4M3 ? launch<__bf16, E4m3>(a, blocks, to, lse, s) : launch<__bf16, __bf16>(a, blocks, to, lse, s);
  return cache_dtype == BSGA_E4M3 ? launch<float, E4m3>(a, blocks, to, lse, s) : launch<float, float>(a, blocks, to, lse, s);
}

}  // extern "C"
