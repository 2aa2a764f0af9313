// What the kernels of attention over pages share: operands of 16x16 products for every type of queries and caches, where the keys of a sequence lie, and the
// loop in which a wave goes over its pieces of them.
//
// Query i of a workgroup is column i of S^T = K Q^T and O^T = V^T P^T, in which the weights are operands as they lie in the results.  A piece of keys and
// values goes from memory straight into the wave's own LDS, two pieces ahead; no wave waits for another.
#pragma once

#include "e4m3.h"
#include "window.h"

namespace bsga {
namespace {

constexpr int kTable = 2048;   // page numbers of a stretch
constexpr int kHeads = 16;     // queries of a workgroup
constexpr int kWaves = 4;

// T: type of the queries and results, C: of the cache.
template <typename T, typename C>
struct Ops16;

template <>
struct Ops16<__bf16, __bf16> {
  typedef bf16x8 A;
  typedef __bf16 Cache;
  static constexpr int kRow = 128;   // bytes of a key
  static constexpr bool kScaled = false;
  static constexpr int kKeys = 32;   // of a piece
  static constexpr int kBlocks = 2;  // of 16 keys
  static constexpr int kSteps = 2;   // products over the 64 numbers of a row
  static __device__ __forceinline__ f32x4 product(A a, A b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
  static __host__ __device__ constexpr int swizzle_k(int r) { return swz_k(r); }
  static __host__ __device__ constexpr int swizzle_v(int r) { return swz_v(r); }
  static __device__ __forceinline__ f32x4 value(const unsigned char* tile, const unsigned*, int r, int d) {  // numbers d .. d + 3 of a value, d a multiple of 4
    const u32x2 x = *LDS_PTR(u32x2, tile + r * kRow + (((d >> 3) ^ swizzle_v(r)) << 4) + (d & 4) * 2);
    return f32x4{__uint_as_float(x[0] << 16), __uint_as_float(x[0] & 0xffff0000u), __uint_as_float(x[1] << 16), __uint_as_float(x[1] & 0xffff0000u)};
  }
  static __device__ __forceinline__ void row(const unsigned char* p, int q, A (&a)[kSteps]) {
#pragma unroll
    for (int c = 0; c < 2; ++c) a[c] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(p + (4 * c + q) * 16));
  }
  static __device__ __forceinline__ void rows(const unsigned char* tile, const unsigned*, int r, int q, A (&a)[kSteps]) {
#pragma unroll
    for (int c = 0; c < 2; ++c) a[c] = *LDS_PTR(bf16x8, tile + r * 128 + (((4 * c + q) ^ swz_k(r)) << 4));
  }
  // a lane's values of a piece, as they are read
  struct Raw {
    bf16x8 a[4];
  };
  static __device__ __forceinline__ void fetch(const unsigned char* tile, const unsigned*, int lane, Raw& raw) {
    const int m = (lane & 15) >> 2, j = lane & 3, q = lane >> 4;
#pragma unroll
    for (int db = 0; db < 4; ++db) {
      u32x2 x[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = 16 * e + 4 * q + m;
        const unsigned char* p = tile + r * 128 + (((2 * db + (j >> 1)) ^ swz_v(r)) << 4) + (j & 1) * 8;
        x[e] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(p)));
      }
      raw.a[db] = __builtin_bit_cast(bf16x8, u32x4{x[0][0], x[0][1], x[1][0], x[1][1]});
    }
  }
  // o += V^T P^T: the weights' products in w[block][r], of keys 16 block + 4 q + r
  static __device__ __forceinline__ void update(const Raw& raw, const f32x4 (&w)[kBlocks], f32x4 (&o)[4]) {
    const bf16x8 b = __builtin_bit_cast(
        bf16x8, u32x4{pack_bf16(w[0][0], w[0][1]), pack_bf16(w[0][2], w[0][3]), pack_bf16(w[1][0], w[1][1]), pack_bf16(w[1][2], w[1][3])});
#pragma unroll
    for (int db = 0; db < 4; ++db) o[db] = product(raw.a[db], b, o[db]);
  }
};

template <>
struct Ops16<float, float> {
  typedef float A;
  typedef float Cache;
  static constexpr int kRow = 256;
  static constexpr bool kScaled = false;
  static constexpr int kKeys = 16;
  static constexpr int kBlocks = 1;
  static constexpr int kSteps = 16;
  static __device__ __forceinline__ f32x4 product(A a, A b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }
  static __host__ __device__ constexpr int swizzle_k(int r) { return r & 15; }
  static __host__ __device__ constexpr int swizzle_v(int r) { return r & 15; }
  static __device__ __forceinline__ f32x4 value(const unsigned char* tile, const unsigned*, int r, int d) {
    return *LDS_PTR(f32x4, tile + r * kRow + (((d >> 2) ^ swizzle_v(r)) << 4));
  }
  static __device__ __forceinline__ void row(const unsigned char* p, int q, A (&a)[kSteps]) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(p + (4 * c + q) * 16);
#pragma unroll
      for (int e = 0; e < 4; ++e) a[4 * c + e] = x[e];
    }
  }
  static __device__ __forceinline__ void rows(const unsigned char* tile, const unsigned*, int r, int q, A (&a)[kSteps]) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const f32x4 x = *LDS_PTR(f32x4, tile + r * 256 + (((4 * c + q) ^ swizzle_k(r)) << 4));
#pragma unroll
      for (int e = 0; e < 4; ++e) a[4 * c + e] = x[e];
    }
  }
  struct Raw {
    float a[4][4];
  };
  static __device__ __forceinline__ void fetch(const unsigned char* tile, const unsigned*, int lane, Raw& raw) {
    const int q = lane >> 4;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = 4 * q + e, d = 16 * db + (lane & 15);
        raw.a[db][e] = *LDS_PTR(float, tile + r * 256 + (((d >> 2) ^ swizzle_v(r)) << 4) + (d & 3) * 4);
      }
  }
  static __device__ __forceinline__ void update(const Raw& raw, const f32x4 (&w)[kBlocks], f32x4 (&o)[4]) {
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[db] = product(raw.a[db][e], w[0][e], o[db]);
  }
};

// Rows of 64 bytes.  A lane takes 16 numbers of a key at once, so that its products go over the numbers 16 q .. 16 q + 15 in two steps, or in sixteen; queries
// are laid out for that.  Keys are multiplied by their scale, which is exact; a value's scale goes to its weight, which is in 32 bits there.  Rows are four to
// the 64 banks: the swizzles keep apart the rows r, r + 4, r + 8, r + 12 that are read whole, and r, r + 4, r + 16, r + 20 that are read transposed.
struct Ops16E4m3 {
  typedef E4m3 Cache;
  static constexpr int kRow = 64;
  static constexpr bool kScaled = true;
  static constexpr int kKeys = 64;
  static constexpr int kBlocks = 4;
  static __host__ __device__ constexpr int swizzle_k(int r) { return (r >> 2) & 3; }
  static __host__ __device__ constexpr int swizzle_v(int r) { return ((r >> 2) & 1) | ((r >> 3) & 2); }
  static __device__ __forceinline__ f32x4 value(const unsigned char* tile, const unsigned* scales, int r, int d) {
    return unpack_f32(*LDS_PTR(unsigned, tile + r * kRow + (((d >> 4) ^ swizzle_v(r)) << 4) + (d & 12))) * scale_of(*LDS_PTR(unsigned, scales + r));
  }
  static __device__ __forceinline__ u32x4 codes(const unsigned char* tile, int r, int q) { return *LDS_PTR(u32x4, tile + r * kRow + ((q ^ swizzle_k(r)) << 4)); }
  // number 16 db + (lane & 15) of the keys 32 h + 4 q .. + 3 and 32 h + 16 + 4 q .. + 3
  static __device__ __forceinline__ u32x2 column(const unsigned char* tile, int lane, int h, int db) {
    const int m = (lane & 15) >> 1, q = lane >> 4;
    const int r = 32 * h + 4 * q + (m & 3) + 4 * (m & 4);
    const unsigned char* p = tile + r * kRow + ((db ^ swizzle_v(r)) << 4) + (lane & 1) * 8;
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((s32x2 __attribute__((address_space(3)))*)(p)));
  }
  struct Raw {
    u32x2 a[2][4];
    u32x4 scale[4];  // of the keys 16 block + 4 q + r
  };
  static __device__ __forceinline__ void fetch(const unsigned char* tile, const unsigned* scales, int lane, Raw& raw) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int db = 0; db < 4; ++db) raw.a[h][db] = column(tile, lane, h, db);
#pragma unroll
    for (int blk = 0; blk < 4; ++blk) raw.scale[blk] = *LDS_PTR(u32x4, scales + 16 * blk + 4 * (lane >> 4));
  }
  // weights times their values' scales
  static __device__ __forceinline__ f32x4 scaled(const u32x4& scale, const f32x4& w) {
    f32x4 y;
#pragma unroll
    for (int r = 0; r < 4; ++r) y[r] = w[r] * scale_of(scale[r]);
    return y;
  }
};

template <>
struct Ops16<__bf16, E4m3> : Ops16E4m3 {
  typedef bf16x8 A;
  static constexpr int kSteps = 2;
  static __device__ __forceinline__ f32x4 product(A a, A b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ void row(const unsigned char* p, int q, A (&a)[kSteps]) {
#pragma unroll
    for (int e = 0; e < 2; ++e) a[e] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(p + q * 32 + e * 16));
  }
  static __device__ __forceinline__ void rows(const unsigned char* tile, const unsigned* scales, int r, int q, A (&a)[kSteps]) {
    const u32x4 x = codes(tile, r, q);
    const float f = scale_of(*LDS_PTR(unsigned, scales + r));
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const u32x2 y0 = unpack_bf16(x[2 * e], f), y1 = unpack_bf16(x[2 * e + 1], f);
      a[e] = __builtin_bit_cast(bf16x8, u32x4{y0[0], y0[1], y1[0], y1[1]});
    }
  }
  static __device__ __forceinline__ void update(const Raw& raw, const f32x4 (&w)[kBlocks], f32x4 (&o)[4]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const f32x4 w0 = scaled(raw.scale[2 * h], w[2 * h]), w1 = scaled(raw.scale[2 * h + 1], w[2 * h + 1]);
      const bf16x8 b = __builtin_bit_cast(bf16x8, u32x4{pack_bf16(w0[0], w0[1]), pack_bf16(w0[2], w0[3]), pack_bf16(w1[0], w1[1]), pack_bf16(w1[2], w1[3])});
#pragma unroll
      for (int db = 0; db < 4; ++db) {
        const u32x2 x = raw.a[h][db];
        const u32x2 y0 = unpack_bf16(x[0], 1.f), y1 = unpack_bf16(x[1], 1.f);
        o[db] = product(__builtin_bit_cast(bf16x8, u32x4{y0[0], y0[1], y1[0], y1[1]}), b, o[db]);
      }
    }
  }
};

template <>
struct Ops16<float, E4m3> : Ops16E4m3 {
  typedef float A;
  static constexpr int kSteps = 16;
  static __device__ __forceinline__ f32x4 product(A a, A b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ void row(const unsigned char* p, int q, A (&a)[kSteps]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(p + q * 64 + e * 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) a[4 * e + i] = x[i];
    }
  }
  static __device__ __forceinline__ void rows(const unsigned char* tile, const unsigned* scales, int r, int q, A (&a)[kSteps]) {
    const u32x4 x = codes(tile, r, q);
    const float f = scale_of(*LDS_PTR(unsigned, scales + r));
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const f32x4 y = unpack_f32(x[e]);
#pragma unroll
      for (int i = 0; i < 4; ++i) a[4 * e + i] = y[i] * f;
    }
  }
  static __device__ __forceinline__ void update(const Raw& raw, const f32x4 (&w)[kBlocks], f32x4 (&o)[4]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const f32x4 w0 = scaled(raw.scale[2 * h], w[2 * h]), w1 = scaled(raw.scale[2 * h + 1], w[2 * h + 1]);
#pragma unroll
      for (int db = 0; db < 4; ++db) {
        const u32x2 x = raw.a[h][db];
        const f32x4 y0 = unpack_f32(x[0]), y1 = unpack_f32(x[1]);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[db] = product(y0[e], w0[e], o[db]);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[db] = product(y1[e], w1[e], o[db]);
      }
    }
  }
};

// Whether one of the 16 bytes' numbers is not finite.
template <typename C>
__device__ __forceinline__ bool any_bad(u32x4 x) {
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (std::is_same<C, float>::value) bad = bad || (x[i] & 0x7f800000u) == 0x7f800000u;
    else if constexpr (std::is_same<C, __bf16>::value) bad = bad || (x[i] & 0x7f80u) == 0x7f80u || (x[i] & 0x7f800000u) == 0x7f800000u;
    else
#pragma unroll
      for (int e = 0; e < 32; e += 8) bad = bad || ((x[i] >> e) & 0x7fu) == 0x7fu;
  }
  return bad;
}

// The pages of a cache.
struct Pages {
  const unsigned char *k, *v;          // [n_pages, kv_heads, page, 64]
  const unsigned char *k_scale, *v_scale;  // [n_pages, kv_heads, page] exponent bytes, of a cache in 8 bits
  int kv_heads, n_pages, page;
  unsigned magic;                      // j / page = umulhi(2 j, magic) >> shift, for j < 2^31
  int shift;
  __device__ __forceinline__ int of(int j) const { return static_cast<int>(__umulhi(static_cast<unsigned>(j) << 1, magic) >> shift); }
};

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

// The same from an address that all lanes share and a 32-bit offset for each.
__device__ __forceinline__ void dma16_from(const unsigned char* base, unsigned offset, unsigned lds) {
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %1, %2"
      :
      : "s"(lds), "v"(offset), "s"(base)
      : "memory", "m0");
}

__device__ __forceinline__ void dma_byte_from(const unsigned char* base, unsigned offset, unsigned lds) {
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 0\n\t"
      "global_load_lds_ubyte %1, %2"
      :
      : "s"(lds), "v"(offset), "s"(base)
      : "memory", "m0");
}

// A byte per lane, as 32 bits at lds + 4 * lane.
__device__ __forceinline__ void dma_byte_at(const unsigned char* p, unsigned lds) {
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 0\n\t"
      "global_load_lds_ubyte %1, off"
      :
      : "s"(lds), "v"(p)
      : "memory", "m0");
}

// Over the four lanes of a column, without the way through LDS.
template <bool MAXIMUM>
__device__ __forceinline__ float across(float x) {
  const unsigned u = __float_as_uint(x);
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  x = MAXIMUM ? fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1])) : __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const unsigned v = __float_as_uint(x);
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return MAXIMUM ? fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1])) : __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// The keys that a workgroup goes over: those that a sequence sees, numbered through (x < s is key x, the others lo + x - s), from x0 to x1.  Their page
// numbers lie in LDS, those of the first tokens before those of the window.
struct Stretch {
  int s, lo, x0, x1, a0, a_pages, b0;
  __device__ __forceinline__ int key(int x) const { return x < s ? x : lo + x - s; }
  // from x0 to x1, x0 < x1; all threads of the workgroup; a barrier has to follow
  __device__ __forceinline__ void fill(const Pages& a, const int32_t* pages, int* table) {
    a0 = a.of(x0), a_pages = x0 < min(x1, s) ? a.of(min(x1, s) - 1) - a0 + 1 : 0;
    b0 = a.of(lo + max(x0, s) - s);
    const int b_pages = max(x0, s) < x1 ? a.of(lo + x1 - 1 - s) - b0 + 1 : 0;
    for (int i = threadIdx.x; i < min(a_pages + b_pages, kTable); i += 64 * kWaves)
      table[i] = min(max(pages[i < a_pages ? a0 + i : b0 + i - a_pages], 0), a.n_pages - 1);  // a bad entry cannot read out of bounds
  }
  // The same without a window, where nothing of it goes by the sequence's length, which then is on its way at the same time; x0 is set, s and lo are 0.
  __device__ __forceinline__ void fill_ahead(const Pages& a, const int32_t* pages, int width, int stretch, int* table) {
    b0 = a.of(x0);
    for (int i = threadIdx.x; i < min(min(width - b0, (stretch + a.page - 2) / a.page + 1), kTable); i += 64 * kWaves)
      table[i] = min(max(pages[b0 + i], 0), a.n_pages - 1);
  }
  // the cache row, of head hk, of the x-th key
  __device__ __forceinline__ int64_t row(const Pages& a, const int* table, int hk, int x) const {
    const int j = key(x);
    const int page = a.of(j);
    const int at = table[min(x < s ? page - a0 : a_pages + page - b0, kTable - 1)];
    return (int64_t(at) * a.kv_heads + hk) * a.page + (j - page * a.page);
  }
};

// Pieces of keys and values on their way into a wave's LDS: kKeys keys, then as many values, then the exponents of both.  A piece that lies in one page has one address for
// all lanes, and its lanes' offsets are known beforehand: no vector instructions; others look their rows up lane by lane.
template <typename P>
struct PieceLoad {
  static constexpr int kChunks = P::kRow / 16, kRowsOfLoad = 64 / kChunks, kLoads = P::kKeys / kRowsOfLoad, kBytes = P::kKeys * P::kRow;
  static constexpr int kInFlight = 2 * kLoads + (P::kScaled ? 2 : 0);  // loads of a piece
  static_assert(kLoads == 4, "eight loads of keys and values");
  // loads whose lanes have the same places in them, 1024 bytes further: their swizzles are those of rows kRowsOfLoad * (1, 2 or 4) apart
  static constexpr int patterns(int (*swizzle)(int)) {
    for (int n = 1; n < kLoads; n *= 2) {
      bool same = true;
      for (int r = 0; r + n * kRowsOfLoad < P::kKeys; ++r) same = same && swizzle(r) == swizzle(r + n * kRowsOfLoad);
      if (same) return n;
    }
    return kLoads;
  }
  static constexpr int kPlacesK = patterns(P::swizzle_k), kPlacesV = patterns(P::swizzle_v);
  unsigned k[kPlacesK], v[kPlacesV];
  int lane, r_in, pos;

  __device__ __forceinline__ explicit PieceLoad(int lane) : lane(lane), r_in(lane / kChunks), pos(lane % kChunks) {
#pragma unroll
    for (int i = 0; i < kPlacesK; ++i) k[i] = r_in * P::kRow + ((pos ^ P::swizzle_k(i * kRowsOfLoad + r_in)) << 4);
#pragma unroll
    for (int i = 0; i < kPlacesV; ++i) v[i] = r_in * P::kRow + ((pos ^ P::swizzle_v(i * kRowsOfLoad + r_in)) << 4);
  }
  // the keys from the x-th on; FRESH: places are not kept in registers for the lanes' own ways
  template <bool FRESH = false>
  __device__ __forceinline__ void issue(const Pages& a, const Stretch& st, const int* table, int hk, int x, unsigned lds) const {
    x = scalar(x);
    const int j = st.key(x), page = a.of(j), inside = j - page * a.page;
    if (x + P::kKeys <= st.x1 && (x >= st.s || x + P::kKeys <= st.s) && inside + P::kKeys <= a.page) {
      const int at = scalar(table[min(x < st.s ? page - st.a0 : st.a_pages + page - st.b0, kTable - 1)]);
      const int64_t row = (int64_t(at) * a.kv_heads + hk) * a.page + inside;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        dma16_from(a.k + row * P::kRow + i * 1024, k[i % kPlacesK], lds + i * 1024);
        dma16_from(a.v + row * P::kRow + i * 1024, v[i % kPlacesV], lds + kBytes + i * 1024);
      }
      if constexpr (P::kScaled) {
        dma_byte_from(a.k_scale + row, lane, lds + 2 * kBytes);
        dma_byte_from(a.v_scale + row, lane, lds + 2 * kBytes + 256);
      }
      return;
    }
    const int l = FRESH ? fresh_lane() : lane, in = l / kChunks, chunk = l % kChunks;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int r = i * kRowsOfLoad + in;
      const int64_t row = st.row(a, table, hk, min(x + r, st.x1 - 1));  // rows past the end are the last one again, with no weight
      dma16_at(a.k + row * P::kRow + ((chunk ^ P::swizzle_k(r)) << 4), lds + i * 1024);
      dma16_at(a.v + row * P::kRow + ((chunk ^ P::swizzle_v(r)) << 4), lds + kBytes + i * 1024);
    }
    if constexpr (P::kScaled) {
      static_assert(P::kKeys == 64, "a lane to a key");
      const int64_t row = st.row(a, table, hk, min(x + l, st.x1 - 1));
      dma_byte_at(a.k_scale + row, lds + 2 * kBytes);
      dma_byte_at(a.v_scale + row, lds + 2 * kBytes + 256);
    }
  }
  // The keys of a piece in LDS whose values (or their exponents) are not finite.
  __device__ __forceinline__ unsigned long long bad_keys(const unsigned char* piece) const {
    unsigned long long in[kLoads], any = 0;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      in[i] = __ballot(any_bad<typename P::Cache>(*LDS_PTR(u32x4, piece + kBytes + i * 1024 + lane * 16)));
      any |= in[i];
    }
    bool bad = false;
    if (any != 0) {
      const int i = lane / kRowsOfLoad;
      const unsigned long long of = i == 0 ? in[0] : i == 1 ? in[1] : i == 2 ? in[2] : in[3];
      bad = lane < P::kKeys && ((of >> (lane % kRowsOfLoad * kChunks)) & ((1ull << kChunks) - 1)) != 0;
    }
    if constexpr (P::kScaled) bad = bad || LDS_PTR(unsigned, piece + 2 * kBytes)[64 + lane] == 255u;
    return __ballot(bad);
  }
  __device__ __forceinline__ void clear_keys(unsigned char* piece, unsigned long long keys) const {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int r = i * kRowsOfLoad + r_in;
      if ((keys >> r) & 1) *reinterpret_cast<u32x4*>(piece + kBytes + r * P::kRow + pos * 16) = u32x4{0u, 0u, 0u, 0u};
    }
    if constexpr (P::kScaled)
      if ((keys >> lane) & 1) reinterpret_cast<unsigned*>(piece + 2 * kBytes)[64 + lane] = 0u;
  }
  // until the piece that was asked for first is there, of two (or one, the last)
  static __device__ __forceinline__ void wait(bool last) {
    static_assert(kInFlight == 8 || kInFlight == 10, "counts below");
    if (last) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    else if constexpr (kInFlight == 10) asm volatile("s_waitcnt vmcnt(10)" ::: "memory");
    else asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
  }
  // values that only fill the last piece become zeros (of scale 1): their weights are zero, which is not nothing if the one that is repeated is infinite
  __device__ __forceinline__ void clear_from(unsigned char* piece, int left) const {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int r = i * kRowsOfLoad + r_in;
      if (r >= left) *reinterpret_cast<u32x4*>(piece + kBytes + r * P::kRow + pos * 16) = u32x4{0u, 0u, 0u, 0u};
    }
    if constexpr (P::kScaled)
      if (lane >= left) reinterpret_cast<unsigned*>(piece + 2 * kBytes)[64 + lane] = 127u;
  }
};

template <typename P>
constexpr int kPiece = P::kKeys * P::kRow;
template <typename P>
constexpr int kBuf = 2 * kPiece<P> + (P::kScaled ? 2 * P::kKeys * 4 : 0);  // keys, values, the exponents of both
template <typename P>
constexpr int kWaveLds = 2 * kBuf<P>;

// Values that are not finite must not reach columns that do not see them, where a weight of zero would still make NaN of them: such keys are added here, for
// the columns that see them, and are zeros for the matrix product.  Only pieces of which some columns see a part come here.
template <typename P, typename SeenI>
__device__ __forceinline__ void leave_bad_out(const PieceLoad<P>& load, unsigned char* piece, SeenI seen, const f32x4 (&w)[P::kBlocks], f32x4 (&o)[4]) {
  unsigned long long bad = load.bad_keys(piece);
  if (bad == 0) return;
  const int c = load.lane & 15, q = load.lane >> 4;
  const unsigned* const scales = reinterpret_cast<const unsigned*>(piece + 2 * PieceLoad<P>::kBytes);
  for (unsigned long long left = bad; left != 0; left &= left - 1) {
    const int i = __builtin_ctzll(left);
    float weight = 0.f;
#pragma unroll
    for (int blk = 0; blk < P::kBlocks; ++blk)
#pragma unroll
      for (int r = 0; r < 4; ++r) weight = blk == i >> 4 && r == (i & 3) ? w[blk][r] : weight;
    weight = __shfl(weight, c + 16 * ((i >> 2) & 3));
    if (!seen(i)) continue;
#pragma unroll
    for (int db = 0; db < 4; ++db) o[db] += P::value(piece + PieceLoad<P>::kBytes, scales + 64, i, 16 * db + 4 * q) * weight;
  }
  load.clear_keys(piece, bad);
}

// Queries are waited for here, and not at their first use in the loop, where that would be waiting for the pieces on their way as well, each time.
template <typename A, int N>
__device__ __forceinline__ void have(A (&q)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+v"(q[i]));
}

// One wave over its pieces: what its columns have of maxima, sums (those of a column's four lanes are still to be added) and weighted values.  seen(key, x) tells
// whether the lane's column sees the key, where MASKED.
template <typename P, bool MASKED, bool STEADY, typename Seen1>
__device__ __forceinline__ void go_over(const Pages& a, const Stretch& st, const int* table, int hk, int wave, int lane, unsigned char* mine, float scale_log2,
                                        const typename P::A (&qf)[P::kSteps], Seen1 seen, f32x4 (&o)[4], float& m, float& l) {
  const int c = lane & 15, q = lane >> 4;
  const unsigned lds = __builtin_amdgcn_readfirstlane(lds_address(mine));
  const int pieces = (st.x1 - st.x0 + P::kKeys - 1) / P::kKeys;
  const PieceLoad<P> load(lane);
  auto issue = [&](int p, int buf) { load.issue(a, st, table, hk, st.x0 + p * P::kKeys, lds + buf * kBuf<P>); };
  if (wave < pieces) issue(wave, 0);
  if (wave + kWaves < pieces) issue(wave + kWaves, 1);

  m = -INFINITY, l = 0.f;
#pragma unroll
  for (int db = 0; db < 4; ++db) o[db] = f32x4{0.f, 0.f, 0.f, 0.f};
  int buf = 0;
  for (int p = wave; p < pieces; p += kWaves, buf ^= 1) {
    load.wait(p + kWaves >= pieces);  // the next piece's loads may be on their way
    unsigned char* const kt = mine + buf * kBuf<P>;
    unsigned* const scales = reinterpret_cast<unsigned*>(kt + 2 * kPiece<P>);
    const int left = st.x1 - st.x0 - p * P::kKeys;
    if (left < P::kKeys) load.clear_from(kt, left);
    f32x4 w[P::kBlocks];
#pragma unroll
    for (int blk = 0; blk < P::kBlocks; ++blk) {
      typename P::A ka[P::kSteps];
      P::rows(kt, scales, 16 * blk + c, q, ka);
      w[blk] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < P::kSteps; ++e) w[blk] = P::product(ka[e], qf[e], w[blk]);
    }
    typename P::Raw raw;
    constexpr bool kEarly = STEADY && !MASKED;
    if constexpr (!MASKED) P::fetch(kt + kPiece<P>, scales + 64, lane, raw);
    if constexpr (kEarly) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // all of the piece is in registers: the buffer is free
      if (p + 2 * kWaves < pieces) issue(p + 2 * kWaves, buf);
    }
    if (MASKED || left < P::kKeys) {
#pragma unroll
      for (int blk = 0; blk < P::kBlocks; ++blk)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int i = 16 * blk + 4 * q + r;
          if (i >= left || (MASKED && !seen(st.key(st.x0 + p * P::kKeys + i)))) w[blk][r] = -INFINITY;
        }
    }
    auto highest = [&]() {
      float top = -INFINITY;
#pragma unroll
      for (int blk = 0; blk < P::kBlocks; ++blk)
#pragma unroll
        for (int r = 0; r < 4; ++r) top = fmaxf(top, w[blk][r]);
      return across<true>(top) * scale_log2;
    };
    auto follow = [&](float to) {
      const float keep = to == -INFINITY ? 1.f : exp2f(m - to);
      m = to;
      l *= keep;
#pragma unroll
      for (int db = 0; db < 4; ++db) o[db] *= keep;
    };
    if constexpr (STEADY) {
      // The reference m stays until the sum of a column's weights passes 2^24, then it follows the largest logit and the sum: no maximum, and no way across lanes, in
      // the piece's chain of operations, which is what few workgroups wait for (96 sequences of up to 4,100 keys 43.6 -> 40.8 us, and 39.5 since the next piece is
      // asked for before this one's weights).
      f32x4 x[P::kBlocks];
      float sum;
      auto take = [&]() {
        const float minus = m == -INFINITY ? 0.f : -m;
        sum = l;
#pragma unroll
        for (int blk = 0; blk < P::kBlocks; ++blk)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            x[blk][r] = __builtin_amdgcn_exp2f(fmaf(w[blk][r], scale_log2, minus));
            sum += x[blk][r];
          }
      };
      take();
      if (__any(!(sum <= 0x1p24f) | (m == -INFINITY))) {
        float to = fmaxf(m, highest());
        const float grown = across<true>(l);
        if (grown > 0x1p16f) to = fmaxf(to, m + log2f(grown));
        follow(to);
        take();
      }
      l = sum;
#pragma unroll
      for (int blk = 0; blk < P::kBlocks; ++blk) w[blk] = x[blk];
    } else {
      const float top = highest();
      if (__any(top > m)) follow(fmaxf(m, top));
      const float from = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int blk = 0; blk < P::kBlocks; ++blk)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          w[blk][r] = __builtin_amdgcn_exp2f(fmaf(w[blk][r], scale_log2, -from));
          l += w[blk][r];
        }
    }
    if constexpr (MASKED) {
      leave_bad_out<P>(load, kt, [&](int i) { return seen(st.key(st.x0 + p * P::kKeys + i)); }, w, o);
      P::fetch(kt + kPiece<P>, scales + 64, lane, raw);
    }
    P::update(raw, w, o);
    if (!kEarly && p + 2 * kWaves < pieces) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the operands are in registers: the buffer is free
      issue(p + 2 * kWaves, buf);
    }
  }
}

// The waves' sums together, each through its own LDS (none of its loads are on their way any more): thread t of the workgroup has numbers 4 (t % 16) .. + 3 of column
// t / 16, not divided by the sum yet.
template <typename P>
__device__ __forceinline__ void join_waves(unsigned char* smem, float (&sums)[kWaves][2][kHeads], int wave, int lane, const f32x4 (&o)[4], float m, float l,
                                           f32x4& y, float& top, float& sum) {
  static_assert(kWaveLds<P> >= kHeads * 64 * 4, "sixteen columns in 32 bits");
  const int c = lane & 15, q = lane >> 4;
  unsigned char* const mine = smem + wave * kWaveLds<P>;
  l = across<false>(l);
#pragma unroll
  for (int db = 0; db < 4; ++db) *reinterpret_cast<f32x4*>(mine + (c * 64 + 16 * db + 4 * q) * 4) = o[db];
  if (q == 0) {
    sums[wave][0][c] = m;
    sums[wave][1][c] = l;
  }
  __syncthreads();
  const int head = threadIdx.x >> 4, d = (threadIdx.x & 15) * 4;
  top = -INFINITY;
  bool nan = false;
#pragma unroll
  for (int x = 0; x < kWaves; ++x) {
    top = fmaxf(top, sums[x][0][head]);
    nan = nan || sums[x][1][head] != sums[x][1][head];
  }
  sum = 0.f;
  y = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int x = 0; x < kWaves; ++x) {
    const float weight = sums[x][0][head] == -INFINITY ? 0.f : exp2f(sums[x][0][head] - top);
    sum += sums[x][1][head] * weight;
    y += *reinterpret_cast<const f32x4*>(smem + x * kWaveLds<P> + (head * 64 + d) * 4) * weight;
  }
  if (nan) sum = NAN;
}

// Keys of a workgroup, and workgroups of a sequence's (or prefix's) keys, `units` of which there are, with at most `most` keys that are seen.  The chip holds
// 512, and 300 with 64 KB on their way each draw what the memory gives; stretches cost a second
// kernel, and each wave should have a few pieces.  Measured, us, for at least 512 / 1024 / 2048 / 4096 workgroups: one sequence of 10,992 bf16 keys and 16
// key heads 14.6 / 15.2 / 15.3 / 15.2; two of 412,200 and 312,300 508 / 482 / 487 / 495; 96 of up to 4,100 keys and 4 key heads 60 (no
// stretches) / 70 / 64 / 67.  The host knows the most that a sequence can see, not its length: one long sequence among short ones must not be left to one
// workgroup (4,608 keys take one about 30 us), and the workgroups that find nothing to do have to stay few.
// Up to 8 pieces for each wave are one workgroup's whatever the launch: 1,024 bf16 keys 9.9 us a call and 27.2 alone, in stretches of 256 with
// their second kernel 13.8 and 26.7; 512 fp32 keys 13.0 and 30.3, 14.2 and 29.7.
// places: so many workgroups, if that is not 0.
inline void cut(int64_t most, int64_t units, int keys_of_piece, int page, int& stretch_out, int& splits_out, int64_t places = 0) {
  most = larger(most, int64_t(1));
  const int64_t step = kWaves * keys_of_piece;
  if (most <= 8 * step) {
    stretch_out = static_cast<int>(ceil_div(most, step) * step);
    splits_out = 1;
    return;
  }
  int64_t splits = larger(int64_t(units > 256 || most * units < 512 * 1024 ? 512 : 1024) / units, int64_t(1));
  if (units > 256) splits = larger(splits, smaller(ceil_div(most, 4608), int64_t(4096) / units));
  if (places > 0) splits = larger(places / units, int64_t(1));
  const int64_t stretch = ceil_div(larger(ceil_div(most, splits), 2 * step), step) * step;
  const int64_t fits = int64_t(kTable - 4) * page / step * step;
  stretch_out = static_cast<int>(smaller(smaller(stretch, fits), ceil_div(most, step) * step));
  splits_out = static_cast<int>(ceil_div(most, stretch_out));
}

inline int check_pages(const char* fn, int kv_heads, int64_t n_pages, int page, Pages& a) {
  if (page < 1 || page > 65536) return fail(BSGA_ERR_INVALID_ARG, "%s: page must be in [1, 65536] tokens, got %d", fn, page);
  if (n_pages < 0 || n_pages > (int64_t(1) << 30)) return fail(BSGA_ERR_INVALID_ARG, "%s: n_pages must be in [0, 2^30], got %lld", fn, (long long)n_pages);
  a.kv_heads = kv_heads;
  a.n_pages = static_cast<int>(n_pages);
  a.page = page;
  a.shift = 0;
  while ((int64_t(1) << a.shift) < page) ++a.shift;
  a.magic = static_cast<unsigned>(((uint64_t(1) << (31 + a.shift)) + page - 1) / page);
  return BSGA_OK;
}

}  // namespace
}  // namespace bsga
