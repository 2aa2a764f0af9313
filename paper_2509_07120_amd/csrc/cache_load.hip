// Tokens of a sequence out of the pages of a cache, head by head: [kv_heads, n, 64].
//
// HBM-bound: a row of 65 bytes is read and one of 128 written (in 8 bits to bf16).  412,200 tokens of 16 heads, 2.55 GB: 480 us, 5.3 TB/s, where a copy of 1
// GiB reaches 5.2.  A lane moves 16 bytes of a row of the cache; a workgroup takes 64 tokens of one head, keys in one half of the grid and values in the other.
#include "e4m3.h"
#include "bsga_internal.h"

namespace bsga {
namespace {

constexpr int kTokens = 64;  // of a workgroup

struct LoadArgs {
  const unsigned char* cache[2];
  const unsigned char* scale[2];
  const int32_t* pages;
  unsigned char* out[2];
  int64_t out_head[2];  // bytes
  int64_t first, n;
  int kv_heads, n_pages, page, width;
};

// C: of the cache, T: of the result (the same where the cache is not in 8 bits)
template <typename C, typename T>
__global__ __launch_bounds__(256) void cache_load_kernel(const LoadArgs a) {
  constexpr bool kCoded = sizeof(C) == 1;
  constexpr int kRow = 64 * sizeof(C), kChunks = kRow / 16, kPer = kTokens * kChunks / 256;
  const int h = blockIdx.y >> 1, t = blockIdx.y & 1;
  const int64_t t0 = int64_t(blockIdx.x) * kTokens;
  u32x4 x[kPer];
  unsigned byte[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int at = i * 256 + threadIdx.x;
    const int64_t token = smaller(t0 + at / kChunks, a.n - 1) + a.first;
    const int64_t page = token / a.page;
    const int p = page < a.width ? a.pages[page] : -1;
    x[i] = u32x4{0u, 0u, 0u, 0u};
    byte[i] = 0;
    if (p >= 0 && p < a.n_pages) {  // what has no page are zeros
      const int64_t row = (int64_t(p) * a.kv_heads + h) * a.page + (token - page * a.page);
      x[i] = *reinterpret_cast<const u32x4*>(a.cache[t] + row * kRow + at % kChunks * 16);
      if constexpr (kCoded) byte[i] = a.scale[t][row];
    }
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int at = i * 256 + threadIdx.x;
    const int64_t token = t0 + at / kChunks;
    if (token >= a.n) continue;
    unsigned char* p = a.out[t] + h * a.out_head[t] + (token * 64 + at % kChunks * (16 / sizeof(C))) * sizeof(T);
    if constexpr (!kCoded) {
      *reinterpret_cast<u32x4*>(p) = x[i];
    } else {
      const float f = scale_of(byte[i]);
      if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const u32x2 y0 = unpack_bf16(x[i][2 * e], f), y1 = unpack_bf16(x[i][2 * e + 1], f);
          reinterpret_cast<u32x4*>(p)[e] = u32x4{y0[0], y0[1], y1[0], y1[1]};
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) reinterpret_cast<f32x4*>(p)[e] = unpack_f32(x[i][e]) * f;
      }
    }
  }
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace
}  // namespace bsga

using namespace bsga;

extern "C" int bsga_cache_load(const void* k_cache, const void* v_cache, const uint8_t* k_scale, const uint8_t* v_scale, int cache_dtype, int64_t n_pages,
                               int page, int kv_heads, int head_dim, const int32_t* pages, int64_t table_width, int64_t first, int64_t n_tokens, int dtype,
                               void* k_out, void* v_out, int64_t k_head, int64_t v_head, void* stream) {
  const char* fn = "bsga_cache_load";
  clear_error();
  if (dtype != BSGA_BF16 && dtype != BSGA_FP32) return fail(BSGA_ERR_INVALID_ARG, "%s: unknown dtype %d", fn, dtype);
  if (cache_dtype != BSGA_E4M3 && cache_dtype != dtype)
    return fail(BSGA_ERR_INVALID_ARG, "%s: a cache must be in 8 bits or of the outputs' type, got %d and %d", fn, cache_dtype, dtype);
  if (head_dim != 64) return fail(BSGA_ERR_UNSUPPORTED, "%s: head_dim must be 64, got %d", fn, head_dim);
  if (kv_heads < 1 || kv_heads > 32767) return fail(BSGA_ERR_INVALID_ARG, "%s: kv_heads must be in [1, 32767], got %d", fn, kv_heads);
  if (page < 1 || page > 65536) return fail(BSGA_ERR_INVALID_ARG, "%s: page must be in [1, 65536] tokens, got %d", fn, page);
  const int64_t most = int64_t(1) << 30;
  if (n_pages < 0 || n_pages > most) return fail(BSGA_ERR_INVALID_ARG, "%s: n_pages must be in [0, 2^30], got %lld", fn, (long long)n_pages);
  if (table_width < 0 || table_width > most / page)
    return fail(BSGA_ERR_INVALID_ARG, "%s: a sequence's pages must hold up to 2^30 tokens, got %lld pages", fn, (long long)table_width);
  if (first < 0 || n_tokens < 0 || first > most || n_tokens > table_width * page - first)
    return fail(BSGA_ERR_INVALID_ARG, "%s: tokens %lld to %lld + %lld do not lie in the sequence's pages", fn, (long long)first, (long long)first, (long long)n_tokens);
  if (n_tokens == 0) return BSGA_OK;
  if (ceil_div(n_tokens, kTokens) >= (int64_t(1) << 32) / 256)  // (a grid has up to 2^32 - 1 threads)
    return fail(BSGA_ERR_UNSUPPORTED, "%s: too many tokens for one launch, got %lld", fn, (long long)n_tokens);
  const int size = dtype == BSGA_BF16 ? 2 : 4;
  if (!pages || !k_out || !v_out || (n_pages > 0 && (!k_cache || !v_cache)))
    return fail(BSGA_ERR_INVALID_ARG, "%s: k_cache, v_cache, pages, k_out and v_out must be non-null", fn);
  if (cache_dtype == BSGA_E4M3 && n_pages > 0 && (!k_scale || !v_scale))
    return fail(BSGA_ERR_INVALID_ARG, "%s: a cache in 8 bits must come with k_scale and v_scale", fn);
  LoadArgs a = {};
  const void* const cache[2] = {k_cache, v_cache};
  const uint8_t* const scale[2] = {k_scale, v_scale};
  void* const out[2] = {k_out, v_out};
  const int64_t head[2] = {k_head, v_head};
  for (int t = 0; t < 2; ++t) {
    if (!aligned16(cache[t]) || !aligned16(out[t])) return fail(BSGA_ERR_INVALID_ARG, "%s: caches and outputs must be 16-byte aligned", fn);
    if (!whole_stride(head[t], size)) return fail(BSGA_ERR_INVALID_ARG, "%s: strides of the heads must be multiples of 16 bytes and not negative", fn);
    if (kv_heads > 1 && head[t] < n_tokens * 64) return fail(BSGA_ERR_INVALID_ARG, "%s: the outputs' heads must not overlap", fn);
    a.cache[t] = static_cast<const unsigned char*>(cache[t]);
    a.scale[t] = scale[t];
    a.out[t] = static_cast<unsigned char*>(out[t]);
    a.out_head[t] = head[t] * size;
  }
  a.pages = pages;
  a.first = first;
  a.n = n_tokens;
  a.kv_heads = kv_heads;
  a.n_pages = static_cast<int>(n_pages);
  a.page = page;
  a.width = static_cast<int>(table_width);
  const dim3 grid(static_cast<unsigned>(ceil_div(n_tokens, kTokens)), static_cast<unsigned>(2 * kv_heads));
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (cache_dtype == BSGA_E4M3) {
    if (dtype == BSGA_BF16) hipLaunchKernelGGL((cache_load_kernel<unsigned char, __bf16>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((cache_load_kernel<unsigned char, float>), grid, dim3(256), 0, s, a);
  } else {
    if (dtype == BSGA_BF16) hipLaunchKernelGGL((cache_load_kernel<__bf16, __bf16>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((cache_load_kernel<float, float>), grid, dim3(256), 0, s, a);
  }
  return check_hip(hipGetLastError(), fn);
}
