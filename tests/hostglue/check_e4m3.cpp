// Host code of the entry points on caches in 8 bits and shared prefixes under AddressSanitizer and UndefinedBehaviorSanitizer, over arguments of any size; the stubs
// for the HIP runtime and the sizes are those of check_stream.cpp.  Built and run by tests/test_hostglue_e4m3.py.
#define main main_of_stream
#include "check_stream.cpp"
#undef main

static void one_more() {
  void* const A = reinterpret_cast<void*>(0x1000);
  float* const F = reinterpret_cast<float*>(A);
  const int32_t* const I = reinterpret_cast<const int32_t*>(A);
  uint8_t* const U = reinterpret_cast<uint8_t*>(A);
  const int dtype = bits() % 16 == 0 ? size32() : static_cast<int>(bits() % 2);
  const int cache_dtype = bits() % 8 == 0 ? size32() : bits() % 2 ? dtype : BSGA_E4M3;
  const int h = heads(), hk = bits() % 2 == 0 ? h : heads();
  int64_t st[6];
  for (int i = 0; i < 6; ++i) st[i] = mostly(64);
  const int64_t frame = mostly(1), window = mostly(4), sinks = mostly(0), batch = mostly(3), width = size64(), pages = size64();
  const int page = bits() % 2 == 0 ? 16 : size32();
  const float scale = static_cast<float>(number());
  auto room = [](size_t need) { return need == 0 || bits() % 4 != 0 ? need : need - 1; };  // (which is too little)

  size_t need = bsga_paged_attn_e4m3_workspace_bytes(dtype, batch, h, hk, width, pages, page, frame, window, sinks);
  CHECK(need < size_t(1) << 62);
  const size_t has_paged = room(need);
  int rc = bsga_paged_attn_e4m3(A, st[0], st[1], A, A, U, U, dtype, batch, h, hk, 64, I, width, I, pages, page, scale, frame, window, sinks, A, F, A, has_paged,
                                nullptr);
  CHECK(rc != BSGA_OK || has_paged == need);
  g_refused += rc != BSGA_OK;

  const int64_t prefixes = mostly(2), prefix_width = size64();
  need = bsga_prefix_attn_workspace_bytes(dtype, cache_dtype, batch, h, hk, width, prefixes, prefix_width, pages, page, frame, window, sinks);
  CHECK(need < size_t(1) << 62);
  const size_t has_prefix = room(need);
  rc = bsga_prefix_attn(A, st[0], st[1], A, A, U, U, dtype, cache_dtype, batch, h, hk, 64, I, width, I, I, prefix_width, I, I, prefixes, pages, page, scale,
                        frame, window, sinks, A, F, A, has_prefix, nullptr);
  CHECK(rc != BSGA_OK || has_prefix == need);
  g_refused += rc != BSGA_OK;

  g_refused += bsga_cache_load(A, A, U, U, cache_dtype, pages, page, hk, 64, I, width, bits() % 2 ? 0 : size64(), size64(), dtype, A, A, st[0], st[1], nullptr) !=
               BSGA_OK;

  const int axes = static_cast<int>(bits() % 4), norm = static_cast<int>(bits() % 4);
  const int64_t n = bits() % 4 == 0 ? 0 : size64();
  void* x[3] = {bits() % 4 ? A : nullptr, bits() % 4 ? A : nullptr, bits() % 4 ? A : nullptr};
  const void *w = norm == BSGA_NORM_NONE ? nullptr : A, *b = norm == BSGA_NORM_LAYER ? A : nullptr;
  g_refused += bsga_qk_norm_rope_e4m3(x[0], x[1], x[2], st[0], st[1], st[2], st[3], st[4], st[5], dtype, n, h, hk, 64, norm, number(), w, b, w, b,
                                      axes ? I : nullptr, axes, number(), bits() % 8 ? I : nullptr, pages, page, x[0], bits() % 2 ? x[1] : nullptr,
                                      bits() % 2 ? x[2] : nullptr, x[1], bits() % 8 ? x[2] : nullptr, x[1] ? U : nullptr, x[2] ? U : nullptr, nullptr) != BSGA_OK;
}

int main(int argc, char** argv) {
  const int rounds = argc > 1 ? atoi(argv[1]) : 1000;
  g_state = 0x9e3779b97f4a7c15ull;
  for (int i = 0; i < rounds; ++i) one_more();
  printf("%d launches, %d calls refused, %d failed checks\n", g_launches, g_refused, g_fail);
  return g_fail == 0 && g_launches > 0 && g_refused > 0 ? 0 : 1;
}
