// Host code of the streamed layer's entry points (argument checks, how a launch is cut up, workspace sizes) under AddressSanitizer and
// UndefinedBehaviorSanitizer, over arguments of any size.  The HIP runtime is replaced by the stubs below, so that nothing is launched
// wherever this runs: a launch only has to be one that the hardware takes.  Built and run by tests/test_hostglue_stream.py.
#include <hip/hip_runtime.h>
#include <stdarg.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

#include "bsga.h"
#include "bsga_internal.h"

static int g_fail = 0, g_launches = 0, g_refused = 0;
#define CHECK(cond)                                                     \
  do {                                                                  \
    if (!(cond)) {                                                      \
      fprintf(stderr, "FAILED %s:%d: %s\n", __FILE__, __LINE__, #cond); \
      ++g_fail;                                                         \
    }                                                                   \
  } while (0)

namespace bsga {
void clear_error() {}
int fail(int code, const char* fmt, ...) {
  char text[1024];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(text, sizeof(text), fmt, ap);
  va_end(ap);
  CHECK(code != BSGA_OK);
  return code;
}
int check_hip(hipError_t e, const char*) { return e == hipSuccess ? BSGA_OK : BSGA_ERR_INVALID_ARG; }
}  // namespace bsga

static dim3 g_grid, g_block;
extern "C" {
void** __hipRegisterFatBinary(const void*) {
  static void* handle;
  return &handle;
}
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void*, char*, const char*, unsigned, void*, void*, void*, void*, int*) {}
void __hipRegisterVar(void**, void*, char*, char*, int, size_t, int, int) {}
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t, hipStream_t) {
  g_grid = grid;
  g_block = block;
  return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* shared, hipStream_t* stream) {
  *grid = g_grid;
  *block = g_block;
  *shared = 0;
  *stream = nullptr;
  return hipSuccess;
}
hipError_t hipLaunchKernel(const void*, dim3 grid, dim3 block, void**, size_t, hipStream_t) {
  ++g_launches;
  CHECK(grid.x >= 1 && grid.x <= 0x7fffffffu && grid.y >= 1 && grid.y <= 65535 && grid.z >= 1 && grid.z <= 65535);
  CHECK(block.x >= 64 && block.x <= 1024 && block.x % 64 == 0 && block.y == 1 && block.z == 1);
  return hipSuccess;
}
hipError_t hipGetLastError() { return hipSuccess; }
}

static uint64_t g_state;
static uint64_t bits() {  // xorshift
  g_state ^= g_state << 13;
  g_state ^= g_state >> 7;
  g_state ^= g_state << 17;
  return g_state;
}
static int64_t pick(const int64_t* from, int n) { return from[bits() % static_cast<uint64_t>(n)]; }
static int64_t size64() {  // sizes that are met and sizes that nobody has
  static const int64_t edges[] = {0, 1, -1, 2, 3, 63, 64, 65, 100, 1374, 65535, 65536, 1 << 24, (1 << 24) + 1, 1 << 25, 1 << 30, 0x7fffffff,
                                  int64_t(1) << 31, (int64_t(1) << 32) + 5, int64_t(1) << 40, int64_t(1) << 48, int64_t(1) << 61, INT64_MAX, INT64_MIN};
  return bits() % 3 == 0 ? pick(edges, sizeof(edges) / sizeof(edges[0])) : static_cast<int64_t>(bits() % 5000) - 3;
}
static int size32() {
  const int64_t x = size64();
  return static_cast<int>(x > INT32_MAX ? INT32_MAX : x < INT32_MIN ? INT32_MIN : x);
}
static int64_t mostly(int64_t usual) { return bits() % 4 != 0 ? usual : size64(); }
static int heads() { return bits() % 4 != 0 ? 1 << bits() % 5 : size32(); }
static double number() {
  static const double edges[] = {1e4, 100.0, 1.0, 1e-6, 0.125, 1e-300, 1e300, 5e-324, 1e-40, 3e38, 0.0, -1.0, INFINITY, NAN};
  return edges[bits() % (sizeof(edges) / sizeof(edges[0]))];
}

static void one() {
  void* const A = reinterpret_cast<void*>(0x1000);
  float* const F = reinterpret_cast<float*>(A);
  const int32_t* const I = reinterpret_cast<const int32_t*>(A);
  const int dtype = bits() % 16 == 0 ? size32() : static_cast<int>(bits() % 2);
  const int h = heads(), hk = bits() % 2 == 0 ? h : heads();
  int64_t st[6], to[6];
  for (int i = 0; i < 6; ++i) {
    st[i] = mostly(64);
    to[i] = mostly(64);
  }
  const int64_t n_q = size64(), n_k = size64(), start = bits() % 2 == 0 ? 0 : size64(), frame = mostly(1), window = mostly(4), sinks = mostly(0);
  const float scale = static_cast<float>(number());
  auto room = [](size_t need) { return need == 0 || bits() % 4 != 0 ? need : need - 1; };  // (which is too little)

  size_t need = bsga_window_attn_workspace_bytes(dtype, h, n_q, n_k, start, frame, window, sinks);
  CHECK(need < size_t(1) << 62);
  g_refused += bsga_window_attn(A, A, A, st[0], st[1], st[2], st[3], st[4], st[5], dtype, h, hk, n_q, n_k, 64, scale, start, frame, window, sinks, A, F, A,
                                room(need), nullptr) != BSGA_OK;
  need = bsga_window_attn_bwd_workspace_bytes(dtype, h, hk, n_q, n_k, start, frame, window, sinks);
  CHECK(need < size_t(1) << 62);
  const size_t has = room(need);
  int rc = bsga_window_attn_bwd(A, A, A, A, st[0], st[1], st[2], st[3], st[4], st[5], A, F, dtype, h, hk, n_q, n_k, 64, scale, start, frame, window, sinks, A,
                                A, A, A, has, nullptr);
  CHECK(rc != BSGA_OK || has == need);
  g_refused += rc != BSGA_OK;

  const int64_t batch = mostly(3), width = size64(), pages = size64();
  const int page = bits() % 2 == 0 ? 16 : size32();
  need = bsga_paged_attn_workspace_bytes(dtype, batch, h, hk, width, pages, page, frame, window, sinks);
  CHECK(need < size_t(1) << 62);
  const size_t has_paged = room(need);
  rc = bsga_paged_attn(A, st[0], st[1], A, A, dtype, batch, h, hk, 64, I, width, I, pages, page, scale, frame, window, sinks, A, F, A, has_paged, nullptr);
  CHECK(rc != BSGA_OK || has_paged == need);
  g_refused += rc != BSGA_OK;

  const int axes = static_cast<int>(bits() % 4), norm = static_cast<int>(bits() % 4);
  const int64_t n = bits() % 4 == 0 ? 0 : size64();
  const double eps = number(), base = number();
  const void *x[3] = {bits() % 4 ? A : nullptr, bits() % 4 ? A : nullptr, bits() % 4 ? A : nullptr};
  void* y[3];
  for (int i = 0; i < 3; ++i) y[i] = bits() % 8 ? const_cast<void*>(x[i]) : A;
  const void *w = norm == BSGA_NORM_NONE ? nullptr : A, *b = norm == BSGA_NORM_LAYER ? A : nullptr;
  g_refused += bsga_qk_norm_rope(x[0], x[1], x[2], st[0], st[1], st[2], st[3], st[4], st[5], dtype, n, h, hk, 64, norm, eps, w, b, w, b, axes ? I : nullptr,
                                 axes, base, bits() % 2 ? I : nullptr, pages, page, y[0], y[1], y[2], nullptr) != BSGA_OK;
  need = bsga_qk_norm_rope_bwd_workspace_bytes(n, h, hk);
  const size_t has_norm = room(need);
  rc = bsga_qk_norm_rope_bwd(x[0], x[1], x[2], x[0], x[1], st[0], st[1], st[2], st[3], dtype, n, h, hk, 64, norm, eps, w, w, axes ? I : nullptr, axes, base,
                             y[0], y[1], y[2], to[0], to[1], to[2], to[3], to[4], to[5], bits() % 2 ? F : nullptr, A, has_norm, nullptr);
  g_refused += rc != BSGA_OK;
}

int main(int argc, char** argv) {
  const int rounds = argc > 1 ? atoi(argv[1]) : 1000;
  g_state = 0x9e3779b97f4a7c15ull;
  for (int i = 0; i < rounds; ++i) one();
  printf("%d launches, %d calls refused, %d failed checks\n", g_launches, g_refused, g_fail);
  return g_fail == 0 && g_launches > 0 && g_refused > 0 ? 0 : 1;
}
