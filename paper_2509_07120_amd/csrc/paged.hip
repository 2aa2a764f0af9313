// Attention of one new token for each sequence over a cache of pages.
//
// The query of sequence b stands at position lengths[b] - 1, its own key is in the cache.  It sees the keys that window.h describes, in
// the cache rows page_table[b][j / page], j % page.  HBM-bound: every visible key and value is read once for up to 16 of the query heads
// that share it (more of them: once for each 16), at 16 flop to the byte at most (fp32 8).  A workgroup takes a stretch of one sequence's visible keys and one key head; its four waves take
// pieces of it in turn and wait for nobody: a wave moves its pieces straight into LDS of its own, two ahead (16 KB on their way for each
// wave, 128 KB for each CU, where 8 TB/s at 2 us of latency ask for 64).  Up to 16 query heads are the columns of 16x16 products
// S^T = K Q^T and O^T = V^T P^T, in which the weights are operands as they lie in the results.
// The waves' sums are joined through LDS; stretches of one sequence by a second kernel.
// Two sequences of 412,200 and 312,300 keys of 16 heads, 2.97 GB: 480 us, 6.2 TB/s; 96 of 1 to 12,000, window of 4096, 16 query heads to 4 key heads: 66 us, 5.0 TB/s.
// In 8 bits, where pieces are 64 keys of 65 bytes (8 KB on their way for each wave are enough: half the bytes, and two numbers' products to one of them), 1.51 GB 250 us,
// 6.0 TB/s, and 39 us, 4.3 TB/s: 36 in the kernel, 27 of them by bytes, the rest from the lengths over the pages to the first piece, and the longest sequences' end.
#include "paged.h"

#include <math.h>

namespace bsga {
namespace {

struct PagedArgs {
  View q;                             // [batch, heads, 64]: token is the sequence's stride
  Pages pages;
  const int32_t *page_table, *lengths;
  unsigned char* out;                 // [batch, heads, 64]
  float* lse;                         // [batch, heads] or null
  float *part, *part_lse;             // with stretches: [splits][batch, heads, 64] and [splits][batch, heads]
  int batch, heads, group, head_blocks, table_width, frame, window, sinks, splits, stretch;
  int dealt;                          // whether the grid is one row, see attend()
  float scale_log2;
};

template <typename T, typename C>
__global__ __launch_bounds__(64 * kWaves, 2) void paged_kernel(const PagedArgs a) {
  typedef Ops16<T, C> P;
  __shared__ __align__(16) unsigned char smem[kWaves * kWaveLds<P>];
  __shared__ int table[kTable];
  __shared__ float sums[kWaves][2][kHeads];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, q = lane >> 4;
  int b = blockIdx.z, split = blockIdx.x, of = blockIdx.y;
  if (a.dealt) {
    const int heads_of = a.pages.kv_heads * a.head_blocks, turn = blockIdx.x >> 3, eight = turn / heads_of, pair = eight * 8 + ((blockIdx.x - eight) & 7);
    of = turn % heads_of, split = pair / a.batch, b = pair % a.batch;
    if (split >= a.splits) return;
  }
  const int hk = of / a.head_blocks, hb = of - hk * a.head_blocks;
  const int heads = min(kHeads, a.group - hb * kHeads);       // query heads of this workgroup,
  const int h0 = hk * a.group + hb * kHeads;                  // the first of them
  const int64_t rows = int64_t(a.batch) * a.heads, row0 = int64_t(b) * a.heads + h0;

  Stretch st = {};
  st.x0 = split * a.stretch;
  const int32_t* const pages = a.page_table + int64_t(b) * a.table_width;
  if (a.window == 0) st.fill_ahead(a.pages, pages, a.table_width, a.stretch, table);
  const int length = min(max(a.lengths[b], 0), a.table_width * a.pages.page);
  if (a.window > 0 && length > 0) {
    const int f = (length - 1) / a.frame;
    st.lo = f < a.window ? 0 : (f + 1 - a.window) * a.frame;
    st.s = min(a.sinks, st.lo);
  }
  const int count = st.s + length - st.lo;
  st.x1 = min(st.x0 + a.stretch, count);
  if (st.x0 >= st.x1 && a.splits > 1) {  // the whole workgroup: the sequence has no keys here
    if (threadIdx.x < heads) a.part_lse[split * rows + row0 + threadIdx.x] = -INFINITY;
    return;
  }
  if (a.window > 0) st.fill(a.pages, pages, table);
  typename P::A qf[P::kSteps];
  P::row(a.q.p + b * a.q.token + (h0 + min(c, heads - 1)) * a.q.head, q, qf);
  __syncthreads();

  f32x4 o[4];
  float m, l;
  go_over<P, false, P::kScaled>(a.pages, st, table, hk, wave, lane, smem + wave * kWaveLds<P>, a.scale_log2, qf, [](int) { return true; }, o, m, l);
  f32x4 y;
  float top, sum;
  join_waves<P>(smem, sums, wave, lane, o, m, l, y, top, sum);
  const int head = threadIdx.x >> 4, d = (threadIdx.x & 15) * 4;
  if (head >= heads) return;
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  const int64_t row = row0 + head;
  const float total = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
  if (a.splits > 1) {
    *reinterpret_cast<f32x4*>(a.part + (split * rows + row) * 64 + d) = y * inv;
    if (d == 0) a.part_lse[split * rows + row] = total;
  } else {
    Ops<T>::store4(a.out + row * Ops<T>::kRow, d, y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
    if (a.lse != nullptr && d == 0) a.lse[row] = total;
  }
}

int keys_of_piece(int dtype, bool coded) { return coded ? Ops16E4m3::kKeys : dtype == BSGA_BF16 ? Ops16<__bf16, __bf16>::kKeys : Ops16<float, float>::kKeys; }

void shape_of(PagedArgs& a, int keys) {
  int64_t most = int64_t(a.table_width) * a.pages.page;
  if (a.window > 0) most = smaller(most, int64_t(a.window) * a.frame + a.sinks);
  cut(most, int64_t(a.batch) * a.pages.kv_heads * a.head_blocks, keys, a.pages.page, a.stretch, a.splits);
}

size_t part_bytes(const PagedArgs& a) { return a.splits > 1 ? static_cast<size_t>(a.splits) * a.batch * a.heads * 65 * sizeof(float) : 0; }

int check_sizes(const char* fn, int dtype, int64_t batch, int heads, int kv_heads, int64_t table_width, int64_t n_pages, int page, int64_t frame,
                int64_t window, int64_t sinks, PagedArgs& a) {
  if (dtype != BSGA_BF16 && dtype != BSGA_FP32) return fail(BSGA_ERR_INVALID_ARG, "%s: unknown dtype %d", fn, dtype);
  if (batch < 0 || batch > 65535) return fail(BSGA_ERR_INVALID_ARG, "%s: batch must be in [0, 65535], got %lld", fn, (long long)batch);
  if (heads < 1 || heads > 65535 || kv_heads < 1 || heads % kv_heads != 0)
    return fail(BSGA_ERR_INVALID_ARG, "%s: heads must be in [1, 65535] and a multiple of kv_heads, got %d and %d", fn, heads, kv_heads);
  if (int rc = check_pages(fn, kv_heads, n_pages, page, a.pages)) return rc;
  const int64_t most = int64_t(1) << 30;
  if (table_width < 0 || table_width > most / page)
    return fail(BSGA_ERR_INVALID_ARG, "%s: a sequence's pages must hold up to 2^30 tokens, got %lld pages", fn, (long long)table_width);
  if (frame < 1 || frame > (1 << 24)) return fail(BSGA_ERR_INVALID_ARG, "%s: frame must be in [1, 2^24] tokens, got %lld", fn, (long long)frame);
  if (window < 0) return fail(BSGA_ERR_INVALID_ARG, "%s: window must be >= 0 frames (0: no limit), got %lld", fn, (long long)window);
  if (sinks < 0) return fail(BSGA_ERR_INVALID_ARG, "%s: sinks must be >= 0, got %lld", fn, (long long)sinks);
  a.batch = static_cast<int>(batch);
  a.heads = heads;
  a.group = heads / kv_heads;
  a.head_blocks = static_cast<int>(ceil_div(a.group, kHeads));
  a.table_width = n_pages > 0 ? static_cast<int>(table_width) : 0;  // without pages there are no keys
  a.frame = static_cast<int>(frame);
  a.window = static_cast<int>(smaller(window, most));
  a.sinks = static_cast<int>(smaller(sinks, most));
  return BSGA_OK;
}

// Both entry points, with caches of the queries' type or in 8 bits.
int attend(const char* fn, bool coded, const void* q, int64_t q_batch, int64_t q_head, const void* k_cache, const void* v_cache, const uint8_t* k_scale,
           const uint8_t* v_scale, int dtype, int64_t batch, int heads, int kv_heads, int head_dim, const int32_t* page_table, int64_t table_width,
           const int32_t* lengths, int64_t n_pages, int page, float softmax_scale, int64_t frame, int64_t window, int64_t sinks, void* out, float* lse,
           void* workspace, size_t workspace_bytes, void* stream) {
  clear_error();
  PagedArgs a = {};
  if (head_dim != 64) return fail(BSGA_ERR_UNSUPPORTED, "%s: head_dim must be 64, got %d", fn, head_dim);
  if (int rc = check_sizes(fn, dtype, batch, heads, kv_heads, table_width, n_pages, page, frame, window, sinks, a)) return rc;
  if (!(softmax_scale > 0.0f) || !isfinite(softmax_scale)) return fail(BSGA_ERR_INVALID_ARG, "%s: softmax_scale must be finite and > 0", fn);
  if (int64_t(kv_heads) * a.head_blocks > 65535) return fail(BSGA_ERR_UNSUPPORTED, "%s: too many heads", fn);
  if (batch == 0) return BSGA_OK;
  if (int rc = check_view(fn, "q", q, q_batch, q_head, dtype == BSGA_BF16 ? 2 : 4, a.q)) return rc;
  if (!lengths || (a.table_width > 0 && (!page_table || !k_cache || !v_cache)))
    return fail(BSGA_ERR_INVALID_ARG, "%s: k_cache, v_cache, page_table and lengths must be non-null", fn);
  if (coded && a.table_width > 0 && (!k_scale || !v_scale)) return fail(BSGA_ERR_INVALID_ARG, "%s: k_scale and v_scale must be non-null", fn);
  if (!out || !aligned16(out) || !aligned16(k_cache) || !aligned16(v_cache))
    return fail(BSGA_ERR_INVALID_ARG, "%s: out must be non-null, it and the caches 16-byte aligned", fn);
  a.pages.k = static_cast<const unsigned char*>(k_cache);
  a.pages.v = static_cast<const unsigned char*>(v_cache);
  a.pages.k_scale = k_scale;
  a.pages.v_scale = v_scale;
  a.page_table = page_table;
  a.lengths = lengths;
  a.out = static_cast<unsigned char*>(out);
  a.lse = lse;
  a.scale_log2 = softmax_scale * kLog2e;
  shape_of(a, keys_of_piece(dtype, coded));
  const int64_t rows = batch * heads;
  if (a.splits > 1 && workgroups_of_join(rows, a.splits) >= (int64_t(1) << 32) / 256)  // (a grid has up to 2^32 - 1 threads)
    return fail(BSGA_ERR_UNSUPPORTED, "%s: too many keys of too many queries for one launch", fn);
  const size_t need = part_bytes(a);
  if (need > 0 && (!workspace || workspace_bytes < need))
    return fail(BSGA_ERR_WORKSPACE, "%s: workspace has %zu bytes, %zu needed", fn, workspace ? workspace_bytes : 0, need);
  if (!aligned16(workspace)) return fail(BSGA_ERR_INVALID_ARG, "%s: workspace must be 16-byte aligned", fn);
  a.part = static_cast<float*>(workspace);
  a.part_lse = a.part + int64_t(a.splits) * rows * 64;
  hipStream_t s = static_cast<hipStream_t>(stream);
  // Workgroup w runs on XCD w % 8.  From four sequences on, first stretches, which more of them have, come first, and each sequence's and each number's stretches are
  // dealt out to all XCDs; a stretch's heads, which read the same pages, follow each other on one.  Against a row of stretches for each head and sequence, us in bf16
  // and 8 bits: 16 sequences of 12,000 tokens on 4 key heads in a table for 192,512 160 -> 74, 124 -> 51; 16 of 1,000 to 100,000 177 -> 163, 100 -> 88; on 8 key heads, 12
  // of 60,000 in a table for 128,000 301 -> 248, 160 -> 133; 4 of 20,000 to 100,000 46 -> 47, 32 -> 32.  Two of 412,200 and 312,300 478 -> 485, 251 -> 256: fewer than
  // four are as they were.
  const int64_t of = int64_t(kv_heads) * a.head_blocks, pairs = batch * a.splits, blocks = 8 * ceil_div(pairs, 8) * of;
  a.dealt = batch >= 4 && pairs >= 64 && blocks < (int64_t(1) << 32) / (64 * kWaves);  // (a grid has up to 2^32 - 1 threads)
  const dim3 grid = a.dealt ? dim3(static_cast<unsigned>(blocks)) : dim3(static_cast<unsigned>(a.splits), static_cast<unsigned>(of), static_cast<unsigned>(batch));
  if (dtype == BSGA_BF16) {
    if (coded) hipLaunchKernelGGL((paged_kernel<__bf16, E4m3>), grid, dim3(64 * kWaves), 0, s, a);
    else hipLaunchKernelGGL((paged_kernel<__bf16, __bf16>), grid, dim3(64 * kWaves), 0, s, a);
  } else {
    if (coded) hipLaunchKernelGGL((paged_kernel<float, E4m3>), grid, dim3(64 * kWaves), 0, s, a);
    else hipLaunchKernelGGL((paged_kernel<float, float>), grid, dim3(64 * kWaves), 0, s, a);
  }
  if (int rc = check_hip(hipGetLastError(), fn)) return rc;
  if (a.splits == 1) return BSGA_OK;
  return dtype == BSGA_BF16 ? launch_join<__bf16>(a.part, a.part_lse, rows, a.splits, a.out, a.lse, s)
                            : launch_join<float>(a.part, a.part_lse, rows, a.splits, a.out, a.lse, s);
}

size_t workspace_of(bool coded, int dtype, int64_t batch, int heads, int kv_heads, int64_t table_width, int64_t n_pages, int page, int64_t frame,
                    int64_t window, int64_t sinks) {
  PagedArgs a = {};
  if (check_sizes("", dtype, batch, heads, kv_heads, table_width, n_pages, page, frame, window, sinks, a) || batch == 0) return 0;
  shape_of(a, keys_of_piece(dtype, coded));
  return part_bytes(a);
}

}  // namespace
}  // namespace bsga

using namespace bsga;

extern "C" {

size_t bsga_paged_attn_workspace_bytes(int dtype, int64_t batch, int heads, int kv_heads, int64_t table_width, int64_t n_pages, int page,
                                       int64_t frame, int64_t window, int64_t sinks) {
  return workspace_of(false, dtype, batch, heads, kv_heads, table_width, n_pages, page, frame, window, sinks);
}

int bsga_paged_attn(const void* q, int64_t q_batch, int64_t q_head, const void* k_cache, const void* v_cache, int dtype, int64_t batch, int heads,
                    int kv_heads, int head_dim, const int32_t* page_table, int64_t table_width, const int32_t* lengths, int64_t n_pages, int page,
                    float softmax_scale, int64_t frame, int64_t window, int64_t sinks, void* out, float* lse, void* workspace, size_t workspace_bytes,
                    void* stream) {
  return attend("bsga_paged_attn", false, q, q_batch, q_head, k_cache, v_cache, nullptr, nullptr, dtype, batch, heads, kv_heads, head_dim, page_table,
                table_width, lengths, n_pages, page, softmax_scale, frame, window, sinks, out, lse, workspace, workspace_bytes, stream);
}

size_t bsga_paged_attn_e4m3_workspace_bytes(int dtype, int64_t batch, int heads, int kv_heads, int64_t table_width, int64_t n_pages, int page,
                                            int64_t frame, int64_t window, int64_t sinks) {
  return workspace_of(true, dtype, batch, heads, kv_heads, table_width, n_pages, page, frame, window, sinks);
}

int bsga_paged_attn_e4m3(const void* q, int64_t q_batch, int64_t q_head, const void* k_cache, const void* v_cache, const uint8_t* k_scale,
                         const uint8_t* v_scale, int dtype, int64_t batch, int heads, int kv_heads, int head_dim, const int32_t* page_table,
                         int64_t table_width, const int32_t* lengths, int64_t n_pages, int page, float softmax_scale, int64_t frame, int64_t window,
                         int64_t sinks, void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  return attend("bsga_paged_attn_e4m3", true, q, q_batch, q_head, k_cache, v_cache, k_scale, v_scale, dtype, batch, heads, kv_heads, head_dim, page_table,
                table_width, lengths, n_pages, page, softmax_scale, frame, window, sinks, out, lse, workspace, workspace_bytes, stream);
}

}  // extern "C"
