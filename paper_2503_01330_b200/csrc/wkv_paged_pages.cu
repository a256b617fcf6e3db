// Host side of choosing pages and of decode attention over chosen ones.
#include <algorithm>

#include "wkv_paged_host.cuh"
#include "wkv_paged_choose.cuh"
#include "wkv_paged_decode.cuh"

namespace wkv {
namespace host {
namespace {

template <typename T, int D, int G>
cudaError_t pick(wkv_paged* c) {
  auto kernel = paged_decode_kernel<T, D, G, true>;
  c->pages_kernel = (const void*)kernel;
  return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, decode_smem<T, D, G>());
}
template <typename T, int D>
cudaError_t pick_by_group(wkv_paged* c) {
  switch (c->group) {
    case 1: return pick<T, D, 1>(c);
    case 2: return pick<T, D, 2>(c);
    case 4: return pick<T, D, 4>(c);
    default: return pick<T, D, 8>(c);
  }
}

}  // namespace

namespace {
typedef void (*choose_fn)(const ChooseParams);
choose_fn choose_kernel(const wkv_paged* c) {
  const bool wide = c->cfg.head_dim == 128;
  return c->cfg.dtype == WKV_F32 ? (wide ? paged_choose_kernel<float, 128> : paged_choose_kernel<float, 64>)
                                 : (wide ? paged_choose_kernel<__nv_bfloat16, 128> : paged_choose_kernel<__nv_bfloat16, 64>);
}
}  // namespace

cudaError_t pick_pages(wkv_paged* c) {
  const bool wide = c->cfg.head_dim == 128;
  if (c->cfg.dtype == WKV_BF16) return wide ? pick_by_group<__nv_bfloat16, 128>(c) : pick_by_group<__nv_bfloat16, 64>(c);
  return wide ? pick_by_group<float, 128>(c) : pick_by_group<float, 64>(c);
}

}  // namespace host
}  // namespace wkv

using namespace wkv::host;

extern "C" {

int wkv_paged_select(wkv_paged* c, int32_t layer, int32_t batch, const void* q, int64_t q_stride, const int32_t* block_table,
                     int32_t table_width, const int32_t* seq_lens, const int8_t* page_bounds, const float* page_scale, int32_t n_select,
                     int32_t recent, int32_t sink, float* page_scores, int64_t page_score_stride, int32_t* pages) {
  if (!c) return WKV_ERR_INVALID;
  DeviceGuard on(c->device);
  WKV_CUDA(c, on.err);
  const wkv_paged_config& f = c->cfg;
  wkv::ChooseParams P;
  std::memset(&P, 0, sizeof(P));
  int rc = cache_params(c, P.A, layer, batch, batch, nullptr, nullptr, 0, block_table, table_width, seq_lens);
  if (rc == WKV_OK) rc = query_params(c, P.A, q, q_stride, const_cast<void*>(q), nullptr);
  if (rc != WKV_OK) return rc;
  if (n_select < 1 || n_select > (1 << 20)) return fail(c, WKV_ERR_INVALID, "n_select must be in [1, 2^20]");
  if (recent < 1 || sink < 0 || (int64_t)recent + sink > n_select) return fail(c, WKV_ERR_INVALID, "recent must be >= 1, sink >= 0 and recent + sink <= n_select");
  if (page_score_stride < table_width) return fail(c, WKV_ERR_INVALID, "page_score_stride must be >= table_width");
  if (batch == 0) return WKV_OK;
  if (!page_bounds || !page_scale || !page_scores || !pages)
    return fail(c, WKV_ERR_INVALID, "page_bounds, page_scale, page_scores and pages must not be NULL");
  if (!aligned16(page_bounds)) return fail(c, WKV_ERR_INVALID, "page_bounds must be 16-byte aligned");
  const size_t chunks = (size_t)layer * f.n_pages * f.n_kv_heads;
  P.bounds = page_bounds + chunks * 2 * f.head_dim;
  P.bound_scale = page_scale + chunks;
  P.page_scores = page_scores; P.page_score_stride = page_score_stride; P.pages = pages; P.arrived = c->arrived;
  P.n_select = n_select; P.recent = recent; P.sink = sink;
  // CTAs per lane: 64 pages each at least, two CTAs an SM in all where the lanes are few
  const long long lanes = (long long)batch * f.n_kv_heads;
  P.splits = (int)std::max<long long>(1, std::min<long long>((table_width + 63) / 64, 2 * c->sm_count / lanes));
  WKV_CUDA(c, launch(c, choose_kernel(c), lanes * P.splits, wkv::kChooseThreads, 0, P));
  return WKV_OK;
}

int wkv_paged_decode_pages(wkv_paged* c, int32_t layer, int32_t batch, const void* q, int64_t q_stride, const int32_t* block_table,
                           int32_t table_width, const int32_t* seq_lens, const int32_t* pages, int32_t n_select, void* out, float* lse) {
  if (!c) return WKV_ERR_INVALID;
  DeviceGuard on(c->device);
  WKV_CUDA(c, on.err);
  const wkv_paged_config& f = c->cfg;
  wkv::PagedParams A;
  int rc = cache_params(c, A, layer, batch, batch, nullptr, nullptr, 0, block_table, table_width, seq_lens);
  if (rc == WKV_OK) rc = query_params(c, A, q, q_stride, out, lse);
  if (rc != WKV_OK) return rc;
  if (n_select < 1 || n_select > (1 << 20)) return fail(c, WKV_ERR_INVALID, "n_select must be in [1, 2^20]");
  if (batch == 0) return WKV_OK;
  if (!pages) return fail(c, WKV_ERR_INVALID, "pages must not be NULL");
  if (f.dtype == WKV_KV4) return decode_kv4(c, A, pages, n_select);
  wkv::DecodeParams P;
  std::memset(&P, 0, sizeof(P));
  P.A = A;
  P.part = c->part; P.part_ml = c->part_ml; P.arrived = c->arrived;
  P.pages = pages; P.n_select = n_select;
  P.oob_chunk = f.n_layers * f.n_pages * f.n_kv_heads;
  P.chunk0 = chunk0(c, A);
  std::memcpy(P.kmap, c->page_kmap, 128);
  std::memcpy(P.vmap, c->page_vmap, 128);
  typedef void (*decode_fn)(const wkv::DecodeParams);
  WKV_CUDA(c, launch(c, (decode_fn)c->pages_kernel, c->decode_ctas, wkv::kDecodeThreads, c->decode_smem, P));
  return WKV_OK;
}

}  // extern "C"
