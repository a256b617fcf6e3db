// Host side of appending with rotation and of spreading 4-bit rows out.
#include <algorithm>

#include "wkv_paged_host.cuh"
#include "wkv_paged_rows.cuh"

namespace wkv {
namespace host {
namespace {

template <typename T, int D, bool FOUR>
int append_typed(wkv_paged* c, AppendParams& P) {
  const PagedParams& A = P.A;
  constexpr int kSlots = RowsShape<D>::kSlots;
  static_assert(rows_smem<D, FOUR>() >= RowsShape<D>::kOffsets, "the queries' CTAs hold offsets and lengths there");
  long long entries = 0;
  if (A.q) {
    // heads per CTA: sixteen rows a thread where that leaves four CTAs an SM, else eight, four, two or one
    const int tokens = std::min(A.rows, kSlots), at_once = kSlots / tokens;
    const long long tiles = ((long long)A.rows + tokens - 1) / tokens;
    int steps = 16;
    while (steps > 1 && tiles * ((A.n_q_heads + at_once * steps - 1) / (at_once * steps)) < 4 * c->sm_count) steps >>= 1;
    P.q_heads = at_once * steps;
    const long long blocks = tiles * ((A.n_q_heads + P.q_heads - 1) / P.q_heads);
    if (blocks > 0x7fffffffLL) return fail(c, WKV_ERR_INVALID, "total_q * heads is too large");
    P.q_blocks = (int)blocks;
  }
  if (A.k) {
    P.kv_slots = A.q_start ? (A.rows >> A.page_shift) + 2 * A.batch : A.batch;
    if constexpr (FOUR) {
      P.kv_heads = 8;
      while (P.kv_heads > 1 && (long long)P.kv_slots * ((A.n_kv_heads + P.kv_heads - 1) / P.kv_heads) < 4 * c->sm_count) P.kv_heads >>= 1;
      P.kv_splits = (A.n_kv_heads + P.kv_heads - 1) / P.kv_heads;
      entries = (long long)P.kv_slots * P.kv_splits;
    } else {
      entries = ((long long)P.kv_slots * A.n_kv_heads + kRowsThreads / 32 - 1) / (kRowsThreads / 32);
    }
  }
  if (P.q_blocks + entries > 0x7fffffffLL) return fail(c, WKV_ERR_INVALID, "total_q * heads is too large");
  WKV_CUDA(c, launch(c, paged_rows_kernel<T, D, FOUR>, P.q_blocks + entries, kRowsThreads, (size_t)rows_smem<D, FOUR>(), P));
  return WKV_OK;
}
int append(wkv_paged* c, AppendParams& P) {
  if (P.A.batch == 0 || P.A.rows == 0 || (!P.A.q && !P.A.k)) return WKV_OK;
  const bool wide = c->cfg.head_dim == 128;
  switch (c->cfg.dtype) {
    case WKV_KV4: return wide ? append_typed<__nv_bfloat16, 128, true>(c, P) : append_typed<__nv_bfloat16, 64, true>(c, P);
    case WKV_BF16: return wide ? append_typed<__nv_bfloat16, 128, false>(c, P) : append_typed<__nv_bfloat16, 64, false>(c, P);
    default: return wide ? append_typed<float, 128, false>(c, P) : append_typed<float, 64, false>(c, P);
  }
}

}  // namespace

cudaError_t prepare_rows(wkv_paged* c) {
  if (c->cfg.dtype != WKV_KV4) return cudaSuccess;
  return c->cfg.head_dim == 128 ? cudaFuncSetAttribute(paged_rows_kernel<__nv_bfloat16, 128, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, rows_smem<128, true>())
                                : cudaFuncSetAttribute(paged_rows_kernel<__nv_bfloat16, 64, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, rows_smem<64, true>());
}

int append_rows(wkv_paged* c, const PagedParams& A) {
  AppendParams P;
  std::memset(&P, 0, sizeof(P));
  P.A = A;
  P.A.q = nullptr;
  return append(c, P);
}

}  // namespace host
}  // namespace wkv

using namespace wkv::host;

extern "C" {

int wkv_paged_append(wkv_paged* c, int32_t layer, int32_t batch, const void* q, int64_t q_stride, const void* k, const void* v,
                     int64_t kv_stride, const int32_t* q_start, int32_t total_q, const int32_t* block_table, int32_t table_width,
                     const int32_t* seq_lens, const float* rope, int32_t rope_rows, int32_t rope_dim, int32_t rope_paired,
                     const int32_t* positions, void* q_out, int64_t q_out_stride, int8_t* page_bounds, float* page_scale) {
  if (!c) return WKV_ERR_INVALID;
  DeviceGuard on(c->device);
  WKV_CUDA(c, on.err);
  const wkv_paged_config& f = c->cfg;
  wkv::AppendParams P;
  std::memset(&P, 0, sizeof(P));
  int rc = cache_params(c, P.A, layer, batch, total_q, k, v, kv_stride, block_table, table_width, seq_lens);
  if (rc != WKV_OK) return rc;
  if (total_q > (1 << 24)) return fail(c, WKV_ERR_INVALID, "total_q must be at most 2^24");
  if (!q_start && total_q != batch) return fail(c, WKV_ERR_INVALID, "without q_start there is one token per sequence: total_q must be batch");
  if ((q == nullptr) != (q_out == nullptr)) return fail(c, WKV_ERR_INVALID, "q and q_out must both be given or both be NULL");
  if (q) {
    const int64_t row = (int64_t)f.n_q_heads * f.head_dim;
    if (q_stride == 0) q_stride = row;
    if (q_out_stride == 0) q_out_stride = row;
    if (q_stride < row || q_out_stride < row) return fail(c, WKV_ERR_INVALID, "a row stride is smaller than the row");
    if (q_stride * (int64_t)c->elem % 16 || q_out_stride * (int64_t)c->elem % 16 || !aligned16(q) || !aligned16(q_out))
      return fail(c, WKV_ERR_INVALID, "rows of q and q_out must be 16-byte aligned");
    if (q == q_out && q_stride != q_out_stride) return fail(c, WKV_ERR_INVALID, "queries turned in place keep their row stride");
    P.A.q = q; P.A.q_stride = q_stride; P.q_out = q_out; P.q_out_stride = q_out_stride;
  }
  if (rope) {
    if (!aligned16(rope)) return fail(c, WKV_ERR_INVALID, "rope must be 16-byte aligned");
    if (rope_rows < 1) return fail(c, WKV_ERR_INVALID, "rope_rows must be >= 1");
    if (rope_dim < 16 || rope_dim > f.head_dim || rope_dim % 16) return fail(c, WKV_ERR_INVALID, "rope_dim must be a multiple of 16 in [16, head_dim]");
    if (rope_paired != 0 && rope_paired != 1) return fail(c, WKV_ERR_INVALID, "rope_paired must be 0 or 1");
    P.rope = rope; P.rope_rows = rope_rows; P.rope_dim = rope_dim; P.paired = rope_paired;
    P.positions = positions;
  }
  if ((page_bounds == nullptr) != (page_scale == nullptr)) return fail(c, WKV_ERR_INVALID, "page_bounds and page_scale must both be given or both be NULL");
  if (page_bounds) {
    if (!k && total_q > 0) return fail(c, WKV_ERR_INVALID, "page bounds need k and v");      // (an empty tensor's address may be NULL)
    if (!aligned16(page_bounds)) return fail(c, WKV_ERR_INVALID, "page_bounds must be 16-byte aligned");
    const size_t chunks = (size_t)layer * f.n_pages * f.n_kv_heads;
    P.bounds = page_bounds + chunks * 2 * f.head_dim;
    P.bound_scale = page_scale + chunks;
  }
  P.A.q_start = q_start;
  return append(c, P);
}

int wkv_paged_expand(wkv_paged* c, int32_t layer, int32_t batch, const int32_t* block_table, int32_t table_width, const int32_t* seq_lens,
                     wkv_paged* dst, int32_t dst_layer, const int32_t* dst_table, int32_t dst_width) {
  if (!c) return WKV_ERR_INVALID;
  DeviceGuard on(c->device);
  WKV_CUDA(c, on.err);
  const wkv_paged_config& f = c->cfg;
  if (f.dtype != WKV_KV4) return fail(c, WKV_ERR_INVALID, "the cache that is spread out must hold rows in 4 bits");
  if (!dst) return fail(c, WKV_ERR_INVALID, "dst must not be NULL");
  const wkv_paged_config& g = dst->cfg;
  if (g.dtype != WKV_BF16 || g.n_kv_heads != f.n_kv_heads || g.head_dim != f.head_dim || dst->device != c->device)
    return fail(c, WKV_ERR_INVALID, "dst must hold bf16 rows with the same kv heads and head_dim on the same device");
  if (dst_layer < 0 || dst_layer >= g.n_layers) return fail(c, WKV_ERR_INVALID, "dst_layer out of range");
  wkv::ExpandParams P;
  std::memset(&P, 0, sizeof(P));
  const int rc = cache_params(c, P.A, layer, batch, batch, nullptr, nullptr, 0, block_table, table_width, seq_lens);
  if (rc != WKV_OK) return rc;
  if (dst_width < 1) return fail(c, WKV_ERR_INVALID, "dst_width must be >= 1");
  if (batch == 0) return WKV_OK;
  if (!dst_table) return fail(c, WKV_ERR_INVALID, "dst_table must not be NULL");
  const size_t layer_bytes = (size_t)g.n_pages * g.n_kv_heads * dst->chunk_bytes;
  P.k_to = reinterpret_cast<__nv_bfloat16*>((char*)dst->k_pool + dst_layer * layer_bytes);
  P.v_to = reinterpret_cast<__nv_bfloat16*>((char*)dst->v_pool + dst_layer * layer_bytes);
  P.to_table = dst_table; P.to_width = dst_width; P.to_pages = g.n_pages; P.to_page = g.page_size; P.to_shift = dst->page_shift;
  P.blocks = (table_width * f.page_size + 63) / 64;
  const long long grid = (long long)batch * f.n_kv_heads * P.blocks;
  if (grid > 0x7fffffffLL) return fail(c, WKV_ERR_INVALID, "batch * n_kv_heads * table_width is too large");
  WKV_CUDA(c, f.head_dim == 128 ? launch(c, wkv::paged_expand_kernel<128>, grid, wkv::kRowsThreads, 0, P)
                                : launch(c, wkv::paged_expand_kernel<64>, grid, wkv::kRowsThreads, 0, P));
  return WKV_OK;
}

}  // extern "C"
