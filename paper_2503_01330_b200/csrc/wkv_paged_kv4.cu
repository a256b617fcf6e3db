// Host side of decode attention on rows in 4 bits.
#include "wkv_paged_host.cuh"
#include "wkv_paged_decode_kv4.cuh"

namespace wkv {
namespace host {
namespace {

template <int D, int G>
cudaError_t pick(wkv_paged* c) {
  auto whole = paged_decode_kv4_kernel<D, G, false>, chosen = paged_decode_kv4_kernel<D, G, true>;
  c->decode_kernel = (const void*)whole;
  c->pages_kernel = (const void*)chosen;
  c->decode_smem = Kv4Shape<D, G>::kSmem;
  cudaError_t e = cudaFuncSetAttribute(whole, cudaFuncAttributeMaxDynamicSharedMemorySize, c->decode_smem);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(chosen, cudaFuncAttributeMaxDynamicSharedMemorySize, c->decode_smem);
  int per_sm = 0;
  if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, whole, kKv4Threads, c->decode_smem);
  c->decode_ctas = c->sm_count * (per_sm < 1 ? 1 : per_sm);
  return e;
}
template <int D>
cudaError_t pick_by_group(wkv_paged* c) {
  switch (c->group) {
    case 1: return pick<D, 1>(c);
    case 2: return pick<D, 2>(c);
    case 4: return pick<D, 4>(c);
    default: return pick<D, 8>(c);
  }
}

}  // namespace

cudaError_t pick_kv4(wkv_paged* c) { return c->cfg.head_dim == 128 ? pick_by_group<128>(c) : pick_by_group<64>(c); }

int decode_kv4(wkv_paged* c, const PagedParams& A, const int32_t* pages, int n_select) {
  DecodeParams P;
  std::memset(&P, 0, sizeof(P));
  P.A = A;
  P.part = c->part; P.part_ml = c->part_ml; P.arrived = c->arrived;
  P.pages = pages; P.n_select = n_select;
  typedef void (*decode_fn)(const DecodeParams);
  WKV_CUDA(c, launch(c, (decode_fn)(pages ? c->pages_kernel : c->decode_kernel), c->decode_ctas, kKv4Threads, c->decode_smem, P));
  return WKV_OK;
}

}  // namespace host
}  // namespace wkv
