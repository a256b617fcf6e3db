// Host side of the paged cache declared in include/wkv.h: configuration checks, workspaces, launches.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <new>
#include <string>
#include <vector>

#include <cuda.h>                      // tensor-map types only; the driver entry point is looked up at run time

#include "../../include/wkv.h"
#include "wkv_paged.cuh"
#include "wkv_paged_decode.cuh"
#include "wkv_paged_prefill.cuh"
#include "wkv_paged_f32.cuh"

struct wkv_paged {
  wkv_paged_config cfg;
  int device = 0;
  int sm_count = 148;
  int group = 1;
  int page_shift = 4;
  float scale = 0.f;
  size_t elem = 2;
  cudaStream_t stream = nullptr;
  void* k_pool = nullptr;
  void* v_pool = nullptr;
  uint32_t* status = nullptr;
  float* logits = nullptr;             // [max_batch][Hq][max_pages * page_size]: a decode step's; kept indexes of an eviction
  float2* head_ml = nullptr;           // [max_batch][Hq]: a decode step's (max, 1 / sum), for the weights
  // decode: partials of the pieces, arrivals per lane
  const void* decode_kernel = nullptr;
  const void* fold_kernel = nullptr;
  int decode_ctas = 0, decode_smem = 0;
  float* part = nullptr;
  float2* part_ml = nullptr;
  uint32_t* arrived = nullptr;
  // prompts: the runs' outputs, next item
  float4* run_part = nullptr;
  float2* run_ml = nullptr;
  uint32_t* item_counter = nullptr;
  // the pools as [chunk][part][row][128 bytes], boxes of a page's rows (at most a decode tile's) x all parts
  alignas(64) unsigned char page_kmap[128] = {};
  alignas(64) unsigned char page_vmap[128] = {};
  // ... in boxes of one part, for prompts on bf16 rows
  alignas(64) unsigned char part_kmap[128] = {};
  alignas(64) unsigned char part_vmap[128] = {};
  void* encode = nullptr;              // the driver's cuTensorMapEncodeTiled
  int32_t* n_moved = nullptr;          // [max_batch][Hkv]
  std::vector<void*> owned;
  long long device_bytes = 0;
  long long launches = 0;
  std::string last_error;
};

namespace {

int fail(wkv_paged* c, int code, const std::string& msg) {
  if (c) c->last_error = msg;
  return code;
}
int cuda_fail(wkv_paged* c, cudaError_t e, const char* what) {
  return fail(c, WKV_ERR_CUDA, std::string(what) + ": " + cudaGetErrorString(e));
}
#define WKV_CUDA(ctx, expr)                                   \
  do {                                                        \
    cudaError_t e_ = (expr);                                  \
    if (e_ != cudaSuccess) return cuda_fail(ctx, e_, #expr);  \
  } while (0)

// Calls may come with another device current than the handle's.
struct DeviceGuard {
  int was = -1;
  cudaError_t err;
  explicit DeviceGuard(int device) {
    err = cudaGetDevice(&was);
    if (err == cudaSuccess && was != device) err = cudaSetDevice(device); else was = -1;
  }
  ~DeviceGuard() { if (was >= 0) cudaSetDevice(was); }
};

void* default_alloc(size_t bytes, void*) {
  void* p = nullptr;
  if (cudaMalloc(&p, bytes) != cudaSuccess) return nullptr;
  return p;
}
void default_release(void* p, void*) { cudaFree(p); }

template <typename P>
int take(wkv_paged* c, P** dst, size_t bytes) {
  bytes = (bytes + 255) & ~(size_t)255;
  void* p = c->cfg.alloc(bytes, c->cfg.user);
  if (!p) return fail(c, WKV_ERR_ALLOC, "device memory provider returned NULL for " + std::to_string(bytes) + " bytes");
  c->owned.push_back(p);
  c->device_bytes += (long long)bytes;
  *dst = reinterpret_cast<P*>(p);
  return WKV_OK;
}

const char* check_config(const wkv_paged_config* c) {
  if (!c) return "config is NULL";
  if (c->n_layers < 1 || c->n_pages < 1) return "n_layers and n_pages must be >= 1";
  if (c->page_size != 16 && c->page_size != 32 && c->page_size != 64) return "page_size must be 16, 32 or 64";
  if (c->n_kv_heads < 1 || c->n_q_heads < 1 || c->n_q_heads % c->n_kv_heads) return "n_q_heads must be a positive multiple of n_kv_heads";
  const int g = c->n_q_heads / c->n_kv_heads;
  if (g != 1 && g != 2 && g != 4 && g != 8) return "n_q_heads / n_kv_heads must be 1, 2, 4 or 8";
  if (c->n_q_heads > 1024) return "n_q_heads must be <= 1024";
  if (c->head_dim != 64 && c->head_dim != 128) return "head_dim must be 64 or 128";
  if (c->max_batch < 1 || c->max_batch > 1024) return "max_batch must be in [1, 1024]";
  if (c->max_pages < 1 || (long long)c->max_pages * c->page_size > (1 << 24)) return "max_pages must be >= 1 and max_pages * page_size at most 2^24";
  if ((long long)c->n_layers * c->n_pages >= 0x7fffffffLL / c->n_kv_heads) return "n_layers * n_pages * n_kv_heads must stay below 2^31";
  if (c->dtype != WKV_F32 && c->dtype != WKV_BF16) return "dtype must be WKV_F32 or WKV_BF16";
  if (!(c->scale >= 0.f) || std::isinf(c->scale)) return "scale must be finite and >= 0";
  if (c->scores != 0 && c->scores != 1) return "scores must be 0 or 1";
  if ((c->k_pool == nullptr) != (c->v_pool == nullptr)) return "k_pool and v_pool must both be set or both be NULL";
  if (((uintptr_t)c->k_pool | (uintptr_t)c->v_pool) & 15) return "k_pool and v_pool must be 16-byte aligned";
  if ((c->alloc == nullptr) != (c->release == nullptr)) return "alloc and release must both be set or both be NULL";
  return nullptr;
}

// Tensor maps: 4-d, the innermost dimension 128 bytes wide, 128-byte swizzle, zeros outside.
int encode_map(wkv_paged* c, unsigned char* out128, const void* base, const cuuint64_t (&dims)[4], const cuuint64_t (&strides)[3],
               const cuuint32_t (&box)[4]) {
  typedef CUresult (*encode_fn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  static_assert(sizeof(CUtensorMap) == 128, "tensor map size");
  if (!c->encode) {
    cudaDriverEntryPointQueryResult qr = cudaDriverEntryPointSymbolNotFound;
    const cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &c->encode, cudaEnableDefault, &qr);
    if (e != cudaSuccess) return cuda_fail(c, e, "cudaGetDriverEntryPoint(cuTensorMapEncodeTiled)");
    if (qr != cudaDriverEntryPointSuccess || !c->encode) return fail(c, WKV_ERR_CUDA, "the driver has no cuTensorMapEncodeTiled");
  }
  const cuuint32_t estr[4] = {1u, 1u, 1u, 1u};
  CUtensorMap m;
  const CUresult r = reinterpret_cast<encode_fn>(c->encode)(
      &m, c->cfg.dtype == WKV_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, const_cast<void*>(base), dims, strides,
      box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) return fail(c, WKV_ERR_CUDA, "cuTensorMapEncodeTiled failed with code " + std::to_string((int)r));
  std::memcpy(out128, &m, sizeof(m));
  return WKV_OK;
}
// A pool: 128 bytes of a row, rows of a chunk, the row's 128-byte parts, chunks; boxes of box_rows rows x box_parts parts.
int encode_pool(wkv_paged* c, unsigned char* out128, void* pool, int box_rows, int box_parts) {
  const wkv_paged_config& f = c->cfg;
  const cuuint64_t row = (cuuint64_t)f.head_dim * c->elem;
  const cuuint32_t elems = (cuuint32_t)(128 / c->elem);
  return encode_map(c, out128, pool, {elems, (cuuint64_t)f.page_size, row / 128, (cuuint64_t)f.n_layers * f.n_pages * f.n_kv_heads},
                    {row, 128, row * f.page_size}, {elems, (cuuint32_t)box_rows, (cuuint32_t)box_parts, 1u});
}
// A call's q, k or v ([tokens][heads][D], tokens `stride` elements apart): 128 bytes of a row, heads, tokens, parts; boxes of
// box_heads x box_tokens rows x one part.
int encode_rows(wkv_paged* c, unsigned char* out128, const void* base, int64_t stride, int heads, int tokens, int box_heads, int box_tokens) {
  const cuuint64_t row = (cuuint64_t)c->cfg.head_dim * c->elem;
  const cuuint32_t elems = (cuuint32_t)(128 / c->elem);
  return encode_map(c, out128, base, {elems, (cuuint64_t)heads, (cuuint64_t)tokens, row / 128}, {row, (cuuint64_t)stride * c->elem, 128},
                    {elems, (cuuint32_t)box_heads, (cuuint32_t)box_tokens, 1u});
}

// Rows of partial outputs that the runs of a prompt call may have: two row blocks per SM on bf16 rows, eight of the smaller ones on
// fp32 rows.
size_t run_rows(const wkv_paged* c) {
  return (size_t)c->sm_count * (c->cfg.dtype == WKV_BF16 ? 2 * wkv::kPrefillRows : 8 * wkv::kF32Rows);
}

// Picks this handle's instantiations and how many decode CTAs the GPU holds at once.
template <typename T, int D, int G>
cudaError_t pick_kernels(wkv_paged* c) {
  auto kernel = wkv::paged_decode_kernel<T, D, G>;
  c->decode_kernel = (const void*)kernel;
  c->fold_kernel = (const void*)wkv::paged_fold_kernel<G>;
  c->decode_smem = wkv::decode_smem<T, D, G>();
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, c->decode_smem);
  int per_sm = 0;
  if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, wkv::kDecodeThreads, c->decode_smem);
  c->decode_ctas = c->sm_count * (per_sm < 1 ? 1 : per_sm);
  if constexpr (sizeof(T) == 4) {
    if (e == cudaSuccess) e = cudaFuncSetAttribute(wkv::paged_prefill_f32_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, wkv::F32Shape<D>::kSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(wkv::paged_weights_f32_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, wkv::F32Shape<D>::kWeightsSmem);
  }
  if constexpr (sizeof(T) == 2) {
    if (e == cudaSuccess)
      e = cudaFuncSetAttribute(wkv::paged_prefill_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, wkv::PrefillShape<D>::kSmem);
    if (e == cudaSuccess)
      e = cudaFuncSetAttribute(wkv::paged_weights_tc_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, wkv::WeightsShape<D>::kSmem);
  }
  return e;
}
template <typename T, int D>
cudaError_t pick_by_group(wkv_paged* c) {
  switch (c->group) {
    case 1: return pick_kernels<T, D, 1>(c);
    case 2: return pick_kernels<T, D, 2>(c);
    case 4: return pick_kernels<T, D, 4>(c);
    default: return pick_kernels<T, D, 8>(c);
  }
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// Arguments that decode and prefill share; fills P.  `rows`: rows of q.
int attention_params(wkv_paged* c, wkv::PagedParams& P, int32_t layer, int32_t batch, int32_t rows, const void* q, int64_t q_stride,
                     const void* k, const void* v, int64_t kv_stride, const int32_t* table, int32_t width, const int32_t* seq_lens,
                     int32_t window, int32_t sink, float* scores, int64_t score_stride, void* out, float* lse) {
  const wkv_paged_config& f = c->cfg;
  if (layer < 0 || layer >= f.n_layers) return fail(c, WKV_ERR_INVALID, "layer out of range");
  if (batch < 0 || batch > f.max_batch) return fail(c, WKV_ERR_INVALID, "batch must be in [0, max_batch]");
  if (rows < 0) return fail(c, WKV_ERR_INVALID, "the number of rows must be >= 0");
  if (width < 1 || width > f.max_pages) return fail(c, WKV_ERR_INVALID, "table_width must be in [1, max_pages]");
  if (window < 0 || sink < 0) return fail(c, WKV_ERR_INVALID, "window and sink must be >= 0");
  if ((k == nullptr) != (v == nullptr)) return fail(c, WKV_ERR_INVALID, "k and v must both be given or both be NULL");
  if (batch > 0 && rows > 0 && (!q || !table || !seq_lens || !out)) return fail(c, WKV_ERR_INVALID, "q, block_table, seq_lens and out must not be NULL");
  const int64_t q_row = (int64_t)f.n_q_heads * f.head_dim, kv_row = (int64_t)f.n_kv_heads * f.head_dim;
  if (q_stride == 0) q_stride = q_row;
  if (kv_stride == 0) kv_stride = kv_row;
  if (q_stride < q_row || kv_stride < kv_row) return fail(c, WKV_ERR_INVALID, "a row stride is smaller than the row");
  if (q_stride * (int64_t)c->elem % 16 || kv_stride * (int64_t)c->elem % 16 || !aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out))
    return fail(c, WKV_ERR_INVALID, "rows of q, k, v and out must be 16-byte aligned");
  if (scores) {
    if (!f.scores) return fail(c, WKV_ERR_INVALID, "scores need a handle created with scores = 1");
    if (score_stride < (int64_t)width * f.page_size) return fail(c, WKV_ERR_INVALID, "score_stride must be >= table_width * page_size");
  }
  std::memset(&P, 0, sizeof(P));
  const size_t layer_bytes = (size_t)f.n_pages * f.n_kv_heads * f.page_size * f.head_dim * c->elem;
  P.k_pool = (char*)c->k_pool + layer * layer_bytes;
  P.v_pool = (char*)c->v_pool + layer * layer_bytes;
  P.q = q; P.k = k; P.v = v; P.q_stride = q_stride; P.kv_stride = kv_stride;
  P.table = table; P.seq_lens = seq_lens; P.out = out; P.lse = lse; P.scores = scores; P.score_stride = score_stride;
  P.status = c->status; P.batch = batch; P.rows = rows; P.width = width; P.n_pages = f.n_pages;
  P.n_q_heads = f.n_q_heads; P.n_kv_heads = f.n_kv_heads; P.page = f.page_size; P.page_shift = c->page_shift;
  P.window = window; P.sink = sink; P.scale_log2 = c->scale * wkv::kLog2e;
  return WKV_OK;
}

// All launches: programmatic stream serialization, each kernel waits for its predecessor first thing.
template <typename... A, typename... B>
cudaError_t launch(wkv_paged* c, void (*kernel)(A...), long long grid, int threads, size_t smem, B&&... args) {
  if (grid < 1 || grid > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
  cudaLaunchConfig_t lc = {};
  lc.gridDim = dim3((unsigned)grid);
  lc.blockDim = dim3((unsigned)threads);
  lc.dynamicSmemBytes = smem;
  lc.stream = c->stream;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  lc.attrs = at;
  lc.numAttrs = 1;
  c->launches++;
  return cudaLaunchKernelEx(&lc, kernel, std::forward<B>(args)...);
}

// The layer's first chunk.
int chunk0(const wkv_paged* c, const wkv::PagedParams& P) {
  return (int)(((char*)P.k_pool - (char*)c->k_pool) / ((size_t)P.page * c->cfg.head_dim * c->elem));
}

int decode(wkv_paged* c, const wkv::PagedParams& A) {
  if (A.batch == 0) return WKV_OK;
  wkv::DecodeParams P;
  std::memset(&P, 0, sizeof(P));
  P.A = A;
  P.part = c->part; P.part_ml = c->part_ml; P.arrived = c->arrived;
  P.logits = A.scores ? c->logits : nullptr;
  P.head_ml = c->head_ml;
  P.fold_inside = A.scores && A.width * A.page <= wkv::kFoldInside;
  P.oob_chunk = c->cfg.n_layers * c->cfg.n_pages * c->cfg.n_kv_heads;
  P.chunk0 = chunk0(c, A);
  std::memcpy(P.kmap, c->page_kmap, 128);
  std::memcpy(P.vmap, c->page_vmap, 128);
  typedef void (*decode_fn)(const wkv::DecodeParams);
  typedef void (*fold_fn)(const wkv::DecodeParams, int);
  cudaError_t e = launch(c, (decode_fn)c->decode_kernel, c->decode_ctas, wkv::kDecodeThreads, c->decode_smem, P);
  if (e == cudaSuccess && A.scores && !P.fold_inside) {
    const int per_lane = (A.width * A.page + wkv::kFoldEntries - 1) / wkv::kFoldEntries;
    e = launch(c, (fold_fn)c->fold_kernel, (long long)A.batch * A.n_kv_heads * per_lane, wkv::kFoldEntries / 4, 0, P, per_lane);
  }
  WKV_CUDA(c, e);
  return WKV_OK;
}

// What the prompt kernels share.  units: row blocks (of `rows` rows) x kv heads, at most; items: with the runs that they may be cut
// into (see work_plan), at most.  A call whose tokens alone make row blocks enough for half the slots is not cut.
int prefill_params(wkv_paged* c, wkv::PrefillParams& P, const wkv::PagedParams& A, int rows, int keys, long long* units, long long* items) {
  std::memset(&P, 0, sizeof(P));
  P.A = A;
  P.g_shift = c->group == 1 ? 0 : c->group == 2 ? 1 : c->group == 4 ? 2 : 3;
  const long long slots = (long long)(run_rows(c) / rows), full = (long long)A.rows * c->group / rows;
  if (2 * A.n_kv_heads * std::max(1LL, full - A.batch) <= slots) P.slots = (int)slots;
  *units = (full + A.batch) * A.n_kv_heads;
  if (*units > 0x3fffffff) return fail(c, WKV_ERR_INVALID, "total_q * n_q_heads is too large");
  const long long tiles = ((long long)A.width * A.page + keys - 1) / keys;
  *items = std::max<long long>(*units, std::min<long long>(P.slots, *units * tiles));
  // An item may walk the whole table, at 1.6 us a tile of 128 entries and more at low clocks: 20 us a tile, 131072 tiles at most.
  P.polls = wkv::kWaitPolls + (uint32_t)((long long)A.width * A.page / 128 * 4);
  P.counter = c->item_counter; P.part = c->run_part; P.part_ml = c->run_ml;
  P.oob_chunk = c->cfg.n_layers * c->cfg.n_pages * c->cfg.n_kv_heads;
  P.chunk0 = chunk0(c, A);
  return WKV_OK;
}

// Prompt attention on bf16 rows (tensor cores) ...
template <int D>
int prefill_bf16(wkv_paged* c, const wkv::PagedParams& A) {
  wkv::PrefillParams P;
  long long units, items;
  int rc = prefill_params(c, P, A, wkv::kPrefillRows, wkv::kPrefillKeys, &units, &items);
  if (rc == WKV_OK) rc = encode_rows(c, P.qmap, A.q, A.q_stride, A.n_q_heads, A.rows, c->group, 128 / c->group);
  if (rc == WKV_OK && A.k) {
    P.append = 1;
    rc = encode_rows(c, P.kinmap, A.k, A.kv_stride, A.n_kv_heads, A.rows, 1, A.page);
    if (rc == WKV_OK) rc = encode_rows(c, P.vinmap, A.v, A.kv_stride, A.n_kv_heads, A.rows, 1, A.page);
  }
  if (rc != WKV_OK) return rc;
  if (A.k) WKV_CUDA(c, launch(c, wkv::paged_append_edge_kernel<__nv_bfloat16, D>, (long long)A.batch * A.page, wkv::kAppendThreads, 0, A));
  std::memcpy(P.kmap, c->part_kmap, 128);
  std::memcpy(P.vmap, c->part_vmap, 128);
  WKV_CUDA(c, launch(c, wkv::paged_prefill_kernel<D>, (int)std::min<long long>(items, c->sm_count), wkv::kPrefillThreads, wkv::PrefillShape<D>::kSmem, P));
  if (P.slots) WKV_CUDA(c, launch(c, wkv::paged_prefill_join_kernel<__nv_bfloat16, D, wkv::kPrefillRows, wkv::kPrefillKeys>, units * (wkv::kPrefillRows / 32), 256, 0, P));
  if (A.scores) {
    const long long blocks = ((long long)A.width * A.page + 255) / 256;
    WKV_CUDA(c, launch(c, wkv::paged_weights_tc_kernel<D>, blocks * A.batch * A.n_kv_heads, wkv::kWeightsThreads, wkv::WeightsShape<D>::kSmem, P));
  }
  return WKV_OK;
}
// ... and on fp32 rows.
template <int D>
int prefill_f32(wkv_paged* c, const wkv::PagedParams& A) {
  wkv::PrefillParams P;
  long long units, items;
  const int rc = prefill_params(c, P, A, wkv::kF32Rows, wkv::kF32Keys, &units, &items);
  if (rc != WKV_OK) return rc;
  if (A.k) WKV_CUDA(c, launch(c, wkv::paged_append_kernel<float, D>, A.rows, wkv::kAppendThreads, 0, A));
  WKV_CUDA(c, launch(c, wkv::paged_prefill_f32_kernel<D>, items, wkv::kF32Threads, wkv::F32Shape<D>::kSmem, P));
  if (P.slots) WKV_CUDA(c, launch(c, wkv::paged_prefill_join_kernel<float, D, wkv::kF32Rows, wkv::kF32Keys>, units * (wkv::kF32Rows / 32), 256, 0, P));
  if (A.scores) {
    const long long blocks = ((long long)A.width * A.page + wkv::kF32Rows - 1) / wkv::kF32Rows;
    WKV_CUDA(c, launch(c, wkv::paged_weights_f32_kernel<D>, blocks * A.batch * A.n_kv_heads, wkv::kF32Groups * wkv::kF32Threads, wkv::F32Shape<D>::kWeightsSmem, P));
  }
  return WKV_OK;
}

int prefill(wkv_paged* c, const wkv::PagedParams& P) {
  if (P.batch == 0 || P.rows == 0) return WKV_OK;
  const bool wide = c->cfg.head_dim == 128;
  if (c->cfg.dtype == WKV_BF16) return wide ? prefill_bf16<128>(c, P) : prefill_bf16<64>(c, P);
  return wide ? prefill_f32<128>(c, P) : prefill_f32<64>(c, P);
}

}  // namespace

extern "C" {

const char* wkv_paged_config_error(const wkv_paged_config* cfg) { return check_config(cfg); }

int wkv_paged_create(const wkv_paged_config* cfg, wkv_paged** out) {
  if (!out) return WKV_ERR_INVALID;
  *out = nullptr;
  if (check_config(cfg) != nullptr) return WKV_ERR_INVALID;
  wkv_paged* c = new (std::nothrow) wkv_paged;
  if (!c) return WKV_ERR_ALLOC;
  c->cfg = *cfg;
  if (!c->cfg.alloc) { c->cfg.alloc = default_alloc; c->cfg.release = default_release; c->cfg.user = nullptr; }
  cudaError_t e = cudaGetDevice(&c->device);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&c->sm_count, cudaDevAttrMultiProcessorCount, c->device);
  if (e != cudaSuccess) { delete c; return WKV_ERR_CUDA; }
  c->group = cfg->n_q_heads / cfg->n_kv_heads;
  c->page_shift = cfg->page_size == 16 ? 4 : cfg->page_size == 32 ? 5 : 6;
  c->scale = cfg->scale != 0.f ? cfg->scale : (float)(1.0 / std::sqrt((double)cfg->head_dim));
  c->elem = cfg->dtype == WKV_BF16 ? 2 : 4;
  c->stream = reinterpret_cast<cudaStream_t>(cfg->stream);
  c->k_pool = cfg->k_pool;
  c->v_pool = cfg->v_pool;
  const size_t pool = (size_t)cfg->n_layers * cfg->n_pages * cfg->n_kv_heads * cfg->page_size * cfg->head_dim * c->elem;
  const size_t lanes = (size_t)cfg->max_batch * cfg->n_kv_heads, heads = (size_t)cfg->max_batch * cfg->n_q_heads;
  const bool wide = cfg->head_dim == 128;
  e = cudaFuncSetAttribute(wkv::paged_select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, wkv::kSelectStaged * 4);
  if (e != cudaSuccess) { delete c; return WKV_ERR_CUDA; }
  if (cfg->dtype == WKV_BF16) e = wide ? pick_by_group<__nv_bfloat16, 128>(c) : pick_by_group<__nv_bfloat16, 64>(c);
  else e = wide ? pick_by_group<float, 128>(c) : pick_by_group<float, 64>(c);
  if (e != cudaSuccess) { delete c; return WKV_ERR_CUDA; }
  int rc = WKV_OK;
#define WKV_TAKE(dst, bytes) do { if (rc == WKV_OK) rc = take(c, dst, bytes); } while (0)
  WKV_TAKE(&c->status, 256);
  if (cfg->scores) {
    WKV_TAKE(&c->logits, heads * cfg->max_pages * cfg->page_size * 4);
    WKV_TAKE(&c->head_ml, heads * 8);
    WKV_TAKE(&c->n_moved, lanes * 4);
  }
  WKV_TAKE(&c->part, ((size_t)c->decode_ctas + lanes) * c->group * cfg->head_dim * 4);
  WKV_TAKE(&c->part_ml, ((size_t)c->decode_ctas + lanes) * c->group * 8);
  WKV_TAKE(&c->arrived, lanes * 4);
  WKV_TAKE(&c->run_part, run_rows(c) * cfg->head_dim * 4);
  WKV_TAKE(&c->run_ml, run_rows(c) * 8);
  WKV_TAKE(&c->item_counter, 12);
  const bool own_pools = !c->k_pool;
  if (own_pools) {
    WKV_TAKE(&c->k_pool, pool);
    WKV_TAKE(&c->v_pool, pool);
  }
#undef WKV_TAKE
  if (rc == WKV_OK) {
    e = cudaMemsetAsync(c->status, 0, 4, c->stream);
    if (e == cudaSuccess) e = cudaMemsetAsync(c->arrived, 0, lanes * 4, c->stream);
    if (e == cudaSuccess) e = cudaMemsetAsync(c->item_counter, 0, 8, c->stream);
    if (e == cudaSuccess && own_pools) e = cudaMemsetAsync(c->k_pool, 0, pool, c->stream);
    if (e == cudaSuccess && own_pools) e = cudaMemsetAsync(c->v_pool, 0, pool, c->stream);
    if (e != cudaSuccess) rc = WKV_ERR_CUDA;
  }
  {
    const int rows = cfg->dtype == WKV_BF16 ? cfg->page_size : std::min(cfg->page_size, 32), parts = (int)(cfg->head_dim * c->elem / 128);
    if (rc == WKV_OK) rc = encode_pool(c, c->page_kmap, c->k_pool, rows, parts);
    if (rc == WKV_OK) rc = encode_pool(c, c->page_vmap, c->v_pool, rows, parts);
    if (rc == WKV_OK && cfg->dtype == WKV_BF16) rc = encode_pool(c, c->part_kmap, c->k_pool, cfg->page_size, 1);
    if (rc == WKV_OK && cfg->dtype == WKV_BF16) rc = encode_pool(c, c->part_vmap, c->v_pool, cfg->page_size, 1);
  }
  if (rc != WKV_OK) {
    wkv_paged_destroy(c);
    return rc;
  }
  *out = c;
  return WKV_OK;
}

void wkv_paged_destroy(wkv_paged* c) {
  if (!c) return;
  for (void* p : c->owned) c->cfg.release(p, c->cfg.user);
  delete c;
}

int wkv_paged_set_stream(wkv_paged* c, void* stream) {
  if (!c) return WKV_ERR_INVALID;
  c->stream = reinterpret_cast<cudaStream_t>(stream);
  return WKV_OK;
}

int wkv_paged_pools(const wkv_paged* c, void** k_pool, void** v_pool) {
  if (!c || !k_pool || !v_pool) return WKV_ERR_INVALID;
  *k_pool = c->k_pool;
  *v_pool = c->v_pool;
  return WKV_OK;
}

int wkv_paged_decode(wkv_paged* c, int32_t layer, int32_t batch, const void* q, int64_t q_stride, const void* k, const void* v,
                     int64_t kv_stride, const int32_t* block_table, int32_t table_width, const int32_t* seq_lens,
                     int32_t window, int32_t sink, float* scores, int64_t score_stride, void* out, float* lse) {
  if (!c) return WKV_ERR_INVALID;
  DeviceGuard on(c->device);
  WKV_CUDA(c, on.err);
  wkv::PagedParams P;
  const int rc = attention_params(c, P, layer, batch, batch, q, q_stride, k, v, kv_stride, block_table, table_width, seq_lens, window,
                                  sink, scores, score_stride, out, lse);
  if (rc != WKV_OK) return rc;
  return decode(c, P);
}

int wkv_paged_prefill(wkv_paged* c, int32_t layer, int32_t batch, const void* q, int64_t q_stride, const void* k, const void* v,
                      int64_t kv_stride, const int32_t* q_start, int32_t total_q, const int32_t* block_table,
                      int32_t table_width, const int32_t* seq_lens, int32_t window, int32_t sink, float* scores,
                      int64_t score_stride, void* out, float* lse) {
  if (!c) return WKV_ERR_INVALID;
  DeviceGuard on(c->device);
  WKV_CUDA(c, on.err);
  wkv::PagedParams P;
  const int rc = attention_params(c, P, layer, batch, total_q, q, q_stride, k, v, kv_stride, block_table, table_width, seq_lens, window,
                                  sink, scores, score_stride, out, lse);
  if (rc != WKV_OK) return rc;
  if (total_q > (1 << 24)) return fail(c, WKV_ERR_INVALID, "total_q must be at most 2^24");
  if (batch > 0 && total_q > 0 && !q_start) return fail(c, WKV_ERR_INVALID, "q_start must not be NULL");
  if (scores && !lse && total_q > 0) return fail(c, WKV_ERR_INVALID, "scores need lse");
  P.q_start = q_start;
  return prefill(c, P);
}

int wkv_paged_evict(wkv_paged* c, int32_t layer, int32_t batch, const int32_t* src_table, int32_t src_width,
                    const int32_t* dst_table, int32_t dst_width, const int32_t* seq_lens, int32_t* new_lens, int32_t budget,
                    int32_t recent, int32_t sink, const float* scores, int64_t score_stride, float* scores_out,
                    int64_t out_stride, int32_t* kept) {
  if (!c) return WKV_ERR_INVALID;
  DeviceGuard on(c->device);
  WKV_CUDA(c, on.err);
  const wkv_paged_config& f = c->cfg;
  if (!f.scores) return fail(c, WKV_ERR_INVALID, "eviction needs a handle created with scores = 1");
  if (layer < 0 || layer >= f.n_layers) return fail(c, WKV_ERR_INVALID, "layer out of range");
  if (batch < 0 || batch > f.max_batch) return fail(c, WKV_ERR_INVALID, "batch must be in [0, max_batch]");
  if (src_width < 1 || src_width > f.max_pages || dst_width < 1) return fail(c, WKV_ERR_INVALID, "src_width must be in [1, max_pages], dst_width >= 1");
  if (budget < 1 || recent < 0 || sink < 0 || (int64_t)recent + sink > budget) return fail(c, WKV_ERR_INVALID, "budget must be >= 1 and >= sink + recent, both >= 0");
  const int64_t most = (int64_t)src_width * f.page_size, left = budget < most ? budget : most;
  if ((int64_t)dst_width * f.page_size < left) return fail(c, WKV_ERR_INVALID, "dst_table has too few pages for min(budget, src_width * page_size) entries");
  if (score_stride < most) return fail(c, WKV_ERR_INVALID, "score_stride must be >= src_width * page_size");
  if (scores_out && out_stride < left) return fail(c, WKV_ERR_INVALID, "out_stride must be >= min(budget, src_width * page_size)");
  if (batch == 0) return WKV_OK;
  if (!src_table || !dst_table || !seq_lens || !new_lens || !scores) return fail(c, WKV_ERR_INVALID, "src_table, dst_table, seq_lens, new_lens and scores must not be NULL");
  if (scores_out == scores || (const int32_t*)new_lens == seq_lens) return fail(c, WKV_ERR_INVALID, "scores_out and new_lens must not be the arrays that the call reads");
  wkv::EvictParams P;
  std::memset(&P, 0, sizeof(P));
  const size_t layer_bytes = (size_t)f.n_pages * f.n_kv_heads * f.page_size * f.head_dim * c->elem;
  P.k_pool = (char*)c->k_pool + layer * layer_bytes;
  P.v_pool = (char*)c->v_pool + layer * layer_bytes;
  P.src_table = src_table; P.dst_table = dst_table; P.seq_lens = seq_lens; P.new_lens = new_lens;
  P.scores = scores; P.score_stride = score_stride; P.scores_out = scores_out; P.out_stride = out_stride;
  P.kept = kept ? kept : reinterpret_cast<int32_t*>(c->logits);
  P.kept_stride = kept ? budget : left;
  P.n_moved = c->n_moved; P.status = c->status;
  P.batch = batch; P.src_width = src_width; P.dst_width = dst_width; P.n_pages = f.n_pages; P.n_kv_heads = f.n_kv_heads;
  P.page = f.page_size; P.page_shift = c->page_shift; P.budget = budget; P.recent = recent; P.sink = sink;
  const long long lanes = (long long)batch * f.n_kv_heads;
  const int staged = (int)std::min<int64_t>((most + wkv::kSelectThreads - 1) / wkv::kSelectThreads * wkv::kSelectThreads, wkv::kSelectStaged);
  cudaError_t e = launch(c, wkv::paged_select_kernel, lanes, wkv::kSelectThreads, (size_t)staged * 4, P, staged);
  if (e == cudaSuccess) {
    const int per_lane = (int)((left + wkv::kMoveEntries - 1) / wkv::kMoveEntries);
    const bool wide = f.head_dim == 128;
    auto kernel = f.dtype == WKV_BF16 ? (wide ? wkv::paged_move_kernel<__nv_bfloat16, 128> : wkv::paged_move_kernel<__nv_bfloat16, 64>)
                                      : (wide ? wkv::paged_move_kernel<float, 128> : wkv::paged_move_kernel<float, 64>);
    e = launch(c, kernel, lanes * per_lane, wkv::kMoveThreads, 0, P, per_lane);
  }
  WKV_CUDA(c, e);
  return WKV_OK;
}

int wkv_paged_status(wkv_paged* c) {
  if (!c) return WKV_ERR_INVALID;
  DeviceGuard on(c->device);
  WKV_CUDA(c, on.err);
  uint32_t w = 0;
  WKV_CUDA(c, cudaStreamSynchronize(c->stream));        // first: a stream that is being captured is refused here
  WKV_CUDA(c, cudaMemcpyAsync(&w, c->status, 4, cudaMemcpyDeviceToHost, c->stream));
  WKV_CUDA(c, cudaStreamSynchronize(c->stream));
  if (w) {
    // On the handle's stream, ahead of the next call: a clear on the default stream is not ordered with streams that do not wait for
    // that one, and could take back the next call's report, or its counts.
    WKV_CUDA(c, cudaMemsetAsync(c->status, 0, 4, c->stream));
    // a call that gave up may have left arrivals, items or rows uncounted
    if (w & wkv::kStatusWaitTimeout) {
      WKV_CUDA(c, cudaMemsetAsync(c->arrived, 0, (size_t)c->cfg.max_batch * c->cfg.n_kv_heads * 4, c->stream));
      WKV_CUDA(c, cudaMemsetAsync(c->item_counter, 0, 8, c->stream));
    }
    if (w & wkv::kStatusWaitTimeout) return fail(c, WKV_ERR_TIMEOUT, "a bounded wait inside a kernel gave up");
    return fail(c, WKV_ERR_STATE, "a page number, length or row offset was out of range, or an eviction's tables overlap");
  }
  return WKV_OK;
}

int wkv_paged_selftest_wait_timeout(wkv_paged* c) {
  if (!c) return WKV_ERR_INVALID;
  DeviceGuard on(c->device);
  WKV_CUDA(c, on.err);
  WKV_CUDA(c, launch(c, wkv::paged_wait_selftest_kernel, 1, 64, 0, c->status));
  return WKV_OK;
}

int64_t wkv_paged_launch_count(const wkv_paged* c) { return c ? c->launches : 0; }
int64_t wkv_paged_device_bytes(const wkv_paged* c) { return c ? c->device_bytes : 0; }
const char* wkv_paged_last_error(const wkv_paged* c) { return c ? c->last_error.c_str() : ""; }

}  // extern "C"
