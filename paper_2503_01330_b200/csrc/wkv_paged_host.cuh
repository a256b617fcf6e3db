// What the host sides of the paged calls share: the handle, errors, argument checks, launches.
#pragma once
#include <cmath>
#include <cstdint>
#include <cstring>
#include <string>
#include <utility>
#include <vector>

#include "../../include/wkv.h"
#include "wkv_paged.cuh"

struct wkv_paged {
  wkv_paged_config cfg;
  int device = 0;
  int sm_count = 148;
  int group = 1;
  int page_shift = 4;
  float scale = 0.f;
  size_t elem = 2;                     // of q, k, v, out
  size_t chunk_bytes = 0;              // one kv head's rows of one page, in a pool
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
  // ... over chosen pages, bf16 and fp32 rows (a kernel of its own; the CTAs are at most decode_ctas)
  const void* pages_kernel = nullptr;
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

namespace wkv {
namespace host {

inline int fail(wkv_paged* c, int code, const std::string& msg) {
  if (c) c->last_error = msg;
  return code;
}
inline int cuda_fail(wkv_paged* c, cudaError_t e, const char* what) {
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

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// Arguments that all calls on one cache's rows share; fills P.  `rows`: rows of k and v (which may be NULL).
inline int cache_params(wkv_paged* c, PagedParams& P, int32_t layer, int32_t batch, int32_t rows, const void* k, const void* v, int64_t kv_stride,
                        const int32_t* table, int32_t width, const int32_t* seq_lens) {
  const wkv_paged_config& f = c->cfg;
  if (layer < 0 || layer >= f.n_layers) return fail(c, WKV_ERR_INVALID, "layer out of range");
  if (batch < 0 || batch > f.max_batch) return fail(c, WKV_ERR_INVALID, "batch must be in [0, max_batch]");
  if (rows < 0) return fail(c, WKV_ERR_INVALID, "the number of rows must be >= 0");
  if (width < 1 || width > f.max_pages) return fail(c, WKV_ERR_INVALID, "table_width must be in [1, max_pages]");
  if ((k == nullptr) != (v == nullptr)) return fail(c, WKV_ERR_INVALID, "k and v must both be given or both be NULL");
  if (batch > 0 && rows > 0 && (!table || !seq_lens)) return fail(c, WKV_ERR_INVALID, "block_table and seq_lens must not be NULL");
  const int64_t kv_row = (int64_t)f.n_kv_heads * f.head_dim;
  if (kv_stride == 0) kv_stride = kv_row;
  if (kv_stride < kv_row) return fail(c, WKV_ERR_INVALID, "a row stride is smaller than the row");
  if (kv_stride * (int64_t)c->elem % 16 || !aligned16(k) || !aligned16(v)) return fail(c, WKV_ERR_INVALID, "rows of k and v must be 16-byte aligned");
  std::memset(&P, 0, sizeof(P));
  const size_t layer_bytes = (size_t)f.n_pages * f.n_kv_heads * c->chunk_bytes;
  P.k_pool = (char*)c->k_pool + layer * layer_bytes;
  P.v_pool = (char*)c->v_pool + layer * layer_bytes;
  P.k = k; P.v = v; P.kv_stride = kv_stride;
  P.table = table; P.seq_lens = seq_lens;
  P.status = c->status; P.batch = batch; P.rows = rows; P.width = width; P.n_pages = f.n_pages;
  P.n_q_heads = f.n_q_heads; P.n_kv_heads = f.n_kv_heads; P.page = f.page_size; P.page_shift = c->page_shift;
  P.scale_log2 = c->scale * kLog2e;
  return WKV_OK;
}

// ... and those of queries and what comes out for them.
inline int query_params(wkv_paged* c, PagedParams& P, const void* q, int64_t q_stride, void* out, float* lse) {
  const wkv_paged_config& f = c->cfg;
  if (P.batch > 0 && P.rows > 0 && (!q || !out)) return fail(c, WKV_ERR_INVALID, "q, block_table, seq_lens and out must not be NULL");
  const int64_t q_row = (int64_t)f.n_q_heads * f.head_dim;
  if (q_stride == 0) q_stride = q_row;
  if (q_stride < q_row) return fail(c, WKV_ERR_INVALID, "a row stride is smaller than the row");
  if (q_stride * (int64_t)c->elem % 16 || !aligned16(q) || !aligned16(out)) return fail(c, WKV_ERR_INVALID, "rows of q, k, v and out must be 16-byte aligned");
  P.q = q; P.q_stride = q_stride; P.out = out; P.lse = lse;
  return WKV_OK;
}

// Arguments that decode and prefill share.
inline int attention_params(wkv_paged* c, PagedParams& P, int32_t layer, int32_t batch, int32_t rows, const void* q, int64_t q_stride,
                            const void* k, const void* v, int64_t kv_stride, const int32_t* table, int32_t width, const int32_t* seq_lens,
                            int32_t window, int32_t sink, float* scores, int64_t score_stride, void* out, float* lse) {
  const wkv_paged_config& f = c->cfg;
  int rc = cache_params(c, P, layer, batch, rows, k, v, kv_stride, table, width, seq_lens);
  if (rc == WKV_OK) rc = query_params(c, P, q, q_stride, out, lse);
  if (rc != WKV_OK) return rc;
  if (window < 0 || sink < 0) return fail(c, WKV_ERR_INVALID, "window and sink must be >= 0");
  if (scores) {
    if (!f.scores) return fail(c, WKV_ERR_INVALID, "scores need a handle created with scores = 1");
    if (score_stride < (int64_t)width * f.page_size) return fail(c, WKV_ERR_INVALID, "score_stride must be >= table_width * page_size");
  }
  P.scores = scores; P.score_stride = score_stride; P.window = window; P.sink = sink;
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
inline int chunk0(const wkv_paged* c, const PagedParams& P) {
  return (int)(((char*)P.k_pool - (char*)c->k_pool) / c->chunk_bytes);
}

// Calls of one unit that another one makes.
cudaError_t pick_pages(wkv_paged* c);                       // wkv_paged_pages.cu: the kernel over chosen pages, bf16 and fp32 rows
cudaError_t pick_kv4(wkv_paged* c);                         // wkv_paged_kv4.cu: the kernel on rows in 4 bits
int decode_kv4(wkv_paged* c, const PagedParams& A, const int32_t* pages, int n_select);
cudaError_t prepare_rows(wkv_paged* c);                     // wkv_paged_rows.cu: shared memory of its kernels
int append_rows(wkv_paged* c, const PagedParams& A);        // ... k and v to their pages, nothing turned

}  // namespace host
}  // namespace wkv
