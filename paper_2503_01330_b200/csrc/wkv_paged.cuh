// Device code of the paged cache (include/wkv.h, "Paged caches"): parameters, lookups, appending as prompt calls do it.
//
// Pool: [layers][pages][kv heads][page][D]; the kernels see one layer.  A "chunk" is one kv head's rows of one page,
// page * D contiguous elements; its number inside the layer is page * Hkv + head.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "wkv_ptx.cuh"

namespace wkv {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct PagedParams {
  void* k_pool;              // the layer's pools
  void* v_pool;
  const void* q;             // [rows][Hq][D], rows q_stride elements apart
  const void* k;             // [rows][Hkv][D] or NULL
  const void* v;
  long long q_stride, kv_stride;
  const int32_t* table;      // [batch][width]
  const int32_t* seq_lens;   // [batch]
  const int32_t* q_start;    // [batch + 1], or NULL: one row per sequence (decode)
  void* out;                 // [rows][Hq][D]
  float* lse;                // [rows][Hq]
  float* scores;             // [batch][Hkv][score_stride] or NULL
  long long score_stride;
  uint32_t* status;
  int batch, rows, width, n_pages, n_q_heads, n_kv_heads, page, page_shift;
  int window, sink;
  float scale_log2;          // softmax scale * log2(e)
};

__device__ __forceinline__ void flag_bad_table(uint32_t* status) { atomicOr(status, kStatusBadTable); }

// Sequence length clamped to what its table row can hold.
__device__ __forceinline__ int clamped_len(const PagedParams& P, int b) {
  const int n = P.seq_lens[b];
  const long long most = (long long)P.width << P.page_shift;
  if (n < 0 || n > most) {
    flag_bad_table(P.status);
    return n < 0 ? 0 : (int)most;
  }
  return n;
}
// Page of entry i, -1 if the table holds no valid number there.
__device__ __forceinline__ int page_of(const PagedParams& P, int b, int i) {
  const int pg = P.table[(long long)b * P.width + (i >> P.page_shift)];
  if ((unsigned)pg >= (unsigned)P.n_pages) {
    flag_bad_table(P.status);
    return -1;
  }
  return pg;
}
__device__ __forceinline__ long long row_offset(const PagedParams& P, int pg, int head, int i, int D) {
  return ((((long long)pg * P.n_kv_heads + head) << P.page_shift) + (i & (P.page - 1))) * D;
}

// A sequence's rows of q: [first, first + n), clamped into the call's buffers.
struct SeqRows {
  int first, n, len;         // len: entries of the sequence, the call's own included
};
__device__ __forceinline__ SeqRows seq_rows(const PagedParams& P, int b) {
  SeqRows s;
  s.len = clamped_len(P, b);
  if (!P.q_start) {
    s.first = b;
    s.n = s.len > 0 ? 1 : 0;
    return s;
  }
  const int lo = P.q_start[b], hi = P.q_start[b + 1];
  s.first = min(max(lo, 0), P.rows);
  s.n = min(max(hi, s.first), P.rows) - s.first;
  if (lo != s.first || hi != s.first + s.n || s.n > s.len) flag_bad_table(P.status);
  return s;
}
// The sequence that row r belongs to, -1 if none: the last b with q_start[b] <= r, if its end is behind r.
__device__ __forceinline__ int seq_of_row(const PagedParams& P, int r) {
  if (!P.q_start) return r;
  int lo = 0, hi = P.batch;            // invariant: q_start[lo] <= r (or lo == 0), q_start[hi] > r (or hi == batch)
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (P.q_start[mid] <= r) lo = mid; else hi = mid;
  }
  return (P.q_start[lo] <= r && r < P.q_start[lo + 1]) ? lo : -1;
}

__device__ __forceinline__ bool visible(int i, int pos, int window, int sink) {
  return i <= pos && (window == 0 || i > pos - window || i < sink);
}
// Does any token from position `pos` on see one of the n entries from i on?  Pages of which none does are not looked up.
__device__ __forceinline__ bool seen_from(int i, int n, int pos, int window, int sink) {
  return window == 0 || i + n > pos - window + 1 || i < sink;
}

// ------------------------------------------------------------------------------------------------
// append
// ------------------------------------------------------------------------------------------------
// Where row r of a prompt call's k and v goes: page (-1: nowhere) and entry.  `inner`: nowhere too for the rows of the page that
// their chunk starts in the middle of.
struct NewRow {
  int page, entry;
};
__device__ __forceinline__ NewRow new_row(const PagedParams& P, int r, bool inner) {
  NewRow w{-1, 0};
  const int b = r < P.rows ? seq_of_row(P, r) : -1;
  if (b < 0) return w;
  const SeqRows s = seq_rows(P, b);
  const int old = s.len - s.n;
  w.entry = old + (r - s.first);
  if (r < s.first || r >= s.first + s.n || w.entry < 0) return w;
  if (inner && (w.entry & ~(P.page - 1)) < old) return w;
  w.page = page_of(P, b, w.entry);
  return w;
}
// The row copied by THREADS threads (this one: `me`), 16 bytes a step and STEPS steps in flight.
template <typename T, int D, int THREADS, int STEPS>
__device__ __forceinline__ void append_row(const PagedParams& P, int r, const NewRow& w, int me) {
  if (w.page < 0) return;
  constexpr int kVec = D * (int)sizeof(T) / 16, kEach = 16 / (int)sizeof(T);
  const int per_row = P.n_kv_heads * kVec;              // pieces: the K row, then the V row
  const long long to = row_offset(P, w.page, 0, w.entry, D);
  for (int base = me; base < 2 * per_row; base += STEPS * THREADS) {
    uint4 piece[STEPS];
#pragma unroll
    for (int k = 0; k < STEPS; ++k) {
      const int at = base + k * THREADS, c = at >= per_row ? at - per_row : at;
      if (at < 2 * per_row) piece[k] = *reinterpret_cast<const uint4*>(static_cast<const T*>(at >= per_row ? P.v : P.k) + (long long)r * P.kv_stride + (long long)c * kEach);
    }
#pragma unroll
    for (int k = 0; k < STEPS; ++k) {
      const int at = base + k * THREADS, c = at >= per_row ? at - per_row : at;
      if (at < 2 * per_row)
        *reinterpret_cast<uint4*>(static_cast<T*>(at >= per_row ? P.v_pool : P.k_pool) + to + ((long long)(c / kVec) * P.page) * D + c % kVec * kEach) = piece[k];
    }
  }
}

// All new rows: a CTA per token.
constexpr int kAppendThreads = 128;
template <typename T, int D>
__global__ void __launch_bounds__(kAppendThreads) paged_append_kernel(const PagedParams P) {
  griddep_launch();
  griddep_wait();
  append_row<T, D, kAppendThreads, 8>(P, blockIdx.x, new_row(P, blockIdx.x, false), threadIdx.x);
}
// The new rows of the page that a chunk starts in the middle of: a CTA per sequence and row of a page.
template <typename T, int D>
__global__ void __launch_bounds__(kAppendThreads) paged_append_edge_kernel(const PagedParams P) {
  griddep_launch();
  griddep_wait();
  const int b = blockIdx.x >> P.page_shift, k = blockIdx.x & (P.page - 1);
  const SeqRows s = seq_rows(P, b);
  const int old = s.len - s.n, i = (old & ~(P.page - 1)) + k;      // the k-th entry of the page
  if (i < old || i >= s.len || !(old & (P.page - 1))) return;
  append_row<T, D, kAppendThreads, 8>(P, s.first + i - old, new_row(P, s.first + i - old, false), threadIdx.x);
}

}  // namespace wkv
