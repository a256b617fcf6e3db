// Eviction from a paged cache by accumulated attention weight; the kernel that tests of bounded waits run.
#pragma once
#include "wkv_paged.cuh"

namespace wkv {

// For tests: a warp's and a thread's wait for barriers that nothing arrives at.
__global__ void __launch_bounds__(64) paged_wait_selftest_kernel(uint32_t* status) {
  __shared__ uint64_t bars[2];
  if (threadIdx.x == 0) {
    mbar_init(&bars[0], 1);
    mbar_init(&bars[1], 1);
  }
  griddep_wait();
  __syncthreads();
  const WaitLimit waits{status, 400};
  if (threadIdx.x < 32) (void)warp_wait(&bars[0], 0, waits);
  else if (threadIdx.x == 32) (void)thread_wait(&bars[1], 0, waits);
}

// ------------------------------------------------------------------------------------------------
// eviction
// ------------------------------------------------------------------------------------------------
struct EvictParams {
  void* k_pool;
  void* v_pool;
  const int32_t* src_table;  // [batch][src_width]
  const int32_t* dst_table;  // [batch][dst_width]
  const int32_t* seq_lens;
  int32_t* new_lens;
  const float* scores;       // [batch][Hkv][score_stride]
  float* scores_out;         // [batch][Hkv][out_stride] or NULL
  long long score_stride, out_stride;
  int32_t* kept;             // [batch][Hkv][kept_stride]: the caller's, or workspace
  long long kept_stride;
  int32_t* n_moved;          // [batch][Hkv] workspace: rows the move kernel copies
  uint32_t* status;
  int batch, src_width, dst_width, n_pages, n_kv_heads, page, page_shift, budget, recent, sink;
};

// Order of eviction as an unsigned key: smaller score, smaller key; -0 like +0; NaN last, but for the entries that stay anyway.
constexpr uint32_t kKeyNan = 0xfffffffeu, kKeyStays = 0xffffffffu;
__device__ __forceinline__ uint32_t score_key(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return x != x ? kKeyNan : u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

constexpr int kSelectThreads = 1024;
constexpr int kSelectStaged = 32768;   // lanes of up to so many entries are read into shared memory once
constexpr int kBitmapWords = 8192;     // pages per round of the overlap check: 32 times that
static_assert(kBitmapWords == 256 * 32, "a counter per digit and lane");

// Which entries stay, in order: one CTA per (sequence, kv head).  The `leave`-th smallest key among the entries that may leave is
// found by four rounds of counting digits of 8 bits, a counter per digit and lane: scores share a few exponents, and lanes that met
// on one counter would queue (33 us with one counter per digit of 11 bits).  Ties and places: a warp owns a contiguous run of
// entries, so they need one exchange of the warps' totals, and ballots.  All counts are whole numbers: the same result every time.
// Bound by instruction issue and latency: about 65 instructions per 32 entries.
struct StagedKeys {
  const uint32_t* key;
  __device__ __forceinline__ uint32_t operator()(int i) const { return key[i]; }
};
struct GlobalKeys {
  const float* x;
  int lo, hi;
  __device__ __forceinline__ uint32_t operator()(int i) const { return i >= lo && i < hi ? score_key(x[i]) : kKeyStays; }
};

__global__ void __launch_bounds__(kSelectThreads) paged_select_kernel(const EvictParams P, int staged) {
  extern __shared__ __align__(16) uint32_t stage[];     // [staged] keys, where they fit
  __shared__ uint32_t bitmap[kBitmapWords];             // overlap check, then the digit counters
  __shared__ int warp_sum[32], warp_below[32], warp_equal[32], found[2];
  griddep_launch();
  griddep_wait();
  const int bh = blockIdx.x, b = bh / P.n_kv_heads, head = bh % P.n_kv_heads, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int raw = P.seq_lens[b];
  const long long most = (long long)P.src_width << P.page_shift;
  const int len = raw < 0 ? 0 : raw > most ? (int)most : raw;
  const float* x = P.scores + (long long)bh * P.score_stride;
  const int left = min(len, P.budget), leave = len - left;
  const int lo = min(P.sink, len), hi = max(lo, len - P.recent);      // entries that may leave
  const int up = (len + kSelectThreads - 1) & ~(kSelectThreads - 1);  // whole passes of the CTA
  const bool in_stage = up <= staged;
  const GlobalKeys from_memory{x, lo, hi};
  if (in_stage && leave > 0) {
    int i = tid;
    for (; i + 7 * kSelectThreads < up; i += 8 * kSelectThreads) {
      uint32_t y[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) y[k] = from_memory(i + k * kSelectThreads);
#pragma unroll
      for (int k = 0; k < 8; ++k) stage[i + k * kSelectThreads] = y[k];
    }
    for (; i < up; i += kSelectThreads) stage[i] = from_memory(i);
  }
  // does the sequence move into pages that it lies in?
  bool bad = len != raw;
  const int n_src = (len + P.page - 1) >> P.page_shift, n_dst = (left + P.page - 1) >> P.page_shift;
  bool overlap = false;
  for (int base = 0; base < P.n_pages; base += kBitmapWords * 32) {
    const int words = min(kBitmapWords, (P.n_pages - base + 31) / 32);
    for (int w = tid; w < words; w += kSelectThreads) bitmap[w] = 0;
    __syncthreads();
    for (int c = tid; c < n_src; c += kSelectThreads) {
      const int pg = P.src_table[(long long)b * P.src_width + c];
      if ((unsigned)pg >= (unsigned)P.n_pages) bad = true;
      const unsigned at = (unsigned)pg - base;
      if ((unsigned)pg < (unsigned)P.n_pages && at < (unsigned)words * 32) atomicOr(&bitmap[at >> 5], 1u << (at & 31));
    }
    __syncthreads();
    for (int c = tid; c < n_dst; c += kSelectThreads) {
      const int pg = P.dst_table[(long long)b * P.dst_width + c];
      if ((unsigned)pg >= (unsigned)P.n_pages) bad = true;
      const unsigned at = (unsigned)pg - base;
      if ((unsigned)pg < (unsigned)P.n_pages && at < (unsigned)words * 32 && (bitmap[at >> 5] >> (at & 31) & 1)) overlap = true;
    }
    overlap = __syncthreads_or(overlap);
  }
  if (tid == 0) {
    if (head == 0) P.new_lens[b] = overlap ? len : left;
    P.n_moved[bh] = overlap ? 0 : left;
  }
  if (bad || (overlap && tid == 0)) flag_bad_table(P.status);
  if (overlap) return;

  int32_t* kept = P.kept + (long long)bh * P.kept_stride;
  float* scores_out = P.scores_out ? P.scores_out + (long long)bh * P.out_stride : nullptr;
  if (leave == 0) {
    for (int i = tid; i < len; i += kSelectThreads) {
      kept[i] = i;
      if (scores_out) scores_out[i] = x[i];
    }
    return;
  }
  __shared__ uint32_t found_threshold;
  auto select = [&](auto key_of) {
    uint32_t threshold = 0;            // the `leave`-th smallest key, its digits found so far
    int rank = leave;                  // its rank among the keys with these digits
#pragma unroll
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int w = tid; w < kBitmapWords; w += kSelectThreads) bitmap[w] = 0;
      __syncthreads();
#pragma unroll 8
      for (int i = tid; i < up; i += kSelectThreads) {
        const uint32_t key = key_of(i);
        if (shift == 24 || key >> (shift + 8 & 31) == threshold) atomicAdd(&bitmap[(key >> shift & 255) * 32 + lane], 1u);
      }
      __syncthreads();
      // four threads per digit, eight counters each (rotated, so that they sit on different banks), then a scan over the digits
      const int digit = tid >> 2;
      int c = 0;
#pragma unroll
      for (int k = 0; k < 8; ++k) c += bitmap[digit * 32 + (tid & 3) * 8 + ((k + digit) & 7)];
      c += __shfl_xor_sync(~0u, c, 1);
      c += __shfl_xor_sync(~0u, c, 2);
      int upto = (tid & 3) == 3 ? c : 0;
#pragma unroll
      for (int off = 1; off < 32; off <<= 1) {
        const int y = __shfl_up_sync(~0u, upto, off);
        if (lane >= off) upto += y;
      }
      if (lane == 31) warp_sum[warp] = upto;
      __syncthreads();
      upto += __reduce_add_sync(~0u, lane < warp ? warp_sum[lane] : 0);
      if ((tid & 3) == 3 && upto - c < rank && rank <= upto) { found_threshold = (uint32_t)digit; found[0] = upto - c; }
      __syncthreads();
      threshold = threshold << 8 | found_threshold;
      rank -= found[0];
      __syncthreads();
    }
    const int ties = rank;             // of the keys equal to the threshold so many leave, the first ones
    // a warp's entries: `run` times 32 in a row
    const int run = up / kSelectThreads, first = warp * run * 32 + lane;
    int wb = 0, we = 0;
#pragma unroll 8
    for (int j = 0; j < run; ++j) {
      const uint32_t key = key_of(first + j * 32);
      wb += __popc(__ballot_sync(~0u, key < threshold));
      we += __popc(__ballot_sync(~0u, key == threshold));
    }
    if (lane == 0) { warp_below[warp] = wb; warp_equal[warp] = we; }
    __syncthreads();
    int equal = __reduce_add_sync(~0u, lane < warp ? warp_equal[lane] : 0);                        // before this warp's entries
    int at = min(warp * run * 32, len) - __reduce_add_sync(~0u, lane < warp ? warp_below[lane] : 0) - min(equal, ties);
    const uint32_t before = (1u << lane) - 1;
#pragma unroll 4
    for (int j = 0; j < run; ++j) {
      const int i = first + j * 32;
      const uint32_t key = key_of(i), eqs = __ballot_sync(~0u, key == threshold);
      const float xi = i < len && scores_out ? x[i] : 0.f;
      const bool keep = i < len && (key > threshold || (key == threshold && equal + __popc(eqs & before) >= ties));
      const uint32_t ks = __ballot_sync(~0u, keep);
      if (keep) {
        const int to = at + __popc(ks & before);
        kept[to] = i;
        if (scores_out) scores_out[to] = xi;
      }
      equal += __popc(eqs);
      at += __popc(ks);
    }
  };
  if (in_stage) select(StagedKeys{stage}); else select(from_memory);
}

// Rows of K and V to their new pages.  A warp takes 32 entries: each lane looks one up (kept index, page, new page -- the chain of
// loads is what would take the time otherwise), then the warp copies them together, 16 bytes a lane and kMoveSteps steps in flight.
constexpr int kMoveThreads = 256, kMoveEntries = kMoveThreads, kMoveSteps = 8;     // entries per CTA: 32 a warp
template <typename T, int D>
__global__ void __launch_bounds__(kMoveThreads) paged_move_kernel(const EvictParams P, int blocks_per_lane) {
  griddep_wait();
  const int bh = blockIdx.x / blocks_per_lane, part = blockIdx.x % blocks_per_lane, lane = threadIdx.x & 31;
  const int b = bh / P.n_kv_heads, head = bh % P.n_kv_heads, n = P.n_moved[bh];
  const int first = part * kMoveEntries + (threadIdx.x >> 5) * 32, i = first + lane;
  if (first >= n) return;
  constexpr uint32_t kNone = 0xffffffffu;
  uint32_t from = kNone, to = kNone;                   // rows of the layer's pools (a row is 128 bytes at least: 32 bits suffice)
  if (i < n) {
    const int src = P.kept[(long long)bh * P.kept_stride + i];
    const int sp = P.src_table[(long long)b * P.src_width + (src >> P.page_shift)];
    const int dp = P.dst_table[(long long)b * P.dst_width + (i >> P.page_shift)];
    // an entry of a bad page counts as zeros, and its place in the destination must not keep what was there
    if ((unsigned)sp < (unsigned)P.n_pages) from = (((uint32_t)sp * P.n_kv_heads + head) << P.page_shift) + (src & (P.page - 1));
    if ((unsigned)dp < (unsigned)P.n_pages) to = (((uint32_t)dp * P.n_kv_heads + head) << P.page_shift) + (i & (P.page - 1));
  }
  constexpr int kVec = 2 * D * (int)sizeof(T) / 16;    // 16-byte pieces of an entry: K row, then V row
  constexpr int kEach = 16 / (int)sizeof(T);
#pragma unroll 1
  for (int s0 = 0; s0 < kVec; s0 += kMoveSteps) {
    uint4 piece[kMoveSteps];
#pragma unroll
    for (int k = 0; k < kMoveSteps; ++k) {
      const int at = (s0 + k) * 32 + lane, c = at % kVec;
      const uint32_t row = __shfl_sync(~0u, from, at / kVec);
      const T* pool = static_cast<const T*>(c < kVec / 2 ? P.k_pool : P.v_pool);
      piece[k] = row != kNone ? __ldcs(reinterpret_cast<const uint4*>(pool + (long long)row * D + c % (kVec / 2) * kEach)) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int k = 0; k < kMoveSteps; ++k) {
      const int at = (s0 + k) * 32 + lane, c = at % kVec;
      const uint32_t row = __shfl_sync(~0u, to, at / kVec);
      T* pool = static_cast<T*>(c < kVec / 2 ? P.k_pool : P.v_pool);
      if (row != kNone) *reinterpret_cast<uint4*>(pool + (long long)row * D + c % (kVec / 2) * kEach) = piece[k];
    }
  }
}

}  // namespace wkv
