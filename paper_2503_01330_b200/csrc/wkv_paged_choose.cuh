// Which pages a query attends to: a cheap score per page from the bounds of its keys, then the best of them.
//
//   score_p = page_scale_p * sum_c (u_c hi_pc + w_c lo_pc),  u = sum over the kv head's query heads of max(q, 0), w of min(q, 0)
//
// With hi, lo the largest and least key of a channel that is an upper bound on sum_heads q.k over the page's keys k, up to the rounding of
// u and w to 1/127 of their largest.  Everything under the sum is an int8 number: the sum is exact in any order (dp4a), so that which
// pages are chosen does not depend on how the work is cut.
//
// Bound: the bounds, 2 D bytes a page and kv head, 1/32 of a bf16 cache in pages of 16; for one sequence latency: length -> table -> bounds
// -> scores -> choice.  Eight lanes share a page; the pages of a lane (sequence, kv head) are cut over CTAs, of which the last to arrive
// (by a counter that nobody waits on) chooses.  (A cluster whose CTAs put their scores into the first one's shared memory saves 2 us of
// that, and costs them again where the launch follows one that fills the SMs: 2048 pages, then 64 of them attended to, 21.3 us for 20.)
//
// Measured: one sequence of 2048 pages, 8 kv heads, 10.5 us; 16 of 256..512 pages, 32 kv heads, 14 us.  Longer ones, whose scores do not fit
// into shared memory and are read again from L2 by the one CTA that chooses: 2049 pages 16 us, 4096 24, 8192 39, 32768 139 (its bounds: 11).
#pragma once
#include "wkv_paged.cuh"

namespace wkv {

struct ChooseParams {
  PagedParams A;
  const int8_t* bounds;      // the layer's [pages][Hkv][2][D]
  const float* bound_scale;  // [pages][Hkv]
  float* page_scores;        // [batch][Hkv][score_stride]
  long long page_score_stride;
  int32_t* pages;            // [batch][Hkv][n_select]
  uint32_t* arrived;         // [lanes], zero between launches
  int n_select, recent, sink, splits;
};

constexpr int kChooseThreads = 256, kChooseWarps = kChooseThreads / 32;
constexpr int kChooseNear = 2048;      // pages of a lane whose scores are held in shared memory
constexpr int kChooseBins = 1024;

// As the eviction's order of scores: -0 like +0, NaN above all numbers.
__device__ __forceinline__ uint32_t page_key(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return x != x ? 0xfffffffeu : u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

struct ChooseShared {
  int bins[kChooseBins];
  unsigned long long candidates[kChooseThreads];
  unsigned long long cutoff;
  float least[kChooseWarps], most[kChooseWarps];
  int sums[2][3 * kChooseWarps];
  int bin, above, n_candidates;
};

// Exclusive sum over the threads; total: of all.  `at`: the warps' sums.  One barrier.
__device__ __forceinline__ int sum_before(int x, int* at, int& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int y = x;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const int z = __shfl_up_sync(~0u, y, off);
    if (lane >= off) y += z;
  }
  if (lane == 31) at[warp] = y;
  __syncthreads();
  total = 0;
  y -= x;
#pragma unroll
  for (int w = 0; w < kChooseWarps; ++w) {
    if (w < warp) y += at[w];
    total += at[w];
  }
  return y;
}

// Order of pages: better score, then lower index.
__device__ __forceinline__ unsigned long long page_rank(float x, int i) { return (unsigned long long)page_key(x) << 32 | (uint32_t)~i; }

// The cutoff among keys that do not spread well (all equal, not finite, far outliers): the `want`-th best of n, two bits of the key a round.
template <typename Each>
__device__ __forceinline__ unsigned long long cutoff_by_digits(Each each, int n, int want, ChooseShared& sh) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  unsigned long long least = 0;
  int at_least = n, turn = 0;
#pragma unroll 1
  for (int shift = 62; shift >= 0 && at_least != want; shift -= 2) {
    const unsigned long long k1 = least + (1ull << shift), k2 = least + (2ull << shift), k3 = least + (3ull << shift);
    int c1 = 0, c2 = 0, c3 = 0;
    each([&](int i, float x) {
      const unsigned long long k = page_rank(x, i);
      c1 += k >= k1; c2 += k >= k2; c3 += k >= k3;
    });
    int* mine = sh.sums[turn];
    turn ^= 1;
    c1 = __reduce_add_sync(~0u, c1); c2 = __reduce_add_sync(~0u, c2); c3 = __reduce_add_sync(~0u, c3);
    if (lane == 0) { mine[warp] = c1; mine[kChooseWarps + warp] = c2; mine[2 * kChooseWarps + warp] = c3; }
    __syncthreads();
    c1 = c2 = c3 = 0;
#pragma unroll
    for (int w = 0; w < kChooseWarps; ++w) { c1 += mine[w]; c2 += mine[kChooseWarps + w]; c3 += mine[2 * kChooseWarps + w]; }
    if (c3 >= want) { least = k3; at_least = c3; }
    else if (c2 >= want) { least = k2; at_least = c2; }
    else if (c1 >= want) { least = k1; at_least = c1; }
  }
  __syncthreads();
  return least;
}

// The `want` best of n pages (more than that), the first `sink` and the last `recent` among them in any case, in order of their index.  Scores are
// counted in bins of equal width between the least and the largest; the bin that holds the last one to be chosen is settled by comparing
// its few pages with one another (digit by digit over all pages where they are many).  NEAR: the scores are in shared memory.  The loops
// are short and rolled: between other kernels a launch finds none of its code in the instruction caches, and unrolled ones, the faster by
// 3 us when nothing else ran in between, then were no faster at all.
template <bool NEAR, typename ScoreAt>
__device__ __forceinline__ void choose(ScoreAt score_at, int sink, int recent, int n, int want, int32_t* to, ChooseShared& sh) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, hi = n - recent, steps = (n + kChooseThreads - 1) / kChooseThreads;
  auto is_free = [&](int i) { return i >= sink && i < hi; };      // neither behind the last page nor taken anyway
  auto each = [&](auto f) {                                // f(index, score) for the free pages
#pragma unroll 2
    for (int i = tid; i < hi; i += kChooseThreads) {
      const float x = score_at(i);
      if (i >= sink) f(i, x);
    }
  };
  float least = INFINITY, most = -INFINITY;
  bool odd = false;
  each([&](int, float x) {
    least = fminf(least, x);
    most = fmaxf(most, x);
    odd = odd || !(fabsf(x) < INFINITY);
  });
#pragma unroll
  for (int off = 16; off; off >>= 1) {
    least = fminf(least, __shfl_xor_sync(~0u, least, off));
    most = fmaxf(most, __shfl_xor_sync(~0u, most, off));
  }
  if (lane == 0) { sh.least[warp] = least; sh.most[warp] = most; }
#pragma unroll
  for (int i = 0; i < kChooseBins / kChooseThreads; ++i) sh.bins[tid + i * kChooseThreads] = 0;
  if (tid == 0) sh.n_candidates = 0;
  odd = __syncthreads_or(odd);
  want -= sink + recent;
#pragma unroll
  for (int w = 0; w < kChooseWarps; ++w) { least = fminf(least, sh.least[w]); most = fmaxf(most, sh.most[w]); }
  const float range = most - least, per_bin = range > 0.f && range < INFINITY ? kChooseBins / range : 0.f;
  odd = odd || !(per_bin > 0.f && per_bin < INFINITY);
  unsigned long long cutoff = ~0ull;                       // want = 0: none but the taken ones
  bool settled = want == 0;
  if (want > 0 && !odd) {
    // (x - least, times a constant, cut to a whole number: each step keeps the order)
    auto bin_of = [&](float x) { return min(kChooseBins - 1, (int)((x - least) * per_bin)); };
    each([&](int, float x) { atomicAdd(&sh.bins[bin_of(x)], 1); });
    __syncthreads();
    constexpr int kMine = kChooseBins / kChooseThreads;    // bins of this thread, from the top down
    int mine[kMine], sum = 0, total;
#pragma unroll
    for (int i = 0; i < kMine; ++i) { mine[i] = sh.bins[kChooseBins - 1 - (tid * kMine + i)]; sum += mine[i]; }
    int before = sum_before(sum, sh.sums[1], total);
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      if (before < want && want <= before + mine[i]) { sh.bin = kChooseBins - 1 - (tid * kMine + i); sh.above = before; }
      before += mine[i];
    }
    __syncthreads();
    const int bin = sh.bin, need = want - sh.above, in_bin = sh.bins[bin];
    if (in_bin <= kChooseThreads) {
      each([&](int i, float x) { if (bin_of(x) == bin) sh.candidates[atomicAdd(&sh.n_candidates, 1)] = page_rank(x, i); });
      __syncthreads();
      if (tid < in_bin) {
        const unsigned long long me = sh.candidates[tid];
        int better = 0;
        for (int k = 0; k < in_bin; ++k) better += sh.candidates[k] > me;
        if (better == need - 1) sh.cutoff = me;
      }
      __syncthreads();
      cutoff = sh.cutoff;
      settled = true;
    }
  }
  if (!settled) cutoff = cutoff_by_digits(each, n - sink - recent, want, sh);
  auto chosen = [&](int i) { return i < n && (!is_free(i) || (want > 0 && page_rank(score_at(i), i) >= cutoff)); };
  if constexpr (NEAR) {
    // chosen pages by (step, warp), counted and given places in that order
    uint32_t* masks = reinterpret_cast<uint32_t*>(sh.bins);
    if (warp == 0) masks[lane] = masks[32 + lane] = 0;
    __syncthreads();
#pragma unroll 2
    for (int k = 0; k < steps; ++k) {
      const uint32_t in = __ballot_sync(~0u, chosen(tid + k * kChooseThreads));
      if (lane == 0) masks[k * kChooseWarps + warp] = in;
    }
    __syncthreads();
    static_assert(kChooseNear / 32 == 64, "two masks a lane");
    const int c0 = __popc(masks[2 * lane]), c1 = __popc(masks[2 * lane + 1]);
    int y = c0 + c1;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int z = __shfl_up_sync(~0u, y, off);
      if (lane >= off) y += z;
    }
    y -= c0 + c1;                                          // before mask 2 lane
    for (int k = 0; k < steps; ++k) {
      const int of = k * kChooseWarps + warp, before = __shfl_sync(~0u, of & 1 ? y + c0 : y, of >> 1);
      const uint32_t in = masks[of];
      if (in >> lane & 1) to[before + __popc(in & ((1u << lane) - 1))] = tid + k * kChooseThreads;
    }
  } else {
    // a warp's pages lie in a row: their number, then their places by ballots
    const int first = warp * steps * 32 + lane;
    int count = 0;
    for (int k = 0; k < steps; ++k) count += __popc(__ballot_sync(~0u, chosen(first + k * 32)));
    if (lane == 0) sh.sums[0][warp] = count;
    __syncthreads();
    int at = 0;
#pragma unroll
    for (int w = 0; w < kChooseWarps; ++w) at += w < warp ? sh.sums[0][w] : 0;
    for (int k = 0; k < steps; ++k) {
      const int i = first + k * 32;
      const bool mine = chosen(i);
      const uint32_t all = __ballot_sync(~0u, mine);
      if (mine) to[at + __popc(all & ((1u << lane) - 1))] = i;
      at += __popc(all);
    }
  }
}

// `splits` CTAs per lane.
template <typename T, int D>
__global__ void __launch_bounds__(kChooseThreads, 4) paged_choose_kernel(const __grid_constant__ ChooseParams P) {
  __shared__ __align__(16) int8_t code[2][D];
  __shared__ float part[kChooseWarps];
  __shared__ ChooseShared sh;
  __shared__ float near[kChooseNear];
  __shared__ bool is_last;
  griddep_launch();
  griddep_wait();
  const PagedParams& A = P.A;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, sub = lane & 7;
  const int lane_no = blockIdx.x / P.splits, split = blockIdx.x % P.splits, b = lane_no / A.n_kv_heads, h = lane_no % A.n_kv_heads;
  // the query's row is there, whatever the length
  const int G = A.n_q_heads / A.n_kv_heads;
  float up = 0.f, down = 0.f;
  const T* q = static_cast<const T*>(A.q) + (long long)b * A.q_stride + (long long)h * G * D + (tid < D ? tid : 0);
  float q0 = (float)q[0];
  const int len = clamped_len(A, b), n = (len + A.page - 1) >> A.page_shift;
  // bounds: eight lanes a page, D / 8 channels each, kSteps pages in flight, kStride apart; the first ones are on their way while the query's
  // codes are made
  constexpr int kWords = D / 32, kSteps = 4, kStride = kChooseWarps * 4;   // words per lane, of the largest and of the least
  const int each = ((n + P.splits - 1) / P.splits + 31) & ~31, p1 = min(n, (split + 1) * each);
  int hi[kSteps][kWords], lo[kSteps][kWords];
  float scale[kSteps];
  auto load = [&](int base) {
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
      const int p = base + k * kStride;
      const int pg = p < p1 ? page_of(A, b, p << A.page_shift) : -1;
      const long long chunk = (long long)pg * A.n_kv_heads + h;
      scale[k] = 0.f;
#pragma unroll
      for (int i = 0; i < kWords; ++i) hi[k][i] = lo[k][i] = 0;
      if (pg < 0) continue;
      scale[k] = P.bound_scale[chunk];
      const int8_t* at = P.bounds + chunk * 2 * D + sub * kWords * 4;
      if constexpr (kWords == 4) {
        const int4 x = *reinterpret_cast<const int4*>(at), y = *reinterpret_cast<const int4*>(at + D);
        hi[k][0] = x.x; hi[k][1] = x.y; hi[k][2] = x.z; hi[k][3] = x.w;
        lo[k][0] = y.x; lo[k][1] = y.y; lo[k][2] = y.z; lo[k][3] = y.w;
      } else {
        const int2 x = *reinterpret_cast<const int2*>(at), y = *reinterpret_cast<const int2*>(at + D);
        hi[k][0] = x.x; hi[k][1] = x.y;
        lo[k][0] = y.x; lo[k][1] = y.y;
      }
    }
  };
  const int first = split * each + warp * 4;               // of this warp's four pages
  load(first + (lane >> 3));
  {
    // (an eighth of the query: up to eight heads' sums stay finite, and the codes are the same)
    if (tid < D) {
      for (int g = 0; g < G; ++g) {
        const float x = 0.125f * (g == 0 ? q0 : (float)q[g * D]);
        up = __fadd_rn(up, fmaxf(x, 0.f));
        down = __fadd_rn(down, fminf(x, 0.f));
      }
    }
    float most = fmaxf(up, -down);
#pragma unroll
    for (int off = 16; off; off >>= 1) most = fmaxf(most, __shfl_xor_sync(~0u, most, off));
    if (lane == 0) part[warp] = most;
    __syncthreads();
    most = 0.f;
#pragma unroll
    for (int w = 0; w < D / 32; ++w) most = fmaxf(most, part[w]);
    const float step = __fmul_rn(most, 1.f / 127.f), inv = step >= 0x1p-103f ? __frcp_rn(step) : 0.f;
    if (tid < D) {
      code[0][tid] = (int8_t)(int)fminf(fmaxf(rintf(__fmul_rn(up, inv)), 0.f), 127.f);
      code[1][tid] = (int8_t)(int)fmaxf(fminf(rintf(__fmul_rn(down, inv)), 0.f), -127.f);
    }
    __syncthreads();
  }
  float* scores = P.page_scores + (long long)lane_no * P.page_score_stride;
  {
    int u[kWords], w[kWords];
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      u[i] = reinterpret_cast<const int*>(code[0])[sub * kWords + i];
      w[i] = reinterpret_cast<const int*>(code[1])[sub * kWords + i];
    }
    for (int base = first; base < p1; base += kSteps * kStride) {
      if (base != first) load(base + (lane >> 3));
#pragma unroll
      for (int k = 0; k < kSteps; ++k) {
        const int p = base + (lane >> 3) + k * kStride;
        int sum = 0;
#pragma unroll
        for (int i = 0; i < kWords; ++i) sum = __dp4a(u[i], hi[k][i], __dp4a(w[i], lo[k][i], sum));
        sum += __shfl_xor_sync(~0u, sum, 1);
        sum += __shfl_xor_sync(~0u, sum, 2);
        sum += __shfl_xor_sync(~0u, sum, 4);
        if (sub == 0 && p < p1) {
          const float x = __fmul_rn((float)sum, scale[k]);
          scores[p] = x;
          if (p < kChooseNear) near[p] = x;
        }
      }
    }
  }
  if (P.splits > 1) {
    __threadfence();
    __syncthreads();
    if (tid == 0) {
      const bool last = atomicAdd(P.arrived + lane_no, 1u) == (uint32_t)P.splits - 1;
      if (last) P.arrived[lane_no] = 0;
      is_last = last;
    }
    __syncthreads();
    if (!is_last) return;
    __threadfence();
#pragma unroll 4
    for (int i = tid; i < min(n, kChooseNear); i += kChooseThreads) near[i] = __ldcg(scores + i);
  }
  __syncthreads();
  const int want = min(P.n_select, n);
  int32_t* to = P.pages + (long long)lane_no * P.n_select;
  for (int i = want + tid; i < P.n_select; i += kChooseThreads) to[i] = -1;
  if (want == n) {
    for (int i = tid; i < n; i += kChooseThreads) to[i] = i;
    return;
  }
  if (n <= kChooseNear) choose<true>([&](int p) { return near[p]; }, P.sink, P.recent, n, want, to, sh);
  else choose<false>([&](int p) { return __ldcg(scores + p); }, P.sink, P.recent, n, want, to, sh);
}

}  // namespace wkv
