// Which pages a query attends to: a cheap score per page from the bounds of its keys, then the best of them.
//
//   score_p = page_scale_p * sum_c (u_c hi_pc + w_c lo_pc),  u = sum over the kv head's query heads of max(q, 0), w of min(q, 0)
//
// With hi, lo the largest and least key of a channel that is an upper bound on sum_heads q.k over the page's keys k, up to the rounding of
// u and w to 1/127 of their largest.  Everything under the sum is an int8 number: the sum is exact in any order (dp4a), so that which
// pages are chosen does not depend on how the work is cut.
//
// Bound: the bounds, 2 D bytes a page and kv head, 1/32 of a bf16 cache in pages of 16; for one sequence latency: bounds -> scores ->
// choice.  Eight lanes share a page; the pages of a lane (sequence, kv head) are cut over CTAs, of which the last to arrive (by a
// counter that nobody waits on) chooses.
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
constexpr int kChooseHeld = 8;         // scores per thread that stay in registers

// As the eviction's order of scores: -0 like +0, NaN above all numbers; pages that are taken anyway above that.
constexpr uint32_t kTakenKey = 0xffffffffu;
__device__ __forceinline__ uint32_t page_key(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return x != x ? 0xfffffffeu : u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

// The `want` largest of n keys, in order of their index, of equal keys the lowest indexes.  A thread owns `per` consecutive ones: in
// registers (HELD), where there are few, or looked up each time.  sums: [2][3 * warps].
template <bool HELD, typename KeyAt>
__device__ __forceinline__ void choose(KeyAt key_at, int per, int n, int want, int32_t* to, int* sums) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, first = tid * per;
  const int count = min(per, max(0, n - first));
  uint32_t held[kChooseHeld];
  if constexpr (HELD) {
#pragma unroll
    for (int i = 0; i < kChooseHeld; ++i) held[i] = i < count ? key_at(first + i) : 0u;
  }
  auto each = [&](auto f) {                                // f(index, key) for this thread's keys
    if constexpr (HELD) {
#pragma unroll
      for (int i = 0; i < kChooseHeld; ++i)
        if (i < count) f(first + i, held[i]);
    } else {
      for (int i = 0; i < count; ++i) f(first + i, key_at(first + i));
    }
  };
  // the want-th largest key, two bits a round; done as soon as exactly `want` keys are not below the digits found
  uint32_t least = 0;
  int at_least = n, turn = 0;
#pragma unroll 1
  for (int shift = 30; shift >= 0 && at_least != want; shift -= 2) {
    const uint32_t k1 = least + (1u << shift), k2 = least + (2u << shift), k3 = least + (3u << shift);
    int c1 = 0, c2 = 0, c3 = 0;
    each([&](int, uint32_t k) { c1 += k >= k1; c2 += k >= k2; c3 += k >= k3; });
    int* mine = sums + turn * 3 * kChooseWarps;
    turn ^= 1;
    if constexpr (HELD) {
      const int c = __reduce_add_sync(~0u, c1 | c2 << 10 | c3 << 20);     // 256 of a warp's keys at most
      if (lane == 0) mine[warp] = c;
      __syncthreads();
      c1 = c2 = c3 = 0;
#pragma unroll
      for (int w = 0; w < kChooseWarps; ++w) { c1 += mine[w] & 1023; c2 += mine[w] >> 10 & 1023; c3 += mine[w] >> 20; }
    } else {
      c1 = __reduce_add_sync(~0u, c1); c2 = __reduce_add_sync(~0u, c2); c3 = __reduce_add_sync(~0u, c3);
      if (lane == 0) { mine[warp] = c1; mine[kChooseWarps + warp] = c2; mine[2 * kChooseWarps + warp] = c3; }
      __syncthreads();
      c1 = c2 = c3 = 0;
#pragma unroll
      for (int w = 0; w < kChooseWarps; ++w) { c1 += mine[w]; c2 += mine[kChooseWarps + w]; c3 += mine[2 * kChooseWarps + w]; }
    }
    if (c3 >= want) { least = k3; at_least = c3; }
    else if (c2 >= want) { least = k2; at_least = c2; }
    else if (c1 >= want) { least = k1; at_least = c1; }
  }
  // keys above `least`, then of those equal to it the first ones: places by exclusive sums over the threads
  int above = 0, equal = 0;
  each([&](int, uint32_t k) { above += k > least; equal += k == least; });
  int a = above, e = equal;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const int x = __shfl_up_sync(~0u, a, off), y = __shfl_up_sync(~0u, e, off);
    if (lane >= off) { a += x; e += y; }
  }
  int* mine = sums + turn * 3 * kChooseWarps;
  if (lane == 31) { mine[warp] = a; mine[kChooseWarps + warp] = e; }
  __syncthreads();
  int total_above = 0;
  a -= above;
  e -= equal;
#pragma unroll
  for (int w = 0; w < kChooseWarps; ++w) {
    if (w < warp) { a += mine[w]; e += mine[kChooseWarps + w]; }
    total_above += mine[w];
  }
  const int ties = want - total_above;
  each([&](int i, uint32_t k) {
    if (k > least || (k == least && e < ties)) to[a + min(e, ties)] = i;
    a += k > least;
    e += k == least;
  });
}

template <typename T, int D>
__global__ void __launch_bounds__(kChooseThreads) paged_choose_kernel(const __grid_constant__ ChooseParams P) {
  __shared__ __align__(16) int8_t code[2][D];
  __shared__ float part[kChooseWarps];
  __shared__ int sums[6 * kChooseWarps];
  __shared__ int is_last;
  griddep_launch();
  griddep_wait();
  const PagedParams& A = P.A;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int lane_no = blockIdx.x / P.splits, split = blockIdx.x % P.splits, b = lane_no / A.n_kv_heads, h = lane_no % A.n_kv_heads;
  const int len = clamped_len(A, b), n = (len + A.page - 1) >> A.page_shift;
  // the query's codes
  {
    const int G = A.n_q_heads / A.n_kv_heads;
    float up = 0.f, down = 0.f;
    if (tid < D && n > 0) {
      const T* q = static_cast<const T*>(A.q) + (long long)b * A.q_stride + (long long)h * G * D + tid;
      for (int g = 0; g < G; ++g) {
        const float x = (float)q[g * D];
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
    const float step = __fmul_rn(most, 1.f / 127.f), inv = step >= 0x1p-100f ? __frcp_rn(step) : 0.f;
    if (tid < D) {
      code[0][tid] = (int8_t)(int)fminf(fmaxf(rintf(__fmul_rn(up, inv)), 0.f), 127.f);
      code[1][tid] = (int8_t)(int)fmaxf(fminf(rintf(__fmul_rn(down, inv)), 0.f), -127.f);
    }
    __syncthreads();
  }
  float* scores = P.page_scores + (long long)lane_no * P.page_score_stride;
  // scores: eight lanes a page, D / 8 channels each
  {
    constexpr int kWords = D / 32;                         // per lane, of the largest and of the least
    const int sub = lane & 7;
    int u[kWords], w[kWords];
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      u[i] = reinterpret_cast<const int*>(code[0])[sub * kWords + i];
      w[i] = reinterpret_cast<const int*>(code[1])[sub * kWords + i];
    }
    const int each = ((n + P.splits - 1) / P.splits + 31) & ~31, p1 = min(n, (split + 1) * each);
    constexpr int kSteps = 4, kStride = kChooseWarps * 4;  // pages in flight; pages a step apart
    for (int base = split * each + warp * 4 + (lane >> 3); base - (lane >> 3) < p1; base += kSteps * kStride) {
      int hi[kSteps][kWords], lo[kSteps][kWords];
      float scale[kSteps];
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
#pragma unroll
      for (int k = 0; k < kSteps; ++k) {
        const int p = base + k * kStride;
        int sum = 0;
#pragma unroll
        for (int i = 0; i < kWords; ++i) sum = __dp4a(u[i], hi[k][i], __dp4a(w[i], lo[k][i], sum));
        sum += __shfl_xor_sync(~0u, sum, 1);
        sum += __shfl_xor_sync(~0u, sum, 2);
        sum += __shfl_xor_sync(~0u, sum, 4);
        if (sub == 0 && p < p1) scores[p] = __fmul_rn((float)sum, scale[k]);
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
  }
  __syncthreads();
  const int want = min(P.n_select, n);
  int32_t* to = P.pages + (long long)lane_no * P.n_select;
  for (int i = want + tid; i < P.n_select; i += kChooseThreads) to[i] = -1;
  if (want == n) {
    for (int i = tid; i < n; i += kChooseThreads) to[i] = i;
    return;
  }
  auto key_of = [&](int p) { return p < P.sink || p >= n - P.recent ? kTakenKey : page_key(__ldcg(scores + p)); };
  const int per = (n + kChooseThreads - 1) / kChooseThreads;
  if (per <= kChooseHeld) choose<true>(key_of, per, n, want, to, sums);
  else choose<false>(key_of, per, n, want, to, sums);
}

}  // namespace wkv
