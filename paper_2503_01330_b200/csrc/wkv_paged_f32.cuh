// Paged prompt attention and its accumulated weights on fp32 rows: the CUDA cores' version of wkv_paged_prefill.cuh, same row
// blocks and runs, every product in fp32.
//
// Bound: fp32 FMAs, 4 D flops per (query head, visible entry).  A CTA of 128 threads owns 64 rows (token, query head) and walks
// tiles of 32 entries: a thread computes 4 x 4 logits from 16-byte pieces in shared memory (8 loads for 64 FMAs) and 4 rows x D / 8
// channels of the output (20 loads for 256 FMAs at D = 128).  Row statistics stay among the eight threads of a row.  The next tile
// is copied (cp.async, zeros where there is no row) while this one is worked on.
#pragma once
#include "wkv_paged.cuh"
#include "wkv_paged_prefill.cuh"

namespace wkv {

constexpr int kF32Rows = 64;
constexpr int kF32Keys = 32;
constexpr int kF32Threads = 128;
constexpr int kF32Groups = 4;                // of the weights' kernel: 128 threads each

template <int D>
struct F32Shape {
  static constexpr int kStride = D + 4;                                     // rows on different banks
  static constexpr int kPStride = kF32Keys + 4;
  static constexpr int kSmem = ((kF32Rows + 2 * kF32Keys) * kStride + 2 * kF32Keys * D + kF32Rows * kPStride) * 4;
  static constexpr int kWeightsSmem = (kF32Rows * kStride + kF32Groups * 2 * kF32Keys * (kStride + 1)) * 4;
};

// acc[i][j] = a[ty + 16 i] . b[tx + 8 j]
template <int D>
__device__ __forceinline__ void dot_tile(const float* a, const float* b, int ty, int tx, float (&acc)[4][4]) {
  constexpr int S = F32Shape<D>::kStride;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = 0.f;
#pragma unroll 4
  for (int d = 0; d < D; d += 4) {
    float4 x[4], y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const float4*>(a + (ty + 16 * i) * S + d);
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = *reinterpret_cast<const float4*>(b + (tx + 8 * j) * S + d);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        acc[i][j] = fmaf(x[i].x, y[j].x, fmaf(x[i].y, y[j].y, fmaf(x[i].z, y[j].z, fmaf(x[i].w, y[j].w, acc[i][j]))));
  }
}

// 16 bytes of a row into shared memory, asynchronously: zeros where src is NULL.
__device__ __forceinline__ void stage_piece(float* dst, const float* src, const float* any) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src ? src : any), "r"(src ? 16 : 0) : "memory");
}
__device__ __forceinline__ void stage_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void stage_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Query row R = token * G + g of a row block.
__device__ __forceinline__ const float* query_row(const PagedParams& A, int first, int n, int head, int g_shift, int R, int D) {
  const int tok = R >> g_shift;
  if (tok >= n) return nullptr;
  return static_cast<const float*>(A.q) + (long long)(first + tok) * A.q_stride + (long long)((head << g_shift) + (R & ((1 << g_shift) - 1))) * D;
}

template <int D>
__global__ void __launch_bounds__(kF32Threads) paged_prefill_f32_kernel(const __grid_constant__ PrefillParams P) {
  using Sh = F32Shape<D>;
  extern __shared__ __align__(16) float f32_smem[];
  float* sq = f32_smem;                                       // [64][kStride]
  float* sk = sq + kF32Rows * Sh::kStride;                    // [2][32][kStride]
  float* sv = sk + 2 * kF32Keys * Sh::kStride;                // [2][32][D]
  float* sp = sv + 2 * kF32Keys * D;                          // [64][kPStride]
  const PagedParams& A = P.A;
  griddep_launch();
  griddep_wait();
  const WorkPlan plan = work_plan<kF32Rows, kF32Keys>(A, P.g_shift, P.slots);
  if (blockIdx.x == 0 && threadIdx.x == 0) P.counter[2] = (uint32_t)plan.run;      // for the join
  if ((int)blockIdx.x >= plan.items) return;                // the grid is an upper bound
  PrefillBlock B;
  int r, runs, first_item, v0, v1;
  if (!find_item<kF32Rows, kF32Keys, false>(A, P.g_shift, plan.run, blockIdx.x / A.n_kv_heads, blockIdx.x % A.n_kv_heads, B, r, runs, first_item) ||
      !run_of<kF32Keys>(B, r, runs, plan.run, v0, v1))
    return;
  const int tid = threadIdx.x, ty = tid >> 3, tx = tid & 7;
  constexpr int kVec = D / 4, kRowsPerPass = kF32Threads / kVec;
  const int vec = tid % kVec;
#pragma unroll 8
  for (int r = tid / kVec; r < kF32Rows; r += kRowsPerPass) {
    const float* q = query_row(A, B.first, B.n, B.head, P.g_shift, B.row0 + r, D);
    stage_piece(sq + r * Sh::kStride + vec * 4, q ? q + vec * 4 : nullptr, static_cast<const float*>(A.q));
  }
  auto load_tile = [&](int v) {
    const int buf = v & 1;
#pragma unroll
    for (int k = 0; k < kF32Keys / kRowsPerPass; ++k) {
      const int r = tid / kVec + k * kRowsPerPass, at = v * kF32Keys + r, i = B.entry(at);
      long long off = -1;
      if (at < B.entries && i < B.len) {
        const int pg = page_of(A, B.b, i);
        if (pg >= 0) off = row_offset(A, pg, B.head, i, D) + vec * 4;
      }
      const float *kp = static_cast<const float*>(A.k_pool), *vp = static_cast<const float*>(A.v_pool);
      stage_piece(sk + (buf * kF32Keys + r) * Sh::kStride + vec * 4, off < 0 ? nullptr : kp + off, kp);
      stage_piece(sv + (buf * kF32Keys + r) * D + vec * 4, off < 0 ? nullptr : vp + off, vp);
    }
    stage_commit();
  };
  if (v0 < v1) load_tile(v0);
  constexpr int kPieces = D / 32;                             // float4s of a row that a thread accumulates: channels tx * 4 + 32 j
  float4 o[4][kPieces];
  float m[4], l[4];
  int pos[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    m[i] = -INFINITY;
    l[i] = 0.f;
    pos[i] = B.old + ((B.row0 + ty + 16 * i) >> P.g_shift);
#pragma unroll
    for (int j = 0; j < kPieces; ++j) o[i][j] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  for (int v = v0; v < v1; ++v) {
    __syncthreads();                                          // the tile before has been read
    if (v + 1 < v1) load_tile(v + 1);
    if (v + 1 < v1) stage_wait<1>(); else stage_wait<0>();
    __syncthreads();
    const float *tk = sk + (v & 1) * kF32Keys * Sh::kStride, *tv = sv + (v & 1) * kF32Keys * D;
    float x[4][4];
    dot_tile<D>(sq, tk, ty, tx, x);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float mx = m[i];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int at = v * kF32Keys + tx + 8 * j, e = B.entry(at);
        // an entry in the sinks' pages counts as a sink only
        const bool see = at < B.entries && (at < B.sink_rows ? e < A.sink && e <= pos[i] : visible(e, pos[i], A.window, A.sink));
        x[i][j] = see ? x[i][j] * A.scale_log2 : -INFINITY;
        mx = fmaxf(mx, x[i][j]);
      }
#pragma unroll
      for (int w = 1; w < 8; w <<= 1) mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, w));
      const float ref = mx == -INFINITY ? 0.f : mx, f = exp2_fast(m[i] - ref);
      m[i] = mx;
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float p = exp2_fast(x[i][j] - ref);
        sp[(ty + 16 * i) * Sh::kPStride + tx + 8 * j] = p;
        sum += p;
      }
      l[i] = fmaf(l[i], f, sum);
#pragma unroll
      for (int j = 0; j < kPieces; ++j) { o[i][j].x *= f; o[i][j].y *= f; o[i][j].z *= f; o[i][j].w *= f; }
    }
    __syncwarp();                                             // a row's weights are written and read by its eight threads
#pragma unroll 2
    for (int e = 0; e < kF32Keys; e += 4) {
      float4 p[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) p[i] = *reinterpret_cast<const float4*>(sp + (ty + 16 * i) * Sh::kPStride + e);
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
          const float4 y = *reinterpret_cast<const float4*>(tv + (e + k) * D + j * 32 + tx * 4);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float w = k == 0 ? p[i].x : k == 1 ? p[i].y : k == 2 ? p[i].z : p[i].w;
            o[i][j].x = fmaf(w, y.x, o[i][j].x); o[i][j].y = fmaf(w, y.y, o[i][j].y);
            o[i][j].z = fmaf(w, y.z, o[i][j].z); o[i][j].w = fmaf(w, y.w, o[i][j].w);
          }
        }
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float sum = l[i];
#pragma unroll
    for (int w = 1; w < 8; w <<= 1) sum += __shfl_xor_sync(~0u, sum, w);
    const int row = ty + 16 * i, R = B.row0 + row;
    if (R >= B.n << P.g_shift) continue;
    const bool seen = !(sum <= 0.f);
    if (plan.run == 0x7fffffff) {
      const float inv = seen ? 1.f / sum : 0.f;
      const long long at = (long long)(B.first + (R >> P.g_shift)) * A.n_q_heads + (B.head << P.g_shift) + (R & ((1 << P.g_shift) - 1));
#pragma unroll
      for (int j = 0; j < kPieces; ++j)
        *reinterpret_cast<float4*>(static_cast<float*>(A.out) + at * D + j * 32 + tx * 4) =
            make_float4(o[i][j].x * inv, o[i][j].y * inv, o[i][j].z * inv, o[i][j].w * inv);
      if (A.lse && tx == 0) A.lse[at] = seen ? (m[i] + log2f(sum)) * kLn2 : -INFINITY;
    } else {
#pragma unroll
      for (int j = 0; j < kPieces; ++j) P.part[((long long)blockIdx.x * (D / 4) + j * 8 + tx) * kF32Rows + row] = o[i][j];
      if (tx == 0) P.part_ml[(long long)blockIdx.x * kF32Rows + row] = make_float2(seen ? m[i] : -INFINITY, seen ? sum : 0.f);
    }
  }
}

// scores of 64 entries of one kv head, over all row tiles (32 rows) that see any of them: four groups of 128 threads take every
// fourth tile each, so that an SM has 16 warps however few blocks of entries there are; their sums are added in the groups' order.
template <int D>
__global__ void __launch_bounds__(kF32Groups * kF32Threads) paged_weights_f32_kernel(const __grid_constant__ PrefillParams P) {
  using Sh = F32Shape<D>;
  extern __shared__ __align__(16) float f32_smem[];
  float* sk = f32_smem;                                       // [64][kStride]
  const int group = threadIdx.x / kF32Threads;
  float* sq = sk + (kF32Rows + group * 2 * kF32Keys) * Sh::kStride;                       // [2][32][kStride] of this group
  float* sl = sk + (kF32Rows + kF32Groups * 2 * kF32Keys) * Sh::kStride + group * 2 * kF32Keys;      // [2][32] base-2 log-sums
  const PagedParams& A = P.A;
  griddep_launch();
  griddep_wait();
  const int head = blockIdx.x % A.n_kv_heads, b = blockIdx.x / A.n_kv_heads % A.batch, e0 = blockIdx.x / A.n_kv_heads / A.batch * kF32Rows;
  const SeqRows s = seq_rows(A, b);
  const int old = s.len - s.n, gs = P.g_shift, tid = threadIdx.x % kF32Threads, ty = tid >> 3, tx = tid & 7;
  auto group_sync = [&] { asm volatile("bar.sync %0, 128;" ::"r"(1 + group) : "memory"); };
  if (e0 >= s.len || s.n == 0 || old < 0) return;
  const int t_lo = max(0, e0 - old), e_last = min(e0 + kF32Rows - 1, s.len - 1);
  const long long t_end = A.window == 0 || e0 < A.sink ? s.n : min((long long)s.n, (long long)e_last - old + A.window);
  if (t_end <= t_lo) return;
  const int tile0 = (t_lo << gs) / kF32Keys, tile1 = (int)(((t_end << gs) + kF32Keys - 1) / kF32Keys);
  constexpr int kVec = D / 4, kRowsPerPass = kF32Threads / kVec;
  const int vec = tid % kVec;
#pragma unroll 8
  for (int r = threadIdx.x / kVec; r < kF32Rows; r += kF32Groups * kRowsPerPass) {
    const int i = e0 + r;
    const int pg = i < s.len && seen_from(i, 1, old, A.window, A.sink) ? page_of(A, b, i) : -1;
    const float* kp = static_cast<const float*>(A.k_pool);
    stage_piece(sk + r * Sh::kStride + vec * 4, pg < 0 ? nullptr : kp + row_offset(A, pg, head, i, D) + vec * 4, kp);
  }
  auto load_tile = [&](int it, int buf) {
#pragma unroll
    for (int k = 0; k < kF32Keys / kRowsPerPass; ++k) {
      const int r = tid / kVec + k * kRowsPerPass;
      const float* q = query_row(A, s.first, s.n, head, gs, it * kF32Keys + r, D);
      stage_piece(sq + (buf * kF32Keys + r) * Sh::kStride + vec * 4, q ? q + vec * 4 : nullptr, static_cast<const float*>(A.q));
    }
    if (tid < kF32Keys) {
      const int R = it * kF32Keys + tid, tok = R >> gs;
      sl[buf * kF32Keys + tid] = tok < s.n ? A.lse[(long long)(s.first + tok) * A.n_q_heads + (head << gs) + (R & ((1 << gs) - 1))] * kLog2e : 0.f;
    }
    stage_commit();
  };
  // copies of a thread: its part of K, then a tile each; `buf` alternates with the group's tiles
  const int it0 = tile0 + group;
  if (it0 < tile1) load_tile(it0, 0);
  else stage_commit();
  stage_wait<0>();
  __syncthreads();                                            // K is complete
  float total[4] = {0.f, 0.f, 0.f, 0.f};
  for (int it = it0, buf = 0; it < tile1; it += kF32Groups, buf ^= 1) {
    if (it != it0) {
      stage_wait<0>();
      group_sync();                                           // this tile is there, and the one before has been read
    }
    if (it + kF32Groups < tile1) load_tile(it + kF32Groups, buf ^ 1);
    const float *tq = sq + buf * kF32Keys * Sh::kStride, *tl = sl + buf * kF32Keys;
    float x[4][4];
    dot_tile<D>(sk, tq, ty, tx, x);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = e0 + ty + 16 * i;
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int R = it * kF32Keys + tx + 8 * j, tok = R >> gs;
        if (tok < s.n && visible(e, old + tok, A.window, A.sink)) sum += exp2_fast(fmaf(x[i][j], A.scale_log2, -tl[tx + 8 * j]));
      }
      total[i] += sum;
    }
  }
  __syncthreads();                                            // K has been read: its place takes the groups' sums
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float w = total[i];
#pragma unroll
    for (int d = 1; d < 8; d <<= 1) w += __shfl_xor_sync(~0u, w, d);
    if (tx == 0) sk[group * kF32Rows + ty + 16 * i] = w;
  }
  __syncthreads();
  const int e = e0 + threadIdx.x;
  if (threadIdx.x < kF32Rows && e < s.len) {
    float w = 0.f;
#pragma unroll
    for (int g = 0; g < kF32Groups; ++g) w += sk[g * kF32Rows + threadIdx.x];
    float* a = A.scores + ((long long)b * A.n_kv_heads + head) * A.score_stride + e;
    *a = (A.k && e >= old ? 0.f : *a) + w / (float)(1 << gs);
  }
}

}  // namespace wkv
