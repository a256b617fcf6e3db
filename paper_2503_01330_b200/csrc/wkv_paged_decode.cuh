// Paged decode attention: one new token per sequence over its pages, cut over the length and joined in one launch.
//
//   o = sum_i p_i v_i,  p = softmax(scale q.k_i) over the visible entries
//
// Bound: HBM.  An entry of one kv head costs 2 D elements of traffic and 4 D G flops, so nothing but the copies may be slow.
// The entries of all lanes (sequence, kv head) are cut into tiles and the tiles, in lane order, dealt to the CTAs in equal
// runs: a ragged batch keeps every SM busy to the end, and lengths are read on the device, so that a captured launch
// serves any of them.  A run's piece of a lane becomes a partial (max, sum, output); the CTA that completes a lane -- the last
// of its pieces to arrive, by a counter that nobody waits on -- joins the partials in the order of the pieces.
//
// A CTA: one producer warp that copies the tiles' pages through a tensor map (a page's rows of one head per copy, 128-byte
// swizzle; pages without a visible entry come out of range and cost no traffic) into a ring, and four consumer warps that
// own a quarter of a tile's entries each, with softmax statistics of their own, so that no barrier is needed inside a piece.
// bf16 rows go through mma.sync m16n8k16: the query heads fill rows 0..7 of A (the rest is zero in q.K), and in P.V rows 8..15
// carry the weights' low halves, p - bf16(p), so that the output keeps fp32-like weights at no extra instruction.
//
// Measured: 16 sequences of 8192..16384 tokens, 32 x 128 heads, 487 us = 6.66 TB/s (1.02 of the measured copy rate); one sequence of
// 611 tokens, 32/8 heads, 8.7 us in a captured graph, the length of its chain of dependent loads.
#pragma once
#include "wkv_paged.cuh"

namespace wkv {

constexpr int kDecodeWarps = 4;                           // consumers
constexpr int kDecodeThreads = (kDecodeWarps + 1) * 32;
constexpr int kDecodeRing = 96 * 1024;
constexpr int kMaxSequences = 1024;
constexpr int kJoinTiles = 4;

struct DecodeParams {
  PagedParams A;
  float* part;               // [CTAs + lanes][G][D]: piece of lane l on CTA c at slot c + l (unique: walking the pieces in
  float2* part_ml;           // ... [G] (max, sum)      order, each step moves on to the next CTA or the next lane)
  uint32_t* arrived;         // [lanes], zero between launches
  float* logits;             // [lanes][G][width * page] base-2 logits, or NULL
  float2* head_ml;           // [rows][Hq] (max, 1 / sum) for the fold
  int fold_inside;           // the CTA that completes a lane folds its weights, no second kernel
  int oob_chunk;             // a chunk number outside the pool
  int chunk0;                // the layer's first chunk
  alignas(64) unsigned char kmap[128];   // pool as [chunk][part][row][128 bytes], boxes of one page (or tile) x all parts
  alignas(64) unsigned char vmap[128];
};

__device__ __forceinline__ void tensor_g2s_4d_hint(void* dst, const void* tmap, int x, int y, int z, int w, uint64_t* bar, uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, %3, %4, %5}], [%6], %7;" ::"r"(
          smem_u32(dst)),
      "l"(tmap), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_u32(bar)), "l"(policy)
      : "memory");
}
__device__ __forceinline__ void fence_proxy_async() { asm volatile("fence.proxy.async;" ::: "memory"); }
__device__ __forceinline__ void mma_m16n8k16_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldsm_x4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm_x4_trans(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// What a decode step sees of a sequence, in tiles: those with sinks first, then those from the window's first entry on.
struct DecodeSpan {
  int len, lo, sinks, sink_tiles, first_tile, tiles;
  __device__ __forceinline__ bool sees(int i) const { return i < len && (i >= lo || i < sinks); }
  __device__ __forceinline__ int tile(int v) const { return v < sink_tiles ? v : first_tile + v - sink_tiles; }
};
template <int TILE>
__device__ __forceinline__ DecodeSpan decode_span(int len, int window, int sink) {
  DecodeSpan s;
  s.len = len;
  s.lo = window > 0 ? max(0, len - window) : 0;
  s.sinks = min(sink, s.lo);
  s.first_tile = s.lo / TILE;
  s.sink_tiles = min((s.sinks + TILE - 1) / TILE, s.first_tile);
  s.tiles = max(1, s.sink_tiles + (len + TILE - 1) / TILE - s.first_tile);   // a padded row's one tile is empty: it writes zeros
  return s;
}

template <typename T, int D>
struct DecodeShape {
  static constexpr int kTile = sizeof(T) == 2 ? 64 : 32;
  static constexpr int kRowBytes = D * (int)sizeof(T);
  static constexpr int kParts = kRowBytes / 128;
  static constexpr int kTileBytes = kTile * kRowBytes;            // of K, and of V
  static constexpr int kStages = kDecodeRing / (2 * kTileBytes);
  static constexpr int kOutStride = D + 8;                        // floats; the pad keeps eight heads' float2 stores off one bank
  static constexpr int kEach = kTile / kDecodeWarps;              // entries per consumer warp
  template <int G> static constexpr int smem() {
    return 1024 + kDecodeRing + G * kOutStride * 4 + 2 * kDecodeWarps * 8 * 4 + (2 * kMaxSequences + 8) * 4 + 2 * kStages * 8 + 16;
  }
};

// Byte offset of 16-byte piece c (of the row's kRowBytes / 16) of row r in a tile whose pages hold `pr` rows each.
template <int PARTS>
__device__ __forceinline__ uint32_t tile_offset(int r, int c, int pr, int pr_shift) {
  return (uint32_t)(((r >> pr_shift) * PARTS * pr + (c >> 3) * pr + (r & (pr - 1))) * 128 + (((c ^ r) & 7) << 4));
}

// Largest logit of head g over the four warps; sm_m: [warps][8].
__device__ __forceinline__ float piece_max(const float* sm_m, int g) {
  return fmaxf(fmaxf(sm_m[g], sm_m[8 + g]), fmaxf(sm_m[16 + g], sm_m[24 + g]));
}

// A consumer warp's share of a piece, bf16 rows on the tensor cores.
template <int D, int G>
struct DecodeWarpMma {
  using Sh = DecodeShape<__nv_bfloat16, D>;
  uint32_t q[D / 16][2];
  float o[D / 8][4];
  float m, l;                 // of head lane / 4; l: this lane's columns
  int lane;

  __device__ __forceinline__ void begin(const __nv_bfloat16* qrow, float*) {
    lane = threadIdx.x & 31;
    const int g = lane >> 2, c = (lane & 3) * 2;
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      q[k][0] = g < G ? *reinterpret_cast<const uint32_t*>(qrow + g * D + k * 16 + c) : 0u;
      q[k][1] = g < G ? *reinterpret_cast<const uint32_t*>(qrow + g * D + k * 16 + 8 + c) : 0u;
    }
#pragma unroll
    for (int n = 0; n < D / 8; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
    m = -INFINITY;
    l = 0.f;
  }
  // row0: the warp's first row in the tile; i0: its entry number
  __device__ __forceinline__ void tile(uint32_t tk, uint32_t tv, int row0, int i0, int pr, int pr_shift, const DecodeSpan& s, float scale_log2,
                                       float* logits, long long logit_stride) {
    float x[2][4] = {};
    {
      // K rows as the B operand: matrices (entries 0..7 | 8..15) x (channels 0..7 | 8..15)
      const int r = row0 + (lane & 7) + ((lane >> 4) << 3), c0 = (lane >> 3) & 1;
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        uint32_t b[4];
        ldsm_x4(b, tk + tile_offset<Sh::kParts>(r, 2 * k + c0, pr, pr_shift));
        mma_m16n8k16_bf16(x[0], q[k][0], 0u, q[k][1], 0u, b[0], b[1]);
        mma_m16n8k16_bf16(x[1], q[k][0], 0u, q[k][1], 0u, b[2], b[3]);
      }
    }
    const int c = (lane & 3) * 2, g = lane >> 2;
    float mx = -INFINITY;
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float y = s.sees(i0 + n * 8 + c + e) ? x[n][e] * scale_log2 : -INFINITY;
        x[n][e] = y;
        mx = fmaxf(mx, y);
      }
    if (logits && g < G) {
#pragma unroll
      for (int n = 0; n < 2; ++n)
        *reinterpret_cast<float2*>(logits + g * logit_stride + i0 + n * 8 + c) = make_float2(x[n][0], x[n][1]);
    }
    mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, 1));
    mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, 2));
    const float mn = fmaxf(m, mx), ref = mn == -INFINITY ? 0.f : mn;
    if (__any_sync(~0u, mn > m)) {
      const float f = exp2_fast(m - ref);
      l *= f;
#pragma unroll
      for (int n = 0; n < D / 8; ++n) { o[n][0] *= f; o[n][1] *= f; o[n][2] *= f; o[n][3] *= f; }
      m = mn;
    }
    uint32_t a[4];
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const float p0 = exp2_fast(x[n][0] - ref), p1 = exp2_fast(x[n][1] - ref);
      l += p0 + p1;
      const uint32_t hi = pack_bf16(p0, p1);
      a[2 * n] = hi;
      a[2 * n + 1] = pack_bf16(p0 - __uint_as_float(hi << 16), p1 - __uint_as_float(hi & 0xffff0000u));
    }
    {
      const int r = row0 + (lane & 15), c0 = lane >> 4;
#pragma unroll
      for (int n = 0; n < D / 16; ++n) {
        uint32_t b[4];
        ldsm_x4_trans(b, tv + tile_offset<Sh::kParts>(r, 2 * n + c0, pr, pr_shift));
        mma_m16n8k16_bf16(o[2 * n], a[0], a[1], a[2], a[3], b[0], b[1]);
        mma_m16n8k16_bf16(o[2 * n + 1], a[0], a[1], a[2], a[3], b[2], b[3]);
      }
    }
  }
  __device__ __forceinline__ void stats(float* sm_m, float* sm_l) {     // [8] of this warp
    l += __shfl_xor_sync(~0u, l, 1);
    l += __shfl_xor_sync(~0u, l, 2);
    if ((lane & 3) == 0) { sm_m[lane >> 2] = m; sm_l[lane >> 2] = l; }
  }
  __device__ __forceinline__ void add(float* out, const float* sm_m, bool first) const {
    const int g = lane >> 2, c = (lane & 3) * 2;
    if (g >= G) return;
    const float f = m == -INFINITY ? 0.f : exp2_fast(m - piece_max(sm_m, g));
#pragma unroll
    for (int n = 0; n < D / 8; ++n) {
      float2* at = reinterpret_cast<float2*>(out + g * Sh::kOutStride + n * 8 + c);
      const float2 w = first ? make_float2(0.f, 0.f) : *at;
      *at = make_float2(fmaf(o[n][0] + o[n][2], f, w.x), fmaf(o[n][1] + o[n][3], f, w.y));
    }
  }
};

// ... and fp32 rows on the CUDA cores: four lanes share an entry's dot product, then every lane owns D / 32 output channels.
template <int D, int G>
struct DecodeWarpF32 {
  using Sh = DecodeShape<float, D>;
  static constexpr int kQ = D / 4;          // channels per lane of a quad
  static constexpr int kV = D / 32;
  static constexpr int kQPad = kQ + 4;      // quads' slices start on different banks
  float o[G][kV];
  float m[G], l[G];
  const float* qs;            // this warp's copy in shared memory: [G][4][kQPad]
  int lane;

  __device__ __forceinline__ void begin(const float* qrow, float* scratch) {
    lane = threadIdx.x & 31;
    __syncwarp();
    for (int e = lane; e < G * D; e += 32) scratch[(e / kQ) * kQPad + e % kQ] = qrow[e];
    __syncwarp();
    qs = scratch;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      m[g] = -INFINITY;
      l[g] = 0.f;
#pragma unroll
      for (int e = 0; e < kV; ++e) o[g][e] = 0.f;
    }
  }
  __device__ __forceinline__ static float4 lds4(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
  }
  __device__ __forceinline__ void tile(uint32_t tk, uint32_t tv, int row0, int i0, int pr, int pr_shift, const DecodeSpan& s, float scale_log2,
                                       float* logits, long long logit_stride) {
    const int r = lane >> 2, j = lane & 3;
    float x[G];
#pragma unroll
    for (int g = 0; g < G; ++g) x[g] = 0.f;
#pragma unroll
    for (int c = 0; c < kQ / 4; ++c) {
      const float4 k = lds4(tk + tile_offset<Sh::kParts>(row0 + r, j * (kQ / 4) + c, pr, pr_shift));
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const float4 q = *reinterpret_cast<const float4*>(qs + (g * 4 + j) * kQPad + c * 4);
        x[g] = fmaf(q.x, k.x, fmaf(q.y, k.y, fmaf(q.z, k.z, fmaf(q.w, k.w, x[g]))));
      }
    }
    const bool on = s.sees(i0 + r);
    float ref[G];
#pragma unroll
    for (int g = 0; g < G; ++g) {
      x[g] += __shfl_xor_sync(~0u, x[g], 1);
      x[g] += __shfl_xor_sync(~0u, x[g], 2);
      x[g] = on ? x[g] * scale_log2 : -INFINITY;
      if (logits && j == 0) logits[g * logit_stride + i0 + r] = x[g];
      float mx = x[g];
      mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, 4));
      mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, 8));
      mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, 16));
      const float mn = fmaxf(m[g], mx);
      ref[g] = mn == -INFINITY ? 0.f : mn;
      const float f = exp2_fast(m[g] - ref[g]);
      l[g] *= f;
#pragma unroll
      for (int e = 0; e < kV; ++e) o[g][e] *= f;
      m[g] = mn;
      x[g] = exp2_fast(x[g] - ref[g]);
      l[g] += x[g];
    }
#pragma unroll
    for (int row = 0; row < 8; ++row) {
      float v[kV];
      if constexpr (kV == 4) {
        const float4 t = lds4(tv + tile_offset<Sh::kParts>(row0 + row, lane, pr, pr_shift));
        v[0] = t.x; v[1] = t.y; v[2] = t.z; v[3] = t.w;
      } else {
        asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(v[0]), "=f"(v[1])
                     : "r"(tv + tile_offset<Sh::kParts>(row0 + row, lane >> 1, pr, pr_shift) + (lane & 1) * 8) : "memory");
      }
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const float p = __shfl_sync(~0u, x[g], row * 4);
#pragma unroll
        for (int e = 0; e < kV; ++e) o[g][e] = fmaf(p, v[e], o[g][e]);
      }
    }
  }
  __device__ __forceinline__ void stats(float* sm_m, float* sm_l) {
#pragma unroll
    for (int g = 0; g < G; ++g) {
      float x = l[g];
      x += __shfl_xor_sync(~0u, x, 4);
      x += __shfl_xor_sync(~0u, x, 8);
      x += __shfl_xor_sync(~0u, x, 16);
      if (lane == 0) { sm_m[g] = m[g]; sm_l[g] = x; }
    }
  }
  __device__ __forceinline__ void add(float* out, const float* sm_m, bool first) const {
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const float f = m[g] == -INFINITY ? 0.f : exp2_fast(m[g] - piece_max(sm_m, g));
#pragma unroll
      for (int e = 0; e < kV; ++e) {
        float* at = out + g * Sh::kOutStride + lane * kV + e;
        *at = fmaf(o[g][e], f, first ? 0.f : *at);
      }
    }
  }
};
template <typename T, int D, int G> struct DecodeWarp;
template <int D, int G> struct DecodeWarp<__nv_bfloat16, D, G> : DecodeWarpMma<D, G> {
  static constexpr int kScratch = 0;
};
template <int D, int G> struct DecodeWarp<float, D, G> : DecodeWarpF32<D, G> {
  static constexpr int kScratch = G * 4 * (D / 4 + 4);   // floats per warp
};

// Weights into the running sums: four entries from i0 on, from the parked base-2 logits and the heads' (max, 1 / sum).
template <int G>
__device__ __forceinline__ void fold_entries(const DecodeParams& P, const DecodeSpan& s, long long lane_no, int i0, const float2 (&ml)[G]) {
  const PagedParams& A = P.A;
  if (i0 >= s.len || (i0 + 4 <= s.lo && i0 >= s.sinks)) return;
  const long long stride = (long long)A.width << A.page_shift;
  float w[4] = {};
#pragma unroll
  for (int g = 0; g < G; ++g) {
    const float4 x = __ldcg(reinterpret_cast<const float4*>(P.logits + (lane_no * G + g) * stride + i0));
    w[0] = fmaf(exp2_fast(x.x - ml[g].x), ml[g].y, w[0]);
    w[1] = fmaf(exp2_fast(x.y - ml[g].x), ml[g].y, w[1]);
    w[2] = fmaf(exp2_fast(x.z - ml[g].x), ml[g].y, w[2]);
    w[3] = fmaf(exp2_fast(x.w - ml[g].x), ml[g].y, w[3]);
  }
  float* a = A.scores + lane_no * A.score_stride + i0;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (s.sees(i0 + e)) a[e] = (A.k && i0 + e == s.len - 1 ? 0.f : a[e]) + w[e] * (1.f / G);
}

__device__ __forceinline__ void consumers_sync() { asm volatile("bar.sync 1, 128;" ::: "memory"); }

template <typename T, int D, int G>
constexpr int decode_smem() { return DecodeShape<T, D>::template smem<G>() + kDecodeWarps * DecodeWarp<T, D, G>::kScratch * 4; }

template <typename T, int D, int G>
__global__ void __launch_bounds__(kDecodeThreads, 2) paged_decode_kernel(const __grid_constant__ DecodeParams P) {
  using Sh = DecodeShape<T, D>;
  using Warp = DecodeWarp<T, D, G>;
  constexpr int TILE = Sh::kTile, STAGES = Sh::kStages;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  float* sm_out = reinterpret_cast<float*>(ring + kDecodeRing);                 // [G][kOutStride]
  float* sm_m = sm_out + G * Sh::kOutStride;                                    // [warps][8]
  float* sm_l = sm_m + kDecodeWarps * 8;
  int* lens = reinterpret_cast<int*>(sm_l + kDecodeWarps * 8);                  // [batch]
  int* cum = lens + kMaxSequences;                                              // [batch + 1] tiles of one head before b
  uint64_t* full = reinterpret_cast<uint64_t*>(cum + kMaxSequences + 8);
  uint64_t* empty = full + STAGES;
  int* sm_last = reinterpret_cast<int*>(empty + STAGES);
  float* scratch = reinterpret_cast<float*>(sm_last + 4);

  const PagedParams& A = P.A;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < STAGES; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], kDecodeWarps); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  griddep_launch();
  griddep_wait();
  for (int b = tid; b < A.batch; b += kDecodeThreads) lens[b] = clamped_len(A, b);
  __syncthreads();
  if (warp == 0) {
    int run = 0, most = 0;
    for (int base = 0; base < A.batch; base += 32) {
      const int b = base + lane;
      int n = b < A.batch ? decode_span<TILE>(lens[b], A.window, A.sink).tiles : 0;
      int x = n;
#pragma unroll
      for (int off = 1; off < 32; off <<= 1) {
        const int y = __shfl_up_sync(~0u, x, off);
        if (lane >= off) x += y;
      }
      if (b < A.batch) cum[b] = run + x - n;
      run += __shfl_sync(~0u, x, 31);
      most = max(most, __reduce_max_sync(~0u, n));
    }
    if (lane == 0) { cum[A.batch] = run; cum[A.batch + 1] = most; }
  }
  __syncthreads();
  const int H = A.n_kv_heads, cta = blockIdx.x;
  const long long total = (long long)cum[A.batch] * H;
  const long long chunk = (total + gridDim.x - 1) / gridDim.x;
  long long t0 = cta * chunk, t1 = min(total, t0 + chunk);
  // Few lanes of nearly equal length: a lane each.  Joining a lane costs about as much as four tiles (7000 cycles; under a window of
  // 508, 232 lanes of ten tiles, 21.5 us with lanes cut every eight tiles, 17.2 us whole).
  const long long lanes = (long long)A.batch * H;
  if (lanes <= gridDim.x && cum[A.batch + 1] <= chunk + kJoinTiles) {
    if (cta >= lanes) return;
    const int bb = cta / H, tiles = cum[bb + 1] - cum[bb];
    t0 = (long long)cum[bb] * H + (long long)(cta % H) * tiles;
    t1 = t0 + tiles;
  }
  if (t0 >= t1) return;
  // the first piece: sequence, head, tile
  int b = 0;
  {
    int lo = 0, hi = A.batch;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if ((long long)cum[mid] * H <= t0) lo = mid; else hi = mid;
    }
    b = lo;
  }
  DecodeSpan s = decode_span<TILE>(lens[b], A.window, A.sink);
  int head = (int)((t0 - (long long)cum[b] * H) / s.tiles), v = (int)((t0 - (long long)cum[b] * H) % s.tiles);
  const int pr = min(A.page, TILE), pr_shift = min(A.page_shift, TILE == 64 ? 6 : 5);
  const int boxes = TILE >> pr_shift;
  // No copy is in flight when the CTA ends, without a wait of its own for that: a consumer has waited for each, and where one or the
  // producer gave up, the last copy was issued ahead of that wait, a whole limit ago (a stage that is not released takes no other).
  // (Of a warp's two forms of wait the one by mbar_wait is the faster here: one sequence of 611 tokens 9.0 us, with the other 9.3.)
  auto wait = [&](uint64_t* bar, uint32_t parity) { return (bool)__all_sync(~0u, mbar_wait(bar, parity, A.status, kWaitPolls)); };

  if (warp == kDecodeWarps) {                              // ---- producer
    const uint64_t policy = l2_policy_evict_first();
    fence_proxy_async();                                   // rows that earlier kernels stored are read by the copies
    int it = 0;
    for (long long t = t0; t < t1; ++t, ++it) {
      const int st = it % STAGES;
      // box of this lane: boxes of K first, then of V
      const bool mine = lane < 2 * boxes;
      const int box = lane & (boxes - 1), i = s.tile(v) * TILE + box * pr;
      // does the box hold a visible entry?  [i, i + pr) against [lo, len) and [0, sinks)
      int chunk_no = P.oob_chunk, row = 0;
      if (mine && i < s.len && (i + pr > s.lo || i < s.sinks)) {
        const int pg = page_of(A, b, i);
        if (pg >= 0) { chunk_no = P.chunk0 + pg * H + head; row = i & (A.page - 1); }
      }
      if (it >= STAGES && !wait(&empty[st], ((it / STAGES) & 1) ^ 1)) break;
      unsigned char* dst = ring + st * 2 * Sh::kTileBytes;
      if (lane == 0) mbar_expect_tx(&full[st], 2 * Sh::kTileBytes);
      __syncwarp();
      if (mine)
        tensor_g2s_4d_hint(dst + (lane >= boxes ? Sh::kTileBytes : 0) + box * pr * Sh::kRowBytes, lane >= boxes ? P.vmap : P.kmap, 0, row, 0,
                           chunk_no, &full[st], policy);
      if (++v == s.tiles) {
        v = 0;
        if (++head == H && t + 1 < t1) {
          head = 0;
          s = decode_span<TILE>(lens[++b], A.window, A.sink);
        }
      }
    }
    return;
  }

  // ---- consumers
  Warp w;
  const float scale_log2 = A.scale_log2;
  bool ok = true;          // else a wait gave up: this warp keeps the others' barriers company, and counts its pieces, but reads no more tiles
  int it = 0;
  for (long long t = t0; t < t1;) {
    const int first_v = v;
    const int n = (int)min((long long)(s.tiles - v), t1 - t);            // tiles of this piece
    const long long lane_no = (long long)b * H + head;
    const int hq0 = head * G;
    w.begin(static_cast<const T*>(A.q) + (long long)b * A.q_stride + (long long)hq0 * D, scratch + warp * Warp::kScratch);
    const long long logit_stride = (long long)A.width << A.page_shift;
    float* logits = P.logits ? P.logits + lane_no * G * logit_stride : nullptr;
    // the call's own entry: the warp that owns it in the piece's last tile fetches its rows now, and stores them when it comes to
    // that tile
    constexpr int kPieces = Sh::kRowBytes / 16, kNew = 2 * kPieces / 32 > 0 ? 2 * kPieces / 32 : 1;
    const bool brings = A.k && s.len > 0 && v + n == s.tiles && (s.len - 1) % TILE / Sh::kEach == warp;
    uint4 news[kNew];
    int new_page = -1;
    if (brings) {
      new_page = page_of(A, b, s.len - 1);
      const long long src = (long long)b * A.kv_stride + (long long)head * D;
#pragma unroll
      for (int j = 0; j < kNew; ++j) {
        const int e = lane + 32 * j;
        if (e >= 2 * kPieces) continue;
        const bool is_v = e >= kPieces;
        const int c = (is_v ? e - kPieces : e) * (16 / (int)sizeof(T));
        news[j] = *reinterpret_cast<const uint4*>(static_cast<const T*>(is_v ? A.v : A.k) + src + c);
      }
    }
    for (int k = 0; k < n; ++k, ++it, ++v) {
      const int st = it % STAGES;
      unsigned char* tk = ring + st * 2 * Sh::kTileBytes;
      unsigned char* tv = tk + Sh::kTileBytes;
      ok = ok && wait(&full[st], (it / STAGES) & 1);
      if (!ok) continue;
      const int row0 = warp * Sh::kEach, i0 = s.tile(v) * TILE + row0;
      // entries [i0, i0 + kEach) against the visible ones
      const bool any = i0 < s.len && (i0 + Sh::kEach > s.lo || i0 < s.sinks);
      if (any) {
        const bool all = i0 + Sh::kEach <= s.len && (i0 >= s.lo || i0 + Sh::kEach <= s.sinks);
        const bool fresh = brings && k == n - 1;
        if (!all || fresh) {
          // rows that nobody sees may hold anything: their weight is zero, their values have to be finite
          for (int e = lane; e < Sh::kEach * kPieces; e += 32) {
            const int r = e / kPieces;
            if (!s.sees(i0 + r))
              *reinterpret_cast<uint4*>(tv + tile_offset<Sh::kParts>(row0 + r, e % kPieces, pr, pr_shift)) = make_uint4(0, 0, 0, 0);
          }
          if (fresh) {
#pragma unroll
            for (int j = 0; j < kNew; ++j) {
              const int e = lane + 32 * j;
              if (e >= 2 * kPieces) continue;
              const bool is_v = e >= kPieces;
              *reinterpret_cast<uint4*>((is_v ? tv : tk) + tile_offset<Sh::kParts>(s.len - 1 - i0 + row0, e % kPieces, pr, pr_shift)) =
                  new_page >= 0 ? news[j] : make_uint4(0, 0, 0, 0);
              if (new_page >= 0)
                *reinterpret_cast<uint4*>(static_cast<T*>(is_v ? A.v_pool : A.k_pool) + row_offset(A, new_page, head, s.len - 1, D) +
                                          e % kPieces * (16 / (int)sizeof(T))) = news[j];
            }
          }
          __syncwarp();
        }
        w.tile(smem_u32(tk), smem_u32(tv), row0, i0, pr, pr_shift, s, scale_log2, logits, logit_stride);
        if (!all || fresh) fence_proxy_async();           // plain stores to the stage ahead of the copy that refills it
      }
      release_stage(&empty[st]);
    }
    // join the four warps, in their order
    w.stats(sm_m + warp * 8, sm_l + warp * 8);
    consumers_sync();
    float my_M = 0.f, my_L = 0.f;                          // of head tid
    if (tid < G) {
      my_M = piece_max(sm_m, tid);
#pragma unroll
      for (int i = 0; i < kDecodeWarps; ++i) {
        const float mi = sm_m[i * 8 + tid];
        my_L += mi == -INFINITY ? 0.f : sm_l[i * 8 + tid] * exp2_fast(mi - my_M);
      }
    }
#pragma unroll
    for (int i = 0; i < kDecodeWarps; ++i) {
      if (warp == i) w.add(sm_out, sm_m, i == 0);
      consumers_sync();
    }
    if (tid < G) { sm_m[tid] = my_M; sm_l[tid] = my_L; }      // of the piece
    consumers_sync();
    const bool whole = n == s.tiles;
    if (!whole) {
      const long long slot = cta + lane_no;
      for (int e = tid; e < G * D / 4; e += 128) {
        const int g = e / (D / 4), c = e % (D / 4) * 4;
        reinterpret_cast<float4*>(P.part + slot * G * D)[e] = *reinterpret_cast<const float4*>(sm_out + g * Sh::kOutStride + c);
      }
      if (tid < G) P.part_ml[slot * G + tid] = make_float2(sm_m[tid], sm_l[tid]);
      __threadfence();
      consumers_sync();
      // pieces of the lane: its tiles lie at [off, off + tiles) of the deal
      const long long off = (long long)cum[b] * H + (long long)head * s.tiles;
      const int c0 = (int)(off / chunk), pieces = (int)((off + s.tiles - 1) / chunk) - c0 + 1;
      if (tid == 0) {
        const bool last = atomicAdd(P.arrived + lane_no, 1u) == (uint32_t)pieces - 1;
        if (last) P.arrived[lane_no] = 0;
        *sm_last = last;
      }
      consumers_sync();
      if (*sm_last) {
        __threadfence();
        const long long slot0 = c0 + lane_no;
        for (int e = tid; e < G * D / 4; e += 128) {
          const int g = e / (D / 4), c = e % (D / 4) * 4;
          float mm = -INFINITY, sum = 0.f;
          float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
          for (int i0 = 0; i0 < pieces; i0 += 8) {         // eight pieces' loads in flight together
            float2 ml[8];
            float4 x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const bool in = i0 + i < pieces;
              ml[i] = in ? __ldcg(&P.part_ml[(slot0 + i0 + i) * G + g]) : make_float2(-INFINITY, 0.f);
              x[i] = in ? __ldcg(&reinterpret_cast<const float4*>(P.part + (slot0 + i0 + i) * G * D)[e]) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
            float mn = mm;
#pragma unroll
            for (int i = 0; i < 8; ++i) mn = fmaxf(mn, ml[i].x);
            const float f0 = mm == -INFINITY ? 0.f : exp2_fast(mm - mn);
            sum *= f0;
            acc.x *= f0; acc.y *= f0; acc.z *= f0; acc.w *= f0;
            mm = mn;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float f = ml[i].x == -INFINITY ? 0.f : exp2_fast(ml[i].x - mm);
              sum = fmaf(ml[i].y, f, sum);
              acc.x = fmaf(x[i].x, f, acc.x); acc.y = fmaf(x[i].y, f, acc.y); acc.z = fmaf(x[i].z, f, acc.z); acc.w = fmaf(x[i].w, f, acc.w);
            }
          }
          *reinterpret_cast<float4*>(sm_out + g * Sh::kOutStride + c) = acc;
          if (c == 0) { sm_m[g] = mm; sm_l[g] = sum; }
        }
      }
      consumers_sync();
    }
    if (whole || *sm_last) {
      for (int e = tid; e < G * D / 4; e += 128) {
        const int g = e / (D / 4), c = e % (D / 4) * 4;
        const float4 x = *reinterpret_cast<const float4*>(sm_out + g * Sh::kOutStride + c);
        const float inv = sm_l[g] > 0.f ? 1.f / sm_l[g] : 0.f;
        T* out = static_cast<T*>(A.out) + ((long long)b * A.n_q_heads + hq0 + g) * D + c;
        if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf16(x.x * inv, x.y * inv), pack_bf16(x.z * inv, x.w * inv));
        else *reinterpret_cast<float4*>(out) = make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv);
      }
      if (tid < G) {
        const long long at = (long long)b * A.n_q_heads + hq0 + tid;
        if (A.lse) A.lse[at] = sm_l[tid] > 0.f ? (sm_m[tid] + log2f(sm_l[tid])) * kLn2 : -INFINITY;
        if (P.logits && !P.fold_inside) P.head_ml[at] = make_float2(sm_m[tid], sm_l[tid] > 0.f ? 1.f / sm_l[tid] : 0.f);
      }
      if (P.fold_inside) {
        float2 ml[G];
#pragma unroll
        for (int g = 0; g < G; ++g) ml[g] = make_float2(sm_m[g], sm_l[g] > 0.f ? 1.f / sm_l[g] : 0.f);
        for (int i0 = tid * 4; i0 < s.len; i0 += 512) fold_entries<G>(P, s, lane_no, i0, ml);
      }
    }
    consumers_sync();                                      // sm_* are free for the next piece
    t += n;
    if (first_v + n == s.tiles) {
      v = 0;
      if (++head == H && t < t1) {
        head = 0;
        s = decode_span<TILE>(lens[++b], A.window, A.sink);
      }
    }
  }
}

// The fold as a kernel of its own, for lanes that may be long: 1024 entries a CTA.
constexpr int kFoldEntries = 1024;
constexpr int kFoldInside = 2048;      // entries that the decode kernel folds itself: 512 a consumer warp, less than a launch takes
template <int G>
__global__ void __launch_bounds__(kFoldEntries / 4) paged_fold_kernel(const __grid_constant__ DecodeParams P, int blocks_per_lane) {
  griddep_wait();
  const PagedParams& A = P.A;
  const int lane_no = blockIdx.x / blocks_per_lane, b = lane_no / A.n_kv_heads, head = lane_no % A.n_kv_heads;
  const int i0 = blockIdx.x % blocks_per_lane * kFoldEntries + threadIdx.x * 4;
  float2 ml[G];
#pragma unroll
  for (int g = 0; g < G; ++g) ml[g] = P.head_ml[(long long)b * A.n_q_heads + head * G + g];
  fold_entries<G>(P, decode_span<64>(clamped_len(A, b), A.window, A.sink), lane_no, i0, ml);
}

}  // namespace wkv
