// Paged decode attention on rows in 4 bits: one token per sequence over its pages, or over a list of chosen pages.
//
//   o = sum_i p_i v_i,  p = softmax(scale q.k_i),  k_i = s_ig (n - z_ig) per group g of 32 channels, v_i likewise
//
// Bound: HBM at 4.5 bits a number; instruction issue close behind it, since a number may cost no more than about three lane instructions.
// Codes are never converted: a masked word is two fp16 subnormals n 2^-24 (or n 2^-20), which mma.sync m16n8k16 takes exactly.  Scales and
// zero points stay outside of the products:
//   q.k_i  = sum_g s_ig (q_g.n_ig - z_ig sum q_g)        groups' products in accumulators of their own
//   o_g    = sum_i (p_i s_ig) n_ig - sum_i (p_i s_ig) z_ig   the weights p s in fp16, the same rounded ones in both sums
// Rounding p s to fp16 costs 2^-11 of it, an eighth of what rounding the output to bf16 does.  The weights are kept in fp16's range
// by a power of two that follows the largest value scale seen.  Queries become fp16 by a power of two per head (exact down to 2^-28 of the
// head's largest channel).
//
// The deal of tiles to CTAs, pieces of a lane and their join are those of the bf16 rows' kernel.  A CTA: one producer warp, which looks up 32
// pages at a time and copies their chunks into a ring (cp.async.bulk), and eight consumer warps with 16 of a tile's 128 entries each.
#pragma once
#include "wkv_paged_decode.cuh"
#include "wkv_paged_kv4.cuh"

namespace wkv {

constexpr int kKv4Warps = 8;                              // consumers
constexpr int kKv4Threads = (kKv4Warps + 1) * 32;
constexpr int kKv4Tile = 16 * kKv4Warps;
constexpr int kKv4MaxSlots = kKv4Tile / 16;               // pages of a tile

template <int D, int G>
struct Kv4Shape {
  using Row = Kv4Row<D>;
  static constexpr int kHalf = kKv4Tile * Row::kBytes;    // keys of a tile; values
  static constexpr int kStage = 2 * kHalf;
  static constexpr int kStages = (G == 8 && D == 128 ? 54 : 72) * 1024 / kStage;
  static constexpr int kOut = kKv4Warps * G * D * 4;      // the warps' outputs
  static constexpr int kScratch = kKv4Warps * 16 * G * 4; // weights of a warp's 16 entries
  static constexpr int kSmem = kStages * kStage + kOut + kScratch + 2 * kKv4Warps * 8 * 4 + (2 * kMaxSequences + 8) * 4 + 2 * kStages * 8 +
                               kStages * kKv4MaxSlots * 4 + 16;
};

__device__ __forceinline__ void mma_m16n8k16_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float pow2f(int e) { return __int_as_float((e + 127) << 23); }       // -126 <= e <= 127
__device__ __forceinline__ uint32_t half_pair(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float2 half_pair_f(uint32_t x) { return __half22float2(*reinterpret_cast<const __half2*>(&x)); }

// A consumer warp's share of a piece.  Lane 4 r + j.  Columns of the products' results are heads n % G (repeated where G < 8): a lane's
// statistics are those of heads 2j % G and (2j + 1) % G.
template <int D, int G>
struct Kv4Warp {
  using Row = Kv4Row<D>;
  static constexpr int kGroups = Row::kGroups;
  static constexpr int kFrags = G <= 2 ? 1 : kGroups * G / 8 > 0 ? kGroups * G / 8 : 1;   // weights' fragments: columns are (group, head) pairs
  static constexpr float kHeadroom = 256.f;
  uint32_t q[kGroups][4];      // key products' B operand: two steps of 16 channels per group
  float qsum[kGroups][2];      // sum of a group's channels, heads 2j and 2j + 1
  float factor[2];             // accumulator -> base-2 logit
  float o[D / 16][4];          // values' products: tile (group, half): channels 4r + 2 half and + 1, columns 2j and 2j + 1
  float zsum[kFrags];          // sum of (p s) z for column r of a fragment, this lane's entries
  float m[2], l[2];
  uint32_t largest;            // scale byte that the weights' power of two follows
  float shift;
  int lane;

  // Group and head of column n of fragment f.
  __device__ __forceinline__ static int group_of(int f, int n) { return G == 1 ? n % kGroups : (f * (8 / G) + n / G) % kGroups; }
  __device__ __forceinline__ static int head_of(int n) { return n % G; }
  __device__ __forceinline__ static int frag_of(int g) { return G <= 2 ? 0 : g * G / 8; }

  __device__ __forceinline__ void begin(const __nv_bfloat16* qrow, float scale_log2) {
    lane = threadIdx.x & 31;
    const int r = lane >> 2, j = lane & 3;
    float x[kGroups][8], most = 0.f;
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      const uint4 u = *reinterpret_cast<const uint4*>(qrow + (r % G) * D + g * 32 + 8 * j);
      const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) { x[g][2 * i] = __uint_as_float(w[i] << 16); x[g][2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
#pragma unroll
      for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(x[g][i]));
    }
    most = fmaxf(most, __shfl_xor_sync(~0u, most, 1));
    most = fmaxf(most, __shfl_xor_sync(~0u, most, 2));
    // the head's largest channel comes to [2^14, 2^15)
    const int e = max(-100, min(100, 14 - ((int)(__float_as_uint(most) >> 23) - 127)));
    const float up = pow2f(e);
    float f = scale_log2 * pow2f(-e) * 0x1p24f;
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        q[g][i] = half_pair(x[g][2 * i] * up, x[g][2 * i + 1] * up);
        const float2 back = half_pair_f(q[g][i]);
        sum += back.x + back.y;
        if (i & 1) q[g][i] = half_pair(back.x * 0.0625f, back.y * 0.0625f);   // meets codes in bits 4..7
      }
      sum += __shfl_xor_sync(~0u, sum, 1);
      sum += __shfl_xor_sync(~0u, sum, 2);
      qsum[g][0] = __shfl_sync(~0u, sum, 8 * j) * 0x1p-24f;
      qsum[g][1] = __shfl_sync(~0u, sum, 8 * j + 4) * 0x1p-24f;
    }
    factor[0] = __shfl_sync(~0u, f, 8 * j);
    factor[1] = __shfl_sync(~0u, f, 8 * j + 4);
#pragma unroll
    for (int n = 0; n < D / 16; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
#pragma unroll
    for (int n = 0; n < kFrags; ++n) zsum[n] = 0.f;
    m[0] = m[1] = -INFINITY;
    l[0] = l[1] = 0.f;
    largest = 0;
    shift = 0.f;
  }

  // 16 entries from i0 on, rows row0 .. of their page; tk, tv: the page's chunks; weights: scratch of this warp, [G][16].
  // bad: the page's number is none, its entries count as zeros.
  __device__ __forceinline__ void tile(const unsigned char* tk, const unsigned char* tv, int page, int row0, int i0, bool all, bool bad, const DecodeSpan& s, float* weights) {
    const int r = lane >> 2, j = lane & 3;
    float x[4] = {};                                       // rows r and r + 8, heads 2j and 2j + 1
    {
      const unsigned char* at = tk + Row::pairs(page, row0 + r);
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
        float d[4] = {};
        uint32_t a[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t w = *reinterpret_cast<const uint32_t*>(tk + Row::k_piece(row0 + r + 8 * h, g) + 4 * j);
          a[h][0] = w & 0x000f000fu;
          a[h][1] = w & 0x00f000f0u;
          a[h][2] = w >> 8 & 0x000f000fu;
          a[h][3] = w >> 8 & 0x00f000f0u;
        }
        mma_m16n8k16_f16(d, a[0][0], a[1][0], a[0][1], a[1][1], q[g][0], q[g][1]);
        mma_m16n8k16_f16(d, a[0][2], a[1][2], a[0][3], a[1][3], q[g][2], q[g][3]);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t pair = *reinterpret_cast<const uint16_t*>(at + h * 8 * Row::kPairs + 2 * g);
          const float sc = kv4_scale(pair & 255), z = (float)(pair >> 8);
          x[2 * h] = fmaf(sc, fmaf(-z, qsum[g][0], d[2 * h]), x[2 * h]);
          x[2 * h + 1] = fmaf(sc, fmaf(-z, qsum[g][1], d[2 * h + 1]), x[2 * h + 1]);
        }
      }
    }
    float mx[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float y = bad ? 0.f : x[2 * h + c] * factor[c];
        if (!all) y = s.sees(i0 + r + 8 * h) ? y : -INFINITY;
        x[2 * h + c] = y;
      }
      mx[c] = fmaxf(x[c], x[2 + c]);
#pragma unroll
      for (int off = 4; off < 32; off <<= 1) mx[c] = fmaxf(mx[c], __shfl_xor_sync(~0u, mx[c], off));
      mx[c] = fmaxf(m[c], mx[c]);
    }
    // scales and zero points of the values: entries j + 4t, the group of column r
    uint32_t pair[kFrags][4];
    uint32_t top = 0;
#pragma unroll
    for (int f = 0; f < kFrags; ++f)
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        uint32_t y = *reinterpret_cast<const uint16_t*>(tv + Row::pairs(page, row0 + j + 4 * t) + 2 * group_of(f, r));
        if (!all || bad) y = s.sees(i0 + j + 4 * t) && !bad ? y : 0u;
        pair[f][t] = y;
        top = max(top, y & 255);
      }
    top = max(__reduce_max_sync(~0u, top), largest);
    if (__any_sync(~0u, mx[0] > m[0] || mx[1] > m[1]) || top != largest) {
      // 2^15-e: the largest scale comes to [1, 2)
      const float to = pow2f(15 - max(1, (int)(top >> 3))) * kHeadroom, ratio = largest ? to / shift : 0.f;
      float f[2];
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const float ref = mx[c] == -INFINITY ? 0.f : mx[c];
        const float g = exp2_fast(m[c] - ref);
        l[c] *= g;
        f[c] = g * ratio;
        m[c] = mx[c];
      }
#pragma unroll
      for (int n = 0; n < D / 16; ++n) { o[n][0] *= f[0]; o[n][1] *= f[1]; o[n][2] *= f[0]; o[n][3] *= f[1]; }
      // column r's head is head r % G: its factor is with lane j = (r % 8) / 2
      const float f0 = __shfl_sync(~0u, f[0], r >> 1), f1 = __shfl_sync(~0u, f[1], r >> 1);
#pragma unroll
      for (int n = 0; n < kFrags; ++n) zsum[n] *= r & 1 ? f1 : f0;
      if (top) { largest = top; shift = to; }
    }
    // weights: entry e of a head at place (e % 4) * 4 + e / 4
    __syncwarp();
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const float ref = m[c] == -INFINITY ? 0.f : m[c];
      const float p0 = exp2_fast(x[c] - ref), p1 = exp2_fast(x[2 + c] - ref);
      l[c] += p0 + p1;
      if (2 * j + c < G) {
        weights[(2 * j + c) * 16 + (r & 3) * 4 + (r >> 2)] = p0;
        weights[(2 * j + c) * 16 + (r & 3) * 4 + (r >> 2) + 2] = p1;
      }
    }
    __syncwarp();
    const float4 p = *reinterpret_cast<const float4*>(weights + head_of(r) * 16 + 4 * j);
    uint32_t b[kFrags][2];
#pragma unroll
    for (int f = 0; f < kFrags; ++f) {
      const float w0 = p.x * shift * kv4_scale(pair[f][0] & 255), w1 = p.y * shift * kv4_scale(pair[f][1] & 255);
      const float w2 = p.z * shift * kv4_scale(pair[f][2] & 255), w3 = p.w * shift * kv4_scale(pair[f][3] & 255);
      b[f][0] = half_pair(w0, w1);
      b[f][1] = half_pair(w2, w3);
      const float2 x0 = half_pair_f(b[f][0]), x1 = half_pair_f(b[f][1]);
      zsum[f] = fmaf(x0.x, (float)(pair[f][0] >> 8), fmaf(x0.y, (float)(pair[f][1] >> 8), fmaf(x1.x, (float)(pair[f][2] >> 8), fmaf(x1.y, (float)(pair[f][3] >> 8), zsum[f]))));
    }
    // values: units r of every group, of entries j + 4t
    uint32_t w[4][kGroups / 2];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const unsigned char* at = tv + Row::v_unit(row0 + j + 4 * t, 0, r);
      if constexpr (kGroups == 4) {
        const uint2 y = *reinterpret_cast<const uint2*>(at);
        w[t][0] = y.x;
        w[t][1] = y.y;
      } else {
        w[t][0] = *reinterpret_cast<const uint32_t*>(at);
      }
    }
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      // entries j | j + 4 and j + 8 | j + 12 side by side
      const uint32_t lo = __byte_perm(w[0][g / 2], w[1][g / 2], g & 1 ? 0x7632 : 0x5410), hi = __byte_perm(w[2][g / 2], w[3][g / 2], g & 1 ? 0x7632 : 0x5410);
      const uint32_t lo8 = lo >> 8, hi8 = hi >> 8;
      const int f = frag_of(g);
      mma_m16n8k16_f16(o[2 * g], lo & 0x000f000fu, lo & 0x00f000f0u, hi & 0x000f000fu, hi & 0x00f000f0u, b[f][0], b[f][1]);
      mma_m16n8k16_f16(o[2 * g + 1], lo8 & 0x000f000fu, lo8 & 0x00f000f0u, hi8 & 0x000f000fu, hi8 & 0x00f000f0u, b[f][0], b[f][1]);
    }
  }

  // (max, sum) of the heads over this warp's entries to [8] each
  __device__ __forceinline__ void stats(float* sm_m, float* sm_l) {
    const int j = lane & 3;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
#pragma unroll
      for (int off = 4; off < 32; off <<= 1) l[c] += __shfl_xor_sync(~0u, l[c], off);
      if (lane < 4 && 2 * j + c < G) { sm_m[2 * j + c] = m[c]; sm_l[2 * j + c] = l[c]; }
    }
  }
  // The warp's output [G][D], relative to the heads' maxima big[G]; zeros: scratch, [groups][G].
  __device__ __forceinline__ void write(float* out, const float* big, float* zeros) {
    const int r = lane >> 2, j = lane & 3;
    __syncwarp();
#pragma unroll
    for (int f = 0; f < kFrags; ++f) {
      float z = zsum[f];
      z += __shfl_xor_sync(~0u, z, 1);
      z += __shfl_xor_sync(~0u, z, 2);
      // column r of fragment f, once
      if (j == 0 && (G > 1 || r < kGroups) && (f * (8 / G) + r / G < kGroups || G == 1)) zeros[group_of(f, r) * G + head_of(r)] = z;
    }
    __syncwarp();
    const float back = largest ? 1.f / shift : 0.f;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int col = 2 * j + c, head = head_of(col);
      const float f = m[c] == -INFINITY ? 0.f : exp2_fast(m[c] - big[head]) * back;
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
        if (G == 1 ? col != g : frag_of(g) * (8 / G) + col / G != g) continue;
        const float z = zeros[g * G + head];
#pragma unroll
        for (int half = 0; half < 2; ++half)
          *reinterpret_cast<float2*>(out + head * D + g * 32 + 4 * r + 2 * half) =
              make_float2((o[2 * g + half][c] * 0x1p24f - z) * f, (o[2 * g + half][2 + c] * 0x1p20f - z) * f);
      }
    }
  }
};

__device__ __forceinline__ void kv4_consumers_sync() { asm volatile("bar.sync 1, %0;" ::"n"(kKv4Warps * 32) : "memory"); }

template <int D, int G, bool CHOSEN>
__global__ void __launch_bounds__(kKv4Threads, 2) paged_decode_kv4_kernel(const __grid_constant__ DecodeParams P) {
  using Sh = Kv4Shape<D, G>;
  using Row = Kv4Row<D>;
  using Warp = Kv4Warp<D, G>;
  constexpr int TILE = kKv4Tile, STAGES = Sh::kStages;
  extern __shared__ __align__(128) unsigned char ring[];
  float* sm_out = reinterpret_cast<float*>(ring + STAGES * Sh::kStage);         // [warps][G][D]
  float* scratch = sm_out + kKv4Warps * G * D;                                  // [warps][G][16]
  float* sm_m = scratch + kKv4Warps * 16 * G;                                   // [warps][8]
  float* sm_l = sm_m + kKv4Warps * 8;
  int* lens = reinterpret_cast<int*>(sm_l + kKv4Warps * 8);                     // [batch]
  int* cum = lens + kMaxSequences;                                              // [batch + 1] tiles of one head before b, then the most
  int* slot_entry = cum + kMaxSequences + 8;                                    // [stages][slots] first entry of a page, see below
  uint64_t* full = reinterpret_cast<uint64_t*>(slot_entry + STAGES * kKv4MaxSlots);
  uint64_t* empty = full + STAGES;
  int* sm_last = reinterpret_cast<int*>(empty + STAGES);

  const PagedParams& A = P.A;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  auto span = [&](int len) {
    if constexpr (CHOSEN) return chosen_span<TILE>(A, len, P.n_select);
    else return decode_span<TILE>(len, A.window, A.sink);
  };
  if (tid == 0) {
    for (int i = 0; i < STAGES; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], kKv4Warps); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  griddep_launch();
  griddep_wait();
  for (int b = tid; b < A.batch; b += kKv4Threads) lens[b] = clamped_len(A, b);
  __syncthreads();
  if (warp == 0) {
    int run = 0, most = 0;
    for (int base = 0; base < A.batch; base += 32) {
      const int b = base + lane;
      int n = b < A.batch ? span(lens[b]).tiles : 0;
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
  // few lanes of nearly equal length: a lane each, as in the bf16 rows' kernel
  const long long lanes = (long long)A.batch * H;
  if (lanes <= gridDim.x && cum[A.batch + 1] <= chunk + kJoinTiles) {
    if (cta >= lanes) return;
    const int bb = cta / H, tiles = cum[bb + 1] - cum[bb];
    t0 = (long long)cum[bb] * H + (long long)(cta % H) * tiles;
    t1 = t0 + tiles;
  }
  if (t0 >= t1) return;
  int b = 0;
  {
    int lo = 0, hi = A.batch;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if ((long long)cum[mid] * H <= t0) lo = mid; else hi = mid;
    }
    b = lo;
  }
  DecodeSpan s = span(lens[b]);
  int head = (int)((t0 - (long long)cum[b] * H) / s.tiles), v = (int)((t0 - (long long)cum[b] * H) % s.tiles);
  const int slots = TILE >> A.page_shift, slot_shift = 7 - A.page_shift;
  const uint32_t chunk_bytes = (uint32_t)A.page * Row::kBytes;
  // copies in flight at the end: as in the bf16 rows' kernel, there are none
  auto wait = [&](uint64_t* bar, uint32_t parity) { return (bool)__all_sync(~0u, mbar_wait(bar, parity, A.status, kWaitPolls)); };
  // Where page `slot` of a tile starts: its first entry, which is seen or not; of a bad page ~entry; the sequence's length if the page
  // holds nothing visible (so that no entry in it is).
  if (warp == kKv4Warps) {                                 // ---- producer
    const uint64_t policy = l2_policy_evict_first();
    fence_proxy_async();                                   // rows that earlier kernels stored are read by the copies
    int it = 0;
    for (long long t = t0; t < t1;) {
      const int n = (int)min((long long)(s.tiles - v), t1 - t);
      const int per = 32 >> slot_shift;                    // tiles whose pages are looked up together
      const long long lane_no = (long long)b * H + head;
      for (int k0 = 0; k0 < n; k0 += per) {
        int entry = s.len, page_no = -1;
        {
          const int k = k0 + (lane >> slot_shift), slot = lane & (slots - 1);
          if (k < n) {
            int i = s.tile(v + k) * TILE + (slot << A.page_shift);
            if constexpr (CHOSEN) {
              const int at = i >> A.page_shift, pages = (s.len + A.page - 1) >> A.page_shift;
              const int pg = at < min(P.n_select, pages) ? P.pages[lane_no * P.n_select + at] : -1;
              i = (unsigned)pg < (unsigned)pages ? pg << A.page_shift : s.len;
            }
            if (i < s.len && (i + A.page > s.lo || i < s.sinks)) {
              page_no = page_of(A, b, i);
              entry = page_no < 0 ? ~i : i;
            }
          }
        }
        for (int k = k0; k < min(n, k0 + per); ++k, ++it) {
          const int st = it % STAGES;
          const int mine = (k - k0) << slot_shift | (lane & (slots - 1));
          const int e = __shfl_sync(~0u, entry, mine), pg = __shfl_sync(~0u, page_no, mine);
          if (it >= STAGES && !wait(&empty[st], ((it / STAGES) & 1) ^ 1)) return;
          const bool copies = lane < 2 * slots && pg >= 0;
          const uint32_t bytes = __popc(__ballot_sync(~0u, copies)) * chunk_bytes;
          if (lane < slots) slot_entry[st * kKv4MaxSlots + lane] = e;
          __threadfence_block();
          __syncwarp();
          if (lane == 0) mbar_expect_tx(&full[st], bytes);
          __syncwarp();
          if (copies) {
            const bool is_v = lane >= slots;
            const unsigned char* src = static_cast<const unsigned char*>(is_v ? A.v_pool : A.k_pool) + ((long long)pg * H + head) * chunk_bytes;
            bulk_g2s_hint(ring + st * Sh::kStage + (is_v ? Sh::kHalf : 0) + (lane & (slots - 1)) * chunk_bytes, src, chunk_bytes, &full[st], policy);
          }
        }
      }
      t += n;
      v += n;
      if (v == s.tiles) {
        v = 0;
        if (++head == H && t < t1) {
          head = 0;
          s = span(lens[++b]);
        }
      }
    }
    return;
  }

  // ---- consumers
  Warp w;
  bool ok = true;          // else a wait gave up: this warp keeps the others' barriers company, and counts its pieces, but reads no more tiles
  int it = 0;
  float* weights = scratch + warp * 16 * G;
  const int row = warp * 16, my_slot = row >> A.page_shift, row0 = row & (A.page - 1);
  for (long long t = t0; t < t1;) {
    const int first_v = v;
    const int n = (int)min((long long)(s.tiles - v), t1 - t);            // tiles of this piece
    const long long lane_no = (long long)b * H + head;
    const int hq0 = head * G;
    w.begin(static_cast<const __nv_bfloat16*>(A.q) + (long long)b * A.q_stride + (long long)hq0 * D, A.scale_log2);
    for (int k = 0; k < n; ++k, ++it, ++v) {
      const int st = it % STAGES;
      ok = ok && wait(&full[st], (it / STAGES) & 1);
      if (!ok) continue;
      const int e = slot_entry[st * kKv4MaxSlots + my_slot];
      const bool bad = e < 0;
      const int i0 = (bad ? ~e : e) + row0;
      if (i0 < s.len && (i0 + 16 > s.lo || i0 < s.sinks)) {
        const bool all = i0 + 16 <= s.len && (i0 >= s.lo || i0 + 16 <= s.sinks);
        const unsigned char* tk = ring + st * Sh::kStage + my_slot * chunk_bytes;
        w.tile(tk, tk + Sh::kHalf, A.page, row0, i0, all, bad, s, weights);
      }
      release_stage(&empty[st]);
    }
    // join the eight warps
    w.stats(sm_m + warp * 8, sm_l + warp * 8);
    kv4_consumers_sync();
    float big[G], sum[G];
#pragma unroll
    for (int g = 0; g < G; ++g) {
      big[g] = -INFINITY;
      sum[g] = 0.f;
#pragma unroll
      for (int i = 0; i < kKv4Warps; ++i) big[g] = fmaxf(big[g], sm_m[i * 8 + g]);
#pragma unroll
      for (int i = 0; i < kKv4Warps; ++i) sum[g] += sm_m[i * 8 + g] == -INFINITY ? 0.f : sm_l[i * 8 + g] * exp2_fast(sm_m[i * 8 + g] - big[g]);
    }
    kv4_consumers_sync();
    if (tid < G) {
      // of the piece (a choice among registers: no local memory)
      float bm = big[0], sl = sum[0];
#pragma unroll
      for (int g = 1; g < G; ++g) { bm = tid == g ? big[g] : bm; sl = tid == g ? sum[g] : sl; }
      sm_m[tid] = bm;
      sm_l[tid] = sl;
    }
    kv4_consumers_sync();
    w.write(sm_out + warp * G * D, sm_m, weights);
    kv4_consumers_sync();
    const bool whole = n == s.tiles;
    constexpr int kVecs = G * D / 4;                       // float4s of a lane's output
    auto warps_sum = [&](int e) {
      float4 x = reinterpret_cast<const float4*>(sm_out)[e];
#pragma unroll
      for (int i = 1; i < kKv4Warps; ++i) {
        const float4 y = reinterpret_cast<const float4*>(sm_out + i * G * D)[e];
        x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
      }
      return x;
    };
    auto finish = [&](int e, float4 x, float total_l) {
      const float inv = total_l > 0.f ? 1.f / total_l : 0.f;
      __nv_bfloat16* out = static_cast<__nv_bfloat16*>(A.out) + ((long long)b * A.n_q_heads + hq0) * D + e * 4;
      *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf16(x.x * inv, x.y * inv), pack_bf16(x.z * inv, x.w * inv));
    };
    auto finish_lse = [&](int g, float mm, float ll) {
      if (A.lse) A.lse[(long long)b * A.n_q_heads + hq0 + g] = ll > 0.f ? (mm + log2f(ll)) * kLn2 : -INFINITY;
    };
    if (whole) {
      for (int e = tid; e < kVecs; e += kKv4Warps * 32) finish(e, warps_sum(e), sm_l[e / (D / 4)]);
      if (tid < G) finish_lse(tid, sm_m[tid], sm_l[tid]);
    } else {
      const long long slot = cta + lane_no;
      for (int e = tid; e < kVecs; e += kKv4Warps * 32) reinterpret_cast<float4*>(P.part + slot * G * D)[e] = warps_sum(e);
      if (tid < G) P.part_ml[slot * G + tid] = make_float2(sm_m[tid], sm_l[tid]);
      __threadfence();
      kv4_consumers_sync();
      // pieces of the lane: its tiles lie at [off, off + tiles) of the deal
      const long long off = (long long)cum[b] * H + (long long)head * s.tiles;
      const int c0 = (int)(off / chunk), pieces = (int)((off + s.tiles - 1) / chunk) - c0 + 1;
      if (tid == 0) {
        const bool last = atomicAdd(P.arrived + lane_no, 1u) == (uint32_t)pieces - 1;
        if (last) P.arrived[lane_no] = 0;
        *sm_last = last;
      }
      kv4_consumers_sync();
      if (*sm_last) {
        __threadfence();
        const long long slot0 = c0 + lane_no;
        for (int e = tid; e < kVecs; e += kKv4Warps * 32) {
          const int g = e / (D / 4);
          float mm = -INFINITY, ll = 0.f;
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
            ll *= f0;
            acc.x *= f0; acc.y *= f0; acc.z *= f0; acc.w *= f0;
            mm = mn;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float f = ml[i].x == -INFINITY ? 0.f : exp2_fast(ml[i].x - mm);
              ll = fmaf(ml[i].y, f, ll);
              acc.x = fmaf(x[i].x, f, acc.x); acc.y = fmaf(x[i].y, f, acc.y); acc.z = fmaf(x[i].z, f, acc.z); acc.w = fmaf(x[i].w, f, acc.w);
            }
          }
          finish(e, acc, ll);
          if (e % (D / 4) == 0) finish_lse(g, mm, ll);
        }
      }
    }
    kv4_consumers_sync();                                  // sm_* are free for the next piece
    t += n;
    if (first_v + n == s.tiles) {
      v = 0;
      if (++head == H && t < t1) {
        head = 0;
        s = span(lens[++b]);
      }
    }
  }
}

}  // namespace wkv
