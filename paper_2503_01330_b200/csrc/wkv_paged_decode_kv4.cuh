// Paged decode attention on rows in 4 bits: one token per sequence over its pages, or over a list of chosen pages.
//
//   o = sum_i p_i v_i,  p = softmax(scale q.k_i),  k_i = s_ig (n - z_ig) per group g of 32 channels, v_i likewise
//
// Bound: HBM at 4.5 bits a number; instruction issue close behind it, since a number may cost no more than about three lane instructions.
// Codes are never converted: a masked word is two fp16 subnormals n 2^-24 (or n 2^-20), which mma.sync m16n8k16 takes exactly.  Scales and
// zero points stay outside of the products:
//   q.k_i  = sum_g s_ig (q_g.n_ig - z_ig sum q_g)        groups' products in accumulators of their own
//   o_g    = sum_i (p_i s_ig) n_ig - sum_i (p_i s_ig) z_ig   the weights p s in fp16, the same rounded ones in both sums
// p and p s are rounded to fp16, 2^-11 each, together a quarter of what rounding the output to bf16 costs.  The weights are kept in fp16's
// range by a power of two that follows the largest value scale seen.  Queries become fp16 by a power of two per head (exact down to 2^-28 of the
// head's largest channel).
//
// The deal of tiles to CTAs, pieces of a lane and their join are those of the bf16 rows' kernel.  A CTA: one producer warp, which looks up 32
// pages at a time and copies their chunks into a ring (cp.async.bulk), and eight consumer warps, four for a tile of 128 entries.
#pragma once
#include "wkv_paged_decode.cuh"
#include "wkv_paged_kv4.cuh"

namespace wkv {

constexpr int kKv4Warps = 8;                              // consumers
constexpr int kKv4Threads = (kKv4Warps + 1) * 32;
constexpr int kKv4Tile = 128;                             // of four warps, 32 entries each: odd and even tiles have their own warps
constexpr int kKv4Share = 32, kKv4TileWarps = kKv4Tile / kKv4Share;
constexpr int kKv4MaxSlots = kKv4Tile / 16;               // pages of a tile

template <int D, int G>
struct Kv4Shape {
  using Row = Kv4Row<D>;
  static constexpr int kHalf = kKv4Tile * Row::kBytes;    // keys of a tile; values
  static constexpr int kStage = 2 * kHalf;
  static constexpr int kStages = (G == 8 && D == 128 ? 54 : 72) * 1024 / kStage;
  static constexpr int kOut = kKv4Warps * G * D * 4;      // the warps' outputs
  static constexpr int kScratch = kKv4Warps * 32 * G * 4; // a warp's weights, then zero points' sums
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
__device__ __forceinline__ uint32_t half_mul(uint32_t a, uint32_t b) {
  const __half2 x = __hmul2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&x);
}
__device__ __forceinline__ float2 half_pair_f(uint32_t x) { return __half22float2(*reinterpret_cast<const __half2*>(&x)); }

// A consumer warp's share of a piece: 32 entries of a tile at a time.  Lane 4 r + j.
//
// Keys: entries are rows of the product.  A lane's 16 channels of two, D / 4 in all, are the quarter j of an entry's channels.
//   G <= 2: the columns of q are (quarter, head) pairs -- (quarter, even or odd steps) for one head -- with zeros in the other quarters'
//   channels, so that a lane gets the products of quarter j alone and applies that quarter's scale and zero point only.  Sums over the
//   quarters by an exchange among four lanes that leaves each with the logit of one entry.
//   G >= 4: the columns are heads (repeated where G = 4); every group of channels has an accumulator, scaled by all lanes.
// Values: channels are rows, entries the inner dimension, and the columns of the weights are (group, head) pairs, G = 1: groups.  The zero
// points' part of the sum is one more product, of the zero points of the columns' groups with the weights.
template <int D, int G>
struct Kv4Warp {
  using Row = Kv4Row<D>;
  static constexpr bool kMasked = G <= 2;
  static constexpr int kGroups = Row::kGroups, kSteps = D / 16;
  static constexpr int kFrags = G * kGroups > 8 ? G * kGroups / 8 : 1;
  static constexpr int kHeads = kMasked ? G : 2;           // heads of a lane's statistics: all, or 2j and 2j + 1 (of G)
  static constexpr float kHeadroom = 14.f;                 // weights are held times 2^14: fp16 numbers down to 2^-28
  uint32_t q[kSteps][2];       // keys' products: the B operand of a step
  float qsum[kMasked ? 1 : kGroups][kHeads];   // sum of the quarter's, or a group's, channels
  float factor[kHeads];        // accumulator -> base-2 logit
  float o[D / 16][4];          // values' products: tile (group, half): channels 4r + 2 half and + 1, columns 2j and 2j + 1
  float zo[kFrags][4];         // zero points' products: row r is the group of column r; rows 8 .. 15 are nothing
  float m[kHeads], l[kHeads];
  uint32_t largest;            // twice the bits of the largest value scale seen, which the weights' power of two follows
  uint32_t shift;              // that power of two, twice
  int lane;

  // Group and head of column n of fragment f.
  __device__ __forceinline__ static int group_of(int f, int n) { return G == 1 ? n % kGroups : (f * (8 / G) + n / G) % kGroups; }
  __device__ __forceinline__ static int head_of(int n) { return n % G; }
  __device__ __forceinline__ static int frag_of(int g) { return kFrags == 1 ? 0 : g * G / 8; }

  __device__ __forceinline__ void begin(const __nv_bfloat16* qrow, float scale_log2) {
    lane = threadIdx.x & 31;
    const int r = lane >> 2, j = lane & 3;
    // column r: its head, and 16-channel pieces of it: of a quarter's, or of every group
    const __nv_bfloat16* mine = qrow + (kMasked ? (G == 2 ? r & 1 : 0) : r % G) * D;
    float x[kSteps][4], most = 0.f;
#pragma unroll
    for (int t = 0; t < kSteps; t += 2) {
      const uint4 u = *reinterpret_cast<const uint4*>(mine + (kMasked ? j * (D / 4) + 4 * t : 16 * t + 8 * j));
      const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[t + i / 2][i % 2 * 2] = __uint_as_float(w[i] << 16);
        x[t + i / 2][i % 2 * 2 + 1] = __uint_as_float(w[i] & 0xffff0000u);
      }
    }
#pragma unroll
    for (int t = 0; t < kSteps; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) most = fmaxf(most, fabsf(x[t][i]));
    most = fmaxf(most, __shfl_xor_sync(~0u, most, 1));
    most = fmaxf(most, __shfl_xor_sync(~0u, most, 2));
    // the head's largest channel comes to [2^14, 2^15)
    const int e = max(-100, min(100, 14 - ((int)(__float_as_uint(most) >> 23) - 127)));
    const float up = pow2f(e), f = scale_log2 * pow2f(-e) * 0x1p24f;
    const bool here = !kMasked || r >> 1 == j;             // does column r hold the lane's quarter?
    float sum = 0.f;
#pragma unroll
    for (int t = 0; t < kSteps; ++t) {
      if (!kMasked && t % 2 == 0) sum = 0.f;
      q[t][0] = half_pair(x[t][0] * up, x[t][1] * up);
      const uint32_t odd = half_pair(x[t][2] * up, x[t][3] * up);
      const float2 a = half_pair_f(q[t][0]), b = half_pair_f(odd);
      sum += (a.x + a.y) + (b.x + b.y);
      q[t][1] = half_pair(b.x * 0.0625f, b.y * 0.0625f);  // meets codes in bits 4..7
      if (!here || (G == 1 && (r & 1) != (t & 1))) q[t][0] = q[t][1] = 0u;
      if (!kMasked && t % 2 == 1) {
        sum += __shfl_xor_sync(~0u, sum, 1);
        sum += __shfl_xor_sync(~0u, sum, 2);
        qsum[t / 2][0] = __shfl_sync(~0u, sum, 8 * j);
        qsum[t / 2][kHeads - 1] = __shfl_sync(~0u, sum, 8 * j + 4);
      }
    }
#pragma unroll
    for (int c = 0; c < kHeads; ++c) {
      if (kMasked) qsum[0][c] = __shfl_sync(~0u, sum, 4 * c + j);          // column c is head c; every column has the lane's quarter's sum
      factor[c] = __shfl_sync(~0u, f, kMasked ? 4 * c : 8 * j + 4 * c);
      m[c] = -INFINITY;
      l[c] = 0.f;
    }
#pragma unroll
    for (int n = 0; n < D / 16; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
#pragma unroll
    for (int n = 0; n < kFrags; ++n) zo[n][0] = zo[n][1] = zo[n][2] = zo[n][3] = 0.f;
    largest = shift = 0;
  }

  // Products of two steps: words a and b hold eight codes each of rows r and r + 8.
  __device__ __forceinline__ void two_steps(float (&d)[4], uint32_t a, uint32_t b, int t) const {
    const uint32_t a8 = a >> 8, b8 = b >> 8;
    mma_m16n8k16_f16(d, a & 0x000f000fu, b & 0x000f000fu, a & 0x00f000f0u, b & 0x00f000f0u, q[t][0], q[t][1]);
    mma_m16n8k16_f16(d, a8 & 0x000f000fu, b8 & 0x000f000fu, a8 & 0x00f000f0u, b8 & 0x00f000f0u, q[t + 1][0], q[t + 1][1]);
  }
  // Scale, and zero point times 2^-24, of a pair.
  __device__ __forceinline__ static float pair_scale(uint32_t pair) { return kv4_scale(pair & 255); }
  __device__ __forceinline__ static float pair_zero(uint32_t pair) { return __half2float(__ushort_as_half((unsigned short)(pair >> 8 & 255))); }

  // 32 entries from i0 on.  at[sub]: where each half's 16 entries lie: the page's chunk of keys in shared memory (that of the values is
  // `half` bytes behind) and the first row in it.  bad: the page's number is none, its entries count as zeros.
  struct Place {
    const unsigned char* chunk;
    int row, entry;
    bool any, all, bad;
  };
  __device__ __forceinline__ void tile(const Place (&at)[2], int half, int page, const DecodeSpan& s, __half* weights) {
    const int r = lane >> 2, j = lane & 3;
    constexpr int kMine = kMasked ? 1 : 4;                 // logits per lane and head: entries of sub 0: r, r + 8; of sub 1
    float x[kMine][kHeads];
    if constexpr (kMasked) {
      float v[4][G];
#pragma unroll
      for (int sub = 0; sub < 2; ++sub) {
        const unsigned char* tk = at[sub].chunk;
        const int row = at[sub].row + r;
        float d[4] = {};
        if constexpr (kGroups == 4) {
          const uint4 a = *reinterpret_cast<const uint4*>(tk + Row::k_piece(row, j)), b = *reinterpret_cast<const uint4*>(tk + Row::k_piece(row + 8, j));
          two_steps(d, a.x, b.x, 0);
          two_steps(d, a.y, b.y, 2);
          two_steps(d, a.z, b.z, 4);
          two_steps(d, a.w, b.w, 6);
        } else {
          const uint2 a = *reinterpret_cast<const uint2*>(tk + Row::k_piece(row, j >> 1) + (j & 1) * 8),
                      b = *reinterpret_cast<const uint2*>(tk + Row::k_piece(row + 8, j >> 1) + (j & 1) * 8);
          two_steps(d, a.x, b.x, 0);
          two_steps(d, a.y, b.y, 2);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t pair = *reinterpret_cast<const uint16_t*>(tk + Row::pairs(page, row + 8 * h) + 2 * (j * kGroups / 4));
          const float sc = pair_scale(pair), z = pair_zero(pair);
#pragma unroll
          for (int c = 0; c < G; ++c) v[2 * sub + h][c] = sc * fmaf(-z, qsum[0][c], G == 1 ? d[2 * h] + d[2 * h + 1] : d[2 * h + c]);
        }
      }
      // sums over the quarters: lane j keeps entry r + 8 (j % 2) of sub j / 2
#pragma unroll
      for (int c = 0; c < G; ++c) {
        const float a0 = j & 1 ? v[1][c] : v[0][c], b0 = j & 1 ? v[0][c] : v[1][c], a1 = j & 1 ? v[3][c] : v[2][c], b1 = j & 1 ? v[2][c] : v[3][c];
        const float s0 = a0 + __shfl_xor_sync(~0u, b0, 1), s1 = a1 + __shfl_xor_sync(~0u, b1, 1);
        x[0][c] = (j & 2 ? s1 : s0) + __shfl_xor_sync(~0u, j & 2 ? s0 : s1, 2);
      }
    } else {
#pragma unroll
      for (int sub = 0; sub < 2; ++sub) {
        const unsigned char* tk = at[sub].chunk;
        const int row = at[sub].row + r;
        uint32_t pairs[2][kGroups / 2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const unsigned char* p = tk + Row::pairs(page, row + 8 * h);
          if constexpr (kGroups == 4) {
            const uint2 y = *reinterpret_cast<const uint2*>(p);
            pairs[h][0] = y.x;
            pairs[h][1] = y.y;
          } else {
            pairs[h][0] = *reinterpret_cast<const uint32_t*>(p);
          }
          x[2 * sub + h][0] = x[2 * sub + h][1] = 0.f;
        }
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
          float d[4] = {};
          two_steps(d, *reinterpret_cast<const uint32_t*>(tk + Row::k_piece(row, g) + 4 * j), *reinterpret_cast<const uint32_t*>(tk + Row::k_piece(row + 8, g) + 4 * j), 2 * g);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t pair = g & 1 ? pairs[h][g / 2] >> 16 : pairs[h][g / 2];
            const float sc = pair_scale(pair), z = pair_zero(pair);
#pragma unroll
            for (int c = 0; c < 2; ++c) x[2 * sub + h][c] = fmaf(sc, fmaf(-z, qsum[g][c], d[2 * h + c]), x[2 * sub + h][c]);
          }
        }
      }
    }
    const bool every = at[0].all && at[1].all && !at[0].bad && !at[1].bad;
    auto entry = [&](int k) {                              // of logit k
      const int sub = kMasked ? j >> 1 : k >> 1, h = kMasked ? j & 1 : k & 1;
      return (sub ? at[1].entry : at[0].entry) + r + 8 * h;
    };
#pragma unroll
    for (int k = 0; k < kMine; ++k)
#pragma unroll
      for (int c = 0; c < kHeads; ++c) {
        x[k][c] *= factor[c];
        if (!every) {
          const bool second = kMasked ? j >> 1 : k >> 1;
          if (second ? at[1].bad : at[0].bad) x[k][c] = 0.f;
          if (!s.sees(entry(k))) x[k][c] = -INFINITY;
        }
      }
    // scales of the values: entries j + 4t, the group of column r, two entries to a word
    uint32_t scale2[2][kFrags][2], zero2[2][kFrags][2], top = largest;
#pragma unroll
    for (int sub = 0; sub < 2; ++sub) {
      const unsigned char* tv = at[sub].chunk + half;
#pragma unroll
      for (int f = 0; f < kFrags; ++f) {
        uint32_t pair[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          pair[t] = *reinterpret_cast<const uint16_t*>(tv + Row::pairs(page, at[sub].row + j + 4 * t) + 2 * group_of(f, r));
          if (!every && (at[sub].bad || !s.sees(at[sub].entry + j + 4 * t))) pair[t] = 0u;
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          scale2[sub][f][t] = __byte_perm(pair[2 * t], pair[2 * t + 1], 0x4302) >> 1;
          zero2[sub][f][t] = __byte_perm(pair[2 * t], pair[2 * t + 1], 0x3521);
          top = __vmaxu2(top, scale2[sub][f][t]);
        }
      }
    }
    bool more = top != largest;
#pragma unroll
    for (int k = 0; k < kMine; ++k)
#pragma unroll
      for (int c = 0; c < kHeads; ++c) more = more || x[k][c] > m[c];
    if (__any_sync(~0u, more)) raise(x, top);
    // weights: entry e of a half at place (e % 4) * 4 + e / 4
    __syncwarp();
#pragma unroll
    for (int k = 0; k < kMine; ++k)
#pragma unroll
      for (int c = 0; c < kHeads; ++c) {
        const float p = exp2_fast(x[k][c] - (m[c] == -INFINITY ? 0.f : m[c] - kHeadroom));
        l[c] += p;
        const int sub = kMasked ? j >> 1 : k >> 1, h = kMasked ? j & 1 : k & 1;
        if (kMasked || 2 * j + c < G) weights[(kMasked ? c : 2 * j + c) * 32 + sub * 16 + (r & 3) * 4 + (r >> 2) + 2 * h] = __float2half_rn(p);
      }
    __syncwarp();
#pragma unroll
    for (int sub = 0; sub < 2; ++sub) {
      const uint2 p = *reinterpret_cast<const uint2*>(weights + head_of(r) * 32 + sub * 16 + 4 * j);
      uint32_t b[kFrags][2];
#pragma unroll
      for (int f = 0; f < kFrags; ++f) {
        b[f][0] = half_mul(p.x, half_mul(scale2[sub][f][0], shift));
        b[f][1] = half_mul(p.y, half_mul(scale2[sub][f][1], shift));
        mma_m16n8k16_f16(zo[f], zero2[sub][f][0], 0u, zero2[sub][f][1], 0u, b[f][0], b[f][1]);
      }
      // units r of every group, of entries j + 4t
      const unsigned char* tv = at[sub].chunk + half;
      uint32_t w[4][kGroups / 2];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const unsigned char* p4 = tv + Row::v_unit(at[sub].row + j + 4 * t, 0, r);
        if constexpr (kGroups == 4) {
          const uint2 y = *reinterpret_cast<const uint2*>(p4);
          w[t][0] = y.x;
          w[t][1] = y.y;
        } else {
          w[t][0] = *reinterpret_cast<const uint32_t*>(p4);
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
  }

  // A larger logit, or value scale, than any before: sums so far follow.
  template <int K>
  __device__ __forceinline__ void raise(const float (&x)[K][kHeads], uint32_t top) {
    top = __reduce_max_sync(~0u, max(top & 0xffffu, top >> 16));
    // the largest scale comes to [1, 2): 2^(15 - its exponent field), as a half
    const float was = half_pair_f(shift).x, to = pow2f(15 - max(1, (int)(top >> 10))), ratio = largest ? to / was : 0.f;
    float f[kHeads];
#pragma unroll
    for (int c = 0; c < kHeads; ++c) {
      float mx = x[0][c];
#pragma unroll
      for (int k = 1; k < K; ++k) mx = fmaxf(mx, x[k][c]);
#pragma unroll
      for (int off = kMasked ? 1 : 4; off < 32; off <<= 1) mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, off));
      mx = fmaxf(mx, m[c]);
      const float g = exp2_fast(m[c] - (mx == -INFINITY ? 0.f : mx));
      l[c] *= g;
      f[c] = g * ratio;
      m[c] = mx;
    }
    const float f0 = f[0], f1 = f[kHeads - 1];             // of columns 2j and 2j + 1
#pragma unroll
    for (int n = 0; n < D / 16; ++n) { o[n][0] *= f0; o[n][1] *= f1; o[n][2] *= f0; o[n][3] *= f1; }
#pragma unroll
    for (int n = 0; n < kFrags; ++n) { zo[n][0] *= f0; zo[n][1] *= f1; }
    if (top) {
      largest = top | top << 16;
      shift = half_pair(to, to);
    }
  }

  // (max, sum) of the heads over this warp's entries to [8] each
  __device__ __forceinline__ void stats(float* sm_m, float* sm_l) {
    const int j = lane & 3;
#pragma unroll
    for (int c = 0; c < kHeads; ++c) {
#pragma unroll
      for (int off = kMasked ? 1 : 4; off < 32; off <<= 1) l[c] += __shfl_xor_sync(~0u, l[c], off);
      const int head = kMasked ? c : 2 * j + c;
      if (lane < (kMasked ? 1 : 4) && head < G) { sm_m[head] = m[c]; sm_l[head] = l[c] * 0x1p-14f; }
    }
  }
  // The warp's output [G][D], relative to the heads' maxima big[G]; zeros: scratch, [groups][G].
  __device__ __forceinline__ void write(float* out, const float* big, float* zeros) {
    const int r = lane >> 2, j = lane & 3;
    __syncwarp();
#pragma unroll
    for (int f = 0; f < kFrags; ++f)                       // column r meets its own group in row r
      if (j == r >> 1 && (G == 1 ? r < kGroups : f * (8 / G) + r / G < kGroups)) zeros[group_of(f, r) * G + head_of(r)] = r & 1 ? zo[f][1] : zo[f][0];
    __syncwarp();
    const float back = largest ? 0x1p10f / half_pair_f(shift).x : 0.f;     // codes' 2^24, weights' 2^-14
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int col = 2 * j + c, head = head_of(col);
      const float mm = m[c < kHeads ? c : 0], f = mm == -INFINITY ? 0.f : exp2_fast(mm - big[head]) * back;
      // of a fragment's groups the one of this column, by selection: registers have no indexes
      constexpr int kPer = kGroups / kFrags;
      const int which = G == 1 ? col : col / G;
#pragma unroll
      for (int f8 = 0; f8 < kFrags; ++f8) {
        float a[4] = {};
#pragma unroll
        for (int i = 0; i < kPer; ++i)
#pragma unroll
          for (int h = 0; h < 4; ++h) a[h] = i == which ? o[2 * (f8 * kPer + i) + h / 2][c + h % 2 * 2] : a[h];
        if (which >= kPer) continue;
        const int g = f8 * kPer + which;
        const float z = zeros[g * G + head];
        float2* to = reinterpret_cast<float2*>(out + head * D + g * 32 + 4 * r);
        to[0] = make_float2((a[0] - z) * f, (a[1] * 0x1p-4f - z) * f);
        to[1] = make_float2((a[2] - z) * f, (a[3] * 0x1p-4f - z) * f);
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
  float* scratch = sm_out + kKv4Warps * G * D;                                  // [warps][G][32]
  float* sm_m = scratch + kKv4Warps * 32 * G;                                   // [warps][8]
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
    for (int i = 0; i < STAGES; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], kKv4TileWarps); }
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
  float* mine = scratch + warp * 32 * G;
  const int team = warp / kKv4TileWarps, row = warp % kKv4TileWarps * kKv4Share;       // the tiles, and rows of a tile, that are this warp's
  for (long long t = t0; t < t1;) {
    const int first_v = v;
    const int n = (int)min((long long)(s.tiles - v), t1 - t);            // tiles of this piece
    const long long lane_no = (long long)b * H + head;
    const int hq0 = head * G;
    w.begin(static_cast<const __nv_bfloat16*>(A.q) + (long long)b * A.q_stride + (long long)hq0 * D, A.scale_log2);
    for (int k = 0; k < n; ++k, ++it) {
      if ((it & 1) != team) continue;
      const int st = it % STAGES;
      ok = ok && wait(&full[st], (it / STAGES) & 1);
      if (!ok) continue;
      typename Warp::Place at[2];
#pragma unroll
      for (int sub = 0; sub < 2; ++sub) {
        const int from = row + 16 * sub, slot = from >> A.page_shift, e = slot_entry[st * kKv4MaxSlots + slot];
        at[sub].bad = e < 0;
        at[sub].row = from & (A.page - 1);
        at[sub].entry = (e < 0 ? ~e : e) + at[sub].row;
        at[sub].chunk = ring + st * Sh::kStage + slot * chunk_bytes;
        at[sub].any = at[sub].entry < s.len && (at[sub].entry + 16 > s.lo || at[sub].entry < s.sinks);
        at[sub].all = at[sub].entry + 16 <= s.len && (at[sub].entry >= s.lo || at[sub].entry + 16 <= s.sinks);
      }
      if (at[0].any || at[1].any) w.tile(at, Sh::kHalf, A.page, s, reinterpret_cast<__half*>(mine));
      release_stage(&empty[st]);
    }
    v += n;
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
    w.write(sm_out + warp * G * D, sm_m, mine);
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
