// Paged decode attention on rows in 4 bits: one token per sequence over its pages, or over a list of chosen pages.
//
//   o = sum_i p_i v_i,  p = softmax(scale q.k_i),  k_i = s_ig (n - z_ig) per group g of 32 channels, v_i likewise
//
// Bound: HBM at 4.5 bits a number, and arithmetic close behind it, since a number may cost no more than about three lane instructions: issue is
// active in 62 to 67 % of the cycles and the ALU pipe in 55 to 57 %, with four to five warps a scheduler that wait for fixed latencies, memory and
// that pipe in turn; no pipe is full.
// Keys: a masked word is four bytes for mma.sync m16n8k32 on integers, against queries of 23 bits in three columns of eight; exact, until
// a group's product becomes fp32.  Values: a masked word is two fp16 subnormals n 2^-24 (or n 2^-20), and one multiplication by 2^14 (2^10)
// makes them normal numbers for m16n8k16.  (That takes subnormals too, but lines products up as if theirs had no leading zeros, and cuts the
// sum 25 bits below: weights below 2^-15 of a step's largest were gone from the zero points' sum and from half of the codes', and, beside an
// entry of nearly all weight, the rest of the output with them.  Normal numbers cost 6 us of 160, and 4 of 99.)
// Scales and zero points stay outside of the products:
//   q.k_i  = sum_g s_ig (q_g.n_ig - z_ig sum q_g)
//   o_g    = sum_i (p_i s_ig) n_ig - sum_i (p_i s_ig) z_ig   the weights p s in fp16, the same rounded ones in both sums
// A query head becomes whole numbers by a power of two that brings its largest channel to [2^21, 2^22), the largest that a group's sum leaves
// room for in 32 bits: bf16 channels down to 2^-14 of it stay exact, smaller ones are off by up to 2^-22 of it.  (Fewer bits show in the
// log-sums, which are fp32: 14 in two columns, 12 us of 174 faster, and 17 with the high halves' codes taken times 16 instead of shifted, 3
// us, were 1e-6 and more off in sequences of one token.)
// p and p s are rounded to fp16, 2^-11 each, together a quarter of what rounding the output to bf16 costs.  Weights are held times 2^9 and
// scales times a power of two that brings the largest one seen, whatever weight its row has, to [2^5, 2^6): all scales of the format are
// exact beside it, and p s is also off by up to 2^-39 of that scale times the largest weight, p by 2^-34 of the latter: below what fp32 sums
// keep beside codes of that weight, and the largest is a warp's own.  (Weights times 2^14 unless a scale of 256 or more comes: 167 us for 166.)
// (Keys as fp16 subnormals: 163 us of arithmetic in the 16 x 8192..16384 case, masks at half rate above all.  As e4m3 numbers the matrix
// instruction is split into fp16 ones with conversions.)
//
// The deal of tiles to CTAs, pieces of a lane and their join are those of the bf16 rows' kernel.  A CTA: eight consumer warps in
// two teams, which take tiles of 128 entries in turn, and a producer warp for each team, which looks up 32 pages at a time and copies their
// chunks into the team's stages of a ring (cp.async.bulk).  (One producer for both: 174 us where two take 167, 40 where they take 32 in pages
// of 16: a tile costs it some 700 cycles.)
//
// Measured: 16 sequences of 8192..16384 tokens, 32 x 128 heads, 166 us = 5.5 TB/s (0.84 of the measured copy rate; 190 us at the power limit
// under load); 16 of 12000..32768, 32/8 heads, 102 us = 4.1 TB/s (108 under load); one of 611 tokens 10.3 us in a captured graph.
#pragma once
#include "wkv_paged_decode.cuh"
#include "wkv_paged_kv4.cuh"

namespace wkv {

constexpr int kKv4Warps = 8;                              // consumers
constexpr int kKv4Threads = (kKv4Warps + 2) * 32;         // and a producer for each team
constexpr int kKv4Tile = 128;                             // of four warps, 32 entries each: odd and even tiles have their own warps
constexpr int kKv4Share = 32, kKv4TileWarps = kKv4Tile / kKv4Share;
constexpr int kKv4MaxSlots = kKv4Tile / 16;               // pages of a tile

template <int D, int G>
struct Kv4Shape {
  using Row = Kv4Row<D>;
  static constexpr int kHalf = kKv4Tile * Row::kBytes;    // keys of a tile; values
  static constexpr int kStage = 2 * kHalf;
  static constexpr int kOuts = G >= 4 ? kKv4Warps / 2 : kKv4Warps;      // outputs side by side in the join: the warps', or of pairs of them
  static constexpr int kOut = kOuts * G * D * 4;
  static constexpr int kScratch = kKv4Warps * 16 * G * 4; // a warp's weights, then zero points' sums
  static constexpr int kQuery = (G == 2 || G == 8 ? 3 : 2) * D / 64 * 512;      // Kv4Warp::kQuery
  static constexpr int kOther = kOut + kScratch + kQuery + 2 * kKv4Warps * 8 * 4 + (2 * kMaxSequences + 8) * 4 + 64;
  // CTAs an SM: one where eight heads' sums of 128 channels would not fit into half of the registers (64 sequences of 8192..16384 tokens,
  // 8 heads on one: 50 us, 64 with two); a stage's slot entries and barriers beside it.  An even number: a stage then belongs to one team of warps, which cannot
  // be more than one of its barrier's phases ahead (with an odd one the teams take turns on it, and a wait that looks at the
  // phase's parity could be let through by the phase before the other team's).
  static constexpr int kCtas = G == 8 && D == 128 ? 1 : 2;
  static constexpr int kStages = (226 / kCtas * 1024 - kOther) / (kStage + kKv4MaxSlots * 4 + 16) / 2 * 2;
  static_assert(kKv4Warps == 2 * kKv4TileWarps && kStages >= 2, "two teams");
  static constexpr int kSmem = kStages * (kStage + kKv4MaxSlots * 4 + 16) + kOther;
};

__device__ __forceinline__ void mma_m16n8k16_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_m16n8k32_u8s8(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k32.row.col.s32.u8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float pow2f(int e) { return __int_as_float((e + 127) << 23); }       // -126 <= e <= 127
__device__ __forceinline__ uint32_t half_pair(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// Shared memory by 32-bit address: a generic pointer would double the address arithmetic.
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t lds32(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t lds16(uint32_t a) {
  uint16_t v;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ void sts16(uint32_t a, __half x) {
  asm volatile("st.shared.u16 [%0], %1;" ::"r"(a), "h"(__half_as_ushort(x)) : "memory");
}
__device__ __forceinline__ uint32_t half_mul(uint32_t a, uint32_t b) {
  const __half2 x = __hmul2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&x);
}
__device__ __forceinline__ uint32_t half_max(uint32_t a, uint32_t b) {
  const __half2 x = __hmax2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&x);
}
__device__ __forceinline__ float2 half_pair_f(uint32_t x) { return __half22float2(*reinterpret_cast<const __half2*>(&x)); }

// Largest logit of a head over the warps, and its sum relative to that.  (A sum is 0 where nothing is seen; logits that are no numbers, and
// so never the largest, leave one that is none either, which goes on into outputs and log-sums.)
__device__ __forceinline__ float warps_max(const float* sm_m, int head) {
  float m = sm_m[head];
#pragma unroll
  for (int i = 1; i < kKv4Warps; ++i) m = fmaxf(m, sm_m[i * 8 + head]);
  return m;
}
__device__ __forceinline__ float warps_l(const float* sm_m, const float* sm_l, int head, float big) {
  float l = 0.f;
#pragma unroll
  for (int i = 0; i < kKv4Warps; ++i) l += sm_l[i * 8 + head] == 0.f ? 0.f : sm_l[i * 8 + head] * exp2_fast(sm_m[i * 8 + head] - big);
  return l;
}

// A consumer warp's share of a piece: 32 entries of a tile at a time.  Lane 4 r + j.
//
// Keys: entries are rows of the product, and columns bytes of the queries: the highest two of a head side by side, the lowest ones in a tile
// of columns of their own.
//   G <= 2: a head's eight columns have a quarter of its channels each, zeros elsewhere, so that a lane gets the products of quarter j alone
//   and applies that quarter's scale and zero point only.  Sums over the quarters by an exchange among four lanes that leaves each with
//   the logit of one entry.
//   G >= 4: eight columns are four heads; every group of channels has an accumulator.  A lane has the logits of head j (and j + 4) and
//   four entries.
// Values: channels are rows, entries the inner dimension, and the columns of the weights are (group, head) pairs.  The products of a
// fragment's groups share accumulators: each takes the weights of its own columns and zeros for the others (with accumulators of their
// own, mostly of columns that nobody reads, a third of the registers went there).  The zero points' part
// of the sum is one more product, of the zero points of the columns' groups with the weights.
template <int D, int G>
struct Kv4Warp {
  using Row = Kv4Row<D>;
  static constexpr bool kMasked = G <= 2;
  static constexpr int kGroups = Row::kGroups, kHeads = kMasked ? G : G / 4;       // heads of a lane's statistics: all; j and j + 4
  static constexpr int kFrags = G * kGroups > 8 ? G * kGroups / 8 : 1, kPer = kGroups / kFrags;   // fragments of weights; groups of one
  // The keys' products' B operands (a step: 32 channels, 8 of each lane's) are made once for all warps, in shared memory, two steps to a
  // lane's 16 bytes.  One head keeps them in registers (3 us of 180 under load); more heads read them for each tile (four heads: 101 us, 104
  // with them in registers, which then spill).
  static constexpr bool kHolds = G == 1;
  static constexpr int kTiles = kHeads + 1;                // of columns
  static constexpr int kQuery = kTiles * kGroups / 2 * 32 * 16;          // bytes
  static constexpr float kHeadroom = 9.f;                  // weights are held times 2^9: normal fp16 numbers down to 2^-23
  int qsum[kHeads][kMasked ? 1 : kGroups];     // sum of the quarter's, or a group's, channels
  uint32_t q[kTiles][kGroups][2];
  float factor[kHeads];        // whole numbers -> base-2 logits
  float o[kFrags][2][4];       // values' products: channels 4r + 2 half and + 1 of the column's group, columns 2j and 2j + 1
  float zo[kFrags][4];         // zero points' products: row r is the group of column r; rows 8 .. 15 are nothing
  float m[kHeads], l[kHeads];
  uint32_t largest;            // twice the bits of the largest value scale seen, which the weights' power of two follows
  uint32_t shift;              // that power of two, twice: 2^-7 or more, so that scales, multiples of 2^-17 of four bits, stay exact

  // Where the lane's words lie in a stage: codes and pairs of its first 16 entries' keys (values: `half` bytes behind), and how far behind
  // them those of the other 16 are.
  struct Offsets {
    int kc, kp, vc, vp, next_c, next_p;
  };
  __device__ __forceinline__ static Offsets offsets(int page, int page_shift, int row, int half) {
    const int lane = threadIdx.x & 31, r = lane >> 2, j = lane & 3, first = row & (page - 1), chunk = page * Row::kBytes;
    const int codes = (row >> page_shift) * chunk + first * Row::kCodes, pairs = (row >> page_shift) * chunk + Row::pairs(page, first);
    Offsets a;
    // (swizzles depend on rows mod 16 only)
    a.kc = codes + (!kMasked ? r * Row::kCodes + 4 * j : kGroups == 4 ? Row::k_piece(r, j) : Row::k_piece(r, j >> 1) + (j & 1) * 8);
    a.kp = pairs + r * Row::kPairs + (kMasked ? 2 * (j * kGroups / 4) : 0);
    a.vc = half + codes + Row::v_unit(j, 0, r);
    a.vp = half + pairs + j * Row::kPairs + (kFrags == 1 ? 2 * group_of(0, r) : G == 4 ? 2 * (r & 1) : 0);
    a.next_c = page == 16 ? chunk : 16 * Row::kCodes;
    a.next_p = page == 16 ? chunk : 16 * Row::kPairs;
    return a;
  }

  // Group and head of column n of fragment f: a lane's columns 2j and 2j + 1 are of the heads whose statistics it has.
  __device__ __forceinline__ static int group_of(int f, int n) {
    return (G == 1 ? n : G == 2 ? n >> 1 : G == 4 ? 2 * f + (n & 1) : f) % kGroups;
  }
  // Is column n of the i-th group of its fragment?
  __device__ __forceinline__ static bool of_group(int i, int n) { return G == 1 ? n % kGroups == i : G == 2 ? n >> 1 == i : G == 4 ? (n & 1) == i : true; }
  __device__ __forceinline__ static int head_of(int n) { return G == 1 ? 0 : G == 2 ? n & 1 : G == 4 ? n >> 1 : (n >> 1) + 4 * (n & 1); }

  __device__ __forceinline__ void begin(const __nv_bfloat16* qrow, float scale_log2, uint4* query, bool stores) {
    const int lane = threadIdx.x & 31, r = lane >> 2, j = lane & 3;
    const bool here = !kMasked || r >> 1 == j;             // does column r hold the lane's quarter?
    uint32_t low[kGroups][2] = {};                         // of column r of the lowest bytes' tile
#pragma unroll
    for (int u = 0; u < kHeads; ++u) {
      // the head of column r of tile u, and of its channels those that meet this lane's codes
      const __nv_bfloat16* mine = qrow + (kMasked ? u : 4 * u + (r >> 1)) * D + (kMasked ? j * (D / 4) : 8 * j);
      float x[kGroups][8], top = 0.f;
#pragma unroll
      for (int t = 0; t < kGroups; ++t) {
        const uint4 y = *reinterpret_cast<const uint4*>(mine + (kMasked ? 8 : 32) * t);
        const uint32_t w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[t][2 * i] = __uint_as_float(w[i] << 16); x[t][2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, x[t][i] == x[t][i] ? fabsf(x[t][i]) : INFINITY);
      }
      top = fmaxf(top, __shfl_xor_sync(~0u, top, 1));      // of all quarters, or of the lanes that share a head's groups
      top = fmaxf(top, __shfl_xor_sync(~0u, top, 2));
      // (-106: up to the largest finite bf16 number; queries of less than 2^-99 keep fewer bits, so that 2^-e stays clear of subnormals)
      const int e = max(-106, min(120, 21 - ((int)(__float_as_uint(top) >> 23) - 127)));
      const float up = pow2f(e), f = top < INFINITY ? scale_log2 * pow2f(-e) : __int_as_float(0x7fffffff);
      factor[u] = kMasked ? f : __shfl_sync(~0u, f, 8 * j);
      int sum = 0;
#pragma unroll
      for (int t = 0; t < kGroups; ++t) {
        if (!kMasked) sum = 0;
        // in the order of the codes' bytes: channels 0, 4, 1, 5 from the low halves of a word's bytes, 2, 6, 3, 7 from the high ones
        constexpr int kAt[8] = {0, 4, 1, 5, 2, 6, 3, 7};
        uint32_t word[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          word[h] = 0;
          uint32_t rest = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int y = __float2int_rn(x[t][kAt[4 * h + i]] * up), y1 = (y + 128) >> 8, y0 = y - y1 * 256, high = (y1 + 128) >> 8;
            sum += y;
            word[h] |= (uint32_t)((r & 1 ? y1 - high * 256 : high) & 255) << 8 * i;
            rest |= (uint32_t)(y0 & 255) << 8 * i;
          }
          if (!here) word[h] = 0;
          if (here && (r & 1) == u) low[t][h] = rest;
        }
        if (stores) reinterpret_cast<uint2*>(query)[((u * kGroups + t) / 2 * 32 + lane) * 2 + (t & 1)] = make_uint2(word[0], word[1]);
        if constexpr (!kMasked) {
          sum += __shfl_xor_sync(~0u, sum, 1);
          sum += __shfl_xor_sync(~0u, sum, 2);
          qsum[u][t] = __shfl_sync(~0u, sum, 8 * j);
        }
      }
      if constexpr (kMasked) qsum[u][0] = sum;
      m[u] = -INFINITY;
      l[u] = 0.f;
    }
#pragma unroll
    for (int t = 0; t < kGroups; ++t)
      if (stores) reinterpret_cast<uint2*>(query)[((kHeads * kGroups + t) / 2 * 32 + lane) * 2 + (t & 1)] = make_uint2(low[t][0], low[t][1]);
#pragma unroll
    for (int f = 0; f < kFrags; ++f)
#pragma unroll
      for (int i = 0; i < 8; ++i) o[f][i / 4][i % 4] = 0.f;
#pragma unroll
    for (int n = 0; n < kFrags; ++n) zo[n][0] = zo[n][1] = zo[n][2] = zo[n][3] = 0.f;
    largest = shift = 0;
  }

  // A step's products: words a and b hold eight codes each of rows r and r + 8.
  __device__ __forceinline__ static void step(int (&d)[kTiles][4], uint32_t a, uint32_t b, const uint32_t (&q)[kTiles][kGroups][2], int t) {
    constexpr uint32_t kLow = 0x0f0f0f0fu;
    const uint32_t a0 = a & kLow, a1 = b & kLow, a2 = a >> 4 & kLow, a3 = b >> 4 & kLow;
#pragma unroll
    for (int i = 0; i < kTiles; ++i) mma_m16n8k32_u8s8(d[i], a0, a1, a2, a3, q[i][t][0], q[i][t][1]);
  }
  __device__ __forceinline__ void load_query(uint32_t query) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int i = 0; i < kTiles * kGroups / 2; ++i) {
      const uint4 y = lds128(query + (i * 32 + lane) * 16);
      uint32_t (&to)[kGroups][2] = q[2 * i / kGroups];
      to[2 * i % kGroups][0] = y.x; to[2 * i % kGroups][1] = y.y;
      to[2 * i % kGroups + 1][0] = y.z; to[2 * i % kGroups + 1][1] = y.w;
    }
  }
  // q.n - z sum q of row half h, head u: below 2^22 * 15 * 32 < 2^31, whatever its parts, which wrap around, are.
  __device__ __forceinline__ static float part(const int (&d)[kTiles][4], int h, int u, uint32_t zero, int sum) {
    return (float)(int)(((uint32_t)d[u][2 * h] * 256 + (uint32_t)d[u][2 * h + 1]) * 256 + (uint32_t)d[kHeads][2 * h + u] - zero * (uint32_t)sum);
  }

  // 32 entries of the stage at shared memory address `stage`, the halves' first ones entry[0] and entry[1]; ~entry: the page's number is
  // none, its entries count as zeros.  EVERY: all of them are seen (code for the others in the way cost a fifth of all instructions).
  template <bool EVERY>
  __device__ __forceinline__ void tile(uint32_t stage, const Offsets& at, int entry0, int entry1, const DecodeSpan& s, uint32_t weights, uint32_t query) {
    const int lane = threadIdx.x & 31, r = lane >> 2, j = lane & 3;
    constexpr int kMine = kMasked ? 1 : 4;                 // logits per lane and head: entries of sub 0: r, r + 8; of sub 1
    constexpr int k8 = 8 * Row::kCodes, p8 = 8 * Row::kPairs;
    float x[kMine][kHeads];
    if constexpr (!kHolds) load_query(query);
    if constexpr (kMasked) {
      float v[4][G];
#pragma unroll
      for (int sub = 0; sub < 2; ++sub) {
        const uint32_t tk = stage + at.kc + sub * at.next_c, tp = stage + at.kp + sub * at.next_p;
        uint32_t a[kGroups], b[kGroups];
        if constexpr (kGroups == 4) {
          const uint4 y = lds128(tk), w = lds128(tk + k8);
          a[0] = y.x; a[1] = y.y; a[2] = y.z; a[3] = y.w;
          b[0] = w.x; b[1] = w.y; b[2] = w.z; b[3] = w.w;
        } else {
          const uint2 y = lds64(tk), w = lds64(tk + k8);
          a[0] = y.x; a[1] = y.y;
          b[0] = w.x; b[1] = w.y;
        }
        const uint32_t pair0 = lds16(tp), pair1 = lds16(tp + p8);
        int d[kTiles][4] = {};
#pragma unroll
        for (int t = 0; t < kGroups; ++t) step(d, a[t], b[t], q, t);
#pragma unroll
        for (int u = 0; u < G; ++u) {
          v[2 * sub][u] = kv4_scale(pair0 & 255) * part(d, 0, u, pair0 >> 8, qsum[u][0]);
          v[2 * sub + 1][u] = kv4_scale(pair1 & 255) * part(d, 1, u, pair1 >> 8, qsum[u][0]);
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
        const uint32_t tk = stage + at.kc + sub * at.next_c, tp = stage + at.kp + sub * at.next_p;
        const int swizzle = Row::k_piece(r, 0) - r * Row::kCodes;
        uint32_t pairs[2][kGroups / 2];
        float2 scales[2][kGroups / 2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if constexpr (kGroups == 4) {
            const uint2 y = lds64(tp + h * p8);
            pairs[h][0] = y.x;
            pairs[h][1] = y.y;
          } else {
            pairs[h][0] = lds32(tp + h * p8);
          }
#pragma unroll
          for (int i = 0; i < kGroups / 2; ++i) scales[h][i] = half_pair_f((pairs[h][i] & 0x00ff00ffu) << 7);
#pragma unroll
          for (int u = 0; u < kHeads; ++u) x[2 * sub + h][u] = 0.f;
        }
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
          const uint32_t piece = tk + (16 * g ^ swizzle);
          const uint32_t a = lds32(piece), b = lds32(piece + k8);
          int d[kTiles][4] = {};
          step(d, a, b, q, g);
#pragma unroll
          for (int u = 0; u < kHeads; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h)
              x[2 * sub + h][u] = fmaf(g & 1 ? scales[h][g / 2].y : scales[h][g / 2].x,
                                       part(d, h, u, __byte_perm(pairs[h][g / 2], 0u, g & 1 ? 0x4443 : 0x4441), qsum[u][g]), x[2 * sub + h][u]);
        }
      }
    }
    bool more = false;
#pragma unroll
    for (int k = 0; k < kMine; ++k)
#pragma unroll
      for (int c = 0; c < kHeads; ++c) {
        x[k][c] *= factor[c];
        if constexpr (!EVERY) {
          const int e = (kMasked ? j >> 1 : k >> 1) ? entry1 : entry0, i = (e < 0 ? ~e : e) + r + 8 * (kMasked ? j & 1 : k & 1);
          x[k][c] = !s.sees(i) ? -INFINITY : e < 0 ? 0.f : x[k][c];
        }
        more = more || x[k][c] > m[c];
      }
    if (__any_sync(~0u, more)) raise(x);
    // weights: entry e of a half at place (e % 4) * 4 + e / 4
    __syncwarp();
#pragma unroll
    for (int c = 0; c < kHeads; ++c) {
      const float ref = m[c] == -INFINITY ? 0.f : m[c] - kHeadroom;
#pragma unroll
      for (int k = 0; k < kMine; ++k) {
        const float p = exp2_fast(x[k][c] - ref);
        l[c] += p;
        const int sub = kMasked ? j >> 1 : k >> 1, h = kMasked ? j & 1 : k & 1;
        sts16(weights + 2 * ((kMasked ? c : j + 4 * c) * 32 + sub * 16 + (r & 3) * 4 + (r >> 2) + 2 * h), __float2half_rn(p));
      }
    }
    __syncwarp();
#pragma unroll
    for (int sub = 0; sub < 2; ++sub) {
      // scales and zero points of the values: entries j + 4t, the group of column r, two entries to a word
      const uint32_t tp = stage + at.vp + sub * at.next_p;
      uint32_t scale2[kFrags][2], zero2[kFrags][2], top = largest;
#pragma unroll
      for (int f = 0; f < kFrags; ++f) {
        uint32_t pair[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          pair[t] = lds16(tp + 2 * f * kPer + t * 4 * Row::kPairs);
          if constexpr (!EVERY) {
            const int e = sub ? entry1 : entry0;
            pair[t] = e >= 0 && s.sees(e + j + 4 * t) ? pair[t] : 0u;
          }
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          scale2[f][t] = __byte_perm(pair[2 * t], pair[2 * t + 1], 0x4302) >> 1;
          zero2[f][t] = __byte_perm(pair[2 * t], pair[2 * t + 1], 0x3521);
          top = half_max(top, scale2[f][t]);
        }
      }
      if (__any_sync(~0u, top != largest)) widen(top);
      const uint2 p = lds64(weights + 2 * (head_of(r) * 32 + sub * 16 + 4 * j));
      uint32_t b[kFrags][2];
#pragma unroll
      for (int f = 0; f < kFrags; ++f) {
        b[f][0] = half_mul(p.x, half_mul(scale2[f][0], shift));
        b[f][1] = half_mul(p.y, half_mul(scale2[f][1], shift));
        mma_m16n8k16_f16(zo[f], even_codes(zero2[f][0]), 0u, even_codes(zero2[f][1]), 0u, b[f][0], b[f][1]);
      }
      // units r of every group, of entries j + 4t
      const uint32_t tv = stage + at.vc + sub * at.next_c;
      uint32_t w[4][kGroups / 2];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        if constexpr (kGroups == 4) {
          const uint2 y = lds64(tv + t * 4 * Row::kCodes);
          w[t][0] = y.x;
          w[t][1] = y.y;
        } else {
          w[t][0] = lds32(tv + t * 4 * Row::kCodes);
        }
      }
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
        // entries j | j + 4 and j + 8 | j + 12 side by side
        const uint32_t lo = __byte_perm(w[0][g / 2], w[1][g / 2], g & 1 ? 0x7632 : 0x5410), hi = __byte_perm(w[2][g / 2], w[3][g / 2], g & 1 ? 0x7632 : 0x5410);
        const uint32_t lo8 = lo >> 8, hi8 = hi >> 8;
        const int f = g / kPer;
        // (times 1 or 0: the other pipe has room)
        const uint32_t mine = of_group(g % kPer, r) ? 0x3c003c00u : 0u, b0 = kPer > 1 ? half_mul(b[f][0], mine) : b[f][0],
                       b1 = kPer > 1 ? half_mul(b[f][1], mine) : b[f][1];
        mma_m16n8k16_f16(o[f][0], even_codes(lo), odd_codes(lo), even_codes(hi), odd_codes(hi), b0, b1);
        mma_m16n8k16_f16(o[f][1], even_codes(lo8), odd_codes(lo8), even_codes(hi8), odd_codes(hi8), b0, b1);
      }
    }
  }

  // Codes (or zero points) in bits 0 .. 3, or 4 .. 7, of both halves as n 2^-10.
  __device__ __forceinline__ static uint32_t even_codes(uint32_t w) { return half_mul(w & 0x000f000fu, 0x74007400u); }
  __device__ __forceinline__ static uint32_t odd_codes(uint32_t w) { return half_mul(w & 0x00f000f0u, 0x64006400u); }
  __device__ __forceinline__ void scale_sums(float f0, float f1) {         // of columns 2j and 2j + 1
#pragma unroll
    for (int f = 0; f < kFrags; ++f) {
#pragma unroll
      for (int i = 0; i < 8; ++i) o[f][i / 4][i % 4] *= i & 1 ? f1 : f0;
      zo[f][0] *= f0;
      zo[f][1] *= f1;
    }
  }
  // A larger logit than any before: sums so far follow.
  template <int K>
  __device__ __forceinline__ void raise(const float (&x)[K][kHeads]) {
    float f[kHeads];
#pragma unroll
    for (int c = 0; c < kHeads; ++c) {
      float mx = x[0][c];
#pragma unroll
      for (int k = 1; k < K; ++k) mx = fmaxf(mx, x[k][c]);
#pragma unroll
      for (int off = kMasked ? 1 : 4; off < 32; off <<= 1) mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, off));
      mx = fmaxf(mx, m[c]);
      f[c] = exp2_fast(m[c] - (mx == -INFINITY ? 0.f : mx));
      l[c] *= f[c];
      m[c] = mx;
    }
    scale_sums(f[0], f[kHeads - 1]);
  }
  // The power of two that brings the largest value scale to [2^5, 2^6), or as near as fp16 has one.
  __device__ __forceinline__ static float power(uint32_t largest) { return pow2f(20 - max(5, (int)(largest >> 26))); }
  // A larger value scale.
  __device__ __forceinline__ void widen(uint32_t top) {
    top = __reduce_max_sync(~0u, max(top & 0xffffu, top >> 16));
    top |= top << 16;
    const float to = power(top), ratio = largest ? to / power(largest) : 0.f;
    scale_sums(ratio, ratio);
    largest = top;
    shift = half_pair(to, to);
  }

  // (max, sum) of the heads over this warp's entries to [8] each
  __device__ __forceinline__ void stats(float* sm_m, float* sm_l) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int c = 0; c < kHeads; ++c) {
#pragma unroll
      for (int off = kMasked ? 1 : 4; off < 32; off <<= 1) l[c] += __shfl_xor_sync(~0u, l[c], off);
      if (lane < (kMasked ? 1 : 4)) {
        sm_m[kMasked ? c : lane + 4 * c] = m[c];
        sm_l[kMasked ? c : lane + 4 * c] = l[c] * 0x1p-9f;
      }
    }
  }
  // The warp's output [G][D], relative to the heads' maxima over the warps (sm_m), to `out` or (ADD) on top of what is there; zeros: scratch, [groups][G].
  template <bool ADD>
  __device__ __forceinline__ void write(float* out, const float* sm_m, float* zeros) const {
    const int lane = threadIdx.x & 31, r = lane >> 2, j = lane & 3;
    __syncwarp();
#pragma unroll
    for (int f = 0; f < kFrags; ++f)                       // column r meets its own group in row r
      if (j == r >> 1 && (G == 1 ? r < kGroups : G == 2 ? r >> 1 < kGroups : true)) zeros[group_of(f, r) * G + head_of(r)] = r & 1 ? zo[f][1] : zo[f][0];
    __syncwarp();
    const float back = largest ? 0x1p1f / power(largest) : 0.f;      // codes' 2^10, weights' 2^-9
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int head = head_of(2 * j + c), which = G == 1 ? 2 * j + c : G == 2 ? j : G == 4 ? c : 0;     // the column's group in its fragment
      const float mm = m[kHeads == 2 ? c : 0], f = mm == -INFINITY ? 0.f : exp2_fast(mm - warps_max(sm_m, head)) * back;
#pragma unroll
      for (int f8 = 0; f8 < kFrags; ++f8) {
        if (which >= kPer) continue;
        const int g = f8 * kPer + which;
        const float z = zeros[g * G + head];
        float4* to = reinterpret_cast<float4*>(out + head * D + g * 32 + 4 * r);
        const float (&a)[2][4] = o[f8];
        float4 y = make_float4((a[0][c] - z) * f, (a[0][2 + c] - z) * f, (a[1][c] - z) * f, (a[1][2 + c] - z) * f);
        if constexpr (ADD) {
          const float4 was = *to;
          y.x += was.x; y.y += was.y; y.z += was.z; y.w += was.w;
        }
        *to = y;
      }
    }
  }
};

struct Kv4Piece {
  long long chunk;           // tiles per CTA of the deal, or
  int cut;                   // CTAs for each lane
  int b, head, v, left;      // lane, first tile, tiles until the end of the CTA's run
  int last;                  // is it the last piece of its lane?
  DecodeSpan s;
};
static_assert(sizeof(Kv4Piece) <= 64, "Kv4Shape::kOther");

__device__ __forceinline__ void kv4_consumers_sync() { asm volatile("bar.sync 1, %0;" ::"n"(kKv4Warps * 32) : "memory"); }

template <int D, int G, bool CHOSEN>
__global__ void __launch_bounds__(kKv4Threads, (Kv4Shape<D, G>::kCtas)) paged_decode_kv4_kernel(const __grid_constant__ DecodeParams P) {
  using Sh = Kv4Shape<D, G>;
  using Row = Kv4Row<D>;
  using Warp = Kv4Warp<D, G>;
  constexpr int TILE = kKv4Tile, STAGES = Sh::kStages;
  extern __shared__ __align__(128) unsigned char ring[];
  float* sm_out = reinterpret_cast<float*>(ring + STAGES * Sh::kStage);         // [outs][G][D]
  uint4* query = reinterpret_cast<uint4*>(sm_out + Sh::kOuts * G * D);
  float* scratch = reinterpret_cast<float*>(query + Sh::kQuery / 16);           // [warps][G][16]
  float* sm_m = scratch + kKv4Warps * 16 * G;                                   // [warps][8]
  float* sm_l = sm_m + kKv4Warps * 8;
  int* lens = reinterpret_cast<int*>(sm_l + kKv4Warps * 8);                     // [batch]
  int* cum = lens + kMaxSequences;                                              // [batch + 1] tiles of one head before b, then the most
  int* slot_entry = cum + kMaxSequences + 8;                                    // [stages][slots] first entry of a page, see below
  uint64_t* full = reinterpret_cast<uint64_t*>(slot_entry + STAGES * kKv4MaxSlots);
  uint64_t* empty = full + STAGES;
  // the consumers' piece: little of it is needed inside the loop over tiles, whose registers are short
  Kv4Piece* piece = reinterpret_cast<Kv4Piece*>(empty + STAGES);

  const PagedParams& A = P.A;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  auto span = [&](int len) {
    DecodeSpan x;
    if constexpr (CHOSEN) x = chosen_span<TILE>(A, len, P.n_select);
    else x = decode_span<TILE>(len, A.window, A.sink);
    if (len == 0) x.tiles = 0;                             // padding costs no piece
    return x;
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
  const long long chunk = quotient(total + gridDim.x - 1, gridDim.x);
  long long t0 = cta * chunk, t1 = min(total, t0 + chunk);
  const long long lanes = (long long)A.batch * H;
  for (int e = cta; e < (int)lanes; e += gridDim.x) {      // padded rows
    if (lens[e / H] != 0) continue;
    const long long to = ((long long)(e / H) * A.n_q_heads + e % H * G) * D;
    for (int i = tid; i < G * D / 8; i += kKv4Threads) reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(A.out) + to)[i] = make_uint4(0, 0, 0, 0);
    if (A.lse && tid < G) A.lse[to / D + tid] = -INFINITY;
  }
  const int cut = lane_ctas(lanes, total, cum[A.batch + 1], chunk, true);
  if (cut && !own_tiles(cta, cut, H, lanes, cum, t0, t1)) return;
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
  const long long into = t0 - (long long)cum[b] * H;
  int head = (int)quotient(into, s.tiles), v = (int)(into - (long long)head * s.tiles);
  const int slots = TILE >> A.page_shift, slot_shift = 7 - A.page_shift;
  const uint32_t chunk_bytes = (uint32_t)A.page * Row::kBytes;
  // copies in flight at the end: as in the bf16 rows' kernel, there are none
  auto wait = [&](uint64_t* bar, uint32_t parity) { return (bool)__all_sync(~0u, mbar_wait(bar, parity, A.status, kWaitPolls)); };
  if (tid == 0) {
    piece->chunk = chunk;
    piece->cut = cut;
    piece->b = b; piece->head = head; piece->v = v; piece->left = (int)(t1 - t0);
    piece->s = s;
  }
  // Where page `slot` of a tile starts: its first entry, which is seen or not; of a bad page ~entry; the sequence's length if the page
  // holds nothing visible (so that no entry in it is).
  if (warp >= kKv4Warps) {                                 // ---- a team's producer: every second tile
    const uint64_t policy = l2_policy_evict_first();
    fence_proxy_async();                                   // rows that earlier kernels stored are read by the copies
    const int team = warp - kKv4Warps;
    int st = team, skip = team;                            // the next tile's stage; tiles of the piece before it
    uint32_t round = 0;                                    // how often the ring was filled
    for (int left = (int)(t1 - t0); left > 0;) {
      const int n = min(s.tiles - v, left);
      const int per = 32 >> slot_shift;                    // tiles whose pages are looked up together
      const long long lane_no = (long long)b * H + head;
      int k0 = skip;
      for (; k0 < n; k0 += 2 * per) {
        int entry = s.len, page_no = -1;
        {
          const int k = k0 + 2 * (lane >> slot_shift), slot = lane & (slots - 1);
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
        for (int i = 0; i < per && k0 + 2 * i < n; ++i) {
          const int mine = i << slot_shift | (lane & (slots - 1));
          const int e = __shfl_sync(~0u, entry, mine), pg = __shfl_sync(~0u, page_no, mine);
          if (round > 0 && !wait(&empty[st], (round & 1) ^ 1)) return;
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
          st += 2;
          if (st >= STAGES) { st -= STAGES; ++round; }
        }
      }
      skip = (skip + n) & 1;
      left -= n;
      v += n;
      if (v == s.tiles && left > 0) {
        v = 0;
        if (++head == H) {
          head = 0;
          do s = span(lens[++b]); while (s.tiles == 0);
        }
      }
    }
    return;
  }

  // ---- consumers
  Warp w;
  bool ok = true;          // else a wait gave up: this warp keeps the others' barriers company, and counts its pieces, but reads no more tiles
  float* mine = scratch + warp * 16 * G;
  const int team = warp / kKv4TileWarps, row = warp % kKv4TileWarps * kKv4Share;       // the tiles, and rows of a tile, that are this warp's
  const typename Warp::Offsets at = Warp::offsets(A.page, A.page_shift, row, Sh::kHalf);
  const int first = row & (A.page - 1), second = A.page == 16 ? 0 : first + 16;        // of the halves' pages
  int st = team, skip = team;                              // stage and parity of this warp's next tile; tiles of a piece before it
  uint32_t phase = 0;
  const uint32_t ring0 = smem_u32(ring), entry0 = smem_u32(slot_entry + (row >> A.page_shift)), entry1 = entry0 + (A.page == 16 ? 4 : 0);
  for (;;) {
    kv4_consumers_sync();                                  // the piece is there, sm_* are free
    if (piece->left <= 0) break;
    const int n = min(piece->s.tiles - piece->v, piece->left);           // tiles of this piece
    w.begin(static_cast<const __nv_bfloat16*>(A.q) + (long long)piece->b * A.q_stride + (long long)piece->head * G * D, A.scale_log2, query, warp == 0);
    kv4_consumers_sync();
    if constexpr (Warp::kHolds) w.load_query(smem_u32(query));
    const int lo = piece->s.lo;
    const unsigned fit = (unsigned)max(0, piece->s.len - 15 - lo);       // places for 16 entries, all of them seen, from lo on
    int k = skip;
    for (; k < n; k += 2) {
      const int at_stage = st;
      ok = ok && wait(&full[at_stage], phase);
      st += 2;
      if (st >= STAGES) { st -= STAGES; phase ^= 1; }
      if (!ok) continue;
      const int e0 = (int)lds32(entry0 + at_stage * (kKv4MaxSlots * 4)), e1 = (int)lds32(entry1 + at_stage * (kKv4MaxSlots * 4));
      const uint32_t stage = ring0 + at_stage * Sh::kStage;
      // (no bad page: the complement of a first entry 0 would be a place like others, 31 or 47 rows into a page of 64)
      if ((e0 | e1) >= 0 && (unsigned)(e0 + first - lo) < fit && (unsigned)(e1 + second - lo) < fit) {
        w.template tile<true>(stage, at, 0, 0, DecodeSpan(), smem_u32(mine), smem_u32(query));
      } else {
        // first entries, complements for bad pages
        const int i0 = e0 < 0 ? e0 - first : e0 + first, i1 = e1 < 0 ? e1 - second : e1 + second;
        const DecodeSpan s = piece->s;
        auto any = [&](int e) { const int i = e < 0 ? ~e : e; return i < s.len && (i + 16 > s.lo || i < s.sinks); };
        if (any(i0) || any(i1)) w.template tile<false>(stage, at, i0, i1, s, smem_u32(mine), smem_u32(query));
      }
      release_stage(&empty[at_stage]);
    }
    skip = k - n;
    // join the eight warps
    w.stats(sm_m + warp * 8, sm_l + warp * 8);
    kv4_consumers_sync();
    if (warp < Sh::kOuts) w.template write<false>(sm_out + warp * G * D, sm_m, mine);
    kv4_consumers_sync();
    if constexpr (Sh::kOuts < kKv4Warps) {
      if (warp >= Sh::kOuts) w.template write<true>(sm_out + (warp - Sh::kOuts) * G * D, sm_m, mine);
      kv4_consumers_sync();
    }
    const int b = piece->b, head = piece->head, hq0 = head * G, tiles = piece->s.tiles;
    const long long lane_no = (long long)b * H + head;
    const bool whole = n == tiles;
    constexpr int kVecs = G * D / 4;                       // float4s of a lane's output
    auto warps_sum = [&](int e) {
      float4 x = reinterpret_cast<const float4*>(sm_out)[e];
#pragma unroll
      for (int i = 1; i < Sh::kOuts; ++i) {
        const float4 y = reinterpret_cast<const float4*>(sm_out + i * G * D)[e];
        x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
      }
      return x;
    };
    auto finish = [&](int e, float4 x, float total_l) {
      const float inv = total_l == 0.f ? 0.f : 1.f / total_l;
      __nv_bfloat16* out = static_cast<__nv_bfloat16*>(A.out) + ((long long)b * A.n_q_heads + hq0) * D + e * 4;
      *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf16(x.x * inv, x.y * inv), pack_bf16(x.z * inv, x.w * inv));
    };
    auto finish_lse = [&](int g, float mm, float ll) {
      if (A.lse) A.lse[(long long)b * A.n_q_heads + hq0 + g] = ll == 0.f ? -INFINITY : (mm + log2f(ll)) * kLn2;
    };
    if (whole) {
      for (int e = tid; e < kVecs; e += kKv4Warps * 32) {
        const int g = e / (D / 4);
        const float big = warps_max(sm_m, g), l = warps_l(sm_m, sm_l, g, big);
        finish(e, warps_sum(e), l);
        if (e % (D / 4) == 0) finish_lse(g, big, l);
      }
    } else {
      const long long slot = cta + lane_no;
      for (int e = tid; e < kVecs; e += kKv4Warps * 32) reinterpret_cast<float4*>(P.part + slot * G * D)[e] = warps_sum(e);
      if (tid < G) {
        const float big = warps_max(sm_m, tid);
        P.part_ml[slot * G + tid] = make_float2(big, warps_l(sm_m, sm_l, tid, big));
      }
      __threadfence();
      kv4_consumers_sync();
      // pieces of the lane: its tiles lie at [off, off + tiles) of the deal
      const long long off = (long long)cum[b] * H + (long long)head * tiles, chunk = piece->chunk;
      const int cut = piece->cut, per = cut ? (tiles + cut - 1) / cut : 1;
      const int c0 = cut ? (int)lane_no * cut : (int)quotient(off, chunk), pieces = cut ? (tiles + per - 1) / per : (int)quotient(off + tiles - 1, chunk) - c0 + 1;
      if (tid == 0) {
        const bool last = atomicAdd(P.arrived + lane_no, 1u) == (uint32_t)pieces - 1;
        if (last) P.arrived[lane_no] = 0;
        piece->last = last;
      }
      kv4_consumers_sync();
      if (piece->last) {
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
    kv4_consumers_sync();
    if (tid == 0) {                                        // the next piece
      piece->left -= n;
      piece->v += n;
      if (piece->v == tiles && piece->left > 0) {
        piece->v = 0;
        if (++piece->head == H) {
          piece->head = 0;
          do piece->s = span(lens[++piece->b]); while (piece->s.tiles == 0);
        }
      }
    }
  }
}

}  // namespace wkv
