// New rows into the pages of a cache, with the position rotation applied on the way, and rows in 4 bits spread out to bf16 pages.
//
//   y_2i = x_2i cos - x_2i+1 sin, y_2i+1 = x_2i+1 cos + x_2i sin     (or channels i and i + dim/2), angles by position from a table
//
// Bound: HBM; a number is read once and written once.  One launch does the queries and the new entries.  The part of a page that one call
// fills belongs to one warp for each kv head (which so owns the page's bounds; the warps of a CTA share the rows' angles in L1), or, in 4
// bits, to a CTA for a few kv heads, which writes all rows in full lines.  Products are rounded one by one (no fused multiply-add), so that
// the result is the same as that of elementwise fp32 arithmetic, code for code where rows are held in 4 bits.
//
// Measured: prompts of 2048..8191 tokens, 4 x 32/32 heads x 128, bf16 with bounds, 220 us = 5.6 TB/s (0.86 of the measured copy rate); one
// token each of 19 sequences 3.8 us in a captured graph; chunks of 17..61 tokens in 4 bits 8.6 us; 8 x 1638..8192 entries, 8 heads x 128,
// spread out 40 us = 5.2 TB/s, nearly all of it writes.
#pragma once
#include "wkv_paged_kv4.cuh"

namespace wkv {

struct AppendParams {
  PagedParams A;                 // q NULL: no queries; rows: tokens of the call
  const float* rope;             // [rope_rows][rope_dim] cos | sin, or NULL
  const int32_t* positions;      // [rows] or NULL: the entry's index
  void* q_out;
  long long q_out_stride;
  int8_t* bounds;                // the layer's [pages][Hkv][2][D], or NULL
  float* bound_scale;            // [pages][Hkv]
  int rope_rows, rope_dim, paired;
  int q_blocks, q_heads, kv_heads, kv_splits, kv_slots;   // CTAs for queries; heads per CTA; CTAs per page part; parts, at most
};

constexpr int kRowsThreads = 256, kMostSequences = 1024;

// Eight channels in fp32.
struct Row8 {
  float x[8];
};
__device__ __forceinline__ Row8 load8(const __nv_bfloat16* p) {
  const uint4 u = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
  Row8 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) { r.x[2 * i] = __uint_as_float(w[i] << 16); r.x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
  return r;
}
__device__ __forceinline__ Row8 load8(const float* p) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  return Row8{{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
}
// ... as they lie in memory: rows in flight take half the registers
template <typename T>
struct Piece {
  uint4 w[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) w[i] = reinterpret_cast<const uint4*>(p)[i];
  }
  __device__ __forceinline__ void store(T* p) const {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4*>(p)[i] = w[i];
  }
  __device__ __forceinline__ Row8 row() const { return load8(reinterpret_cast<const T*>(w)); }
};
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const Row8& r) {
  *reinterpret_cast<uint4*>(p) = make_uint4(bf16_pair(r.x[0], r.x[1]), bf16_pair(r.x[2], r.x[3]), bf16_pair(r.x[4], r.x[5]), bf16_pair(r.x[6], r.x[7]));
}
__device__ __forceinline__ void store8(float* p, const Row8& r) {
  reinterpret_cast<float4*>(p)[0] = make_float4(r.x[0], r.x[1], r.x[2], r.x[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(r.x[4], r.x[5], r.x[6], r.x[7]);
}

// A row is eight or four units of two pieces of eight channels: unit u < dim/16 holds a turned pair of pieces (u, u + dim/16), the others
// two neighbouring pieces that stay.
template <int D>
__device__ __forceinline__ int2 unit_pieces(int u, int dim) {
  const int h = dim >> 4;
  return u < h ? make_int2(u, u + h) : make_int2(2 * u, 2 * u + 1);
}
__device__ __forceinline__ void turn(float& a, float& b, float c, float s) {
  const float y = __fsub_rn(__fmul_rn(a, c), __fmul_rn(b, s));
  b = __fadd_rn(__fmul_rn(b, c), __fmul_rn(a, s));
  a = y;
}
// A unit's angles: of channel i of both pieces cos c[i], sin s[i]; paired: of channels 2i, 2i + 1 of the first piece c[i], s[i], of the
// second one's c[4 + i], s[4 + i].
struct Turn {
  bool on;
  Row8 c, s;
  __device__ __forceinline__ void load(const float* angles, int u, int dim, int paired) {      // angles: the position's row, or NULL
    const int h = dim >> 4;
    on = angles && u < h;
    if (!on) return;
    const float* sines = angles + (dim >> 1);
    const float4* at[4] = {reinterpret_cast<const float4*>(angles + (paired ? 4 * u : 8 * u)), reinterpret_cast<const float4*>(angles + (paired ? 4 * (u + h) : 8 * u + 4)),
                           reinterpret_cast<const float4*>(sines + (paired ? 4 * u : 8 * u)), reinterpret_cast<const float4*>(sines + (paired ? 4 * (u + h) : 8 * u + 4))};
    const float4 y[4] = {*at[0], *at[1], *at[2], *at[3]};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      c.x[4 * k] = y[k].x; c.x[4 * k + 1] = y[k].y; c.x[4 * k + 2] = y[k].z; c.x[4 * k + 3] = y[k].w;
      s.x[4 * k] = y[2 + k].x; s.x[4 * k + 1] = y[2 + k].y; s.x[4 * k + 2] = y[2 + k].z; s.x[4 * k + 3] = y[2 + k].w;
    }
  }
  __device__ __forceinline__ void turn_unit(Row8& a, Row8& b, int paired) const {
    if (!on) return;
    if (!paired) {
#pragma unroll
      for (int i = 0; i < 8; ++i) turn(a.x[i], b.x[i], c.x[i], s.x[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        turn(a.x[2 * i], a.x[2 * i + 1], c.x[i], s.x[i]);
        turn(b.x[2 * i], b.x[2 * i + 1], c.x[4 + i], s.x[4 + i]);
      }
    }
  }
};
// The table's row for token r with entry index i; NULL, reported, if the position is outside of it.
__device__ __forceinline__ const float* angles_of(const AppendParams& P, int r, int i) {
  if (!P.rope) return nullptr;
  const int pos = P.positions ? P.positions[r] : i;
  if ((unsigned)pos >= (unsigned)P.rope_rows) {
    flag_bad_table(P.A.status);
    return nullptr;
  }
  return P.rope + (long long)pos * P.rope_dim;
}

// First of the slots for parts of pages that sequence b has: as many as its tokens may touch, whatever its length.  Sequence b's tokens,
// n of them, lie in (n - 2) / page + 2 pages at most, rounded down.
__device__ __forceinline__ int first_slot(int row, int b, int page_shift) { return (row >> page_shift) + 2 * b; }

// ---- queries: 32 (token, head) rows at once, a unit per thread.  The rows that a thread takes do not depend on whose they are: the first
// ones are on their way while that is found out, then always the next ones while some are turned.
template <typename T, int D>
__device__ __forceinline__ void turn_queries(const AppendParams& P, int block, int* starts) {
  const PagedParams& A = P.A;
  constexpr int kUnits = D / 16, kSlots = kRowsThreads / kUnits, kSteps = sizeof(T) == 2 ? 2 : 1;
  const int per = (A.n_q_heads + P.q_heads - 1) / P.q_heads;
  const int tokens = min(A.rows, kSlots), t0 = block / per * tokens, h0 = block % per * P.q_heads, h1 = min(A.n_q_heads, h0 + P.q_heads);
  const int u = threadIdx.x % kUnits, slot = threadIdx.x / kUnits, lanes = kSlots / tokens;     // heads at once
  const int r = t0 + slot % tokens;
  const bool on = slot < lanes * tokens && r < A.rows;
  const int2 at = unit_pieces<D>(u, P.rope ? P.rope_dim : 0);
  const T* from = static_cast<const T*>(A.q) + (long long)r * A.q_stride;
  T* to = static_cast<T*>(P.q_out) + (long long)r * P.q_out_stride;
  struct Rows {
    Piece<T> a[kSteps], b[kSteps];
  } x0, x1;
  auto load = [&](Rows& x, int base) {
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
      const int h = base + k * lanes;
      if (h >= h1) continue;
      x.a[k].load(from + h * D + 8 * at.x);
      x.b[k].load(from + h * D + 8 * at.y);
    }
  };
  int base = h0 + slot / tokens;
  if (on) load(x0, base);
  int entry;
  if (A.q_start) {
    int* lens = starts + kMostSequences + 1;
    for (int b = threadIdx.x; b <= A.batch; b += kRowsThreads) {
      starts[b] = A.q_start[b];
      if (b < A.batch) lens[b] = A.seq_lens[b];
    }
    __syncthreads();
    if (!on) return;
    int lo = 0, hi = A.batch;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (starts[mid] <= r) lo = mid; else hi = mid;
    }
    const int s0 = max(0, starts[lo]), s1 = min(starts[lo + 1], A.rows);   // as seq_rows has them; the appending CTAs, or this, report
    const long long most = (long long)A.width << A.page_shift;
    const int len = lens[lo] < 0 ? 0 : lens[lo] > most ? (int)most : lens[lo];
    if (s0 != starts[lo] || s1 != starts[lo + 1] || s1 < s0 || len != lens[lo] || s1 - s0 > len) flag_bad_table(A.status);
    if (r < s0 || r >= s1) return;
    entry = len - (s1 - s0) + (r - s0);
  } else {
    if (!on) return;
    entry = clamped_len(A, r) - 1;
    if (entry < 0) return;
  }
  Turn angles;
  angles.load(angles_of(P, r, entry), u, P.rope_dim, P.paired);
  auto store = [&](const Rows& x, int at_head) {
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
      const int h = at_head + k * lanes;
      if (h >= h1) continue;
      Row8 a = x.a[k].row(), b = x.b[k].row();
      angles.turn_unit(a, b, P.paired);
      store8(to + h * D + 8 * at.x, a);
      store8(to + h * D + 8 * at.y, b);
    }
  };
  const int step = kSteps * lanes;
  for (; base < h1; base += 2 * step) {
    load(x1, base + step);
    store(x0, base);
    load(x0, base + 2 * step);
    store(x1, base + step);
  }
}

// ---- bounds of the n keys of a page: key(row, pair of channels) in shared memory.  Pairs of channels as they lie in a row:
__device__ __forceinline__ __nv_bfloat162 pair_max(__nv_bfloat162 a, __nv_bfloat162 b) { return __hmax2(a, b); }
__device__ __forceinline__ __nv_bfloat162 pair_min(__nv_bfloat162 a, __nv_bfloat162 b) { return __hmin2(a, b); }
__device__ __forceinline__ float2 pair_floats(__nv_bfloat162 a) { return __bfloat1622float2(a); }
__device__ __forceinline__ float2 pair_max(float2 a, float2 b) { return make_float2(fmaxf(a.x, b.x), fmaxf(a.y, b.y)); }
__device__ __forceinline__ float2 pair_min(float2 a, float2 b) { return make_float2(fminf(a.x, b.x), fminf(a.y, b.y)); }
__device__ __forceinline__ float2 pair_floats(float2 a) { return a; }
__device__ __forceinline__ __nv_bfloat162 pair_shuffle(__nv_bfloat162 a, int off) { return __shfl_xor_sync(~0u, a, off); }
__device__ __forceinline__ float2 pair_shuffle(float2 a, int off) { return make_float2(__shfl_xor_sync(~0u, a.x, off), __shfl_xor_sync(~0u, a.y, off)); }
template <typename T> struct PairOf { typedef __nv_bfloat162 type; };
template <> struct PairOf<float> { typedef float2 type; };

// A page's scale and its inverse; a bound in steps of it, outwards.  An infinite key makes the scale infinite and its own products no
// numbers: those end at the outer border, here the largest at 127 and the least at -127 (minima and maxima drop what is no number), all
// others are 0, so that the page's score is infinity or no number, and the page among the chosen.
struct BoundScale {
  float scale, inv;
  __device__ __forceinline__ uint32_t up(float x) const { return (uint32_t)(int)fmaxf(fminf(ceilf(__fmul_rn(x, inv)), 127.f), -127.f) & 255; }
  __device__ __forceinline__ uint32_t down(float x) const { return (uint32_t)(int)fminf(fmaxf(floorf(__fmul_rn(x, inv)), -127.f), 127.f) & 255; }
};

__device__ __forceinline__ BoundScale bound_scale(float most) {
  BoundScale q;
  q.scale = __fmul_rn(most, 1.f / 127.f);
  q.inv = q.scale >= 0x1p-100f ? __frcp_rn(q.scale) : 0.f;
  return q;
}

// By a CTA.  work: [2][threads] pairs and [warps] floats.  A thread owns a pair of channels over a share of the rows; the shares meet in
// shared memory.  One barrier; the caller's next one protects the keys and the work.
template <int D, typename Keys>
__device__ __forceinline__ void write_bounds(const AppendParams& P, Keys key, int n, float2* work, long long chunk) {
  constexpr int kPairs = D / 2, kShares = kRowsThreads / kPairs;
  float2* his = work;
  float2* los = his + kRowsThreads;
  float* mosts = reinterpret_cast<float*>(los + kRowsThreads);
  const int c = threadIdx.x % kPairs, share = threadIdx.x / kPairs;
  float2 hi = key(min(share, n - 1), c), lo = hi;
  for (int r = share + kShares; r < n; r += kShares) {
    const float2 x = key(r, c);
    hi = pair_max(hi, x);
    lo = pair_min(lo, x);
  }
  his[threadIdx.x] = hi;
  los[threadIdx.x] = lo;
  float most = fmaxf(fmaxf(fabsf(hi.x), fabsf(hi.y)), fmaxf(fabsf(lo.x), fabsf(lo.y)));
#pragma unroll
  for (int off = 16; off; off >>= 1) most = fmaxf(most, __shfl_xor_sync(~0u, most, off));
  if ((threadIdx.x & 31) == 0) mosts[threadIdx.x >> 5] = most;
  __syncthreads();
  if (share == 0) {
#pragma unroll
    for (int k = 1; k < kShares; ++k) {
      hi = pair_max(hi, his[threadIdx.x + k * kPairs]);
      lo = pair_min(lo, los[threadIdx.x + k * kPairs]);
    }
    most = 0.f;
#pragma unroll
    for (int k = 0; k < kRowsThreads / 32; ++k) most = fmaxf(most, mosts[k]);
    const BoundScale q = bound_scale(most);
    uint16_t* to = reinterpret_cast<uint16_t*>(P.bounds + chunk * 2 * D);
    to[c] = (uint16_t)(q.up(hi.x) | q.up(hi.y) << 8);
    to[kPairs + c] = (uint16_t)(q.down(lo.x) | q.down(lo.y) << 8);
    if (c == 0) P.bound_scale[chunk] = q.scale;
  }
}

// ---- new entries in the storage type
template <int D>
struct RowsShape {
  static constexpr int kUnits = D / 16, kSlots = kRowsThreads / kUnits;
  static constexpr int kOffsets = (2 * kMostSequences + 1) * 4;         // of the queries' CTAs: offsets and lengths
};
// 4 bits: fp32 keys of a page, then the codes and pairs of its keys and values.  A group's 32 keys lie 36 floats behind the last one's:
// the threads of a row's groups read them from different banks.
template <int D>
struct Rows4Shape {
  static constexpr int kStride = D / 32 * 36;
  __device__ __forceinline__ static int at(int r, int c) { return r * kStride + c / 32 * 36 + c % 32; }
  static constexpr int kKeys = 64 * kStride * 4;
  static constexpr int kImage = 64 * Kv4Row<D>::kBytes;
  static constexpr int kWork = 2 * kRowsThreads * 8 + 32;
};
template <int D, bool FOUR>
constexpr int rows_smem() { return FOUR ? Rows4Shape<D>::kKeys + 2 * Rows4Shape<D>::kImage + Rows4Shape<D>::kWork : RowsShape<D>::kOffsets; }

struct PagePart {
  int b, first;                // sequence; row of the first new entry
  int e0, n, old;              // index of the first new entry, number of new entries, entries of the page before them
};

// A head's rows of a part, by one warp: four (or eight) rows at once, a unit per lane; the next rows are read while these are turned and
// stored.  The largest and least keys of a channel stay in registers until the end: no barriers (a CTA per part, keys staged in shared
// memory, took 203 us for the kv half of 4 x 2048..8191 tokens, 32 heads, where 152 are without bounds).
template <typename T, int D>
__device__ __forceinline__ void append_head(const AppendParams& P, const PagePart& w, int h) {
  typedef typename PairOf<T>::type Pair;
  constexpr int kUnits = D / 16, kRows = 32 / kUnits;
  const PagedParams& A = P.A;
  const int lane = threadIdx.x & 31, u = lane % kUnits, sub = lane / kUnits;
  const int2 at = unit_pieces<D>(u, P.rope ? P.rope_dim : 0);
  struct Unit {
    Piece<T> ka, kb, va, vb;
    Turn angles;
  } x0, x1;
  auto load = [&](Unit& x, int r) {
    if (r >= w.n) return;
    x.angles.load(angles_of(P, w.first + r, w.e0 + r), u, P.rope_dim, P.paired);
    const long long src = (long long)(w.first + r) * A.kv_stride + (long long)h * D;
    x.ka.load(static_cast<const T*>(A.k) + src + 8 * at.x);
    x.kb.load(static_cast<const T*>(A.k) + src + 8 * at.y);
    x.va.load(static_cast<const T*>(A.v) + src + 16 * u);
    x.vb.load(static_cast<const T*>(A.v) + src + 16 * u + 8);
  };
  load(x0, sub);
  const int page = page_of(A, w.b, w.e0);                  // (the first rows are on their way)
  if (page < 0) return;
  const long long dst = row_offset(A, page, h, w.e0, D);
  Pair up[8], down[8];                                     // of pieces at.x and at.y
  {
    const float2 least = make_float2(-INFINITY, -INFINITY), most = make_float2(INFINITY, INFINITY);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (sizeof(T) == 2) { up[i] = __float22bfloat162_rn(least); down[i] = __float22bfloat162_rn(most); }
      else { up[i] = least; down[i] = most; }
    }
  }
  auto look = [&](const Piece<T>& a, const Piece<T>& b) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const Pair y = reinterpret_cast<const Pair*>(i < 4 ? a.w : b.w)[i & 3];
      up[i] = pair_max(up[i], y);
      down[i] = pair_min(down[i], y);
    }
  };
  auto store = [&](const Unit& x, int r) {
    if (r >= w.n) return;
    Row8 a = x.ka.row(), b = x.kb.row();
    x.angles.turn_unit(a, b, P.paired);
    Piece<T> pa, pb;
    store8(reinterpret_cast<T*>(pa.w), a);
    store8(reinterpret_cast<T*>(pb.w), b);
    const long long to = dst + (long long)r * D;
    pa.store(static_cast<T*>(A.k_pool) + to + 8 * at.x);
    pb.store(static_cast<T*>(A.k_pool) + to + 8 * at.y);
    x.va.store(static_cast<T*>(A.v_pool) + to + 16 * u);
    x.vb.store(static_cast<T*>(A.v_pool) + to + 16 * u + 8);
    if (P.bounds) look(pa, pb);
  };
  if (P.bounds) {
    constexpr int kSteps = sizeof(T) == 2 ? 4 : 2;         // entries of the page that are there already
    for (int base = sub; base < w.old; base += kSteps * kRows) {
      Piece<T> a[kSteps], b[kSteps];
#pragma unroll
      for (int k = 0; k < kSteps; ++k) {
        const T* from = static_cast<const T*>(A.k_pool) + row_offset(A, page, h, min(base + k * kRows, w.old - 1), D);      // (one twice: no matter)
        a[k].load(from + 8 * at.x);
        b[k].load(from + 8 * at.y);
      }
#pragma unroll
      for (int k = 0; k < kSteps; ++k) look(a[k], b[k]);
    }
  }
  if constexpr (sizeof(T) == 2) {
    for (int r = sub; r < w.n; r += 2 * kRows) {
      load(x1, r + kRows);
      store(x0, r);
      load(x0, r + 2 * kRows);
      store(x1, r + kRows);
    }
  } else {
    // (two fp32 rows would not fit into the registers)
    for (int r = sub; r < w.n; r += kRows) {
      store(x0, r);
      load(x0, r + kRows);
    }
  }
  if (!P.bounds) return;
  __syncwarp();
  float most = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
#pragma unroll
    for (int off = kUnits; off < 32; off <<= 1) {
      up[i] = pair_max(up[i], pair_shuffle(up[i], off));
      down[i] = pair_min(down[i], pair_shuffle(down[i], off));
    }
    const float2 a = pair_floats(up[i]), b = pair_floats(down[i]);
    most = fmaxf(most, fmaxf(fmaxf(fabsf(a.x), fabsf(a.y)), fmaxf(fabsf(b.x), fabsf(b.y))));
  }
#pragma unroll
  for (int off = 1; off < kUnits; off <<= 1) most = fmaxf(most, __shfl_xor_sync(~0u, most, off));
  const BoundScale q = bound_scale(most);
  const long long chunk = (long long)page * A.n_kv_heads + h;
  // the rows' lanes share the writing: largest and least of piece at.x, of piece at.y
  if (sub < 4) {
    uint32_t word[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 hi = pair_floats(sub & 2 ? up[4 + i] : up[i]), lo = pair_floats(sub & 2 ? down[4 + i] : down[i]);
      const uint32_t two = sub & 1 ? q.down(lo.x) | q.down(lo.y) << 8 : q.up(hi.x) | q.up(hi.y) << 8;
      word[i / 2] |= two << 16 * (i & 1);
    }
    *reinterpret_cast<uint2*>(P.bounds + (chunk * 2 + (sub & 1)) * D + 8 * (sub & 2 ? at.y : at.x)) = make_uint2(word[0], word[1]);
    if (lane == 0) P.bound_scale[chunk] = q.scale;
  }
}

// A group of 32 channels: codes and the pair of its row.
template <bool KEY>
__device__ __forceinline__ void pack_group(const float (&x)[32], uint32_t (&words)[4], uint32_t& pair, Kv4Scale& q) {
  float lo = 0.f, hi = 0.f;
#pragma unroll
  for (int i = 0; i < 32; ++i) { lo = fminf(lo, x[i]); hi = fmaxf(hi, x[i]); }
  q = kv4_scale_of(lo, hi);
  pair = q.byte | q.zero << 8;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    words[w] = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t n = kv4_code(x[8 * w + i], q);
      words[w] |= n << (KEY ? (i >> 1) * 4 + (i & 1) * 16 : 4 * i);      // values: unit 2w in the low half, unit 2w + 1 in the high one
    }
  }
}

template <typename T, int D>
__device__ __forceinline__ void append_part4(const AppendParams& P, const PagePart& w, int h0, int h1, unsigned char* smem) {
  using Sh = RowsShape<D>;
  using Row = Kv4Row<D>;
  using R4 = Rows4Shape<D>;
  constexpr int G = Row::kGroups;
  const PagedParams& A = P.A;
  float* keys = reinterpret_cast<float*>(smem);
  unsigned char* image = smem + Rows4Shape<D>::kKeys;      // codes [n][kCodes] and pairs [n][kPairs] of the keys, then of the values
  float2* work = reinterpret_cast<float2*>(smem + Rows4Shape<D>::kKeys + 2 * Rows4Shape<D>::kImage);
  const int u = threadIdx.x % Sh::kUnits, slot = threadIdx.x / Sh::kUnits;
  const int2 at = unit_pieces<D>(u, P.rope ? P.rope_dim : 0);
  const int i0 = w.e0 & (A.page - 1);
  const long long chunk_bytes = (long long)A.page * Row::kBytes;
  const int page = page_of(A, w.b, w.e0);
  if (page < 0) return;
  for (int h = h0; h < h1; ++h) {
    const long long chunk = (long long)page * A.n_kv_heads + h;
    unsigned char* kc = static_cast<unsigned char*>(A.k_pool) + chunk * chunk_bytes;
    unsigned char* vc = static_cast<unsigned char*>(A.v_pool) + chunk * chunk_bytes;
    for (int r = slot; r < w.n; r += Sh::kSlots) {
      const T* src = static_cast<const T*>(A.k) + (long long)(w.first + r) * A.kv_stride + (long long)h * D;
      Row8 a = load8(src + 8 * at.x), b = load8(src + 8 * at.y);
      Turn angles;
      angles.load(angles_of(P, w.first + r, w.e0 + r), u, P.rope_dim, P.paired);
      angles.turn_unit(a, b, P.paired);
      store8(keys + R4::at(w.old + r, 8 * at.x), a);
      store8(keys + R4::at(w.old + r, 8 * at.y), b);
    }
    __syncthreads();
    // a thread per group: the keys', then the values'
    for (int k = threadIdx.x; k < 2 * w.n * G; k += kRowsThreads) {
      const bool key = k < w.n * G;
      const int r = (key ? k : k - w.n * G) / G, g = k % G;
      float x[32];
      uint32_t words[4], pair;
      Kv4Scale q;
      unsigned char* to = image + (key ? 0 : Rows4Shape<D>::kImage);
      if (key) {
        float* from = keys + R4::at(w.old + r, g * 32);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const Row8 y = load8(from + 8 * i);
#pragma unroll
          for (int e = 0; e < 8; ++e) x[8 * i + e] = y.x[e];
        }
        pack_group<true>(x, words, pair, q);
        *reinterpret_cast<uint4*>(to + Row::k_piece(i0 + r, g) - i0 * Row::kCodes) = make_uint4(words[0], words[1], words[2], words[3]);
        if (P.bounds) {
          // the bounds are those of the values that the codes stand for
#pragma unroll
          for (int i = 0; i < 32; ++i) from[i] = ((float)kv4_code(x[i], q) - q.z) * q.s;
        }
      } else {
        const T* from = static_cast<const T*>(A.v) + (long long)(w.first + r) * A.kv_stride + (long long)h * D + g * 32;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const Row8 y = load8(from + 8 * i);
#pragma unroll
          for (int e = 0; e < 8; ++e) x[8 * i + e] = y.x[e];
        }
        pack_group<false>(x, words, pair, q);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          *reinterpret_cast<uint16_t*>(to + Row::v_unit(i0 + r, g, i) - i0 * Row::kCodes) = (uint16_t)(words[i >> 1] >> (i & 1) * 16);
      }
      *reinterpret_cast<uint16_t*>(to + w.n * Row::kCodes + r * Row::kPairs + 2 * g) = (uint16_t)pair;
    }
    if (P.bounds) {
      for (int k = threadIdx.x; k < w.old * G; k += kRowsThreads) {
        const int r = k / G, g = k % G;
        const uint4 c = *reinterpret_cast<const uint4*>(kc + Row::k_piece(r, g));
        const uint32_t pair = *reinterpret_cast<const uint16_t*>(kc + Row::pairs(A.page, r) + 2 * g), words[4] = {c.x, c.y, c.z, c.w};
        const float s = kv4_scale(pair & 255), z = (float)(pair >> 8);
#pragma unroll
        for (int i = 0; i < 32; ++i)
          keys[R4::at(r, g * 32 + i)] = ((float)(words[i >> 3] >> ((i & 7) >> 1) * 4 + (i & 1) * 16 & 15) - z) * s;
      }
    }
    __syncthreads();
    // the image to the page: rows lie end to end, in both parts
    const int code16 = w.n * Row::kCodes / 16, pair4 = w.n * Row::kPairs / 4;
    for (int k = threadIdx.x; k < 2 * code16; k += kRowsThreads) {
      const bool key = k < code16;
      const int e = key ? k : k - code16;
      *reinterpret_cast<uint4*>((key ? kc : vc) + i0 * Row::kCodes + e * 16) = *reinterpret_cast<const uint4*>(image + (key ? 0 : Rows4Shape<D>::kImage) + e * 16);
    }
    for (int k = threadIdx.x; k < 2 * pair4; k += kRowsThreads) {
      const bool key = k < pair4;
      const int e = key ? k : k - pair4;
      *reinterpret_cast<uint32_t*>((key ? kc : vc) + Row::pairs(A.page, i0) + e * 4) =
          *reinterpret_cast<const uint32_t*>(image + (key ? 0 : Rows4Shape<D>::kImage) + w.n * Row::kCodes + e * 4);
    }
    if (P.bounds)
      write_bounds<D>(P, [&](int r, int c) { return *reinterpret_cast<const float2*>(keys + R4::at(r, 2 * c)); }, w.old + w.n, work, chunk);
    __syncthreads();
  }
}

// The part that slot `slot` stands for; n = 0: none.  count: of `n` sequences those for which f(b) holds, by the whole CTA or a warp.
template <typename Count>
__device__ __forceinline__ PagePart find_part(const PagedParams& A, int slot, Count count) {
  PagePart w;
  int part = 0;
  w.b = slot;
  w.n = 0;
  if (A.q_start) {
    // the last sequence whose first slot is not behind this one (offsets that do not rise are reported by seq_rows)
    auto first = [&](int b) { return first_slot(min(max(A.q_start[b], 0), A.rows), b, A.page_shift); };
    w.b = max(0, count([&](int b) { return first(b) <= slot; }) - 1);
    part = slot - first(w.b);
  }
  const SeqRows s = seq_rows(A, w.b);
  const int old = s.len - s.n, p = (max(old, 0) >> A.page_shift) + part;
  if (part < 0 || s.n <= 0 || old < 0) return w;
  w.e0 = max(old, p << A.page_shift);
  w.n = max(0, min(s.len, (p + 1) << A.page_shift) - w.e0);
  w.first = s.first + (w.e0 - old);
  w.old = w.e0 & (A.page - 1);
  return w;
}

// CTAs: queries first, then the slots for parts of pages: in 4 bits kv_splits CTAs each, else a warp for each kv head.  Two CTAs an SM, so
// that the rows in flight and their angles stay in registers (three: 282 us for prompts of 2048..8191 tokens where two take 230).
template <typename T, int D, bool FOUR>
__global__ void __launch_bounds__(kRowsThreads, 2) paged_rows_kernel(const __grid_constant__ AppendParams P) {
  extern __shared__ __align__(16) unsigned char smem[];
  griddep_launch();
  griddep_wait();
  const PagedParams& A = P.A;
  if ((int)blockIdx.x < P.q_blocks) {
    turn_queries<T, D>(P, blockIdx.x, reinterpret_cast<int*>(smem));
    return;
  }
  const int k = (int)blockIdx.x - P.q_blocks;
  if constexpr (FOUR) {
    const PagePart w = find_part(A, k / P.kv_splits, [&](auto f) {
      int n = 0;
      for (int base = 0; base < A.batch; base += kRowsThreads) n += __syncthreads_count(base + (int)threadIdx.x < A.batch && f(base + threadIdx.x));
      return n;
    });
    const int h0 = k % P.kv_splits * P.kv_heads;
    if (w.n > 0) append_part4<T, D>(P, w, h0, min(A.n_kv_heads, h0 + P.kv_heads), smem);
  } else {
    const int warp = k * (kRowsThreads / 32) + (threadIdx.x >> 5), slot = warp / A.n_kv_heads;
    if (slot >= P.kv_slots) return;
    const PagePart w = find_part(A, slot, [&](auto f) {
      int n = 0;
      for (int base = 0; base < A.batch; base += 32) n += __popc(__ballot_sync(~0u, base + (int)(threadIdx.x & 31) < A.batch && f(base + (threadIdx.x & 31))));
      return n;
    });
    if (w.n > 0) append_head<T, D>(P, w, warp % A.n_kv_heads);
  }
}

// ------------------------------------------------------------------------------------------------
// rows in 4 bits to bf16 pages
// ------------------------------------------------------------------------------------------------
struct ExpandParams {
  PagedParams A;                 // the 4-bit cache
  __nv_bfloat16* k_to;           // the other cache's layer
  __nv_bfloat16* v_to;
  const int32_t* to_table;       // [batch][to_width]
  int to_width, to_pages, to_page, to_shift;
  int blocks;                    // CTAs per (sequence, kv head): 64 entries each
};

// Eight channels per thread and row: a word of a key, or one of a value, which has four channels of two groups.  All of it is exact in
// bf16: 128 + n and 128 + z are such numbers, and so are their difference and its product with s.  Bound: the bf16 rows' writes.
__device__ __forceinline__ uint32_t kv4_values(uint32_t codes, uint32_t zeros, uint32_t scales) {      // pairs; zeros: 128 + z
  const uint32_t n = codes | 0x43004300u;
  const __nv_bfloat162 y = __hmul2(__hsub2(*reinterpret_cast<const __nv_bfloat162*>(&n), *reinterpret_cast<const __nv_bfloat162*>(&zeros)),
                                   *reinterpret_cast<const __nv_bfloat162*>(&scales));
  return *reinterpret_cast<const uint32_t*>(&y);
}
template <int D>
__global__ void __launch_bounds__(kRowsThreads) paged_expand_kernel(const __grid_constant__ ExpandParams P) {
  using Row = Kv4Row<D>;
  constexpr int kWords = D / 8, kRows = kRowsThreads / kWords, kSteps = 64 / kRows;
  constexpr uint32_t kLow = 0x000f000fu;
  griddep_launch();
  griddep_wait();
  const PagedParams& A = P.A;
  const int bh = blockIdx.x / P.blocks, b = bh / A.n_kv_heads, h = bh % A.n_kv_heads, first = blockIdx.x % P.blocks * 64;
  const int len = clamped_len(A, b), c = threadIdx.x % kWords, r0 = first + threadIdx.x / kWords;
  if (first >= len) return;
  // 16 entries share a page on both sides: where their codes, pairs and values start, -1 for none
  __shared__ long long codes_at[4], pairs_at[4], to_at[4];
  if (threadIdx.x < 4) {
    const int i = first + threadIdx.x * 16, col = i >> P.to_shift;
    codes_at[threadIdx.x] = to_at[threadIdx.x] = -1;
    if (i < len) {
      const int pg = col < P.to_width ? P.to_table[(long long)b * P.to_width + col] : -1, from = page_of(A, b, i), row = i & (A.page - 1);
      if ((unsigned)pg < (unsigned)P.to_pages) to_at[threadIdx.x] = ((((long long)pg * A.n_kv_heads + h) << P.to_shift) + (i & (P.to_page - 1))) * D;
      else flag_bad_table(A.status);
      const long long chunk = ((long long)from * A.n_kv_heads + h) * A.page * Row::kBytes;
      if (from >= 0) codes_at[threadIdx.x] = chunk + row * Row::kCodes;
      pairs_at[threadIdx.x] = chunk + Row::pairs(A.page, row);
    }
  }
  __syncthreads();
  // of a key: channels 8c .. 8c + 7; of a value: channels 4u .. 4u + 3 of groups g0 and g0 + 1; of the row's 16 (swizzles depend on no more)
  const int g = c / 4, u = c / (Row::kGroups / 2), g0 = 2 * (c % (Row::kGroups / 2)), in16 = (threadIdx.x / kWords) & 15;
  const unsigned char* kc = static_cast<const unsigned char*>(A.k_pool) + Row::k_piece(in16, g) + (c & 3) * 4;
  const unsigned char* kp = static_cast<const unsigned char*>(A.k_pool) + in16 * Row::kPairs + 2 * g;
  const unsigned char* vc = static_cast<const unsigned char*>(A.v_pool) + Row::v_unit(in16, g0, u);
  const unsigned char* vp = static_cast<const unsigned char*>(A.v_pool) + in16 * Row::kPairs + 2 * g0;
  uint32_t key[kSteps], key_pair[kSteps], value[kSteps], value_pairs[kSteps];
  long long to[kSteps];
#pragma unroll
  for (int k = 0; k < kSteps; ++k) {
    const int i = r0 + k * kRows, group = (i - first) >> 4;
    const long long base = to_at[group], at = codes_at[group];
    to[k] = i < len && base >= 0 ? base + in16 * D : -1;
    key[k] = key_pair[k] = value[k] = value_pairs[k] = 0;
    if (to[k] < 0 || at < 0) continue;                     // (a bad page counts as zeros)
    const long long pair_at = pairs_at[group];
    key[k] = *reinterpret_cast<const uint32_t*>(kc + at);
    key_pair[k] = *reinterpret_cast<const uint16_t*>(kp + pair_at);
    value[k] = *reinterpret_cast<const uint32_t*>(vc + at);
    value_pairs[k] = *reinterpret_cast<const uint32_t*>(vp + pair_at);
  }
#pragma unroll
  for (int k = 0; k < kSteps; ++k) {
    if (to[k] < 0) continue;
    {
      const uint32_t s = __float_as_uint(kv4_scale(key_pair[k] & 255)), s2 = __byte_perm(s, s, 0x3232), z2 = __byte_perm(key_pair[k], 0x43u, 0x4141);
      *reinterpret_cast<uint4*>(P.k_to + 8 * c + to[k]) =
          make_uint4(kv4_values(key[k] & kLow, z2, s2), kv4_values(key[k] >> 4 & kLow, z2, s2), kv4_values(key[k] >> 8 & kLow, z2, s2), kv4_values(key[k] >> 12 & kLow, z2, s2));
    }
    {
      const uint32_t s2 = __byte_perm(__float_as_uint(kv4_scale(value_pairs[k] & 255)), __float_as_uint(kv4_scale(value_pairs[k] >> 16 & 255)), 0x7632);
      const uint32_t z2 = (value_pairs[k] >> 8 & 0x00ff00ffu) | 0x43004300u;
      uint32_t y[4];                                       // channel m of group g0 | of group g0 + 1
#pragma unroll
      for (int m = 0; m < 4; ++m) y[m] = kv4_values(value[k] >> 4 * m & kLow, z2, s2);
      __nv_bfloat16* out = P.v_to + 32 * g0 + 4 * u + to[k];
      *reinterpret_cast<uint2*>(out) = make_uint2(__byte_perm(y[0], y[1], 0x5410), __byte_perm(y[2], y[3], 0x5410));
      *reinterpret_cast<uint2*>(out + 32) = make_uint2(__byte_perm(y[0], y[1], 0x7632), __byte_perm(y[2], y[3], 0x7632));
    }
  }
}

}  // namespace wkv
