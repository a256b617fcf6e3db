// New rows into the pages of a cache, with the position rotation applied on the way, and rows in 4 bits spread out to bf16 pages.
//
//   y_2i = x_2i cos - x_2i+1 sin, y_2i+1 = x_2i+1 cos + x_2i sin     (or channels i and i + dim/2), angles by position from a table
//
// Bound: HBM; a number is read once and written once.  One launch does the queries and the new entries.  A CTA takes the part of a page
// that one call fills (so that it owns the page's bounds, and all rows of a 4-bit page are written in full lines), for a few kv heads: the
// angles of its rows then come from L1 after the first.  Products are rounded one by one (no fused multiply-add), so that the result is
// the same as that of elementwise fp32 arithmetic, code for code where rows are held in 4 bits.
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
  int q_blocks, q_heads, kv_heads, kv_splits;   // CTAs for queries; heads per CTA; CTAs per page part
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
// Rotation of a unit's two pieces; `angles`: the position's row of the table.
__device__ __forceinline__ void turn_unit(Row8& a, Row8& b, const float* angles, int u, int dim, int paired) {
  const int h = dim >> 4;
  if (!angles || u >= h) return;
  if (!paired) {
    const Row8 c = load8(angles + 8 * u), s = load8(angles + (dim >> 1) + 8 * u);
#pragma unroll
    for (int i = 0; i < 8; ++i) turn(a.x[i], b.x[i], c.x[i], s.x[i]);
  } else {
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int at = 4 * (u + half * h);
      const float4 c = *reinterpret_cast<const float4*>(angles + at), s = *reinterpret_cast<const float4*>(angles + (dim >> 1) + at);
      Row8& r = half ? b : a;
      turn(r.x[0], r.x[1], c.x, s.x);
      turn(r.x[2], r.x[3], c.y, s.y);
      turn(r.x[4], r.x[5], c.z, s.z);
      turn(r.x[6], r.x[7], c.w, s.w);
    }
  }
}
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
  const float* angles = angles_of(P, r, entry);
  auto store = [&](const Rows& x, int at_head) {
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
      const int h = at_head + k * lanes;
      if (h >= h1) continue;
      Row8 a = x.a[k].row(), b = x.b[k].row();
      turn_unit(a, b, angles, u, P.rope_dim, P.paired);
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

// ---- bounds of the n keys of a page, for several heads at once: keys(head, row, pair of channels) from shared memory
// Pairs of channels as they lie there, with the largest and the least of two of them.
__device__ __forceinline__ __nv_bfloat162 pair_max(__nv_bfloat162 a, __nv_bfloat162 b) { return __hmax2(a, b); }
__device__ __forceinline__ __nv_bfloat162 pair_min(__nv_bfloat162 a, __nv_bfloat162 b) { return __hmin2(a, b); }
__device__ __forceinline__ float2 pair_floats(__nv_bfloat162 a) { return __bfloat1622float2(a); }
__device__ __forceinline__ float2 pair_max(float2 a, float2 b) { return make_float2(fmaxf(a.x, b.x), fmaxf(a.y, b.y)); }
__device__ __forceinline__ float2 pair_min(float2 a, float2 b) { return make_float2(fminf(a.x, b.x), fminf(a.y, b.y)); }
__device__ __forceinline__ float2 pair_floats(float2 a) { return a; }
template <typename T> struct PairOf { typedef __nv_bfloat162 type; };
template <> struct PairOf<float> { typedef float2 type; };

// work: [2][threads] pairs and [warps] floats.  heads: 1, 2 or 4, of which the first `valid` are written; heads * rows at most as many as one pass of the CTA takes.  A thread
// owns a pair of channels of a head over a share of the rows; the shares meet in shared memory.  One barrier; the caller's next one
// protects the keys and the work.
template <typename T, int D, typename Keys>
__device__ __forceinline__ void write_bounds(const AppendParams& P, Keys keys, int n, int heads, int valid, unsigned char* work, long long chunk) {
  typedef typename PairOf<T>::type Pair;
  constexpr int kPairs = D / 2;
  Pair* his = reinterpret_cast<Pair*>(work);
  Pair* los = his + kRowsThreads;
  float* mosts = reinterpret_cast<float*>(los + kRowsThreads);
  const int c = threadIdx.x % kPairs, of = threadIdx.x / kPairs, shares = kRowsThreads / kPairs / heads, head = of / shares, share = of % shares;
  Pair hi = keys(head, min(share, n - 1), c), lo = hi;
  for (int r = share + shares; r < n; r += shares) {
    const Pair x = keys(head, r, c);
    hi = pair_max(hi, x);
    lo = pair_min(lo, x);
  }
  his[threadIdx.x] = hi;
  los[threadIdx.x] = lo;
  float2 up = pair_floats(hi), down = pair_floats(lo);
  float most = fmaxf(fmaxf(fabsf(up.x), fabsf(up.y)), fmaxf(fabsf(down.x), fabsf(down.y)));
#pragma unroll
  for (int off = 16; off; off >>= 1) most = fmaxf(most, __shfl_xor_sync(~0u, most, off));
  if ((threadIdx.x & 31) == 0) mosts[threadIdx.x >> 5] = most;
  __syncthreads();
  if (share == 0 && head < valid) {
    for (int k = 1; k < shares; ++k) {
      hi = pair_max(hi, his[threadIdx.x + k * kPairs]);
      lo = pair_min(lo, los[threadIdx.x + k * kPairs]);
    }
    const int warps = kRowsThreads / 32 / heads;           // of the head
    most = 0.f;
    for (int k = 0; k < warps; ++k) most = fmaxf(most, mosts[head * warps + k]);
    const float scale = __fmul_rn(most, 1.f / 127.f), inv = scale >= 0x1p-100f ? __frcp_rn(scale) : 0.f;
    // outwards; what is not finite ends at the border
    up = pair_floats(hi);
    down = pair_floats(lo);
    auto above = [&](float x) { return (int)fminf(fmaxf(ceilf(__fmul_rn(x, inv)), -127.f), 127.f) & 255; };
    auto below = [&](float x) { return (int)fmaxf(fminf(floorf(__fmul_rn(x, inv)), 127.f), -127.f) & 255; };
    uint16_t* to = reinterpret_cast<uint16_t*>(P.bounds + (chunk + head) * 2 * D);
    to[c] = (uint16_t)(above(up.x) | above(up.y) << 8);
    to[kPairs + c] = (uint16_t)(below(down.x) | below(down.y) << 8);
    if (c == 0) P.bound_scale[chunk + head] = scale;
  }
}

// ---- new entries in the storage type
template <typename T, int D>
struct RowsShape {
  static constexpr int kUnits = D / 16, kSlots = kRowsThreads / kUnits, kVec = 16 / (int)sizeof(T);
  static constexpr int kStride = D + kVec;
  static constexpr int kBounds = 64 * kStride * (int)sizeof(T);         // staged keys of a page
  static constexpr int kWork = 2 * kRowsThreads * 2 * (int)sizeof(T) + 32;
};
// 4 bits: fp32 keys of a page, then the codes and pairs of its keys and values.  A group's 32 keys lie 36 floats behind the last one's:
// the threads of a row's groups read them from different banks.
template <int D>
struct Rows4Shape {
  static constexpr int kStride = D / 32 * 36;
  __device__ __forceinline__ static int at(int r, int c) { return r * kStride + c / 32 * 36 + c % 32; }
  static constexpr int kKeys = 64 * kStride * 4;
  static constexpr int kImage = 64 * Kv4Row<D>::kBytes;
};
template <typename T, int D, bool FOUR>
constexpr int rows_smem() {
  return FOUR ? Rows4Shape<D>::kKeys + 2 * Rows4Shape<D>::kImage + RowsShape<float, D>::kWork : RowsShape<T, D>::kBounds + RowsShape<T, D>::kWork;
}

struct PagePart {
  int b, first, page;          // row of the first new entry; the pool's page (-1: not looked up yet)
  int e0, n, old;              // index of the first new entry, number of new entries, entries of the page before them
};

// One row's unit of a head: read, turned and stored; keys are staged too where `rows` is given.
template <typename T, int D>
struct RowUnit {
  Piece<T> ka, kb, va, vb;
  __device__ __forceinline__ void load(const PagedParams& A, long long src, int2 at, int u) {
    ka.load(static_cast<const T*>(A.k) + src + 8 * at.x);
    kb.load(static_cast<const T*>(A.k) + src + 8 * at.y);
    va.load(static_cast<const T*>(A.v) + src + 16 * u);
    vb.load(static_cast<const T*>(A.v) + src + 16 * u + 8);
  }
  __device__ __forceinline__ void store(const AppendParams& P, long long dst, int2 at, int u, const float* angles, T* row) const {
    Row8 a = ka.row(), b = kb.row();
    turn_unit(a, b, angles, u, P.rope_dim, P.paired);
    store8(static_cast<T*>(P.A.k_pool) + dst + 8 * at.x, a);
    store8(static_cast<T*>(P.A.k_pool) + dst + 8 * at.y, b);
    va.store(static_cast<T*>(P.A.v_pool) + dst + 16 * u);
    vb.store(static_cast<T*>(P.A.v_pool) + dst + 16 * u + 8);
    if (row) {
      store8(row + 8 * at.x, a);
      store8(row + 8 * at.y, b);
    }
  }
};
// Threads are (row of the page, unit), as many heads at once as there are threads for.
template <typename T, int D>
__device__ __forceinline__ void append_part(const AppendParams& P, PagePart w, int h0, int h1, unsigned char* smem) {
  using Sh = RowsShape<T, D>;
  const PagedParams& A = P.A;
  const int u = threadIdx.x % Sh::kUnits, slot = threadIdx.x / Sh::kUnits, page = min(A.page, Sh::kSlots);
  const int at_once = Sh::kSlots / page, mine = slot & (page - 1), sub = slot / page;
  const int2 at = unit_pieces<D>(u, P.rope ? P.rope_dim : 0);
  const long long head_step = (long long)A.page * D;
  T* rows = P.bounds ? reinterpret_cast<T*>(smem) : nullptr;
  unsigned char* work = smem + Sh::kBounds;
  if (w.n <= page) {
    // the next heads' rows are read while these are turned, stored and looked over
    const bool on = mine < w.n;
    const long long src = (long long)(w.first + mine) * A.kv_stride;
    RowUnit<T, D> x0, x1;
    if (on && h0 + sub < h1) x0.load(A, src + (long long)(h0 + sub) * D, at, u);
    w.page = page_of(A, w.b, w.e0);                        // (the first rows are on their way)
    if (w.page < 0) return;
    const float* angles = on ? angles_of(P, w.first + mine, w.e0 + mine) : nullptr;
    const long long dst = row_offset(A, w.page, 0, w.e0, D) + (long long)mine * D;
    auto heads = [&](RowUnit<T, D>& x, RowUnit<T, D>& next, int hb) {
      const int h = hb + sub;
      if (on && h + at_once < h1) next.load(A, src + (long long)(h + at_once) * D, at, u);
      if (on && h < h1) x.store(P, dst + h * head_step, at, u, angles, rows ? rows + (sub * A.page + w.old + mine) * Sh::kStride : nullptr);
      if (!rows) return;
      for (int r = mine; r < w.old && h < h1; r += page) {
        const T* from = static_cast<const T*>(A.k_pool) + row_offset(A, w.page, h, r, D) + 16 * u;
        Piece<T> a, b;
        a.load(from);
        b.load(from + 8);
        a.store(rows + (sub * A.page + r) * Sh::kStride + 16 * u);
        b.store(rows + (sub * A.page + r) * Sh::kStride + 16 * u + 8);
      }
      __syncthreads();
      write_bounds<T, D>(P, [&](int s, int r, int c) { return *reinterpret_cast<const typename PairOf<T>::type*>(rows + (s * A.page + r) * Sh::kStride + 2 * c); },
                         w.old + w.n, at_once, h1 - hb, work, (long long)w.page * A.n_kv_heads + hb);
    };
    for (int hb = h0; hb < h1; hb += 2 * at_once) {
      heads(x0, x1, hb);
      if (hb + at_once < h1) heads(x1, x0, hb + at_once);
    }
    return;
  }
  // a page of more rows than threads for them: one head at a time
  w.page = page_of(A, w.b, w.e0);
  if (w.page < 0) return;
  const long long dst0 = row_offset(A, w.page, 0, w.e0, D);
  for (int h = h0; h < h1; ++h) {
    for (int r = mine; r < w.n; r += page) {
      RowUnit<T, D> x;
      x.load(A, (long long)(w.first + r) * A.kv_stride + (long long)h * D, at, u);
      x.store(P, dst0 + (long long)r * D + h * head_step, at, u, angles_of(P, w.first + r, w.e0 + r), rows ? rows + (w.old + r) * Sh::kStride : nullptr);
    }
    if (!rows) continue;
    for (int r = mine; r < w.old; r += page) {
      const T* from = static_cast<const T*>(A.k_pool) + row_offset(A, w.page, h, r, D) + 16 * u;
      Piece<T> a, b;
      a.load(from);
      b.load(from + 8);
      a.store(rows + r * Sh::kStride + 16 * u);
      b.store(rows + r * Sh::kStride + 16 * u + 8);
    }
    __syncthreads();
    write_bounds<T, D>(P, [&](int, int r, int c) { return *reinterpret_cast<const typename PairOf<T>::type*>(rows + r * Sh::kStride + 2 * c); }, w.old + w.n, 1, 1, work,
                       (long long)w.page * A.n_kv_heads + h);
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
__device__ __forceinline__ void append_part4(const AppendParams& P, PagePart w, int h0, int h1, unsigned char* smem) {
  using Sh = RowsShape<T, D>;
  using Row = Kv4Row<D>;
  using R4 = Rows4Shape<D>;
  constexpr int G = Row::kGroups;
  const PagedParams& A = P.A;
  float* keys = reinterpret_cast<float*>(smem);
  unsigned char* image = smem + Rows4Shape<D>::kKeys;      // codes [n][kCodes] and pairs [n][kPairs] of the keys, then of the values
  float* work = reinterpret_cast<float*>(smem + Rows4Shape<D>::kKeys + 2 * Rows4Shape<D>::kImage);
  const int u = threadIdx.x % Sh::kUnits, slot = threadIdx.x / Sh::kUnits;
  const int2 at = unit_pieces<D>(u, P.rope ? P.rope_dim : 0);
  const int i0 = w.e0 & (A.page - 1);
  const long long chunk_bytes = (long long)A.page * Row::kBytes;
  w.page = page_of(A, w.b, w.e0);
  if (w.page < 0) return;
  for (int h = h0; h < h1; ++h) {
    const long long chunk = (long long)w.page * A.n_kv_heads + h;
    unsigned char* kc = static_cast<unsigned char*>(A.k_pool) + chunk * chunk_bytes;
    unsigned char* vc = static_cast<unsigned char*>(A.v_pool) + chunk * chunk_bytes;
    for (int r = slot; r < w.n; r += Sh::kSlots) {
      const T* src = static_cast<const T*>(A.k) + (long long)(w.first + r) * A.kv_stride + (long long)h * D;
      Row8 a = load8(src + 8 * at.x), b = load8(src + 8 * at.y);
      turn_unit(a, b, angles_of(P, w.first + r, w.e0 + r), u, P.rope_dim, P.paired);
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
      write_bounds<float, D>(P, [&](int, int r, int c) { return *reinterpret_cast<const float2*>(keys + R4::at(r, 2 * c)); }, w.old + w.n, 1, 1,
                             reinterpret_cast<unsigned char*>(work), chunk);
    __syncthreads();
  }
}

// CTAs: queries first, then the slots for parts of pages, kv_splits CTAs each.
template <typename T, int D, bool FOUR>
__global__ void __launch_bounds__(kRowsThreads, sizeof(T) == 2 && !FOUR ? 3 : 2) paged_rows_kernel(const __grid_constant__ AppendParams P) {
  extern __shared__ __align__(16) unsigned char smem[];
  griddep_launch();
  griddep_wait();
  const PagedParams& A = P.A;
  if ((int)blockIdx.x < P.q_blocks) {
    turn_queries<T, D>(P, blockIdx.x, reinterpret_cast<int*>(smem));
    return;
  }
  const int k = blockIdx.x - P.q_blocks, slot = k / P.kv_splits, h0 = k % P.kv_splits * P.kv_heads, h1 = min(A.n_kv_heads, h0 + P.kv_heads);
  PagePart w;
  int part = 0;
  if (A.q_start) {
    // the last sequence whose first slot is not behind this one (offsets that do not rise are reported by seq_rows)
    int below = 0;
    for (int base = 0; base < A.batch; base += kRowsThreads) {
      const int b = base + threadIdx.x;
      below += __syncthreads_count(b < A.batch && first_slot(min(max(A.q_start[min(b, A.batch)], 0), A.rows), b, A.page_shift) <= slot);
    }
    w.b = max(0, below - 1);
    part = slot - first_slot(min(max(A.q_start[w.b], 0), A.rows), w.b, A.page_shift);
  } else {
    w.b = slot;
  }
  const SeqRows s = seq_rows(A, w.b);
  const int old = s.len - s.n, p = (max(old, 0) >> A.page_shift) + part;
  if (part < 0 || s.n <= 0 || old < 0) return;
  w.e0 = max(old, p << A.page_shift);
  w.n = min(s.len, (p + 1) << A.page_shift) - w.e0;
  if (w.n <= 0) return;
  w.first = s.first + (w.e0 - old);
  w.old = w.e0 & (A.page - 1);
  w.page = -1;
  if constexpr (FOUR) append_part4<T, D>(P, w, h0, h1, smem);
  else append_part<T, D>(P, w, h0, h1, smem);
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
  const long long chunk_bytes = (long long)A.page * Row::kBytes;
  // of a key: channels 8c .. 8c + 7; of a value: channels 4u .. 4u + 3 of groups g0 and g0 + 1
  const int g = c / 4, u = c / (Row::kGroups / 2), g0 = 2 * (c % (Row::kGroups / 2));
  uint32_t key[kSteps], key_pair[kSteps], value[kSteps], value_pairs[kSteps];
  long long to[kSteps];
#pragma unroll
  for (int k = 0; k < kSteps; ++k) {
    const int i = r0 + k * kRows;
    to[k] = -1;
    key[k] = key_pair[k] = value[k] = value_pairs[k] = 0;
    if (i >= len) continue;
    const int col = i >> P.to_shift, pg = col < P.to_width ? P.to_table[(long long)b * P.to_width + col] : -1, from = page_of(A, b, i);
    if ((unsigned)pg >= (unsigned)P.to_pages) {
      flag_bad_table(A.status);
      continue;
    }
    to[k] = ((((long long)pg * A.n_kv_heads + h) << P.to_shift) + (i & (P.to_page - 1))) * D;
    if (from < 0) continue;                                // counts as zeros
    const int row = i & (A.page - 1);
    const long long at = ((long long)from * A.n_kv_heads + h) * chunk_bytes;
    const unsigned char* kc = static_cast<const unsigned char*>(A.k_pool) + at;
    const unsigned char* vc = static_cast<const unsigned char*>(A.v_pool) + at;
    key[k] = *reinterpret_cast<const uint32_t*>(kc + Row::k_piece(row, g) + (c & 3) * 4);
    key_pair[k] = *reinterpret_cast<const uint16_t*>(kc + Row::pairs(A.page, row) + 2 * g);
    value[k] = *reinterpret_cast<const uint32_t*>(vc + Row::v_unit(row, g0, u));
    value_pairs[k] = *reinterpret_cast<const uint32_t*>(vc + Row::pairs(A.page, row) + 2 * g0);
  }
#pragma unroll
  for (int k = 0; k < kSteps; ++k) {
    if (to[k] < 0) continue;
    {
      const uint32_t s = __float_as_uint(kv4_scale(key_pair[k] & 255)), s2 = __byte_perm(s, s, 0x3232), z2 = __byte_perm(key_pair[k], 0x43u, 0x4141);
      *reinterpret_cast<uint4*>(P.k_to + to[k] + 8 * c) =
          make_uint4(kv4_values(key[k] & kLow, z2, s2), kv4_values(key[k] >> 4 & kLow, z2, s2), kv4_values(key[k] >> 8 & kLow, z2, s2), kv4_values(key[k] >> 12 & kLow, z2, s2));
    }
    {
      const uint32_t s2 = __byte_perm(__float_as_uint(kv4_scale(value_pairs[k] & 255)), __float_as_uint(kv4_scale(value_pairs[k] >> 16 & 255)), 0x7632);
      const uint32_t z2 = (value_pairs[k] >> 8 & 0x00ff00ffu) | 0x43004300u;
      uint32_t y[4];                                       // channel m of group g0 | of group g0 + 1
#pragma unroll
      for (int m = 0; m < 4; ++m) y[m] = kv4_values(value[k] >> 4 * m & kLow, z2, s2);
      __nv_bfloat16* out = P.v_to + to[k] + 32 * g0 + 4 * u;
      *reinterpret_cast<uint2*>(out) = make_uint2(__byte_perm(y[0], y[1], 0x5410), __byte_perm(y[2], y[3], 0x5410));
      *reinterpret_cast<uint2*>(out + 32) = make_uint2(__byte_perm(y[0], y[1], 0x7632), __byte_perm(y[2], y[3], 0x7632));
    }
  }
}

}  // namespace wkv
