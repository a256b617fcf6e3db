// Paged prompt attention on bf16 rows: chunks of new tokens of a ragged batch against their sequences' pages, under a window
// with sinks.  Same formulas as the decode step, a causal limit per token.
//
// Bound: tensor cores and exponentials, 4 D flops and one exponential per (query head, visible entry); a 128 x 128 tile of
// logits takes the SM's tensor cores 2 x 512 cycles at D = 128 and its 16 exponentials a cycle 1024 cycles, so the two have
// to overlap.
//
// An item of work is 256 rows of one kv head -- a row being (token, query head of the group), token-major: grouped heads share a
// tile, so a row tile spans 128 / G tokens and a window wastes little of it -- and a share of the key tiles that they see: all of
// them, or a run of a few tiles where there are too few row blocks to fill the GPU (chunks of a few tokens behind long contexts);
// paged_prefill_join_kernel then joins the runs.  One CTA per SM takes items from a counter until there are none: the
// copies of the next item run while the last one's outputs are written.
//
// Two row tiles of 128 take turns: while one's logits are in its softmax warps, the tensor cores work on the other's.  Warps 0-3
// and 4-7: softmax of row tile 0 and 1, a thread per row (a TMEM lane), so statistics need no shuffles; warp 8 issues all matrix
// instructions; warp 9 all copies; warp 10 fetches items; warp 11 stores the call's new rows,
// with the softmax warps' help when they have run out of items.
//
// New rows come to the tensor cores straight from the call's k and v; storing them in their pages (41 us for 8192 tokens of 32 x
// 128 by a kernel of its own) runs beside the products, whose time leaves HBM idle.  Only the page that a chunk starts in the middle
// of is read back from the pool: paged_append_edge_kernel has stored its new rows before.
// TMEM, 512 columns: logits of both tiles (fp32, 128 columns each; the weights overwrite them as bf16, 64 columns, and are the A
// operand of P.V straight from TMEM) and both outputs (D columns each).  An output is rescaled in place, and only when a row's
// maximum has grown by more than 2^8 since its reference was taken.
//
// Measured: 8192 tokens, 32 x 128 heads, 495 us = 1110 TFLOP/s in a row of up to 100 passes, 557..586 us on five GPUs in a long series
// at the power limit; a pair of tiles takes 2900..3100 cycles (tensor cores 2048): TMEM holds no third row tile that could hide the
// chain logits, softmax, weights.
#pragma once
#include "wkv_paged.cuh"
#include "wkv_paged_decode.cuh"
#include "wkv_tcgen05.cuh"

namespace wkv {

// Three warpgroups of 168 registers a thread at launch; the softmax ones hold a row of logits (128) and take what the third
// does not need: 2 * 208 + 88 = 3 * 168.
constexpr int kPrefillThreads = 384;
constexpr int kPrefillSoftmaxWarps = 8;
constexpr int kPrefillRows = 256;            // rows of an item
constexpr int kPrefillKeys = 128;            // entries per tile

struct PrefillParams {
  PagedParams A;
  int g_shift;               // log2 of the query heads per kv head
  int slots;                 // items that a call whose row blocks are cut into runs may have; 0: this call is not cut
  uint32_t* counter;         // next item, next eight new rows (zero between launches); tiles of a run
  float4* part;              // [item][D / 4][rows] outputs of runs, four channels of a row together
  float2* part_ml;           // [item][rows] (maximum in base-2 logits, sum)
  int oob_chunk, chunk0;
  int append;                // the call brings k and v, and this kernel stores what paged_append_edge_kernel has not
  uint32_t polls;            // limit of the kernels' waits; some of them last as long as an item, so it grows with the table's width
  alignas(64) unsigned char qmap[128];   // q as [part][token][head][64 elements], boxes of a row tile
  alignas(64) unsigned char kmap[128];   // pool as [chunk][part][row][64 elements], boxes of a page x one part
  alignas(64) unsigned char vmap[128];
  alignas(64) unsigned char kinmap[128]; // the call's k and v as [part][token][head][64 elements], boxes of one head's `page` tokens
  alignas(64) unsigned char vinmap[128];
};

template <int D>
struct PrefillShape {
  static constexpr int kParts = D / 64;
  static constexpr int kPartBytes = 128 * 128;                    // 128 rows x 128 bytes
  static constexpr int kTileBytes = kParts * kPartBytes;          // of Q (one row tile), K or V
  static constexpr int kStages = D == 128 ? 5 : 8;
  static constexpr int kSmem = 2 * kTileBytes + kStages * kTileBytes + (2 * kStages + 17) * 8 + 16 + 2 * 64;
};

__device__ __forceinline__ void tensor_g2s_4d(void* dst, const void* tmap, int x, int y, int z, int w, uint64_t* bar) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(
                   smem_u32(dst)),
               "l"(tmap), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_u32(bar))
               : "memory");
}

// A row block: which sequence, which rows, and the entries it walks -- the pages with sinks, then those from the page of the first
// row's window on, end to end: tile v holds the 128 of them from 128 v on, so neither a few sinks nor a window's start in the
// middle of nowhere takes a tile of its own.
struct PrefillBlock {
  int b, head, first, n, len, old;      // old: entries before the chunk
  int row0;                             // first row (token * G + g) of the block
  int sink_rows, start, entries;        // sink_rows, start: multiples of the page; entries walked
  __device__ __forceinline__ int entry(int i) const { return i < sink_rows ? i : i - sink_rows + start; }
};
// Positions of a row tile's first and last token; none if it has no rows.
struct RowTile {
  bool any;
  int pos_lo, pos_hi;
};
__device__ __forceinline__ RowTile row_tile(const PrefillBlock& B, int row0, int g_shift) {
  RowTile t;
  t.any = row0 < B.n << g_shift;
  t.pos_lo = B.old + (row0 >> g_shift);
  t.pos_hi = min(B.old + ((row0 + 127) >> g_shift), B.len - 1);
  return t;
}
// Does any row of the row tile see an entry of tile v?
__device__ __forceinline__ bool tile_seen(const PrefillBlock& B, const RowTile& t, int v, int window, int sink) {
  const int at = v * kPrefillKeys;
  if (!t.any) return false;
  if (at < B.sink_rows) return true;
  const int e0 = B.entry(at);
  return e0 <= t.pos_hi && (window == 0 || e0 + kPrefillKeys > t.pos_lo - window + 1 || e0 < sink);
}
// Does every row see all of it?
__device__ __forceinline__ bool tile_whole(const PrefillBlock& B, const RowTile& t, int v, int window, int sink) {
  const int at = v * kPrefillKeys;
  if (at < B.sink_rows) return at + kPrefillKeys <= min(sink, B.sink_rows);
  const int e0 = B.entry(at);
  return e0 + kPrefillKeys - 1 <= t.pos_lo && (window == 0 || e0 >= t.pos_hi - window + 1 || e0 + kPrefillKeys <= sink);
}

// How a call's work is cut: row blocks of ROWS rows, and where there are too few of them to fill the GPU, their key tiles (KEYS
// entries) into runs of `run` tiles, so that no more than `slots` items come out: a sequence whose row blocks walk t tiles has
// ceil(t / run) <= t / run + 1 runs each.  Every warp computes it from the lengths, so that a captured call follows new ones, and a
// ragged batch's short sequences are not cut as finely as its longest.
struct WorkPlan {
  int run;                   // tiles of a run; the largest int where nothing is cut
  int items;                 // (row block, run, kv head)
};
// Row blocks of sequence b (0 behind the last), and the tiles that one walks at most.
template <int ROWS, int KEYS>
__device__ __forceinline__ void sequence_work(const PagedParams& A, int g_shift, int b, int& blocks, int& tiles) {
  blocks = tiles = 0;
  if (b >= A.batch) return;
  const int lo = min(max(A.q_start[b], 0), A.rows), hi = min(max(A.q_start[b + 1], lo), A.rows);
  blocks = (int)((((long long)(hi - lo) << g_shift) + ROWS - 1) / ROWS);
  const long long len = clamped_len(A, b), walked = A.window > 0 ? min(len, (long long)A.window + A.sink + ROWS + 2 * A.page) : len;
  tiles = (int)((walked + KEYS - 1) / KEYS);
}
__device__ __forceinline__ int runs_of(int tiles, int run) { return tiles <= run ? 1 : (tiles + run - 1) / run; }

template <int ROWS, int KEYS>
__device__ __forceinline__ WorkPlan work_plan(const PagedParams& A, int g_shift, int slots) {
  const int lane = threadIdx.x & 31;
  WorkPlan w{0x7fffffff, 0};
#pragma unroll 1
  for (int pass = 0; pass < 2; ++pass) {
    long long units = 0, all = 0;                      // row blocks; their tiles, then their runs
    for (int b = lane; b < A.batch; b += 32) {
      int blocks, tiles;
      sequence_work<ROWS, KEYS>(A, g_shift, b, blocks, tiles);
      units += blocks;
      all += (long long)blocks * (pass == 0 ? tiles : runs_of(tiles, w.run));
    }
#pragma unroll
    for (int off = 16; off; off >>= 1) {
      units += __shfl_xor_sync(~0u, units, off);
      all += __shfl_xor_sync(~0u, all, off);
    }
    w.items = (int)((pass == 0 ? units : all) * A.n_kv_heads);
    if (pass == 1) break;
    const long long more = (long long)slots - w.items;
    if (w.items == 0 || more < w.items) break;         // nothing to do, or row blocks enough
    w.run = (int)max(KEYS < 64 ? 2LL : 4LL, (all * A.n_kv_heads + more - 1) / more);
  }
  return w;
}

// Item x of one kv head's -- or, UNIT, the first item of row block x: row block, run r of its `runs`, and that first item's number;
// false if there is none.  Every warp searches for itself.
template <int ROWS, int KEYS, bool UNIT>
__device__ __forceinline__ bool find_item(const PagedParams& A, int g_shift, int run, int x, int head, PrefillBlock& B, int& r, int& runs, int& first_item) {
  const int lane = threadIdx.x & 31;
  int before = 0, items = 0;                           // what x counts, and items, of the sequences before
  for (int base = 0; base < A.batch; base += 32) {
    int blocks, tiles;
    sequence_work<ROWS, KEYS>(A, g_shift, base + lane, blocks, tiles);
    const int n = runs_of(tiles, run), mine = UNIT ? blocks : blocks * n;
    int upto = mine, upto_items = blocks * n;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int y = __shfl_up_sync(~0u, upto, off), z = __shfl_up_sync(~0u, upto_items, off);
      if (lane >= off) { upto += y; upto_items += z; }
    }
    const uint32_t behind = __ballot_sync(~0u, x < before + upto);
    if (behind) {
      const int at = __ffs(behind) - 1;
      const int all = __shfl_sync(~0u, blocks, at), y = x - before - __shfl_sync(~0u, upto - mine, at);
      runs = __shfl_sync(~0u, n, at);
      r = UNIT ? 0 : y % runs;
      const int block = UNIT ? y : y / runs;
      first_item = items + __shfl_sync(~0u, upto_items - blocks * n, at) + block * runs;
      const SeqRows s = seq_rows(A, base + at);
      B.b = base + at; B.head = head; B.first = s.first; B.n = s.n; B.len = s.len; B.old = s.len - s.n;
      B.row0 = (all - 1 - block) * ROWS;               // a sequence's last rows see most: they start first
      const int p0 = B.old + (B.row0 >> g_shift);                              // positions of the block's tokens
      const int p1 = min(B.old + ((B.row0 + ROWS - 1) >> g_shift), B.len - 1);
      const int lo_key = A.window > 0 ? max(0, p0 - A.window + 1) : 0;
      B.start = lo_key & ~(A.page - 1);
      B.sink_rows = (min(A.sink, B.start) + A.page - 1) & ~(A.page - 1);
      B.entries = p1 < 0 ? 0 : B.sink_rows + p1 + 1 - B.start;
      return true;
    }
    before += __shfl_sync(~0u, upto, 31);
    items += __shfl_sync(~0u, upto_items, 31);
  }
  return false;
}
// Run r of a row block: its tiles [v0, v1); false if it has none, but for the first run.
template <int KEYS>
__device__ __forceinline__ bool run_of(const PrefillBlock& B, int r, int runs, int run, int& v0, int& v1) {
  const int tiles = (B.entries + KEYS - 1) / KEYS;
  v0 = (int)min((long long)tiles, (long long)r * run);
  v1 = r == runs - 1 ? tiles : (int)min((long long)tiles, (long long)(r + 1) * run);
  return r == 0 || v0 < v1;
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t fma2_(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t pair(float lo, float hi) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
  return d;
}
__device__ __forceinline__ void unpair(uint64_t d, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(d)); }

// What warp 10 tells the others about an item.
struct PrefillItem {
  PrefillBlock B;
  int v0, v1;                // its key tiles
  int slot;                  // -1: no more items
  int whole;                 // not a run: the output is final
};
static_assert(sizeof(PrefillItem) <= 64, "two of them in 128 bytes of shared memory");

// Visible columns of a 32-column piece as bits: columns 0..top, of these low.. and those below sinks.
__device__ __forceinline__ uint32_t low_bits(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1; }

// Eight lanes with 128 bytes of a row each, in 16-byte pieces: lane i gets piece i of all eight rows.  Stored piece by piece, every
// lane its own row, a row tile's output took 6900 cycles (32 lines a store); now a store writes four rows' full lines.
__device__ __forceinline__ void exchange_pieces(uint32_t (&y)[8][4]) {
#pragma unroll
  for (int s = 1; s < 8; s <<= 1) {
    const bool up = threadIdx.x & s;
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      if (p & s) continue;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint32_t got = __shfl_xor_sync(~0u, up ? y[p][w] : y[p | s][w], s);
        if (up) y[p][w] = got; else y[p | s][w] = got;
      }
    }
  }
}

// New rows into their pages, by one warp of several on every CTA (`takers`): eight tokens at a time from a counter, looked up
// together, then copied one after the other.
template <int D>
__device__ __forceinline__ void append_rows(const PrefillParams& P, int takers) {
  const int lane = threadIdx.x & 31;
  const uint32_t chunks = (uint32_t)(P.A.rows + 7) / 8;
  for (;;) {
    uint32_t w = 0;
    if (lane == 0) w = atomicAdd(P.counter + 1, 1u);
    w = __shfl_sync(~0u, w, 0);
    if (w >= chunks) {
      if (lane == 0 && w == chunks + (uint32_t)takers * gridDim.x - 1) P.counter[1] = 0;      // the last one to ask
      return;
    }
    const int r0 = (int)w * 8;
    const NewRow mine = new_row(P.A, r0 + (lane & 7), true);
#pragma unroll 1
    for (int j = 0; j < 8; ++j) {
      const NewRow row{__shfl_sync(~0u, mine.page, j), __shfl_sync(~0u, mine.entry, j)};
      append_row<__nv_bfloat16, D, 32, 8>(P.A, r0 + j, row, lane);
    }
  }
}

template <int D>
__global__ void __launch_bounds__(kPrefillThreads, 1) paged_prefill_kernel(const __grid_constant__ PrefillParams P) {
  using Sh = PrefillShape<D>;
  constexpr int STAGES = Sh::kStages;
  extern __shared__ __align__(1024) unsigned char sq[];               // Q, then the ring: there is no room to align by hand
  unsigned char* ring = sq + 2 * Sh::kTileBytes;
  uint64_t* full = reinterpret_cast<uint64_t*>(ring + STAGES * Sh::kTileBytes);
  uint64_t* empty = full + STAGES;
  uint64_t* q_full = empty + STAGES;
  uint64_t* q_free = q_full + 1;       // the item's last logits are done
  uint64_t* s_full = q_free + 1;       // [2] logits of a row tile are in TMEM (and its last P.V is done)
  uint64_t* p_ready = s_full + 2;      // [2][2] a half of the weights is in TMEM, the output is rescaled
  uint64_t* o_full = p_ready + 4;      // [2] the item's products of a row tile are done
  uint64_t* o_free = o_full + 2;       // [2] a row tile's output has been read
  uint64_t* item_full = o_free + 2;    // [2]
  uint64_t* item_empty = item_full + 2;
  uint64_t* drained = item_empty + 2;  // all matrix instructions are done
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drained + 1);
  unsigned char* item_smem = reinterpret_cast<unsigned char*>(tmem_slot + 4);

  const PagedParams& A = P.A;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, G = 1 << P.g_shift;
  if (tid == 0) {
    for (int i = 0; i < STAGES; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], 1); }
    mbar_init(q_full, 1);
    mbar_init(q_free, 1);
    mbar_init(drained, 1);
    for (int t = 0; t < 2; ++t) {
      mbar_init(&o_full[t], 1);
      mbar_init(&s_full[t], 1); mbar_init(&p_ready[2 * t], 4); mbar_init(&p_ready[2 * t + 1], 4); mbar_init(&o_free[t], 4);
      mbar_init(&item_full[t], 1); mbar_init(&item_empty[t], 10);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 8) tmem_take(tmem_slot);
  tcgen05_before_sync();
  griddep_wait();
  __syncthreads();
  tcgen05_after_sync();
  // behind the allocation: a kernel that starts early and takes TMEM here first would keep it until this one ends
  griddep_launch();
  const uint32_t tmem = __shfl_sync(~0u, *tmem_slot, 0);

  // A warp's work is a lambda that returns early where a wait gives up.
  const WaitLimit waits{A.status, P.polls};
  // the n-th item of this CTA for a warp, once it is there; every reader tells when it has its copy.  false: there are no more.
  auto take_item = [&](int n, PrefillItem& item) {
    if (!warp_wait(&item_full[n & 1], (n >> 1) & 1, waits)) return false;
    item = *reinterpret_cast<const PrefillItem*>(item_smem + (n & 1) * 64);
    __syncwarp();
    if (lane == 0) mbar_arrive(&item_empty[n & 1]);
    return item.slot >= 0;
  };

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    if (warp == 10) {
      // ---- items
      const WorkPlan plan = work_plan<kPrefillRows, kPrefillKeys>(A, P.g_shift, P.slots);
      if (blockIdx.x == 0 && lane == 0) P.counter[2] = (uint32_t)plan.run;       // for the join
      for (int n = 0;; ++n) {
        PrefillItem item;
        item.slot = -1;
        for (;;) {
          uint32_t w = 0;
          if (lane == 0) w = atomicAdd(P.counter, 1u);
          w = __shfl_sync(~0u, w, 0);
          if (w >= (uint32_t)plan.items) {
            if (lane == 0 && w == (uint32_t)plan.items + gridDim.x - 1) *P.counter = 0;      // the last CTA to ask
            break;
          }
          int r, runs, first_item;
          if (!find_item<kPrefillRows, kPrefillKeys, false>(A, P.g_shift, plan.run, w / A.n_kv_heads, w % A.n_kv_heads, item.B, r, runs, first_item) ||
              !run_of<kPrefillKeys>(item.B, r, runs, plan.run, item.v0, item.v1))
            continue;
          item.whole = plan.run == 0x7fffffff;
          item.slot = (int)w;
          break;
        }
        if (n >= 2 && !warp_wait(&item_empty[n & 1], ((n >> 1) & 1) ^ 1, waits)) break;
        if (lane == 0) {
          *reinterpret_cast<PrefillItem*>(item_smem + (n & 1) * 64) = item;
          mbar_arrive(&item_full[n & 1]);
        }
        __syncwarp();
        if (item.slot < 0) break;
      }
    } else if (warp == 9) {
      // ---- copies
      const int pr = A.page, boxes = kPrefillKeys >> A.page_shift;
      const bool mine = lane < boxes * Sh::kParts;
      const int box = lane & (boxes - 1), part = mine ? lane / boxes : 0;
      fence_proxy_async();                                     // rows that the append kernel stored
      int it = 0, q_fills = 0;                                 // copies issued: ring stages, row blocks
      [&] {
        for (int n = 0;; ++n) {
          PrefillItem item;
          if (!take_item(n, item)) return;
          const PrefillBlock& B = item.B;
          if (n > 0 && !warp_wait(q_free, (n & 1) ^ 1, waits)) return;
          ++q_fills;
          if (lane == 0) {
            const int tiles = B.row0 + 128 < B.n << P.g_shift ? 2 : 1;
            mbar_expect_tx(q_full, tiles * Sh::kTileBytes);
            for (int t = 0; t < tiles; ++t)
              for (int p = 0; p < Sh::kParts; ++p)
                tensor_g2s_4d(sq + t * Sh::kTileBytes + p * Sh::kPartBytes, P.qmap, 0, B.head * G, B.first + ((B.row0 + t * 128) >> P.g_shift), p, q_full);
          }
          __syncwarp();
          for (int v = item.v0; v < item.v1; ++v) {
            const int i = B.entry(v * kPrefillKeys + box * pr);
            const int pg = mine && i < B.len ? page_of(A, B.b, i) : -1;
            const bool fresh = P.append && i >= B.old && pg >= 0;      // a box of the call's own rows (tokens behind the chunk: never used)
            const int chunk = pg >= 0 ? P.chunk0 + pg * A.n_kv_heads + B.head : P.oob_chunk;
#pragma unroll
            for (int kv = 0; kv < 2; ++kv, ++it) {
              const int st = it % STAGES;
              if (it >= STAGES && !warp_wait(&empty[st], ((it / STAGES) & 1) ^ 1, waits)) return;
              if (lane == 0) mbar_expect_tx(&full[st], Sh::kTileBytes);
              __syncwarp();
              unsigned char* dst = ring + st * Sh::kTileBytes + part * Sh::kPartBytes + box * pr * 128;
              if (mine && fresh) tensor_g2s_4d(dst, kv ? P.vinmap : P.kinmap, 0, B.head, B.first + i - B.old, part, &full[st]);
              else if (mine) tensor_g2s_4d(dst, kv ? P.vmap : P.kmap, 0, 0, part, chunk, &full[st]);
            }
          }
        }
      }();
      // they land before the CTA ends, whoever gave up
      bool landed = q_fills == 0 || drain_wait(q_full, (q_fills & 1) ^ 1, A.status);
      for (int f = max(0, it - STAGES); f < it && landed; ++f) landed = drain_wait(&full[f % STAGES], (f / STAGES) & 1, A.status);
    } else if (warp == 11) {
      // ---- the call's new rows into their pages
      if (P.append) append_rows<D>(P, 1 + kPrefillSoftmaxWarps);
    } else if (warp == 8) {
      // ---- matrix instructions, all by one elected thread
      if (elect_one()) {
        const uint32_t s_at[2] = {tmem, tmem + 128}, o_at[2] = {tmem + 256, tmem + 256 + D};
        const uint64_t q_at[2] = {smem_matrix(smem_u32(sq), 16), smem_matrix(smem_u32(sq + Sh::kTileBytes), 16)};
        const uint64_t k_ring = smem_matrix(smem_u32(ring), 16), v_ring = smem_matrix(smem_u32(ring), Sh::kPartBytes);
        uint32_t p_phase[2] = {0, 0};
        int it = 0;
        [&] {
          for (int n = 0;; ++n) {
            PrefillItem item;
            if (!thread_wait(&item_full[n & 1], (n >> 1) & 1, waits)) return;
            item = *reinterpret_cast<const PrefillItem*>(item_smem + (n & 1) * 64);
            mbar_arrive(&item_empty[n & 1]);
            if (item.slot < 0) return;
            const PrefillBlock& B = item.B;
            const RowTile rt[2] = {row_tile(B, B.row0, P.g_shift), row_tile(B, B.row0 + 128, P.g_shift)};
            bool pending[2] = {false, false}, started[2] = {false, false};
            uint64_t vd = 0;                                        // values of the tile before
            auto weights_times_values = [&](int t) {
              if (!started[t] && n > 0 && !thread_wait(&o_free[t], (n & 1) ^ 1, waits)) return false;
#pragma unroll
              for (int half = 0; half < 2; ++half) {
                if (!thread_wait(&p_ready[2 * t + half], p_phase[t], waits)) return false;
                tcgen05_after_sync();
#pragma unroll
                for (int k = half * 4; k < half * 4 + 4; ++k) mma_tmem(o_at[t], s_at[t] + k * 8, vd + k * 128, mma_shape(D, true), started[t] || k > 0);
              }
              p_phase[t] ^= 1;
              started[t] = true;
              pending[t] = false;
              return true;
            };
            if (!thread_wait(q_full, n & 1, waits)) return;
            for (int v = item.v0; v < item.v1; ++v, it += 2) {
              const int st = it % STAGES;
              const uint64_t kd = k_ring + (uint32_t)(st * (Sh::kTileBytes >> 4));
              // both copies ahead of the weights, so that P.V and the next logits of a row tile are issued in one go
              if (!thread_wait(&full[st], (it / STAGES) & 1, waits)) return;
              if (v > item.v0 && !thread_wait(&full[(it - 1) % STAGES], ((it - 1) / STAGES) & 1, waits)) return;
#pragma unroll
              for (int t = 0; t < 2; ++t) {
                if (pending[t] && !weights_times_values(t)) return;
                if (!tile_seen(B, rt[t], v, A.window, A.sink)) continue;
                tcgen05_after_sync();
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                  constexpr int kPart = Sh::kPartBytes >> 4;
                  mma_smem(s_at[t], q_at[t] + (k >> 2) * kPart + (k & 3) * 2, kd + (k >> 2) * kPart + (k & 3) * 2, mma_shape(kPrefillKeys, false), k > 0);
                }
                tcgen05_commit(&s_full[t]);
                pending[t] = true;
              }
              tcgen05_commit(&empty[st]);
              if (v > item.v0) tcgen05_commit(&empty[(it - 1) % STAGES]);
              vd = v_ring + (uint32_t)(((it + 1) % STAGES) * (Sh::kTileBytes >> 4));
            }
            tcgen05_commit(q_free);
            bool told = false;
            if (item.v1 > item.v0) {
              if (!thread_wait(&full[(it - 1) % STAGES], ((it - 1) / STAGES) & 1, waits)) return;
#pragma unroll
              for (int t = 0; t < 2; ++t)
                if (pending[t]) {
                  if (!weights_times_values(t)) return;
                  if (t == 0) tcgen05_commit(&o_full[0]);        // its rows need not wait for the other row tile
                  told = told || t == 0;
                }
              tcgen05_commit(&empty[(it - 1) % STAGES]);
            }
            // a row tile without products in this item: its readers' word on the last item is still due
            for (int t = 0; t < 2; ++t)
              if (!started[t] && n > 0 && !thread_wait(&o_free[t], (n & 1) ^ 1, waits)) return;
            if (!told) tcgen05_commit(&o_full[0]);
            tcgen05_commit(&o_full[1]);
          }
        }();
        // nothing is in flight when the CTA ends
        tcgen05_commit(drained);
        drain_wait(drained, 0, A.status);
      }
      __syncwarp();
    }
  } else {
    // ---- softmax: this thread's row
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    const int t = warp >> 2, row = tid & 127;
    const uint32_t lanes = (uint32_t)(warp & 3) << 21;          // 32 TMEM lanes per warp, lane number in bits 16..
    const uint32_t s_at = tmem + lanes + t * 128, o_at = tmem + lanes + 256 + t * D;
    const float c = A.scale_log2;
    uint32_t phase = 0;
    int it = 1;                                                 // ring position of the item's first values
    [&] {
      for (int n = 0;; ++n) {
        PrefillItem item;
        if (!take_item(n, item)) return;
        const PrefillBlock& B = item.B;
        const int R = B.row0 + t * 128 + row;
        const RowTile my = row_tile(B, B.row0 + t * 128, P.g_shift);
        const int pos = B.old + (R >> P.g_shift);
        const bool live = R < B.n << P.g_shift;
        const int lo_key = A.window > 0 ? max(0, pos - A.window + 1) : 0;
        float m = -INFINITY, l = 0.f;                             // m: reference of the exponentials, in logits
        bool first = true;
        for (int v = item.v0; v < item.v1; ++v) {
          const int v_at = v * kPrefillKeys;
          if (!tile_seen(B, my, v, A.window, A.sink)) continue;
          if (!warp_wait(&s_full[t], phase, waits)) return;
          phase ^= 1;
          tcgen05_after_sync();
          uint32_t x[128];
#pragma unroll
          for (int i = 0; i < 4; ++i) tmem_load32(s_at + i * 32, x + i * 32);
          tmem_wait_loads();
          // a tile that every row of the row tile sees whole needs no mask
          if (!tile_whole(B, my, v, A.window, A.sink)) {
#pragma unroll
            for (int h = 0; h < 4; ++h) {
              const int at = v_at + h * 32, e0 = at - B.sink_rows + B.start;      // of the entries behind the sinks' pages
              uint32_t see = low_bits(pos + 1 - e0) & (~low_bits(lo_key - e0) | low_bits(A.sink - e0));
              if (at < B.sink_rows) {
                const uint32_t front = low_bits(B.sink_rows - at);
                see = (front & low_bits(min(A.sink, pos + 1) - at)) | (~front & see);
              }
#pragma unroll
              for (int i = 0; i < 32; ++i)
                if (!(see >> i & 1)) x[h * 32 + i] = 0xff800000u;
            }
          }
          float mx4[4];                                           // four chains: the latency of one would show
#pragma unroll
          for (int i = 0; i < 4; ++i) mx4[i] = max3(__uint_as_float(x[i]), __uint_as_float(x[4 + i]), __uint_as_float(x[8 + i]));
#pragma unroll
          for (int i = 12; i < 124; i += 8)
#pragma unroll
            for (int e = 0; e < 4; ++e) mx4[e] = max3(mx4[e], __uint_as_float(x[i + e]), __uint_as_float(x[i + 4 + e]));
#pragma unroll
          for (int e = 0; e < 4; ++e) mx4[e] = fmaxf(mx4[e], __uint_as_float(x[124 + e]));
          const float mx = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3]));
          if (first) {
            m = mx;
            first = false;
          } else {
            const bool grow = (mx - m) * c > 8.f;                 // true too where m is still -infinity and mx is not
            if (__any_sync(~0u, grow)) {
              const float f = grow ? exp2_fast((m - mx) * c) : 1.f;
              if (grow) m = mx;
              l *= f;
#pragma unroll
              for (int i = 0; i < D / 16; ++i) {
                uint32_t o[16];
                tmem_load16(o_at + i * 16, o);
                tmem_wait_loads();
#pragma unroll
                for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                tmem_store16(o_at + i * 16, o);
              }
            }
          }
          const int v_len = B.len - B.start + B.sink_rows;          // where the sequence ends
          if (v_at + kPrefillKeys > v_len) {
            // rows behind the sequence may hold anything: their weights are zero, their values have to be finite
            const int at = it + 2 * (v - item.v0), st = at % STAGES;
            if (!warp_wait(&full[st], (at / STAGES) & 1, waits)) return;
            for (int e = row + (v_len - v_at) * 8 * Sh::kParts; e < kPrefillKeys * 8 * Sh::kParts; e += 128) {
              const int r = e / (8 * Sh::kParts), piece = e % (8 * Sh::kParts);
              *reinterpret_cast<uint4*>(ring + st * Sh::kTileBytes + (piece >> 3) * Sh::kPartBytes + r * 128 + (piece & 7) * 16) = make_uint4(0, 0, 0, 0);
            }
            fence_proxy_async();
          }
          const float shift = m == -INFINITY ? 0.f : -m * c;
          const uint64_t c2 = pair(c, c), shift2 = pair(shift, shift);
          uint64_t sum2[4] = {0, 0, 0, 0};
#pragma unroll
          for (int h = 0; h < 4; ++h) {
            uint32_t w[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              // The sum takes the weights in fp32, the products as bf16, half a step (2^-8 of each weight) off at random: the output's
              // relative error against 64 bits is 0.0020..0.0023, where rounding the output alone gives 0.0016.  A second product with
              // the low halves, as in the decode step, would add half as many matrix flops again to a kernel that they bound.
              float p0, p1;
              unpair(fma2_(pair(__uint_as_float(x[h * 32 + 2 * i]), __uint_as_float(x[h * 32 + 2 * i + 1])), c2, shift2), p0, p1);
              p0 = exp2_fast(p0);
              p1 = exp2_fast(p1);
              sum2[i & 3] = add2(sum2[i & 3], pair(p0, p1));
              w[i] = pack_bf16(p0, p1);
            }
            tmem_store16(s_at + h * 16, w);
            if (h & 1) {                                          // half of the weights: its products may start
              tmem_wait_stores();
              tcgen05_before_sync();
              __syncwarp();
              if (lane == 0) mbar_arrive(&p_ready[2 * t + (h >> 1)]);
            }
          }
          float a0, a1;
          unpair(add2(add2(sum2[0], sum2[1]), add2(sum2[2], sum2[3])), a0, a1);
          l += a0 + a1;
        }
        it += 2 * (item.v1 - item.v0);
        // ---- output
        if (!warp_wait(&o_full[t], n & 1, waits)) return;
        tcgen05_after_sync();
        const bool seen = !(l <= 0.f);                            // else the row's TMEM lane may hold anything
        const float inv = seen ? 1.f / l : 0.f;
        // rows of the eight lanes that exchange pieces, and this lane's 16-byte piece of 128
        const int row8 = t * 128 + (row & ~7), piece = lane & 7;
        if (item.whole) {
#pragma unroll 1
          for (int i = 0; i < D / 64; ++i) {
            uint32_t o[64], y[8][4];
            tmem_load32(o_at + i * 64, o);
            tmem_load32(o_at + i * 64 + 32, o + 32);
            tmem_wait_loads();
#pragma unroll
            for (int e = 0; e < 32; ++e)
              y[e >> 2][e & 3] = seen ? pack_bf16(__uint_as_float(o[2 * e]) * inv, __uint_as_float(o[2 * e + 1]) * inv) : 0u;
            exchange_pieces(y);
#pragma unroll
            for (int r = 0; r < 8; ++r) {
              const int Rr = B.row0 + row8 + r, tok = Rr >> P.g_shift;
              if (tok >= B.n) break;
              __nv_bfloat16* out = static_cast<__nv_bfloat16*>(A.out) + ((long long)(B.first + tok) * A.n_q_heads + B.head * G + (Rr & (G - 1))) * D + i * 64;
              reinterpret_cast<uint4*>(out)[piece] = make_uint4(y[r][0], y[r][1], y[r][2], y[r][3]);
            }
          }
          if (live && A.lse) {
            const long long at = (long long)(B.first + (R >> P.g_shift)) * A.n_q_heads + B.head * G + (R & (G - 1));
            A.lse[at] = seen ? (m * c + log2f(l)) * kLn2 : -INFINITY;
          }
        } else {
          // a warp's store covers 32 rows' same four channels, which lie side by side
          float4* part = P.part + (long long)item.slot * (D / 4) * kPrefillRows + t * 128 + row;
#pragma unroll 1
          for (int i = 0; i < D / 32; ++i) {
            uint32_t o[32];
            tmem_load32(o_at + i * 32, o);
            tmem_wait_loads();
            if (live && seen) {
#pragma unroll
              for (int e = 0; e < 8; ++e)
                part[(i * 8 + e) * kPrefillRows] = make_float4(__uint_as_float(o[4 * e]), __uint_as_float(o[4 * e + 1]), __uint_as_float(o[4 * e + 2]),
                                                               __uint_as_float(o[4 * e + 3]));
            }
          }
          if (live) P.part_ml[(long long)item.slot * kPrefillRows + t * 128 + row] = make_float2(seen ? m * c : -INFINITY, seen ? l : 0.f);
        }
        tcgen05_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(&o_free[t]);
      }
    }();
    if (P.append) append_rows<D>(P, 1 + kPrefillSoftmaxWarps);     // what warp 11 has not come to
  }
  tcgen05_before_sync();
  __syncthreads();
  if (warp == 8) {
    tcgen05_after_sync();
    tmem_give_back(tmem);
  }
}

// The runs of a row block (ROWS rows) joined: 32 rows per CTA, eight threads per row, a warp on the same channels of all of them.
// The grid is an upper bound; a call that was not cut leaves nothing to do.
template <typename T, int D, int ROWS, int KEYS>
__global__ void __launch_bounds__(256) paged_prefill_join_kernel(const __grid_constant__ PrefillParams P) {
  griddep_launch();
  griddep_wait();
  const PagedParams& A = P.A;
  const int unit = blockIdx.x / (ROWS / 32), G = 1 << P.g_shift, head = unit % A.n_kv_heads;
  const int run = (int)P.counter[2];
  if (run == 0x7fffffff) return;
  PrefillBlock B;
  int r, runs, first_item;
  if (!find_item<ROWS, KEYS, true>(A, P.g_shift, run, unit / A.n_kv_heads, head, B, r, runs, first_item)) return;
  const int row = blockIdx.x % (ROWS / 32) * 32 + (threadIdx.x & 31), R = B.row0 + row, c0 = threadIdx.x >> 5;
  if (R >= B.n << P.g_shift) return;
  int there = 1, v0, v1;                                          // runs that have tiles
  while (there < runs && run_of<KEYS>(B, there, runs, run, v0, v1)) ++there;
  auto slot = [&](int s) { return (long long)(first_item + s) * A.n_kv_heads + head; };
  float m = -INFINITY;
  for (int s = 0; s < there; ++s) m = fmaxf(m, P.part_ml[slot(s) * ROWS + row].x);
  constexpr int V = D / 32;                                       // float4s per thread
  float4 acc[V] = {};
  float l = 0.f;
  for (int s = 0; s < there; ++s) {
    const float2 ml = P.part_ml[slot(s) * ROWS + row];
    if (ml.x == -INFINITY) continue;                              // a run that the row sees nothing of wrote no output
    const float f = exp2_fast(ml.x - m);
    l = fmaf(ml.y, f, l);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float4 x4 = P.part[(slot(s) * (D / 4) + i * 8 + c0) * ROWS + row];
      acc[i].x = fmaf(x4.x, f, acc[i].x); acc[i].y = fmaf(x4.y, f, acc[i].y); acc[i].z = fmaf(x4.z, f, acc[i].z); acc[i].w = fmaf(x4.w, f, acc[i].w);
    }
  }
  const bool seen = !(l <= 0.f);
  const float inv = seen ? 1.f / l : 0.f;
  const long long tok = B.first + (R >> P.g_shift), hq = B.head * G + (R & (G - 1));
  T* out = static_cast<T*>(A.out) + (tok * A.n_q_heads + hq) * D;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const float4 y = make_float4(acc[i].x * inv, acc[i].y * inv, acc[i].z * inv, acc[i].w * inv);
    if constexpr (sizeof(T) == 2) reinterpret_cast<uint2*>(out)[i * 8 + c0] = make_uint2(pack_bf16(y.x, y.y), pack_bf16(y.z, y.w));
    else reinterpret_cast<float4*>(out)[i * 8 + c0] = y;
  }
  if (A.lse && c0 == 0) A.lse[tok * A.n_q_heads + hq] = seen ? (m + log2f(l)) * kLn2 : -INFINITY;
}

// ------------------------------------------------------------------------------------------------
// accumulated weights of a prompt on bf16 rows
// ------------------------------------------------------------------------------------------------
// scores[i] += 1/G sum over the call's tokens t that see i and the group's heads g of exp(scale q_tg.k_i - lse_tg): column sums of the
// attention matrix, which needs the finished log-sums and so a second pass over the logits.  The transposed product K Q^T puts an
// entry's column into one TMEM lane: a thread adds up its own entry's weights, no shuffles, no atomics, a fixed order (a tile's sum
// first, then the tiles).  A CTA owns 256 entries (two key tiles, loaded once) of one kv head and walks the row tiles that see any
// of them; logits are double buffered (4 x 128 TMEM columns), so the tensor cores run ahead.  Bound: the exponentials, 16 a cycle
// and SM -- half as many matrix flops per exponential as the attention itself.
constexpr int kWeightsThreads = 640;

template <int D>
struct WeightsShape {
  static constexpr int kPartBytes = 128 * 128;
  static constexpr int kTileBytes = D / 64 * kPartBytes;
  static constexpr int kStages = D == 128 ? 4 : 6;
  static constexpr int kSmem = (2 + kStages) * kTileBytes + (2 * kStages + 12) * 8 + 16 + 2 * 128 * 4 + 256 * 4;
};

template <int D>
__global__ void __launch_bounds__(kWeightsThreads, 1) paged_weights_tc_kernel(const __grid_constant__ PrefillParams P) {
  using Sh = WeightsShape<D>;
  constexpr int STAGES = Sh::kStages;
  extern __shared__ __align__(1024) unsigned char sk[];               // two key tiles, then the ring of row tiles
  unsigned char* ring = sk + 2 * Sh::kTileBytes;
  uint64_t* full = reinterpret_cast<uint64_t*>(ring + STAGES * Sh::kTileBytes);
  uint64_t* empty = full + STAGES;
  uint64_t* k_full = empty + STAGES;
  uint64_t* s_full = k_full + 1;       // [key tile][buffer]
  uint64_t* s_empty = s_full + 4;
  uint64_t* lse_full = s_empty + 4;    // [buffer]
  uint64_t* drained = lse_full + 2;    // all matrix instructions are done
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drained + 1);
  float* lse = reinterpret_cast<float*>(tmem_slot + 4);               // [buffer][128] base-2 log-sums of a row tile
  float* sums = lse + 256;                                            // [key tile][128] from the second halves

  const PagedParams& A = P.A;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, G = 1 << P.g_shift;
  griddep_wait();
  const int head = blockIdx.x % A.n_kv_heads, b = blockIdx.x / A.n_kv_heads % A.batch, e0 = blockIdx.x / A.n_kv_heads / A.batch * 256;
  const SeqRows s = seq_rows(A, b);
  const int old = s.len - s.n;
  if (e0 >= s.len || s.n == 0 || old < 0) return;
  // row tiles that see an entry of the block: tokens from the first entry's on, to the window's end of the last one
  const int t_lo = max(0, e0 - old), e_last = min(e0 + 255, s.len - 1);
  const long long t_end = A.window == 0 || e0 < A.sink ? s.n : min((long long)s.n, (long long)e_last - old + A.window);   // first token that sees none
  const int tile0 = (t_lo << P.g_shift) >> 7, tiles = t_end <= t_lo ? 0 : (int)(((t_end << P.g_shift) + 127) >> 7) - tile0;
  if (tiles == 0) return;                                             // entries that came with the call are seen by their own tokens
  if (tid == 0) {
    for (int i = 0; i < STAGES; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], 1); }
    mbar_init(k_full, 1);
    for (int i = 0; i < 4; ++i) { mbar_init(&s_full[i], 1); mbar_init(&s_empty[i], 8); }
    for (int i = 0; i < 2; ++i) mbar_init(&lse_full[i], 1);
    mbar_init(drained, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 16) tmem_take(tmem_slot);
  tcgen05_before_sync();
  __syncthreads();
  tcgen05_after_sync();
  griddep_launch();                                                   // behind the allocation, as in the kernel above
  const uint32_t tmem = __shfl_sync(~0u, *tmem_slot, 0);

  const WaitLimit waits{A.status, P.polls};

  if (warp == 17) {
    // ---- copies
    const int pr = A.page, boxes = 256 >> A.page_shift;
    fence_proxy_async();
    if (lane == 0) mbar_expect_tx(k_full, 2 * Sh::kTileBytes);
    __syncwarp();
    for (int j = lane; j < boxes * (D / 64); j += 32) {
      const int box = j & (boxes - 1), part = j / boxes, i = e0 + box * pr, at = box * pr;      // row of the block
      int chunk = P.oob_chunk;
      if (i < s.len && seen_from(i, pr, old, A.window, A.sink)) {
        const int pg = page_of(A, b, i);
        if (pg >= 0) chunk = P.chunk0 + pg * A.n_kv_heads + head;
      }
      tensor_g2s_4d(sk + (at >> 7) * Sh::kTileBytes + part * Sh::kPartBytes + (at & 127) * 128, P.kmap, 0, 0, part, chunk, k_full);
    }
    int it = 0;
    for (; it < tiles; ++it) {
      const int st = it % STAGES;
      if (it >= STAGES && !warp_wait(&empty[st], ((it / STAGES) & 1) ^ 1, waits)) break;
      if (lane == 0) mbar_expect_tx(&full[st], Sh::kTileBytes);
      __syncwarp();
      if (lane < D / 64)
        tensor_g2s_4d(ring + st * Sh::kTileBytes + lane * Sh::kPartBytes, P.qmap, 0, head * G, s.first + (((tile0 + it) * 128) >> P.g_shift), lane, &full[st]);
    }
    // they land before the CTA ends, whoever gave up
    bool landed = drain_wait(k_full, 0, A.status);
    for (int f = max(0, it - STAGES); f < it && landed; ++f) landed = drain_wait(&full[f % STAGES], (f / STAGES) & 1, A.status);
  } else if (warp == 18) {
    // ---- log-sums of the row tiles
    for (int it = 0; it < tiles; ++it) {
      const int buf = it & 1;
      float x[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int R = (tile0 + it) * 128 + j * 32 + lane, tok = R >> P.g_shift;
        x[j] = tok < s.n ? A.lse[(long long)(s.first + tok) * A.n_q_heads + head * G + (R & (G - 1))] * kLog2e : 0.f;
      }
      if (it >= 2 && (!warp_wait(&s_empty[buf], ((it >> 1) & 1) ^ 1, waits) || !warp_wait(&s_empty[2 + buf], ((it >> 1) & 1) ^ 1, waits))) break;
#pragma unroll
      for (int j = 0; j < 4; ++j) lse[buf * 128 + j * 32 + lane] = x[j];
      __syncwarp();
      if (lane == 0) mbar_arrive(&lse_full[buf]);
    }
  } else if (warp == 16) {
    // ---- matrix instructions, all by one elected thread
    if (elect_one()) {
      const uint64_t k_at[2] = {smem_matrix(smem_u32(sk), 16), smem_matrix(smem_u32(sk + Sh::kTileBytes), 16)}, q_ring = smem_matrix(smem_u32(ring), 16);
      [&] {
        if (!thread_wait(k_full, 0, waits)) return;
        for (int it = 0; it < tiles; ++it) {
          const int st = it % STAGES, buf = it & 1;
          const uint64_t qd = q_ring + (uint32_t)(st * (Sh::kTileBytes >> 4));
          if (!thread_wait(&full[st], (it / STAGES) & 1, waits)) return;
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            if (it >= 2 && !thread_wait(&s_empty[t * 2 + buf], ((it >> 1) & 1) ^ 1, waits)) return;
            tcgen05_after_sync();
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
              constexpr int kPart = Sh::kPartBytes >> 4;
              mma_smem(tmem + (t * 2 + buf) * 128, k_at[t] + (k >> 2) * kPart + (k & 3) * 2, qd + (k >> 2) * kPart + (k & 3) * 2, mma_shape(128, false), k > 0);
            }
            tcgen05_commit(&s_full[t * 2 + buf]);
          }
          tcgen05_commit(&empty[st]);
        }
      }();
      // nothing is in flight when the CTA ends
      tcgen05_commit(drained);
      drain_wait(drained, 0, A.status);
    }
    __syncwarp();
  } else if (warp < 16) {
    // ---- an entry and half of a row tile's rows per thread
    const int t = warp >> 3, half = (warp >> 2) & 1, e = e0 + t * 128 + (tid & 127);
    const uint32_t s_at = tmem + ((uint32_t)(warp & 3) << 21) + t * 256 + half * 64;
    const float c = A.scale_log2;
    // rows [r_lo, r_hi) of the sequence see the entry
    const int r_lo = max(0, e - old) << P.g_shift;
    const long long t_hi = A.window == 0 || e < A.sink ? s.n : min((long long)s.n, (long long)e - old + A.window);
    const int r_hi = e < s.len ? (int)(max(t_hi, 0LL) << P.g_shift) : 0;
    float total = 0.f;
    bool ok = true;
    for (int it = 0; it < tiles; ++it) {
      const int buf = it & 1, row0 = (tile0 + it) * 128 + half * 64;
      ok = warp_wait(&lse_full[buf], (it >> 1) & 1, waits) && warp_wait(&s_full[t * 2 + buf], (it >> 1) & 1, waits);
      if (!ok) break;
      tcgen05_after_sync();
      const bool whole = __all_sync(~0u, row0 >= r_lo && row0 + 64 <= r_hi);
      float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
      for (int h = 0; h < 2; ++h) {
        uint32_t x[32];
        tmem_load32(s_at + buf * 128 + h * 32, x);
        tmem_wait_loads();
        const float4* ls = reinterpret_cast<const float4*>(lse + buf * 128 + half * 64 + h * 32);
        if (whole) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float4 z = ls[i];
            sum[0] += exp2_fast(fmaf(__uint_as_float(x[4 * i]), c, -z.x));
            sum[1] += exp2_fast(fmaf(__uint_as_float(x[4 * i + 1]), c, -z.y));
            sum[2] += exp2_fast(fmaf(__uint_as_float(x[4 * i + 2]), c, -z.z));
            sum[3] += exp2_fast(fmaf(__uint_as_float(x[4 * i + 3]), c, -z.w));
          }
        } else {
          const int lo = r_lo - row0 - h * 32, hi = r_hi - row0 - h * 32;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float4 z = ls[i];
            const float w0 = exp2_fast(fmaf(__uint_as_float(x[4 * i]), c, -z.x)), w1 = exp2_fast(fmaf(__uint_as_float(x[4 * i + 1]), c, -z.y));
            const float w2 = exp2_fast(fmaf(__uint_as_float(x[4 * i + 2]), c, -z.z)), w3 = exp2_fast(fmaf(__uint_as_float(x[4 * i + 3]), c, -z.w));
            sum[0] += 4 * i >= lo && 4 * i < hi ? w0 : 0.f;
            sum[1] += 4 * i + 1 >= lo && 4 * i + 1 < hi ? w1 : 0.f;
            sum[2] += 4 * i + 2 >= lo && 4 * i + 2 < hi ? w2 : 0.f;
            sum[3] += 4 * i + 3 >= lo && 4 * i + 3 < hi ? w3 : 0.f;
          }
        }
      }
      total += (sum[0] + sum[1]) + (sum[2] + sum[3]);
      tcgen05_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(&s_empty[t * 2 + buf]);
    }
    if (half) sums[t * 128 + (tid & 127)] = total;
    asm volatile("bar.sync 1, 512;" ::: "memory");
    if (ok && !half && e < s.len) {
      float* a = A.scores + ((long long)b * A.n_kv_heads + head) * A.score_stride + e;
      *a = (A.k && e >= old ? 0.f : *a) + (total + sums[t * 128 + (tid & 127)]) * (1.f / G);
    }
  }
  tcgen05_before_sync();
  __syncthreads();
  if (warp == 16) {
    tcgen05_after_sync();
    tmem_give_back(tmem);
  }
}

}  // namespace wkv
