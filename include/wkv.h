/* wkv.h -- C ABI of the WeightedKV decode hot path for NVIDIA B200 (sm_100a).
 *
 * The library keeps, for every lane = (layer, sequence, kv-head), a key/value cache of at most
 * `budget` entries and runs one iteration of the paper's Algorithm 1 ("WeightedKV") per incoming
 * token: append k_t, v_t; single-query softmax attention over the cache (Background section:
 * A_t = softmax(q_t^T K_t), o_t = A_t^T V_t); fold A_t into the accumulated scores a; once the cache
 * holds more than `budget` entries, pick the entry with the smallest average score a/n outside the
 * protected regions, merge its value into the right neighbour by the score-weighted convex
 * combination, and drop its key.  Lanes are independent (the paper omits the batch and head
 * dimensions for that reason).  Every step of that path runs in CUDA kernels of this library; there
 * is no CPU fallback.
 *
 * Conventions
 *   - "device" pointers are CUDA device addresses on the context's GPU; "host" pointers are ordinary
 *     (preferably page-locked) host addresses.  The library never takes ownership of caller buffers.
 *   - q, k, v, out hold elements of the context's storage type (fp32 or bf16); scores are fp32.
 *   - All calls on one context must be issued from one host thread at a time and run on the
 *     context's stream; device-pointer calls are asynchronous with respect to the host.
 *   - Every function returning int returns WKV_OK (0) or a negative wkv_error; no exceptions cross the
 *     boundary.  wkv_last_error() gives a text for the most recent failure on that context.
 */
#ifndef WKV_H_
#define WKV_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct wkv_ctx wkv_ctx; /* opaque, library-owned */

typedef enum {
  WKV_F32 = 0,
  WKV_BF16 = 1,
  WKV_KV4 = 4 /* paged caches only: q, k, v, out in bf16, the pool's rows in 4 bits (see "Rows in 4 bits") */
} wkv_dtype;

typedef enum {
  WKV_OK = 0,
  WKV_ERR_INVALID = -1, /* bad configuration or argument                                   */
  WKV_ERR_ALLOC = -2,   /* the memory provider returned NULL                               */
  WKV_ERR_CUDA = -3,    /* a CUDA runtime call or launch failed (text in wkv_last_error)    */
  WKV_ERR_STATE = -4,   /* a lane's bookkeeping found inconsistent (host check of an export,
                           or a kernel's own check of its slot links)                       */
  WKV_ERR_TIMEOUT = -5  /* a bounded device-side wait gave up (device status word)          */
} wkv_error;

typedef enum {
  WKV_SCHEDULE_AUTO = 0,
  WKV_SCHEDULE_SPLIT = 1,  /* two launches: scan every unit, then one CTA per lane finishes it (any n_splits)    */
  WKV_SCHEDULE_CLUSTER = 2,/* one launch: a lane's units form a thread-block cluster (n_splits in {1,2,4,8,16})  */
  WKV_SCHEDULE_FLAT = 3    /* two launches as in SPLIT, but the scan's CTAs take equal runs of the 32-entry tiles of
                              ALL lanes, across lane boundaries (n_splits = CTAs per lane on average, 0 = one wave
                              that fills the GPU); same results                                                  */
} wkv_schedule;

/* Device memory provider.  alloc returns a device address aligned to at least 256 bytes, or NULL. */
typedef void* (*wkv_alloc_fn)(size_t bytes, void* user);
typedef void (*wkv_release_fn)(void* ptr, void* user);

typedef struct {
  int32_t n_layers;   /* >= 1                                                                          */
  int32_t batch;      /* sequences per call, >= 1                                                      */
  int32_t n_q_heads;  /* query heads; a multiple of n_kv_heads; group = n_q_heads/n_kv_heads in {1,2,4,8} */
  int32_t n_kv_heads; /* key/value heads                                                               */
  int32_t head_dim;   /* 64 or 128                                                                     */
  int32_t budget;     /* m of Algorithm 1: entries kept per lane after a step; 1 <= m < 2^20           */
  int32_t window;     /* W >= 1: the W newest entries are never picked (W = 1 is Algorithm 1's range
                         {0..m-1}; the Experiments section keeps 508 / 124 recent tokens)              */
  int32_t sink;       /* S >= 0: the S first tokens are never picked (Experiments section keeps 4);
                         budget >= sink + window is required                                           */
  int32_t dtype;      /* wkv_dtype: storage type of q, k, v, out and the cache                         */
  float scale;        /* softmax scale; 0 selects 1/sqrt(head_dim) (Ideal Merging section)             */
  int32_t merge;      /* 1: WeightedKV; 0: the "Eviction" variant of the Ablation Study (value dropped) */
  int32_t n_splits;   /* units a lane's cache scan is cut into; 0 = choose from the shape; max 64         */
  int32_t schedule;   /* wkv_schedule: how units are mapped to CTAs; 0 = choose from the shape            */
  void* stream;       /* cudaStream_t of the caller; NULL = the legacy default stream                  */
  wkv_alloc_fn alloc; /* NULL = cudaMalloc / cudaFree                                                  */
  wkv_release_fn release;
  void* user;
} wkv_config;

/* Host-only check of a configuration: NULL if wkv_create would accept it, else a static text naming the
 * first violated rule.  Touches no GPU. */
const char* wkv_config_error(const wkv_config* cfg);

/* Validates cfg, allocates the cache and bookkeeping for n_layers*batch*n_kv_heads lanes on the current
 * CUDA device through the provider and clears them (Algorithm 1 starts from empty score and count lists).  *out is
 * NULL on failure; when the provider returns NULL for one of the blocks the call returns WKV_ERR_ALLOC after handing
 * every block it had obtained back to `release`.  On bf16 rows the cache scan with four query heads per key, the value sweep of a blocked prompt tail and the
 * dense prompt kernel take tiles of the cache through tensor maps, which the driver encodes here (cuTensorMapEncodeTiled, looked up at run time): WKV_ERR_CUDA if
 * the driver lacks it, WKV_ERR_INVALID if the value cache would have 2^31 rows or more. */
int wkv_create(const wkv_config* cfg, wkv_ctx** out);

/* Releases everything obtained from the provider.  NULL is accepted. */
void wkv_destroy(wkv_ctx* ctx);

/* Empties every lane (all caches, scores, positions); asynchronous on the stream. */
int wkv_reset(wkv_ctx* ctx);

/* Changes the stream later calls are issued on.  The caller orders work across streams. */
int wkv_set_stream(wkv_ctx* ctx, void* stream);

/* One iteration of Algorithm 1 for every sequence of one layer (one or two kernel launches), asynchronous.
 *   q    device [batch, n_q_heads, head_dim]   query of the new token
 *   k, v device [batch, n_kv_heads, head_dim]  its key and value, appended to the cache first
 *                                              (Background: K_t = [K_{t-1}, k_t], V_t = [V_{t-1}, v_t])
 *   out  device [batch, n_q_heads, head_dim]   o_t = A_t^T V_t over the cache including the new token and
 *                                              before this step's merge
 *   evicted_pos device [batch, n_kv_heads] int32, or NULL: original 0-based position of the token whose
 *                                              key was dropped this step, -1 when the lane did not compress
 *   probs device [batch, n_q_heads, budget+1] fp32, or NULL: A_t in slot order (slot -> position through
 *                                              wkv_export_slots); slots beyond the lane's length get 0
 * Errors: WKV_ERR_INVALID (NULL ctx/q/k/v/out, layer out of range), WKV_ERR_CUDA (launch failure). */
int wkv_decode_step(wkv_ctx* ctx, int32_t layer, const void* q, const void* k, const void* v, void* out,
                    int32_t* evicted_pos, float* probs);

/* All layers of one decode step in one call: wkv_decode_step for layer 0, 1, ..., n_layers-1 (Algorithm 1 per lane;
 * the lanes of different layers are independent).
 *   q   device [n_layers, batch, n_q_heads, head_dim];  k, v device [n_layers, batch, n_kv_heads, head_dim]
 *   out device [n_layers, batch, n_q_heads, head_dim];  evicted_pos device [n_layers, batch, n_kv_heads] or NULL
 * By making this call the caller states that ALL layers' q, k, v are complete on the stream before it; the library
 * uses that to run the lanes of all layers in one launch when a layer alone is small, or else to let each layer's
 * cache scan run while the previous layer's per-lane epilogue is still finishing (results are identical to n_layers
 * separate calls).  Inputs must not overlap the outputs.  Asynchronous. */
int wkv_decode_step_layers(wkv_ctx* ctx, const void* q, const void* k, const void* v, void* out, int32_t* evicted_pos);

/* No counterpart in the paper: this entry point exists for callers that must not allocate device memory.
 *
 * Some hosts of this library cannot call cudaMalloc at the moment they need a decode step: code running
 * inside a region where allocation is forbidden or would stall (a latency-critical serving loop that
 * promised its allocator a fixed footprint, a process whose memory pool has been handed over entirely to
 * another component, a plug-in that is only allowed to use buffers it is given).  wkv_decode_step already
 * allocates nothing per call, but its scratch (parked logits, per-split partial outputs) was obtained from
 * the memory provider at wkv_create.  This variant runs the same two kernels (scan, lane epilogue) with that
 * scratch placed in a fixed array of WKV_STATIC_SCRATCH_BYTES bytes that is part of the library image, so a
 * context created through a provider that only hands out caller-owned memory never causes an allocation.
 * Every GPU that loads the library holds the array until the process exits.
 *
 *   Arguments, shapes and results: exactly those of wkv_decode_step, without `probs`.
 *   Limit: batch*n_kv_heads*(group*4*roundup4(budget+1) + n_splits*group*(head_dim+2)*4) bytes (each
 *          region rounded up to 256) must fit WKV_STATIC_SCRATCH_BYTES; otherwise WKV_ERR_INVALID is returned,
 *          nothing is launched, and wkv_last_error() names both numbers.
 *   First call on a device: looks up the array's device address (cudaGetSymbolAddress) with that device
 *          current and remembers it.  Make that first call outside any stream capture.
 *   Sharing: all contexts and all calls use the one array, which keeps the previous call's contents.  Nothing
 *          in it has to start at zero: every word the second kernel reads has been written by the first
 *          kernel of the same call.  Calls that can overlap on the GPU (different streams, or different contexts
 *          without ordering between them) race on the array: serialise them.
 *   Calls no cudaMalloc, cudaFree or other allocating routine.  (The CUDA runtime may load a kernel's code the
 *          first time that kernel is launched on a device and take device memory for it: run one step of the same
 *          shape outside the region that must not allocate.) */
#define WKV_STATIC_SCRATCH_BYTES (4u << 20)
int wkv_decode_step_static(wkv_ctx* ctx, int32_t layer, const void* q, const void* k, const void* v, void* out,
                           int32_t* evicted_pos);

/* The same step from HOST buffers: copies q, k, v to library-owned device staging, runs the step, copies
 * out (and evicted_pos if not NULL) back and waits for the stream.  Shapes as in wkv_decode_step. */
int wkv_decode_step_host(wkv_ctx* ctx, int32_t layer, const void* q, const void* k, const void* v, void* out,
                         int32_t* evicted_pos);

/* wkv_decode_step_layers from HOST buffers (shapes as there, all layers of one step): three copies in, the step, two
 * copies out, then waits for the stream. */
int wkv_decode_step_layers_host(wkv_ctx* ctx, const void* q, const void* k, const void* v, void* out,
                                int32_t* evicted_pos);

/* Consumes a prompt exactly as Algorithm 1 does: token by token, compressing as soon as a lane exceeds
 * the budget (the algorithm has no separate prompt phase).  One kernel launch per token, asynchronous.
 *   Q    device [batch, T_max, n_q_heads, head_dim], K, V device [batch, T_max, n_kv_heads, head_dim]
 *   seq_lens device [batch] int32 or NULL: sequence b consumes tokens 0..seq_lens[b]-1 (NULL = T_max each)
 *   out  device [batch, T_max, n_q_heads, head_dim] or NULL (outputs discarded into internal staging)
 *   evicted_pos device [batch, T_max, n_kv_heads] int32 or NULL */
int wkv_prefill(wkv_ctx* ctx, int32_t layer, const void* Q, const void* K, const void* V, const int32_t* seq_lens,
                int32_t T_max, void* out, int32_t* evicted_pos);

/* The same prompt, same arguments and same results as wkv_prefill, with the uncompressed part of the prompt done as
 * one dense problem per lane and the rest in blocks of tokens that share two sweeps of the cache.  Algorithm 1 compresses only once a lane holds more than `budget` entries; until then
 * its iterations are causal attention (Background section) plus the running sums of the attention columns.  The
 * library keeps, per layer, an upper bound on the tokens any lane has consumed since wkv_create / wkv_reset (calls of
 * every kind count; an imported lane counts as its token count if nothing of it was removed, as full otherwise).
 * While that bound is below the budget, the first min(T_max, budget - bound) tokens of the call go through one kernel
 * for all lanes of the layer -- on top of what each lane already holds, whose keys and values it reads from the cache
 * -- with every logit, probability and accumulated score computed by the arithmetic of the streamed step and the
 * scores added in the order of the tokens.  The remaining tokens are taken 8 / group at a time where window > 8 / group
 * and a lane's entries fit the register form of the per-lane kernel (budget + 1 <= 4352 for one query head per key):
 * one sweep over the key rows gives the logits of the whole block, the per-token step of Algorithm 1 (probabilities,
 * score fold, pick, merge) then runs on them token after token exactly as when streaming, and one sweep over the value
 * rows gives all outputs; elsewhere they are streamed as in wkv_prefill.  So a prompt may come in one call or in chunks.  K, positions, accumulated scores and removed positions are bit-identical to
 * wkv_prefill's; outputs and merged values agree within rounding.
 * The first call takes 64 * lanes_per_layer * round_up(budget, 128) bytes of scratch from the memory provider (twice that for
 * bf16 layers of at most two lanes per SM, which run blocks of 32 query rows), the first
 * blocked tail about 64 * lanes_per_layer * (budget + 1) bytes more (if the provider refuses those, the tail is streamed);
 * both are kept until wkv_destroy.  Q, K, V, out must be 16-byte aligned (WKV_ERR_INVALID otherwise).  Asynchronous. */
int wkv_prefill_bulk(wkv_ctx* ctx, int32_t layer, const void* Q, const void* K, const void* V, const int32_t* seq_lens,
                     int32_t T_max, void* out, int32_t* evicted_pos);

/* wkv_prefill_bulk for all layers of a prompt in one call (Algorithm 1 per lane; lanes of different layers are as
 * independent as lanes of one layer).
 *   Q device [n_layers, batch, T_max, n_q_heads, head_dim], K, V device [n_layers, batch, T_max, n_kv_heads, head_dim]
 *   seq_lens device [batch] or NULL (shared by the layers); out like Q or NULL; evicted_pos device
 *   [n_layers, batch, T_max, n_kv_heads] int32 or NULL.  Inputs and outputs must not overlap; 16-byte alignment as above.
 * While no lane of any layer can have reached the budget, the dense phase runs over the lanes of all layers at once if its scratch
 * (64 * n_layers * lanes_per_layer * round_up(budget, 128) bytes) stays under 256 MB -- what a single sequence needs to
 * fill the GPU -- and layer by layer otherwise.  The remaining tokens are streamed: one launch per token over the
 * lanes of all layers where wkv_decode_step_layers does the same, else with the layers interleaved so that one layer's
 * scan can run alongside the previous layer's lane epilogues.  Results equal wkv_prefill's. */
int wkv_prefill_bulk_layers(wkv_ctx* ctx, const void* Q, const void* K, const void* V, const int32_t* seq_lens,
                            int32_t T_max, void* out, int32_t* evicted_pos);

/* Copies one lane to HOST memory in position order and checks its bookkeeping (links form one chain of
 * `len` entries with strictly increasing positions); waits for the stream.  Any destination may be NULL.
 *   len, tokens : entries held / tokens consumed so far
 *   pos [len] int32 original positions; a [len] fp32 accumulated scores (n_i = tokens - pos_i);
 *   K, V [len, head_dim] storage type.  Buffers must have room for budget entries.
 * Returns WKV_ERR_STATE if the bookkeeping is inconsistent. */
int wkv_export_state(wkv_ctx* ctx, int32_t layer, int32_t b, int32_t kv_head, int32_t* len, int32_t* tokens,
                     int32_t* pos, float* a, void* K, void* V);

/* Slot-order view of one lane for interpreting `probs`: slot_pos [budget+1] int32 on the HOST, -1 for a
 * free slot.  Waits for the stream. */
int wkv_export_slots(wkv_ctx* ctx, int32_t layer, int32_t b, int32_t kv_head, int32_t* slot_pos);

/* Replaces one lane by the given position-ordered HOST state (len <= budget, pos strictly increasing and
 * < tokens).  Waits for the stream. */
int wkv_import_state(wkv_ctx* ctx, int32_t layer, int32_t b, int32_t kv_head, int32_t len, int32_t tokens,
                     const int32_t* pos, const float* a, const void* K, const void* V);

/* Reads and clears the device status word (waits for the stream): WKV_OK, WKV_ERR_TIMEOUT if a bounded wait inside
 * a kernel gave up since the last call, or WKV_ERR_STATE if a kernel found inconsistent slot links.
 * After WKV_ERR_TIMEOUT the context accepts calls as before (this call also clears the per-lane arrival counters of
 * the kernels), but a lane whose step was abandoned has consumed one token less than the others and its outputs of
 * that step are undefined: wkv_reset the context or wkv_import_state the affected lanes before decoding on. */
int wkv_status(wkv_ctx* ctx);

/* Self-test of the error path for device-side waits.  Every wait inside the kernels is bounded: the waits on a
 * shared-memory barrier fed by a bulk copy, and the lane epilogue's poll of its lane's arrival counter, which the scan
 * kernel in front of it increments (that kernel's CTAs have all started before an epilogue CTA becomes resident, so
 * the poll never waits for work that waits for it; at most 2^22 polls of about 100 ns).  After its limit the waiting
 * thread sets a bit in the device status word and carries on, so a kernel always terminates.  This call launches a
 * one-thread kernel that waits on a barrier nothing will complete (20000 polls, a few milliseconds); afterwards
 * wkv_status returns WKV_ERR_TIMEOUT once and the context is as usable as before.  Nothing faults or hangs.
 * Asynchronous. */
int wkv_selftest_wait_timeout(wkv_ctx* ctx);

/* Number of kernels this context has launched so far, and bytes it obtained from the provider. */
int64_t wkv_launch_count(const wkv_ctx* ctx);
int64_t wkv_device_bytes(const wkv_ctx* ctx);
/* The number of CTAs per lane the context uses (after resolving n_splits = 0); under the flat deal, where runs of tiles
 * cross lane boundaries, the largest number of CTAs that can share one lane. */
int32_t wkv_splits(const wkv_ctx* ctx);

const char* wkv_strerror(int code);
const char* wkv_last_error(const wkv_ctx* ctx);

/* ---------------------------------------------------------------------------------------------------------------------
 * Paged caches: every token kept, or the caches that the paper measures WeightedKV against -- first and newest tokens
 * (StreamingLLM: `sink` + `window`) and heavy hitters (H2O: eviction by accumulated attention weight); Experiments
 * section, baselines.  Keys and values lie in a pool of pages, [n_layers, n_pages, n_kv_heads, page_size, head_dim];
 * sequence b's entry i is row i mod page_size of page block_table[b][i / page_size], for every kv head.  Which pages
 * belong to whom is the caller's business: several sequences may share pages that no call writes to.
 *
 * Conventions of these calls, beside those at the top of this file:
 *   - Tables, lengths and offsets are read on the device, so a captured call can be replayed with new ones.  A page number,
 *     length or offset out of range never leads to an access outside the pool or the call's buffers: that page counts as
 *     zeros (entries that the call brings for it are stored nowhere and count as zeros too), the length or offset is clamped,
 *     and wkv_paged_status reports WKV_ERR_STATE.  Columns of a table behind a sequence's last page are not read; nor are those
 *     of pages of which no token of an attention call sees an entry, so a windowed cache may give back the pages behind its
 *     window (an eviction reads its source table's columns up to the sequence's last page).
 *   - Pool rows behind a sequence's length are never used, whatever bits they hold.  Rows inside it are expected to be finite:
 *     an infinity or NaN in one may make any output of that sequence NaN, also of tokens that do not see the entry.
 *   - out, lse and scores must not overlap a call's other arguments.
 *   - A row that sees no entry (a padded sequence of length 0) gets output 0 and log-sum -infinity; a decode step's whose query has a NaN gets
 *     NaN for both.
 *   - The token at position p sees entry i if i <= p and (window == 0, or i > p - window, or i < sink).
 *   - scores [batch, n_kv_heads, score_stride] fp32, or NULL: the attention weight of every entry, averaged over the kv
 *     head's query heads, is added to it, the sum over the call's tokens in a fixed order.  Entries that the call appends
 *     start from 0.  Needs a handle created with scores = 1 and score_stride >= table_width * page_size.
 *   - A handle has one set of workspaces, taken at creation.  Its calls, and replays of graphs captured from them, must not
 *     overlap on the GPU.
 * ------------------------------------------------------------------------------------------------------------------- */
typedef struct wkv_paged wkv_paged; /* opaque, library-owned */

typedef struct {
  int32_t n_layers;   /* >= 1                                                                                     */
  int32_t n_pages;    /* pages of the pool, per layer; n_layers * n_pages * n_kv_heads < 2^31                     */
  int32_t page_size;  /* entries per page: 16, 32 or 64                                                           */
  int32_t n_q_heads;  /* as in wkv_config: n_q_heads / n_kv_heads in {1,2,4,8}                                    */
  int32_t n_kv_heads;
  int32_t head_dim;   /* 64 or 128                                                                                */
  int32_t max_batch;  /* most sequences of one call, 1..1024                                                      */
  int32_t max_pages;  /* most pages of one sequence (table columns); max_pages * page_size <= 2^24                */
  int32_t dtype;      /* wkv_dtype of q, k, v, out and the pool                                                   */
  float scale;        /* softmax scale; 0 selects 1/sqrt(head_dim)                                                */
  int32_t scores;     /* 1: calls may accumulate weights and evict (adds a workspace of 4 * max_batch * n_q_heads *
                         max_pages * page_size bytes); 0 with WKV_KV4                                             */
  void* stream;       /* cudaStream_t                                                                             */
  void* k_pool;       /* the caller's pools, 16-byte aligned device memory; both NULL: taken from the provider    */
  void* v_pool;
  wkv_alloc_fn alloc; /* as in wkv_config                                                                         */
  wkv_release_fn release;
  void* user;
} wkv_paged_config;

/* Host-only check: NULL if wkv_paged_create would accept it, else a static text naming the first violated rule. */
const char* wkv_paged_config_error(const wkv_paged_config* cfg);

/* Creates a handle on the current CUDA device.  Pools that the library takes from the provider start at zero.  The pools'
 * tensor maps are encoded here (WKV_ERR_CUDA if the driver lacks the encoder).  Workspaces, besides that of `scores`: partial
 * outputs, about 300 KB an SM with bf16 rows of 128 channels. */
int wkv_paged_create(const wkv_paged_config* cfg, wkv_paged** out);
/* Releases what the provider gave; the handle's calls are done by then.  NULL is accepted. */
void wkv_paged_destroy(wkv_paged* c);
int wkv_paged_set_stream(wkv_paged* c, void* stream);
/* The pools' device addresses. */
int wkv_paged_pools(const wkv_paged* c, void** k_pool, void** v_pool);

/* One decode step of a layer: appends the new token of every sequence and attends with it (Background section: A_t, o_t),
 * the cache's length split over CTAs and joined in the same launch.  Asynchronous.
 *   q    device [batch, n_q_heads, head_dim], rows q_stride elements apart (0: packed)
 *   k, v device [batch, n_kv_heads, head_dim], rows kv_stride elements apart (0: packed): stored as entry seq_lens[b] - 1.
 *        Both NULL: the entries are in the pool already and nothing is stored.
 *   block_table device [batch, table_width] int32;  seq_lens device [batch] int32: entries WITH the new one, 0 = padding
 *   out  device [batch, n_q_heads, head_dim] packed;  lse device [batch, n_q_heads] fp32 or NULL: ln sum exp(scale q.k)
 * Rows are 16-byte aligned (pointers, and strides in bytes).  Sequences whose last entry shares a page row with another's
 * must not be in one call that appends. */
int wkv_paged_decode(wkv_paged* c, int32_t layer, int32_t batch, const void* q, int64_t q_stride, const void* k, const void* v,
                     int64_t kv_stride, const int32_t* block_table, int32_t table_width, const int32_t* seq_lens,
                     int32_t window, int32_t sink, float* scores, int64_t score_stride, void* out, float* lse);

/* Chunks of new tokens -- whole prompts, pieces of prompts, a few drafted tokens -- of a ragged batch in one call: appends
 * them and attends with each.  Sequence b's tokens are rows q_start[b] .. q_start[b+1]-1 of q, k, v, out and lse and become
 * its last entries; seq_lens counts them.  Rows behind q_start[batch] are left as they were.  No page that the call stores to
 * may be read by another of its sequences.
 *   q, k, v [total_q, heads, head_dim] and their strides as in wkv_paged_decode;  q_start device [batch + 1] int32
 *   out [total_q, n_q_heads, head_dim];  lse [total_q, n_q_heads] fp32, or NULL where scores is NULL. */
int wkv_paged_prefill(wkv_paged* c, int32_t layer, int32_t batch, const void* q, int64_t q_stride, const void* k, const void* v,
                      int64_t kv_stride, const int32_t* q_start, int32_t total_q, const int32_t* block_table,
                      int32_t table_width, const int32_t* seq_lens, int32_t window, int32_t sink, float* scores,
                      int64_t score_stride, void* out, float* lse);

/* Eviction by accumulated weight, for every (sequence, kv head) by itself: while more than `budget` entries are left, the one
 * with the smallest (score, index) outside of the first `sink` and the newest `recent` entries leaves (the index breaks
 * ties; a NaN counts as the largest score).  The others move, in order, into the pages of dst_table, which must share none
 * with the call's src_table rows: pages that several sequences share stay as they are.  (An overlap inside one sequence is
 * found on the device: nothing of that sequence is moved, its new length is its old one and wkv_paged_status reports
 * WKV_ERR_STATE.)  budget >= sink + recent.  Asynchronous.
 *   src_table [batch, src_width], dst_table [batch, dst_width];  seq_lens [batch];  new_lens [batch] out: min(len, budget)
 *   scores [batch, n_kv_heads, score_stride];  scores_out [batch, n_kv_heads, out_stride] or NULL: the kept entries' scores
 *   kept [batch, n_kv_heads, budget] int32 or NULL: their indexes.  Behind a sequence's new length both are left as they were.
 * out_stride >= min(budget, src_width * page_size); scores_out must not overlap scores.  No page may stand twice among those that
 * dst_table's sequences get. */
int wkv_paged_evict(wkv_paged* c, int32_t layer, int32_t batch, const int32_t* src_table, int32_t src_width,
                    const int32_t* dst_table, int32_t dst_width, const int32_t* seq_lens, int32_t* new_lens, int32_t budget,
                    int32_t recent, int32_t sink, const float* scores, int64_t score_stride, float* scores_out,
                    int64_t out_stride, int32_t* kept);

/* Rows in 4 bits (WKV_KV4).  32 neighbouring channels of a row share a scale s and a zero point z, a code n in 0..15 stands for
 * s (n - z).  With lo = min(0, least) and hi = max(0, largest of the 32): s = (hi - lo) * (1/15) rounded up to four significant
 * bits, and into 2^-17 .. 4096 (below 2^-14 to a multiple of 2^-17); z = rint(-lo * (1/s)), n = rint(x * (1/s)) + z, both clamped to
 * 0..15; all of it in binary32, each operation rounded by itself.  Values beyond 15 * 4096 saturate.  s (n - z) is a bf16 number.
 * A pool is [n_layers, n_pages, n_kv_heads, page_size * (head_dim / 2 + head_dim / 16)] bytes: of one kv head's part of a page first
 * the codes, head_dim / 2 bytes a row, then a pair of bytes per row and group: bits 14..7 of s as a binary16 number; z.
 * With D = head_dim, S = D / 32 groups, row i of the page, channel c = 32 g + r:
 *   keys    r = 8 w + e: in the 32-bit word at byte 16 (g ^ x) + 4 w of the row, bits 4 (e / 2) + 16 (e % 2) and the three above;
 *           x = (i / 2) % 4 for D = 128, (i / 4) % 2 for D = 64
 *   values  r = 4 u + e: in the 16-bit word at byte (2 S u + 2 g) ^ x of the row, bits 4 e and the three above;
 *           x = 32 ((i / 2) % 2) for D = 128, 0 for D = 64
 * A decode step rounds an entry's weight times a value scale by 2^-10 of itself at most, or, where that is more, by 2^-34 of the head's
 * largest weight times the largest value scale in sight.
 * Such a handle takes wkv_paged_append, wkv_paged_decode (k and v, where given, are stored in 4 bits first, and the new token sees its
 * entry as stored), wkv_paged_select, wkv_paged_decode_pages and wkv_paged_expand; prompts run on bf16 rows (wkv_paged_expand). */

/* Appends new entries, turned to their position on the way, and turns the queries that go with them; no attention.  Asynchronous.
 * What follows is a wkv_paged_decode or wkv_paged_prefill with k and v NULL.
 *   q [total_q, n_q_heads, head_dim], k, v [total_q, n_kv_heads, head_dim]: rows q_stride, kv_stride elements apart (0: packed),
 *        16-byte aligned;  q NULL: no queries;  k and v NULL: only the queries
 *   q_start device [batch + 1] int32: sequence b's tokens are rows q_start[b] .. q_start[b+1]-1 and become its last entries
 *        (total_q at most 2^24); NULL: one token per sequence, row b, total_q = batch.  seq_lens counts the new entries; 0 = padding
 *   rope device [rope_rows, rope_dim] fp32, 16-byte aligned: for every position rope_dim / 2 cosines, then as many sines; NULL: nothing is
 *        turned.  The first rope_dim channels of a head (a multiple of 16, <= head_dim) are turned in pairs,
 *        (a, b) -> (a cos - b sin, b cos + a sin), in binary32, each product rounded by itself; rope_paired = 1: angle i turns channels
 *        2i and 2i + 1, 0: channels i and i + rope_dim / 2
 *   positions device [total_q] int32, NULL: a token's position is its entry's index.  A position outside of the table leaves the row as
 *        it is, and wkv_paged_status reports WKV_ERR_STATE
 *   q_out [total_q, n_q_heads, head_dim], rows q_out_stride elements apart (0: packed); may be q itself (same stride), and must
 *        not overlap the call's other arguments otherwise.  Rows of no sequence are left as they were
 *   page_bounds device [n_layers, n_pages, n_kv_heads, 2, head_dim] int8 and page_scale [n_layers, n_pages, n_kv_heads], or both
 *        NULL: of every page that gets an entry the bounds of its keys, as stored, up to the sequence's length: page_scale =
 *        (largest magnitude) * (1/127), and per channel the largest key / page_scale rounded up and the least rounded down (0 where
 *        page_scale is below 2^-100).  Of rows that are not finite: a NaN counts as no key, an infinite key, or a channel without a
 *        number, makes page_scale infinite and the page's score infinity or NaN, which rank above all others.  A page
 *        that another sequence shares must hold the same entries for both.  Calls that store or move entries otherwise (wkv_paged_decode
 *        and wkv_paged_prefill with k and v, wkv_paged_evict) keep no bounds; a page's are whole again once it gets an entry here. */
int wkv_paged_append(wkv_paged* c, int32_t layer, int32_t batch, const void* q, int64_t q_stride, const void* k, const void* v,
                     int64_t kv_stride, const int32_t* q_start, int32_t total_q, const int32_t* block_table, int32_t table_width,
                     const int32_t* seq_lens, const float* rope, int32_t rope_rows, int32_t rope_dim, int32_t rope_paired,
                     const int32_t* positions, void* q_out, int64_t q_out_stride, int8_t* page_bounds, float* page_scale);

/* Chooses the pages that a decode step's query attends to, for every (sequence, kv head) by itself: the first `sink` and the newest
 * `recent` pages, then those with the best scores, of equal scores the lowest page.  Asynchronous.  A page's score is page_scale
 * times the whole number sum over channels of (u hi + w lo), with hi, lo the page's bounds and u, w the sums over the kv head's
 * query heads of max(q, 0) and min(q, 0), both in steps of 1/127 of their largest channel: up to rounding, and a factor per query,
 * a bound on the sum over the heads of q.k.
 *   q as in wkv_paged_decode;  page_bounds, page_scale as wkv_paged_append keeps them: of a page that got entries by another call, an
 *        eviction above all, they are those of what it held before, and nothing reports that
 *   n_select in [1, 2^20]; recent >= 1, recent + sink <= n_select
 *   page_scores [batch, n_kv_heads, page_score_stride] fp32 out: the score of every page (page_score_stride >= table_width);
 *        behind a sequence's last page left as it was
 *   pages [batch, n_kv_heads, n_select] int32 out: indexes into the sequence's table row, rising; -1 behind the last */
int wkv_paged_select(wkv_paged* c, int32_t layer, int32_t batch, const void* q, int64_t q_stride, const int32_t* block_table,
                     int32_t table_width, const int32_t* seq_lens, const int8_t* page_bounds, const float* page_scale, int32_t n_select,
                     int32_t recent, int32_t sink, float* page_scores, int64_t page_score_stride, int32_t* pages);

/* Attention of one token per sequence to the entries of chosen pages, each kv head its own.  Stores nothing.  Asynchronous.
 *   pages [batch, n_kv_heads, n_select] int32: indexes into the sequence's table row; of a list as many places are read as the
 *        sequence has pages.  Numbers outside of the sequence count as none; one that stands twice counts twice
 *   q, block_table, seq_lens, out and lse as in wkv_paged_decode */
int wkv_paged_decode_pages(wkv_paged* c, int32_t layer, int32_t batch, const void* q, int64_t q_stride, const int32_t* block_table,
                           int32_t table_width, const int32_t* seq_lens, const int32_t* pages, int32_t n_select, void* out, float* lse);

/* Spreads rows in 4 bits out to the bf16 pages of another handle on the same device (same n_kv_heads and head_dim; the page size
 * may differ), where prompts can attend to them.  Runs on c's stream; the caller orders dst's.  Asynchronous.
 *   block_table, seq_lens as in wkv_paged_decode;  dst_table device [batch, dst_width] int32, pages for every sequence's length (entries
 *        that it has no page for are stored nowhere, and c's wkv_paged_status reports WKV_ERR_STATE)
 * Rows behind a sequence's length are left as they were.  batch * n_kv_heads * (table_width * page_size / 64, rounded up) must stay
 * below 2^31. */
int wkv_paged_expand(wkv_paged* c, int32_t layer, int32_t batch, const int32_t* block_table, int32_t table_width, const int32_t* seq_lens,
                     wkv_paged* dst, int32_t dst_layer, const int32_t* dst_table, int32_t dst_width);

/* As their namesakes without _paged.  A wait inside a kernel that gave up (WKV_ERR_TIMEOUT) ends its block's work; what the calls
 * since the last status wrote is then undefined, and the handle can be used again. */
int wkv_paged_status(wkv_paged* c);
int wkv_paged_selftest_wait_timeout(wkv_paged* c);
int64_t wkv_paged_launch_count(const wkv_paged* c);
int64_t wkv_paged_device_bytes(const wkv_paged* c);
const char* wkv_paged_last_error(const wkv_paged* c);

#ifdef __cplusplus
}
#endif
#endif /* WKV_H_ */
