/*
 * epikv.h -- C ABI of the EpiKV eviction hot path for NVIDIA GB300 (sm_103a).
 *
 * EpiKV ("Epiphany-Aware KV Cache Eviction Without the Attention Matrix")
 * scores every generated token once, from quantities the forward pass
 * already produces, and keeps the K best tokens of each sequence's KV cache:
 *
 *   score   Band-z ("EpiKV"): g_l(t) = ||h_l(t) - h_l(t-1)||_2 per band layer
 *           (Sec. 3.2, Eq. 1), a causal rolling z-score per layer (Eq. 3),
 *           Band A mean minus Band B mean (Fig. 1).
 *           Lag-KV: each token's K and V vectors normalised by the previous
 *           chunk's per-channel range, variance over the head dimension, key
 *           + value, mean over (layer, head), rolling mean (Sec. 3.3).
 *   select  keep all prefill tokens and the last min(128, K/4) tokens, and
 *           give the rest of the budget K to the highest-scoring tokens
 *           (Sec. 3.1, Sec. 3.3, App. D).
 *   compact rewrite every layer's and head's K/V rows to the kept set, in
 *           token order (App. H).
 *
 * Conventions shared by every call
 *   - Ownership: the caller owns every buffer (the workspace, hidden rows,
 *     the K/V pool, block tables, outputs).  The library never allocates
 *     device memory; epikv_init allocates only its small host-side context.
 *   - Asynchrony: every call except epikv_get_error, epikv_get_stats,
 *     epikv_read_slots and epikv_read_layer_slots only enqueues work on the
 *     given stream and returns (no synchronisation, no allocation), so a
 *     whole decode step can be captured once in a CUDA graph and replayed.
 *     Calls on one context must be ordered on one stream.
 *   - Host validation failures return EPIKV_EINVAL and enqueue nothing.
 *   - Device-side anomalies (an index out of range, a batch larger than
 *     declared, a kept list that is not strictly increasing) never trap:
 *     the kernel records a code in the context's sticky error word and
 *     skips the offending work.  epikv_get_error returns and clears it.
 *   - bf16 data; K/V rows of one token and layer are H*d contiguous
 *     elements (head-major, channel-minor); all pointers 16-byte aligned.
 *   - A sequence id appears at most once in one call's batch.
 *   - A call's kernels are launched with programmatic dependent launch
 *     among themselves (each waits for the results that it reads, and ends
 *     after its predecessor); against the caller's own work on the stream the
 *     order is plain stream order, except that a caller kernel itself
 *     launched with programmatic dependent launch right after a call must,
 *     as with any such launch, wait for its predecessor
 *     (cudaGridDependencySynchronize) before reading the call's results.
 */
#ifndef EPIKV_H_
#define EPIKV_H_

#include <stddef.h>
#include <stdint.h>
#include <cuda_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  EPIKV_OK = 0,
  EPIKV_EINVAL = 1,   /* invalid argument or configuration; nothing enqueued */
  EPIKV_ECUDA = 2,    /* a CUDA runtime call or kernel launch failed */
  EPIKV_EDEVICE = 3,  /* the device error word was set (see epikv_device_error) */
} epikv_status;

/* Codes a kernel writes into the sticky device error word (first one wins). */
typedef enum {
  EPIKV_DEV_OK = 0,
  EPIKV_DEV_BATCH = 1,      /* n_new < 0 or > max_new, or seq id out of range */
  EPIKV_DEV_CAPACITY = 2,   /* n_cache + n_new would exceed max_cache_tokens; epikv_attention: or too much work */
  EPIKV_DEV_SLOT = 3,       /* a slot or block index outside the KV view */
  EPIKV_DEV_KEPT = 4,       /* kept list not strictly increasing / out of range */
  EPIKV_DEV_BUDGET = 5,     /* budget K < 1 or > max_cache_tokens */
  EPIKV_DEV_TIMEOUT = 6,    /* a bounded wait inside a kernel gave up */
  EPIKV_DEV_POSITION = 7,   /* a token's position outside the rotation table */
} epikv_device_error;

/* Score kinds (bit mask in epikv_config.score_kinds, one value as policy).
 *   BANDZ   EpiKV: Band A mean - Band B mean of rolling z-scores of g (Eq. 3)
 *   LAGKV   Lag-KV: lag-normalised key + value head variance (Sec. 3.3)
 *   HSVAR   HS-variance: Band A mean - Band B mean of rolling means of g (Eq. 2)
 *   KVKEY   KV-key: rolling mean of the stored keys' head variance (Sec. 3.3)
 *   KVVAL   KV-val: the same for the values (Sec. 3.3)
 *   LAGKEY  lag-kv-key: Lag-KV's key term only (Tab. "acc-math" rows)
 *   WEIGHT  accumulated attention weight, which needs what attention-free kinds do without: what
 *           epikv_attention_weights finds, added up by epikv_weigh.  Not frozen: a new token's
 *           score is 0 until then
 * The band kinds use z_window as their window; the K/V kinds lag_window. */
enum {
  EPIKV_SCORE_BANDZ = 1,
  EPIKV_SCORE_LAGKV = 2,
  EPIKV_SCORE_HSVAR = 4,
  EPIKV_SCORE_KVKEY = 8,
  EPIKV_SCORE_KVVAL = 16,
  EPIKV_SCORE_LAGKEY = 32,
  EPIKV_SCORE_WEIGHT = 128,   /* (64 is no kind) */
};

/* KV cache layouts. */
enum { EPIKV_LAYOUT_CONTIGUOUS = 0, EPIKV_LAYOUT_PAGED = 1 };

typedef struct {
  int32_t max_seqs;         /* sequence ids are 0..max_seqs-1 */
  int32_t max_cache_tokens; /* cache slots per sequence (T_cap) */
  int32_t max_new_tokens;   /* new tokens per sequence per score update, max */
  int32_t num_layers;       /* L: layers of the K/V cache */
  int32_t num_kv_heads;     /* H */
  int32_t head_dim;         /* d: a power of two in [8, 256]; H*d/8 <= 256 */
  int32_t hidden;           /* D: hidden size, a multiple of 8, <= 8192 */
  int32_t n_band_a;         /* Band A layers passed per update (Sec. 3.2: 7..13) */
  int32_t n_band_b;         /* Band B layers (Sec. 3.2: 18..25); A+B <= 32 */
  int32_t z_window;         /* w of Eq. 2 and 3 (paper: 64), 1..1024 */
  float z_eps;              /* epsilon of Eq. 3 (1e-6) */
  int32_t lag;              /* Lag-KV chunk length (16), >= 1 */
  float lag_eps;            /* epsilon of the range normalisation (1e-6) */
  int32_t lag_window;       /* rolling-mean window of the K/V scores (64), 1..1024 */
  int32_t recency_cap;      /* recency window R = min(recency_cap, K/4) (App. D: 128) */
  int32_t score_kinds;      /* EPIKV_SCORE_* mask computed by every update (WEIGHT: by epikv_weigh; not with
                             * layer_budgets) */
  int32_t select_chunk;     /* C, 0..65536 (0 reads as 1).  1: the paper's token-level top-K.
                             * C > 1: chunk-level selection, which the paper names as future
                             * work (Sec. 5, after ChunkKV's contiguous chunks, Sec. 2): the
                             * candidates fall into fixed position chunks floor(pos / C), a
                             * chunk scores the fp32 mean of its candidate members' scores
                             * (summed in slot order), and whole chunks fill the candidate
                             * budget in rank order (NaN lowest, ties to the earlier chunk);
                             * the first chunk that does not fit keeps its lowest slots. */
  int32_t layer_budgets;    /* 0: one budget per sequence (the paper's method).  1: one budget
                             * per (sequence, layer), which the paper names as future work
                             * (Sec. 5, after PyramidKV's per-layer allocation, Sec. 2): layer
                             * l keeps its own cache of n_l slots and evicts it with its own
                             * budget K_l at the sequence's events; every layer keeps the
                             * prefill and one shared recency window R = min(recency_cap,
                             * K_min/4) (shrunk to K_min - P), K_min the smallest budget.
                             * Needs num_layers <= 64 and select_chunk <= 1.  In this mode
                             * the per-entry budget, kept and length arrays of epikv_select,
                             * epikv_compact and epikv_step gain a layer dimension (see
                             * there), "n_cache" is the largest layer's length, and the new
                             * K/V rows of an update go to slots n_l .. n_l+n_new-1 of each
                             * layer. */
} epikv_config;

/* New hidden-state rows of one update call (Sec. 3.1: the per-layer hidden
 * states of the standard output_hidden_states interface).  band_rows[i] is a
 * device pointer to bf16 rows [total_new][row_stride] of band layer i (the
 * n_band_a Band A layers first, then the Band B layers); batch entry b owns
 * rows cu_new[b] .. cu_new[b+1]-1, in position order. */
typedef struct {
  const void* band_rows[32];
  int64_t row_stride;       /* elements between consecutive rows (>= hidden) */
} epikv_hidden_view;

/* The K/V cache (Sec. 3.1: 2*L*H*d scalars per token).  Element offsets:
 *   contiguous: layer*stride_layer + seq*stride_seq + slot*stride_token
 *   paged:      layer*stride_layer + block_table[layer*stride_table_layer +
 *               seq*max_blocks_per_seq + slot/block_size]*stride_block +
 *               (slot%block_size)*stride_token
 * The same offsets address k and v.  stride_table_layer = 0 shares one block
 * table among the layers; with per-layer budgets, stride_layer = 0 and one
 * table per layer describe a single pool of blocks in which every (layer,
 * sequence) owns its own blocks, so each layer's memory follows its own
 * budget.  The caller keeps distinct (layer, sequence) block lists disjoint. */
typedef struct {
  void* k;
  void* v;
  int32_t layout;               /* EPIKV_LAYOUT_* */
  int64_t stride_layer;
  int64_t stride_seq;           /* contiguous only */
  int64_t stride_block;         /* paged only */
  int64_t stride_token;         /* usually H*d */
  const int32_t* block_table;   /* paged only: device int32 [max_seqs][max_blocks_per_seq] */
  int32_t max_blocks_per_seq;   /* paged only */
  int32_t block_size;           /* paged only: tokens per block */
  int32_t num_blocks;           /* paged only: pool size, for bounds checks */
  int64_t stride_table_layer;   /* paged only: elements between consecutive layers' block
                                 * tables (0: one table for every layer) */
} epikv_kv_view;

typedef struct {
  unsigned long long tokens_scored;  /* new tokens accepted by score updates */
  unsigned long long evictions;      /* (sequence, event) pairs that evicted */
  unsigned long long rows_moved;     /* kept tokens whose slot changed (largest layer) */
  unsigned long long layer_rows_moved; /* (layer, kept token) pairs whose slot changed */
} epikv_stats;

typedef struct epikv_ctx epikv_ctx;

/* Bytes of device workspace epikv_init needs for cfg (0 if cfg is invalid):
 * the per-sequence state (counters, frozen scores and positions per slot,
 * score rings, Lag-KV chunk ranges, kept lists) plus a fixed compaction stash
 * of 512 x min(128, max_cache_tokens) K/V rows of one layer (128 MiB at
 * num_kv_heads * head_dim = 1024). */
size_t epikv_workspace_bytes(const epikv_config* cfg);

/* Create a context over a caller-allocated device workspace of at least
 * epikv_workspace_bytes(cfg) bytes (256-byte aligned), zero it on `stream`
 * and reset every sequence.  *out receives a host-side handle. */
epikv_status epikv_init(epikv_ctx** out, const epikv_config* cfg, void* d_workspace,
                        size_t workspace_bytes, cudaStream_t stream);

/* Start sequence `seq` afresh: empty cache, next position 0, `prefill_len`
 * leading tokens that are never evicted (App. D: all prefill kept), and the
 * score kind that drives its selection (`policy`, one EPIKV_SCORE_* value
 * that is in cfg.score_kinds). */
epikv_status epikv_seq_reset(epikv_ctx* ctx, int32_t seq, int32_t prefill_len, int32_t policy,
                             cudaStream_t stream);

/* Score the new tokens of a batch and append them to each sequence's slots.
 *   d_seq_ids [n_seq]   device: sequence id of each batch entry
 *   d_cu_new  [n_seq+1] device: prefix offsets of the new tokens per entry
 *                       (d_cu_new[0] = 0, non-decreasing)
 *   max_new             host: an upper bound of every entry's new tokens
 *                       (<= cfg.max_new_tokens; sizes the grid)
 *   hidden              band rows of the new tokens (needed for BANDZ, HSVAR)
 *   kv                  the cache; the new tokens' K/V rows must already be
 *                       in slots n_cache .. n_cache+n_new-1 (needed for the
 *                       K/V kinds)
 * Each token's score is computed once, causally, and frozen (Sec. 3.3). */
epikv_status epikv_score_update(epikv_ctx* ctx, int32_t n_seq, const int32_t* d_seq_ids,
                                const int32_t* d_cu_new, int32_t max_new,
                                const epikv_hidden_view* hidden, const epikv_kv_view* kv,
                                cudaStream_t stream);

/* Choose the kept tokens of each batch entry (Sec. 3.1, App. D).
 *   d_budget  [n_seq] device: budget K per entry
 *   d_trigger [n_seq] device or NULL: evict only if n_cache > trigger
 *             (NULL: evict whenever n_cache > K)
 *   d_kept    device int32 [n_seq][kept_stride]: ascending kept slots,
 *             written only for entries that evict
 *   d_n_kept  device int32 [n_seq]: the cache length after the call
 * With cfg.layer_budgets = 1: d_budget is [n_seq][num_layers] (K_l of each
 * layer), an entry evicts if n_cache (its largest layer) exceeds the trigger
 * (NULL: the largest K_l) and the smallest K_l; d_kept is
 * [n_seq][num_layers][kept_stride], each layer's kept slots in its own slot
 * numbering, and d_n_kept is [n_seq][num_layers]; kept_stride must be at
 * least max(K_max, prefill).  A sequence's layer budgets must stay the same
 * from one epikv_seq_reset to the next: the library keeps one ranking for
 * all layers, which is exact because fixed budgets keep the layers' caches
 * nested; a change that would break the nesting is reported as
 * EPIKV_DEV_KEPT.
 * Ties between equal scores go to the lower slot, NaN ranks lowest.  The
 * call commits the eviction to the context's slot metadata (scores and
 * positions move with their tokens); the caller must apply epikv_compact
 * with the same kept lists, once, before the next score update. */
epikv_status epikv_select(epikv_ctx* ctx, int32_t n_seq, const int32_t* d_seq_ids,
                          const int32_t* d_budget, const int32_t* d_trigger, int32_t* d_kept,
                          int32_t kept_stride, int32_t* d_n_kept, cudaStream_t stream);

/* Move every layer's K and V rows of the entries that evicted in the
 * preceding epikv_select to their kept slots, in order, in place (App. H).
 * Rows before the first evicted slot are not touched.  d_kept has the layout
 * epikv_select wrote (per layer with cfg.layer_budgets = 1).  An eviction is
 * applied once: calling epikv_compact again, or with no eviction selected
 * since the last score update, moves nothing; a score update that finds an
 * eviction selected but not yet compacted reports EPIKV_DEV_KEPT. */
epikv_status epikv_compact(epikv_ctx* ctx, int32_t n_seq, const int32_t* d_seq_ids,
                           const int32_t* d_kept, int32_t kept_stride, const epikv_kv_view* kv,
                           cudaStream_t stream);

/* One decode step: epikv_score_update, then a device-side trigger
 * (evict entries with n_cache > trigger), epikv_select into the context's
 * own kept buffer and epikv_compact -- without any host synchronisation.
 *   d_n_cache_out [n_seq] device or NULL: each entry's cache length after
 *                 the step (a paged caller frees blocks past it);
 *                 [n_seq][num_layers], every layer's length, with
 *                 cfg.layer_budgets = 1 (d_budget as in epikv_select). */
epikv_status epikv_step(epikv_ctx* ctx, int32_t n_seq, const int32_t* d_seq_ids,
                        const int32_t* d_cu_new, int32_t max_new, const int32_t* d_budget,
                        const int32_t* d_trigger, const epikv_hidden_view* hidden,
                        const epikv_kv_view* kv, int32_t* d_n_cache_out, cudaStream_t stream);

/* Record events[0..3] on the stream at the phase boundaries of every later
 * epikv_step (before scoring, before select, before compact, after compact);
 * NULL stops it.  The events are the caller's. */
epikv_status epikv_set_phase_events(epikv_ctx* ctx, const cudaEvent_t* events);

/* Per-kernel timing for measurement.  From this call on, every kernel that an
 * entry point of `ctx` launches (epikv_score_update, epikv_select,
 * epikv_compact, epikv_step) is bracketed on its stream by two of the
 * caller's events -- events[2k] before and events[2k+1] after the k-th such
 * kernel -- and h_names[k] receives its name as the CUDA runtime reports it
 * (storage owned by the runtime), for at most n_kernels kernels; later ones
 * are not recorded.  Both arrays are the caller's and must stay valid until
 * the next call.  An event recorded between two kernels also ends the early
 * launch of the second (programmatic dependent launch), so the kernels then
 * run strictly one after another.  events == NULL stops it and, if h_used is
 * not NULL, stores how many kernels were recorded.  Not thread safe with
 * respect to other calls on the same context. */
epikv_status epikv_set_kernel_events(epikv_ctx* ctx, const cudaEvent_t* events, int32_t n_kernels,
                                     const char** h_names, int32_t* h_used);

/* Debug/test read-back (synchronises): the cache length, positions and
 * scores of kind `kind` of `seq`'s slots; at most `cap` entries copied. */
epikv_status epikv_read_slots(epikv_ctx* ctx, int32_t seq, int32_t kind, float* h_score,
                              int32_t* h_pos, int32_t cap, int32_t* h_n);

/* Debug/test read-back (synchronises), cfg.layer_budgets = 1 only: the
 * length n_l of layer `layer` of `seq` and the positions its slots hold, at
 * most `cap` of them. */
epikv_status epikv_read_layer_slots(epikv_ctx* ctx, int32_t seq, int32_t layer, int32_t* h_pos,
                                    int32_t cap, int32_t* h_n);

/* Synchronise the last stream used and return the cumulative counters. */
epikv_status epikv_get_stats(epikv_ctx* ctx, epikv_stats* out);

/* Synchronise; EPIKV_EDEVICE if the device error word is set, with its code
 * in *code (may be NULL); the word is cleared. */
epikv_status epikv_get_error(epikv_ctx* ctx, int32_t* code);

/* Lag-KV scores of positions 0..n-1 of one sequence, in one call that needs
 * no context and no device memory beyond its arguments.  The paper has no
 * counterpart to this entry point: it is for callers that cannot allocate
 * device memory -- a plugin inside an application whose memory pool owns the
 * whole GPU, an embedded caller without a device allocator, or a loop that
 * must never block on cudaMalloc -- and so cannot create the workspace that
 * epikv_init needs.  Its scores agree, to fp32 rounding, with the ones
 * epikv_score_update gives for the same tokens of a fresh sequence.
 *   kv         the caller's cache; slots 0..n-1 of `seq` hold positions 0..n-1
 *   L, H, d    layers, KV heads, head dim (d a power of two in [8, 256],
 *              H <= 32, H*d/8 <= 256)
 *   lag, lag_eps, window   as in epikv_config
 *   d_scores   device float [n]: the output
 * Working memory is a fixed 2 MiB array inside the library (every GPU that
 * loads the library holds it until the process exits), so n * 2 * L must not
 * exceed 524,288 (n <= 8,192 at L = 32): larger requests return EPIKV_EINVAL
 * and launch nothing.  The first call in each CUDA context looks the array's
 * address up (with that context current) and remembers it under the
 * context's unique id, so a context created again after cudaDeviceReset gets
 * a fresh lookup; make the first call in a context before any stream
 * capture.  All calls share the array: calls that overlap on the GPU
 * (unordered streams) race and must be avoided; calls ordered on one stream
 * are independent.  Slots the view does not map (a negative or out-of-range
 * block-table entry) are read as zero rows and are not reported.  A CUDA
 * error already pending on the calling thread is returned as EPIKV_ECUDA
 * before anything is launched, and left in place for its owner. */
epikv_status epikv_lagkv_score_noalloc(const epikv_kv_view* kv, int32_t seq, int32_t n,
                                       int32_t num_layers, int32_t num_kv_heads, int32_t head_dim,
                                       int32_t lag, float lag_eps, int32_t window, float* d_scores,
                                       cudaStream_t stream);

/* ------------------------------------------------------------------------
 * Beside eviction: putting new tokens into the cache and attending over it.
 *
 * After an eviction a token's slot is no longer its position: new rows go to
 * the slots behind the kept ones while the rotation goes on by position, and
 * attention runs over slots.  These calls take both, from device arrays that
 * the caller holds anyway (the lengths that epikv_step returns, the positions
 * that it counts).  They have a context of their own (epikv_attn_ctx), which
 * follows the conventions above: the caller's workspace, no allocation, no
 * synchronisation, EPIKV_EINVAL before anything is enqueued, a sticky device
 * error word.
 * ------------------------------------------------------------------------ */

/* What a cache row holds.
 *   BF16   H*d bf16 values, the rows of every call above
 *   E2M1   4 bits a value: for each head d/2 bytes of E2M1 codes (channel 2i in
 *          the low half of byte i), then for each head d/16 bytes of E4M3
 *          scales, one for every 16 channels; a channel is code * scale * the
 *          head's kv_scale.  4.5 bits a value.  The row is padded to
 *          epikv_cache_row's size.
 * Strides of a view count 2-byte units for both, so a 4-bit cache is described
 * by the same epikv_kv_view, and epikv_select, epikv_compact and epikv_step
 * (with the band kinds or WEIGHT, which do not read K and V) move its rows as they are:
 * their context is configured with the num_kv_heads and head_dim that
 * epikv_cache_row returns. */
enum { EPIKV_CACHE_BF16 = 0, EPIKV_CACHE_E2M1 = 1 };

/* Element types of epikv_rows. */
enum { EPIKV_TYPE_BF16 = 0, EPIKV_TYPE_F16 = 1, EPIKV_TYPE_F32 = 2 };

/* Which channels of a head form the rotated pairs: i and i + dim/2, or 2i and
 * 2i + 1.  Channels from dim on pass unchanged. */
enum { EPIKV_ROPE_HALF = 0, EPIKV_ROPE_INTERLEAVED = 1 };

/* How the frequencies theta^(-2i/dim) are changed for long contexts.
 *   LINEAR   divided by factor
 *   NTK      theta multiplied by factor^(dim/(dim-2))
 *   BYPARTS  freq * ((1-g)/factor + g), g = clamp((rot - low) / (high - low)),
 *            rot = original * freq / 2pi: the turns that the frequency makes
 *            over the original context.  The ramp is linear in turns, as Llama
 *            3.1's is; checkpoints whose ramp is linear over the frequency's
 *            index between two rounded ends (the usual YaRN code) need a table
 *            of their own in epikv_rope_view */
enum { EPIKV_ROPE_PLAIN = 0, EPIKV_ROPE_LINEAR = 1, EPIKV_ROPE_NTK = 2, EPIKV_ROPE_BYPARTS = 3 };

typedef struct {
  int32_t dim;              /* rotated channels of a head: even, >= 2 */
  float theta;              /* base of the frequencies, > 1 */
  int32_t scaling;          /* EPIKV_ROPE_PLAIN .. BYPARTS */
  float factor;             /* >= 1 (read unless PLAIN) */
  float low, high;          /* BYPARTS: 0 <= low < high */
  int32_t original;         /* BYPARTS: tokens of the original context, >= 1 */
  float magnitude;          /* cos and sin are multiplied by it (1: a pure rotation) */
} epikv_rope_config;

/* A table made once by epikv_rope_table (or by the caller): device float
 * [n_pos][dim/2][2], cos and sin of every position and frequency. */
typedef struct {
  const float* table;       /* 16-byte aligned */
  int32_t n_pos;
  int32_t dim;
  int32_t layout;           /* EPIKV_ROPE_HALF or INTERLEAVED */
} epikv_rope_view;

/* Heads of tokens, channels contiguous: element (token, head, channel) at
 * token*stride_token + head*stride_head + channel (strides in elements).  The
 * pointer and the strides are multiples of 16 bytes. */
typedef struct {
  void* ptr;
  int64_t stride_token;
  int64_t stride_head;
  int32_t type;             /* EPIKV_TYPE_* */
} epikv_rows;

typedef struct {
  int32_t max_seqs;         /* sequence ids are 0..max_seqs-1 */
  int32_t max_cache_tokens; /* cache slots per sequence */
  int32_t max_new_tokens;   /* new tokens per sequence and call, max */
  int32_t num_layers;
  int32_t num_heads;        /* query heads: a multiple of num_kv_heads; head h reads KV head
                             * h / (num_heads / num_kv_heads) */
  int32_t num_kv_heads;     /* 1..32 */
  int32_t head_dim;         /* 64, 128 or 256 */
  int32_t cache_format;     /* EPIKV_CACHE_* */
  float softmax_scale;      /* 0: 1/sqrt(head_dim) */
  const float* kv_scale;    /* E2M1: device float [2][num_layers][num_kv_heads], a positive scale of each
                             * head's keys, then values, which the E4M3 scales multiply (E4M3 reaches from
                             * 2^-9 to 448: heads whose values lie far from 1 need one); NULL: 1 */
} epikv_attn_config;

typedef struct epikv_attn_ctx epikv_attn_ctx;

/* The row of one token, layer and of K or V as the eviction calls see it:
 * *heads * *dim 2-byte units (for E2M1 the packed row, padded until it is such
 * a product).  EPIKV_EINVAL if no such row exists (over 2,048 units). */
epikv_status epikv_cache_row(int32_t num_kv_heads, int32_t head_dim, int32_t cache_format, int32_t* heads,
                             int32_t* dim);

/* Bytes of device workspace for cfg (0 if cfg is invalid): room for the partial results of rows that are split between SMs.  32
 * query and 8 KV heads of 128: 10 MB for one new token a sequence, 20 for 8, 40 from 64 on (epikv_attention_chunk's). */
size_t epikv_attn_workspace_bytes(const epikv_attn_config* cfg);

/* Create a context over a caller-allocated workspace (256-byte aligned). */
epikv_status epikv_attn_init(epikv_attn_ctx** out, const epikv_attn_config* cfg, void* d_workspace,
                             size_t workspace_bytes, cudaStream_t stream);

/* Fill d_table, float [n_pos][dim/2][2] (angles in 64 bits, rounded once). */
epikv_status epikv_rope_table(const epikv_rope_config* cfg, int32_t n_pos, float* d_table, cudaStream_t stream);

/* Rotate n_tokens x n_heads heads of ctx's head_dim by their positions
 * d_pos [n_tokens] (32-bit arithmetic, rounded once).  inverse = 1 turns the
 * other way, which is the rotation's gradient.  out may be x.  A token whose
 * position is outside the table is skipped (EPIKV_DEV_POSITION). */
epikv_status epikv_rope(epikv_attn_ctx* ctx, int32_t n_tokens, int32_t n_heads, const epikv_rows* x,
                        const epikv_rows* out, const int32_t* d_pos, const epikv_rope_view* rope, int32_t inverse,
                        cudaStream_t stream);

/* Append the new tokens of a batch to one layer's cache.
 *   d_seq_ids, d_cu_new, max_new   as in epikv_score_update
 *   d_len [n_seq] (every len_stride-th int32 of it): the slots that each entry
 *         holds before the call; token i of entry b goes to slot d_len[b] + i.
 *         A per-layer length array is read with its layer stride.
 *   d_pos [n_seq]  position of each entry's first new token; may be NULL if
 *                  rope is NULL (no rotation)
 *   q, q_out       bf16 queries [total_new][num_heads][d] and where they go,
 *                  rotated (may be the same rows); both NULL: no queries
 *   k, v           bf16 [total_new][num_kv_heads][d]
 * Keys are rotated in 32 bits and rounded to bf16; a 4-bit cache then takes
 * them to 4 bits: for 16 channels, scale = E4M3(min(448, max|x| / 6)), code =
 * E2M1(x / scale), to nearest even, saturating (NaN: the 16 channels read as
 * NaN).  Nothing but the new tokens' rows is written. */
epikv_status epikv_append(epikv_attn_ctx* ctx, int32_t layer, int32_t n_seq, const int32_t* d_seq_ids,
                          const int32_t* d_cu_new, int32_t max_new, const int32_t* d_len, int32_t len_stride,
                          const int32_t* d_pos, const epikv_rows* q, const epikv_rows* q_out, const epikv_rows* k,
                          const epikv_rows* v, const epikv_rope_view* rope, const epikv_kv_view* kv,
                          cudaStream_t stream);

/* Attention of the batch's queries over one layer's cache: bf16 queries and
 * outputs [total_new][num_heads][d], statistics in 32 bits.
 *   d_len     as in epikv_append: the slots held before the new tokens
 *   causal    1: the new tokens' rows are in the cache, query i of entry b
 *             reads slots 0 .. d_len[b] + i.  0: every query reads the d_len[b]
 *             slots (a shared prefix; join with d_lse)
 *   d_lse     float [total_new][num_heads] or NULL: log of the sum of exponentials
 * A probability is held in 16 bits (bf16 cache; below 2^-126 of the row's largest
 * it is 0) or, over a 4-bit cache, in 11 bits down to 2^-21 of about the row's
 * largest and to within 2^-32 of it below: a channel to which only slots of less
 * weight contribute keeps that absolute accuracy, not the relative one.
 * A row that sees no slot, or only slots of score -infinity, gives zeros and
 * -infinity.  An infinite value in a slot that a row sees is the row's output in
 * that channel, however small its probability (NaN beside one of the other sign,
 * or where the slot's score is -infinity).  Slots that a row does not
 * see do not reach it, whatever they hold (memory of the view up to the next
 * multiple of 16 slots may be read: of a block, or of the max_cache_tokens slots
 * of a contiguous sequence; where stride_seq / stride_token is between 1 and
 * max_cache_tokens - 1, only slots that are seen, by a slower way).
 * The work is counted in 32 bits, in tiles of 16 slots or more: an entry has one
 * for every 16 slots that a run of 8 to 32 of its query rows (tokens times
 * num_heads / num_kv_heads) sees, for each group of 8 KV heads (4 at head_dim
 * 256).  The entry that takes a call's sum to 2^31 - 1 and those behind it are
 * skipped (EPIKV_DEV_CAPACITY).  A prompt of 500,000 tokens with 32 query and 8
 * KV heads of 128 has 1.95 * 10^9 tiles. */
epikv_status epikv_attention(epikv_attn_ctx* ctx, int32_t layer, int32_t n_seq, const int32_t* d_seq_ids,
                             const int32_t* d_cu_new, int32_t max_new, const int32_t* d_len, int32_t len_stride,
                             int32_t causal, const epikv_rows* q, const epikv_rows* out, float* d_lse,
                             const epikv_kv_view* kv, cudaStream_t stream);

/* The same attention for many query rows: chunks of prompts, drafts, turns, of one token or more a sequence.
 * Arguments, order of the slots, what a row sees, empty rows and d_lse as in epikv_attention; nothing is split
 * between calls, so a prompt may be taken in by pieces.  out may not overlap q.  It reads the cache once for 256 rows (tokens times
 * num_heads / num_kv_heads; 128 at head_dim 256) where epikv_attention does so for 8 to 32.  It is the faster one from 16 to 64
 * such rows of an entry on; a single token of many sequences is slower here (64 sequences over a bf16 cache 156 us and 132, over
 * a 4-bit one 213 and 61).
 * A probability is held in 8 significant bits over a bf16 cache, where epikv_attention holds 16: the outputs' error against
 * 64 bits is 0.0023 of their size, there 0.0017, which their own rounding gives.  Over a 4-bit cache it is held as in
 * epikv_attention: in 11 bits down to 2^-21 of about the row's largest and to within 2^-32 of it below.  Sums, maxima and d_lse
 * are held in 32 bits.  In a channel where a slot that a row sees holds an infinity or a NaN the row's output is infinite or NaN
 * (in epikv_attention it is the infinity).  Slots that a row does not see do not reach it, whatever they hold (memory
 * of the view behind them may be read, up to the end of the block, or of the max_cache_tokens slots of a contiguous
 * sequence; where stride_seq / stride_token is between 1 and max_cache_tokens - 1, only slots that are seen).
 * Where an item of rows is cut between the SMs depends on the whole batch, and with it how a row's parts are rounded: the
 * same batch gives the same bits, an entry of another batch may differ in its last ones.  The work is counted in 32 bits,
 * in tiles of 128 slots (64 at head_dim 256) of an item and four more for each item; the entry that takes the sum to 2^31 - 1
 * and those behind it are skipped (EPIKV_DEV_CAPACITY). */
epikv_status epikv_attention_chunk(epikv_attn_ctx* ctx, int32_t layer, int32_t n_seq, const int32_t* d_seq_ids,
                                   const int32_t* d_cu_new, int32_t max_new, const int32_t* d_len, int32_t len_stride,
                                   int32_t causal, const epikv_rows* q, const epikv_rows* out, float* d_lse,
                                   const epikv_kv_view* kv, cudaStream_t stream);

/* A number for every slot and KV head: device float, that of (sequence, head, slot) at seq*stride_seq +
 * head*stride_head + slot (strides in elements; the caller keeps the rows of max_cache_tokens slots apart). */
typedef struct {
  float* ptr;               /* 4-byte aligned */
  int64_t stride_seq;
  int64_t stride_head;
} epikv_weights;

/* What each slot of one layer's cache receives of the attention of the batch's queries: for KV head h,
 *   sum over the entry's new tokens and the query heads that read h of exp(scale q.k - lse)
 * over the queries that see the slot.  Sums in 32 bits and in an order that the batch's sizes give: eight partial sums, each of
 * every eighth row (a token's query heads, then the next token's), added up where the batch's work is cut.  The same batch
 * gives the same bits.
 *   d_seq_ids .. causal, q, kv   as in the attention call that gave d_lse
 *   last      only the last so many of each entry's new tokens count; 0: all of them
 *   d_lse     float [total_new][num_heads]: the attention's, or its joined parts'
 *   add       0: store, 1: add to what stands there (the next layer of a step)
 *   w         written for the entries' sequences and all KV heads, slots 0 .. d_len + n - 1 (causal = 0: 0 ..
 *             d_len - 1), nothing else.  An entry without new tokens stores zeros
 * A query whose lse is minus infinity saw nothing and gives nothing; a NaN in what a slot receives is NaN there.
 * A slot outside the view receives nothing (EPIKV_DEV_SLOT).  The work is counted as in epikv_attention_chunk: for each KV head
 * and 256 slots (128 at head_dim 256) the steps of 128 rows that see some of them and four more, or one where no entry has more
 * than 16 rows that count. */
epikv_status epikv_attention_weights(epikv_attn_ctx* ctx, int32_t layer, int32_t n_seq, const int32_t* d_seq_ids,
                                     const int32_t* d_cu_new, int32_t max_new, const int32_t* d_len, int32_t len_stride,
                                     int32_t causal, int32_t last, const epikv_rows* q, const float* d_lse, int32_t add,
                                     const epikv_weights* w, const epikv_kv_view* kv, cudaStream_t stream);

/* Add a step's weights to the WEIGHT scores of a context's slots (its score_kinds hold EPIKV_SCORE_WEIGHT): for slots
 * 0 .. n_cache-1 of each entry's sequence
 *   score = decay * score + sum over h = 0 .. n_heads-1 of w(seq, h, slot)
 * (32 bits, each product and sum rounded, heads first, in order).  decay is in 0 .. 1; 1 accumulates for good.
 * Belongs between epikv_score_update, which registers the step's tokens, and epikv_select; the scores move with their
 * tokens from then on, and epikv_read_slots returns them.  An entry whose eviction is selected but not yet compacted is
 * reported (EPIKV_DEV_KEPT) and keeps its scores: they stand by its new slots already. */
epikv_status epikv_weigh(epikv_ctx* ctx, int32_t n_seq, const int32_t* d_seq_ids, const epikv_weights* w, int32_t n_heads,
                         float decay, cudaStream_t stream);

/* Read n_rows rows of one layer back as bf16 [n_rows][num_kv_heads][d]: slot
 * d_slots[i] of sequence d_seqs[i].  k or v may be NULL.  Rows outside the view
 * are skipped (EPIKV_DEV_SLOT). */
epikv_status epikv_cache_read(epikv_attn_ctx* ctx, int32_t layer, int32_t n_rows, const int32_t* d_seqs,
                              const int32_t* d_slots, const epikv_rows* k, const epikv_rows* v,
                              const epikv_kv_view* kv, cudaStream_t stream);

/* As epikv_get_error. */
epikv_status epikv_attn_get_error(epikv_attn_ctx* ctx, int32_t* code);

void epikv_attn_destroy(epikv_attn_ctx* ctx);

void epikv_destroy(epikv_ctx* ctx);
const char* epikv_status_string(epikv_status s);

#ifdef __cplusplus
}
#endif
#endif /* EPIKV_H_ */
