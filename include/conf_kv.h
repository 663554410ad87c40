/*
 * conf_kv.h -- C ABI of the Conf-KV per-decode-step library for AMD MI355X (gfx950).
 *
 * The library keeps, for every unit (layer, batch, kv-head), a position-sorted KV
 * cache whose oldest tokens are INT8 (per-token, per-kv-head fp16 absmax scales) and
 * whose newest tokens are FP16, plus per-slot metadata (original position, fp32 EMA of
 * attention mass).  One decode step is
 *
 *     for every layer:  conf_kv_attend          (append + attention + mass EMA)
 *     once:             conf_kv_step            (confidence -> tight/loose budget)
 *     once:             conf_kv_evict_compact   (rank, evict, compact, demote)
 *
 * and, where a program wants them, conf_kv_attend_pages and conf_kv_load_pages for a prompt that lies in pages,
 * conf_kv_attend_diff for models with differential attention, conf_kv_prepare_qkv in front of the attention (projection rows ->
 * queries, keys, values), conf_kv_attend_shared in its place (a prefix that sequences share) and
 * conf_kv_constrain in front of conf_kv_step (penalties, biases, grammar masks).
 *
 * The first three are the paper's Algorithm 1 with the append moved in front of the step's own
 * attention (a decode query attends to its own key).
 *
 * Conventions
 *   - "dev" pointers are device memory owned by the CALLER and valid until
 *     conf_kv_destroy; "host" pointers are ordinary host memory.  The library never
 *     allocates or frees device memory.
 *   - The hot calls (those above) only enqueue kernels on the given stream; they never
 *     synchronise.  Lengths and budgets live on the device; the host keeps upper bounds.
 *   - A handle is driven from one host thread, on one stream at a time.
 *   - A whole decode step (the calls above, on one stream) may be recorded into a HIP graph
 *     and replayed: the calls enqueue kernels only (no copies, no memset nodes), and what
 *     changes from step to step (lengths, ring heads, budgets, the positions appended tokens
 *     get, the tags the in-kernel waits compare) lives on the device and is advanced by the
 *     kernels themselves.  The kernel arguments do hold the launch shapes, which the host
 *     derives from upper bounds of the lengths: call conf_kv_static_plan(h, 1) before
 *     recording, so that the shapes cover every later step, and record only after one step has
 *     run outside the graph (first launches set kernel attributes).  The tensors the recorded
 *     calls read and write are the ones given at recording time.  conf_kv_step_static keeps its
 *     tag on the host and is not replayable.
 *   - At most 2^23 attention or confidence launches may lie between two
 *     conf_kv_evict_compact calls (CONF_KV_ERR_BAD_STATE beyond that).
 *   - Every function returns CONF_KV_OK (0) or a negative conf_kv_status; nothing throws.
 *   - Tensors are dense, row-major, in the index order written next to each argument.
 *   - fp16 data is IEEE binary16; "int8" codes are two's complement in [-127, 127].
 */
#ifndef CONF_KV_H
#define CONF_KV_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct conf_kv_handle conf_kv_handle;
typedef void *conf_kv_stream;            /* a hipStream_t; NULL = the default stream */

typedef enum conf_kv_status {
  CONF_KV_OK = 0,
  CONF_KV_ERR_INVALID_ARG = -1,  /* null pointer, negative size, misaligned buffer            */
  CONF_KV_ERR_BAD_SHAPE = -2,    /* a config field outside what the kernels are built for     */
  CONF_KV_ERR_BAD_LAYER = -3,    /* layer index outside [0, n_layers)                          */
  CONF_KV_ERR_CAPACITY = -4,     /* the operation would need more slots than `capacity`       */
  CONF_KV_ERR_BAD_STATE = -5,    /* call order violated (see each function)                    */
  CONF_KV_ERR_HIP = -6,          /* a HIP call failed; see conf_kv_last_hip_error             */
  CONF_KV_ERR_DEVICE = -7        /* a kernel reported an internal error (bounded wait expired) */
} conf_kv_status;

/*
 * Problem statement of Algorithm 1 (its REQUIRE line: thresholds tau, budgets
 * N_high / N_low, protected window P, ranker weight alpha, FP16 window W) plus the
 * shape of the model's attention.  Weights of Eq. 1 are (w_entropy, w_margin, w_top).
 */
typedef struct conf_kv_config {
  int32_t n_layers;          /* L  >= 1                                                        */
  int32_t batch;             /* B  >= 1 sequences, all at the same decode position             */
  int32_t n_q_heads;         /* Hq, a multiple of n_kv_heads; group G = Hq / Hkv in 1..8
                                (1..16 at head_dim 128)                                        */
  int32_t n_kv_heads;        /* Hkv                                                            */
  int32_t head_dim;          /* D in {64, 128}                                                 */
  int32_t vocab;             /* V >= 2                                                         */
  int32_t capacity;          /* slots per unit; a multiple of 16; must exceed every budget     */
  int32_t fp16_window;       /* W >= 0: newest W retained tokens stay FP16; < 0: FP16-only     */
  int32_t protected_window;  /* P >= 0: the newest P tokens are never evicted                  */
  float tau;                 /* tight budget when c >= tau (paper: 0.7)                        */
  float alpha;               /* ranker weight on attention mass (paper: 0.65)                  */
  float ema_decay;           /* lambda of the mass EMA (paper: 0.9)                            */
  float sm_scale;            /* softmax scale, usually 1/sqrt(D)                               */
  float w_entropy, w_margin, w_top; /* Eq. 1 weights (paper: 0.4, 0.3, 0.3)                    */
  const int32_t *n_tight;    /* host [L]: N_high per layer (budget on confident steps)         */
  const int32_t *n_loose;    /* host [L]: N_low  per layer; n_tight[l] <= n_loose[l]           */
  /* Variants of the ranker (the paper's experimental setup and its literal per-layer
   * bookkeeping).  All zeros except mass_gain < 0 give the method as described above. */
  float mass_gain;           /* weight of a step's mass: a <- ema_decay a + mass_gain A;
                                negative = 1 - ema_decay (the paper's EMA); (ema_decay,
                                mass_gain) = (1, 1) is the running sum of the mass         */
  int32_t ranker;            /* conf_kv_ranker                                                 */
  int32_t rank_scope;        /* conf_kv_rank_scope                                             */
  uint64_t ranker_seed;      /* CONF_KV_RANKER_RANDOM: seed of its counter-based draws         */
  int32_t scale_mode;        /* conf_kv_scale_mode: granularity of the INT8 scales             */
  int32_t max_chunk;         /* most tokens one conf_kv_attend_chunk / conf_kv_observe call may
                                carry; 0 or 1 = single-token calls only.  Above 1: head_dim 128
                                and max_chunk * (n_q_heads / n_kv_heads) <= 128 query rows per
                                kv-head; beyond 16 rows per-token scales only                  */
  int32_t evict_page;        /* 0 or 1: tokens are evicted one by one.  g > 1 (at most 1024):
                                coarsened eviction for paged layouts (the remedy the paper names
                                in "Compatibility with serving systems" and "Limitations" for
                                partially dead blocks; it defines no rule) -- a page is the live slots
                                whose original positions share floor(position / g); a page
                                goes whole or not at all, and only when none of its slots lies
                                in the protected window; pages are ranked by the mean of their
                                slots' scores and go lowest first, older first among equal
                                means, until the length is at most the budget (it may end up to
                                g - 1 below it) or no page that can go is left (up to g - 1
                                slots over max(budget, protected_window) then remain).
                                capacity must hold max(n_loose, protected_window + g - 1) plus
                                the appended tokens                                            */
  int32_t layout;            /* conf_kv_layout: where the INT8 slots of a unit live              */
  int32_t max_shared;        /* most tokens of a shared prefix that conf_kv_attend_shared may be given (sizes the scratch
                                buffer: up to 64 partial results per query row), up to 2^30; 0: none         */
  int32_t max_paged;         /* most tokens of a sequence in the pages that conf_kv_attend_pages may be given (above 128: room
                                for 65536 partial results in the scratch buffer), up to 2^30; 0: none     */
} conf_kv_config;

typedef enum conf_kv_layout {
  CONF_KV_LAYOUT_CONTIGUOUS = 0, /* the paper's layout ("Cache manager": gather survivors into
                                    contiguous storage): slots in position order in one ring per
                                    plane; an eviction moves the rows on the cheaper side of
                                    the holes                                                    */
  CONF_KV_LAYOUT_PAGED = 1       /* the alternative "Compatibility with serving systems" and
                                    "Limitations" name for paged serving stacks: the INT8 slots
                                    of a unit live in pages of evict_page slots reached through a
                                    per-unit block table; a page holds the tokens whose original
                                    positions share floor(position / evict_page); attention reads
                                    rows through the table; evicting a page edits the table and
                                    moves no row.  Needs coarsened eviction (evict_page a power
                                    of two, 8 .. 1024), a mixed cache with fp16_window <=
                                    protected_window (so that only whole INT8 pages can go),
                                    per-token scales, the per-kv-head ranking scope, a group of
                                    2 .. 8 query heads and single-token attention calls;
                                    conf_kv_import is not available.  conf_kv_export returns the
                                    same position-sorted view as under the contiguous layout     */
} conf_kv_layout;

typedef enum conf_kv_scale_mode {
  CONF_KV_SCALES_TOKEN = 0,     /* one scale per token and kv-head (absmax over the channels),
                                   separately for K and V                                      */
  CONF_KV_SCALES_CHANNEL = 1    /* the granularity "Tiled attention and mixed precision" names:
                                   one scale per (kv-head, channel), separately for K and V,
                                   s_d = fl16(fl32(max_t |x_{t,d}| / 127)) over ALL T0 prompt
                                   tokens of conf_kv_load_prefill (those that stay FP16
                                   included), fixed from then on; later tokens saturate at
                                   +-127.  Attention folds the K scales into the query and the
                                   V scales into the output.  Needs D = 128 and a mixed cache
                                   (fp16_window >= 0); a layer must be given its scales
                                   (conf_kv_load_prefill or conf_kv_import) before its first
                                   conf_kv_evict_compact, else CONF_KV_ERR_BAD_STATE           */
} conf_kv_scale_mode;

typedef enum conf_kv_ranker {
  CONF_KV_RANKER_COMPOSITE = 0, /* s = alpha * minmax(mass) + (1 - alpha) * minmax(position)  */
  CONF_KV_RANKER_RANDOM = 1     /* s = top 53 bits of splitmix64(seed + unit * 2^32 + position)
                                   as a fraction: which token goes is random, how many go is
                                   still the budget rule's (matched-rate isolation); unit =
                                   (layer * B + b) * Hkv + kv_head, or 2^40 + layer * B + b in
                                   layer scope                                                 */
} conf_kv_ranker;

typedef enum conf_kv_rank_scope {
  CONF_KV_SCOPE_KV_HEAD = 0,    /* one importance value and one kept set per (layer, kv-head)  */
  CONF_KV_SCOPE_LAYER = 1       /* one kept set per (layer, sequence): the importance of a
                                   token is its mass summed over the kv-heads (the head
                                   average up to a factor that min-max removes); every kv-head
                                   of a sequence must hold the same positions                  */
} conf_kv_rank_scope;

typedef struct conf_kv_stats {
  uint64_t evicted;          /* tokens evicted, summed over units                              */
  uint64_t demoted;          /* tokens quantised FP16 -> INT8 by conf_kv_evict_compact         */
  uint64_t tight_steps;      /* sequence-steps that selected the tight budget                  */
  uint64_t loose_steps;      /* sequence-steps that selected the loose budget                  */
  uint64_t device_errors;    /* bounded waits that expired inside kernels, and launches whose plan
                                did not fit what they found (0 in a healthy run)               */
  uint64_t compact_bytes;    /* bytes read + written by the compaction's in-place row moves    */
} conf_kv_stats;

/* Environment variables read once by conf_kv_create (test and measurement hooks; none is
 * needed in normal use): CONF_KV_SPLITS=n asks for n workgroups per unit in conf_kv_attend
 * instead of the planned number (clamped to what the unit's length allows);
 * CONF_KV_TWO_LAUNCH=1 forces the two-launch form of conf_kv_attend; CONF_KV_SHARED_ROWS=1/2/4 the number of
 * wavefronts side by side along the rows of conf_kv_attend_shared's prefix kernel; CONF_KV_NO_MFMA=1 (read
 * at the first plan of the process) keeps every shape on the vector-ALU streaming body (conf_kv_attend_diff then has
 * no kernel: CONF_KV_ERR_BAD_SHAPE);
 * CONF_KV_SPIN_LIMIT=n bounds the in-kernel waits for other workgroups to n polls (default
 * 400000, about 0.4 s; an expired wait ends the kernel early and counts a device error);
 * CONF_KV_TEST_WITHHOLD=1 makes split 0 of every unit (conf_kv_attend) and chunk 0 of every
 * logit row (conf_kv_step) keep their published words to themselves, so that the waits of the
 * others expire (the kernels still end normally; tests of the expiry path);
 * CONF_KV_GRID_KV_MAJOR=0/1 overrides the order of the attention grid (kv-heads first puts all
 * splits of a unit on one XCD and is the default when the number of kv-heads is a multiple of 8);
 * CONF_KV_EVICT_ONE=0 keeps conf_kv_evict_compact in its separate launches (ranking, compaction,
 * demotion) where a decode loop on few units otherwise takes one launch for all of it;
 * CONF_KV_COMPACT_PAIRED=0/1 (read at every conf_kv_evict_compact) forces one of the two grid
 * shapes of the compaction kernel, which is otherwise chosen by the number of units;
 * CONF_KV_TEST_TAG_BASE=n starts the device-side tag bases (see conf_kv_tag_state) at n instead
 * of 0, so that a test reaches the clearing of the exchange words in a few steps. */

/* Bytes of device memory the caller must provide for the cache state and for scratch
 * (tagged exchange words of the splits and chunks, ranking work arrays).  0 on an invalid config. */
size_t conf_kv_state_bytes(const conf_kv_config *cfg);
size_t conf_kv_scratch_bytes(const conf_kv_config *cfg);

/* Validates cfg, copies it, lays the cache out inside dev_state (256-byte aligned, at
 * least conf_kv_state_bytes) and dev_scratch (likewise), zeroes lengths / counters /
 * scratch with synchronous HIP calls on the current device, and sets every budget to the
 * loose one.  All units start empty.  On error *out is NULL. */
int conf_kv_create(conf_kv_handle **out, const conf_kv_config *cfg, void *dev_state,
                   void *dev_scratch);

/* Pyramidal per-layer budgets ("Pyramidal layer budgets": N(l) = max(N_min,
 * N(0) * beta^(l / L))), floored to integers, for filling n_tight / n_loose: host_out int32
 * [n_layers].  The paper uses beta = 0.5 and N_min = 96.  Pure host arithmetic in double;
 * CONF_KV_ERR_INVALID_ARG on n_layers < 1, n0 < 1, n_min < 1 or beta outside (0, 1]. */
int conf_kv_pyramid_budgets(int32_t n0, int32_t n_layers, double beta, int32_t n_min,
                            int32_t *host_out);

/* Frees the host-side handle only (device buffers belong to the caller). */
int conf_kv_destroy(conf_kv_handle *h);

/* Replaces the cache of one layer by T0 prompt tokens at positions 0..T0-1
 * (Algorithm 1's input cache).  dev_k16 / dev_v16: fp16 [B][Hkv][T0][D], 16-byte aligned
 * (CONF_KV_ERR_INVALID_ARG otherwise).
 * dev_ema0: fp32 [B][Hkv][T0] initial EMA importance, or NULL for zeros.
 * All but the newest W tokens are quantised to INT8 ("Tiled attention and mixed
 * precision": symmetric, scale = max|x|/127, per token and kv-head, or per kv-head and
 * channel over the T0 prompt tokens: conf_kv_scale_mode).
 * 0 <= T0 <= capacity - 1, else CONF_KV_ERR_CAPACITY.  Enqueues on `stream`. */
int conf_kv_load_prefill(conf_kv_handle *h, int32_t layer, const void *dev_k16,
                         const void *dev_v16, int32_t T0, const float *dev_ema0,
                         conf_kv_stream stream);

/*
 * Decode attention of one layer with the importance update fused in
 * (Algorithm 1: forward pass attention, "update EMA attention metadata", "append new K/V
 * in FP16"; "Tiled attention and mixed precision"; "Budget and ranker").
 *   1. appends (k_new, v_new) in FP16 at the next position with EMA 0;
 *   2. out[b][h] = softmax_i(sm_scale * q[b][h] . K_i) V_i over ALL stored slots of the
 *      unit (b, h / G), K_i/V_i being the fp16 value or int8 code * fp16 scale, computed
 *      as split-K blockwise online softmax with fp32 accumulation;
 *   3. per slot, A_i = sum over the G query heads of the exact normalised probability
 *      (so sum_i A_i = G), then ema_i <- lambda * ema_i + (1 - lambda) * A_i.
 * dev_q16: fp16 [B][Hq][D]; dev_knew16 / dev_vnew16: fp16 [B][Hkv][D]; dev_out16: fp16
 * [B][Hq][D], written.  All 16-byte aligned.
 * Exactly one conf_kv_attend (conf_kv_attend_chunk, conf_kv_attend_shared, conf_kv_attend_diff) per layer between two conf_kv_evict_compact calls
 * (CONF_KV_ERR_BAD_STATE otherwise); CONF_KV_ERR_CAPACITY, before anything is launched,
 * if the unit could already hold `capacity` tokens.
 * The workgroups that share a unit exchange partial results inside the launch, so the launch
 * is sized to be resident on the device all at once.  Kernels that do not wait for one another,
 * running at the same time, only delay it (its waits are bounded at several hundred
 * milliseconds); a wait that does expire leaves the call's outputs undefined and is reported by
 * conf_kv_counters (device_errors, CONF_KV_ERR_DEVICE).  Two launches of this kind on two streams
 * (other handles: conf_kv_attend, conf_kv_attend_chunk, conf_kv_attend_shared, conf_kv_attend_diff, conf_kv_observe, conf_kv_step) may each
 * hold compute units that the other's workgroups wait for if together they need more than the
 * device has; order such calls by events where their grids are large.  A call of this function
 * takes up to one workgroup per compute unit.  Calls of more than 16 / G tokens
 * (conf_kv_attend_chunk, conf_kv_observe) take more than half of them only while a workgroup has
 * 256 slots and a unit at most eight workgroups, or, with a multiple of eight kv-heads, where two
 * such calls do not stop each other.
 */
int conf_kv_attend(conf_kv_handle *h, int32_t layer, const void *dev_q16, const void *dev_knew16,
                   const void *dev_vnew16, void *dev_out16, conf_kv_stream stream);

/* Several consecutive tokens of every sequence in one call (a chunk of a prompt, or decode
 * tokens that are all kept; "Compatibility with serving systems" names such multi-token
 * steps): 1 <= tq <= max_chunk.  Defined as tq conf_kv_attend calls without eviction in
 * between: token t gets position p0 + t, query t attends the cache and the chunk's tokens
 * 0 .. t (causal), and the importance follows a <- lambda a + gain A_t once per query, i.e.
 * a_i <- lambda^tq a_i + gain * sum_t lambda^(tq-1-t) A_{t,i}, stored once.  The keys and
 * values of the cache are read once for all tq queries.
 * dev_q16 / dev_out16: fp16 [B][tq][Hq][D]; dev_knew16 / dev_vnew16: fp16 [B][tq][Hkv][D].
 * The following conf_kv_evict_compact commits all tq appends.  Same errors as conf_kv_attend;
 * tq outside 1 .. max(1, max_chunk) is CONF_KV_ERR_INVALID_ARG. */
int conf_kv_attend_chunk(conf_kv_handle *h, int32_t layer, int32_t tq, const void *dev_q16,
                         const void *dev_knew16, const void *dev_vnew16, void *dev_out16,
                         conf_kv_stream stream);

/* A prefix that sequences share (a system prompt, a document that many questions are asked about): its keys, rotated, and
 * values, stored once for the whole batch, in no cache and in no budget. */
typedef struct conf_kv_prefix {
  const void *dev_k16;       /* fp16 [Hkv][tokens][D], kv-heads head_stride values apart                        */
  const void *dev_v16;       /* the same                                                                       */
  int64_t head_stride;       /* >= tokens * D, a multiple of 8                                                 */
  int32_t tokens;            /* 0 .. max_shared; 0: the call is conf_kv_attend_chunk's                         */
  const int32_t *dev_seen;   /* int32 [B]: sequence b sees the first dev_seen[b] of them (held within 0 .. tokens;
                                0: none); NULL: all see all                                                    */
} conf_kv_prefix;

/* conf_kv_attend_chunk for sequences behind a shared prefix: tokens of the call attend what they see of the prefix, the
 * cache and the call's own tokens up to themselves, in one softmax,
 *     out[b][t][h] = sum_i p_i V_i,   p = softmax over prefix and cache of sm_scale * q . K_i,
 * and the importance of the cached slots follows the probabilities of that softmax (what goes to the prefix goes to no slot:
 * sum_i A_i = G minus the prefix's share).  The prefix's keys and values are read once for the whole batch; one that is infinite
 * or NaN shows in the sequences that see its token and in no other.  Tensors, errors
 * and rules of conf_kv_attend_chunk (tq = 1: of conf_kv_attend); tq * n_q_heads / n_kv_heads at most 16, and more than
 * max_shared tokens, a null or misaligned prefix are CONF_KV_ERR_INVALID_ARG.  Prefix tensors are 16-byte aligned.
 * Positions are the caller's affair: the handle's count the cache only (conf_kv_prepare_qkv's `first` adds the prefix).
 * conf_kv_observe* see the cache alone: the importance they give sums to G per query, that of a step behind a prefix to G minus
 * the prefix's share, so slots that carry both stand higher than a step would put them until the average has moved on (a lower
 * start can be handed to conf_kv_load_prefill instead).  A recorded call keeps the prefix's place and length and reads dev_seen anew. */
int conf_kv_attend_shared(conf_kv_handle *h, int32_t layer, int32_t tq, const conf_kv_prefix *prefix, const void *dev_q16,
                          const void *dev_knew16, const void *dev_vnew16, void *dev_out16, conf_kv_stream stream);

/* conf_kv_attend_chunk with differential attention: heads 2 j and 2 j + 1 of a kv-head's group are the two maps of pair j, over the
 * pair's keys and values, and the output is their difference,
 *     out[b][t][j] = sum_i w_i V_i,   w_i = p_i - lambda[b][t][j] p'_i,
 * one rounding at its end; importance is the size of the weight that a slot's value had, A_i = sum_j |w_i| (of one query; queries
 * of a call as in conf_kv_attend_chunk).  Tensors, errors and rules of conf_kv_attend_chunk (tq = 1: of conf_kv_attend) but for dev_out16,
 * fp16 [B][tq][Hq / 2][D], and dev_lambda, fp32 [B][tq][Hq / 2] with sequences batch_stride and tokens token_stride values apart
 * (0: the same weights for all).  An odd group, tq * n_q_heads / n_kv_heads above 16 and an output that overlaps what is read are
 * CONF_KV_ERR_INVALID_ARG.
 * conf_kv_observe* see single maps: the importance they give sums to G per query, more than a step's here. */
int conf_kv_attend_diff(conf_kv_handle *h, int32_t layer, int32_t tq, const float *dev_lambda, int64_t batch_stride,
                        int64_t token_stride, const void *dev_q16, const void *dev_knew16, const void *dev_vnew16, void *dev_out16,
                        conf_kv_stream stream);

/* A paged FP16 cache of the caller's, in which prompts are kept while they are worked off: the rows of token t of sequence b
 * lie in page table[b][t / page_tokens], slot t % page_tokens, kv-head g's at page * page_stride + slot * token_stride +
 * g * head_stride (so a page may be [slots][Hkv][D] or [Hkv][slots][D], and keys and values may take turns).  Entries that a
 * sequence's tokens do not reach are not used.  An entry outside 0 .. n_pages - 1 where a token is: its rows are
 * taken from some page, and what would be written there is not written. */
typedef struct conf_kv_pages {
  void *dev_k16;             /* fp16, heads of D values, 16-byte aligned                                        */
  void *dev_v16;             /* the same                                                                       */
  int64_t page_stride, token_stride, head_stride;   /* in values, multiples of 8; rows do not overlap              */
  int32_t page_tokens;       /* a power of two, 8 .. 2^20                                                      */
  int32_t n_pages;           /* pages there are, 1 .. 2^30                                                     */
  const int32_t *dev_table;  /* int32 [B][max_pages], rows table_stride entries apart                          */
  int64_t table_stride;      /* >= max_pages                                                                   */
  int32_t max_pages;         /* entries per sequence, >= 1; max_pages * page_tokens at most 2^30                */
} conf_kv_pages;

/* New tokens of every sequence: rows start .. start + new - 1 of the row tensors, behind `context` tokens that the pages hold. */
typedef struct conf_kv_chunk {
  int32_t tokens;            /* most new tokens of a sequence, >= 0                                             */
  int32_t rows;              /* rows of the row tensors                                                        */
  const int32_t *dev_starts; /* int32 [B]; NULL: b * tokens (rows >= B * tokens)                                */
  const int32_t *dev_new;    /* int32 [B], held within 0 .. tokens, within the rows and within the pages' room;
                                NULL: `tokens` each                                                            */
  const int32_t *dev_context;/* int32 [B], held within 0 .. max_pages * page_tokens                             */
  const void *dev_q16;       /* fp16 [rows][Hq][D]                                                             */
  const void *dev_knew16;    /* fp16 [rows][Hkv][D], or NULL with dev_vnew16: the pages hold the new tokens too  */
  const void *dev_vnew16;
  void *dev_out16;           /* fp16 [rows][Hq][D], or [rows][Hq / 2][D] with dev_lambda; written               */
  const float *dev_lambda;   /* fp32 [rows][Hq / 2], rows lambda_stride values apart, or NULL                   */
  int64_t lambda_stride;     /* >= 0; 0: the same weights for every row                                        */
} conf_kv_chunk;

/*
 * Attention of a chunk of new tokens over a paged cache, of any length per sequence: a prompt's chunks, single tokens and
 * sequences without new tokens in one call.  New keys and values go to their pages (tokens context .. context + new - 1), and
 *     out[start + t][h] = sum_i p_i V_i,   p = softmax over tokens i <= context + t of sm_scale * q . K_i
 * with float32 accumulation.  With dev_lambda, differential attention: heads 2 j and 2 j + 1 of a kv-head's group are the two maps
 * of pair j, the output is their difference sum_i (p_i - lambda p'_i) V_i (conf_kv_attend_diff).
 * The handle gives B, Hq, Hkv, D and the softmax scale; nothing of its cache changes, and the lengths are the caller's, on the
 * device: a recorded call moves on with them.  A token's key that is NaN or scores +infinity leaves no
 * number in the rows that see it (one that scores -infinity has no weight), a value that is none shows in its channel of these rows; no other
 * row shows either.  Rows that no sequence claims are left as they were; two sequences claim no row and write to no page together
 * (pages that both only read are shared freely).
 * CONF_KV_ERR_INVALID_ARG beyond the limits noted above, where max_pages * page_tokens is more than max_paged (rounded up to whole
 * pages), and for tensors that overlap what is written (keys and values may take turns in one tensor, not share a value of it).
 * Tensors are 16-byte aligned, tokens * n_q_heads * B at most 2^30. */
int conf_kv_attend_pages(conf_kv_handle *h, const conf_kv_pages *pages, const conf_kv_chunk *chunk, conf_kv_stream stream);

/* conf_kv_load_prefill from pages: the cache of the layer becomes the first T0 tokens of every sequence (dev_ema0 fp32
 * [B][Hkv][T0], or NULL).  Same result, call order and errors; T0 at most max_pages * page_tokens (CONF_KV_ERR_INVALID_ARG). */
int conf_kv_load_pages(conf_kv_handle *h, int32_t layer, const conf_kv_pages *pages, int32_t T0, const float *dev_ema0,
                       conf_kv_stream stream);

/* Importance from the prompt's own attention (the step before the decode loop: the cache's
 * initial importance comes from an observation window of queries at the end of the prompt
 * instead of starting at zero).  dev_q16: fp16 [B][tq][Hq][D], the queries of the cached slots
 * first .. first + tq - 1 of every unit of the layer; nothing is appended.  Defined like
 * conf_kv_attend_chunk on the stored values: query t sees slots 0 .. first + t, the importance
 * of every slot below first + tq follows a <- lambda a + gain A_t once per query (a window
 * slot counts from 0 at its own query, whatever it held before), slots from first + tq on are
 * neither seen nor changed.  Calls for consecutive windows first = s, s + tq, .. compose.
 * dev_out16: fp16 [B][tq][Hq][D] attention outputs of those queries, or NULL.
 * Allowed between conf_kv_load_prefill of the layer and its first conf_kv_attend
 * (CONF_KV_ERR_BAD_STATE otherwise), with max_chunk >= 2 (or a group of more than 8 heads, then
 * tq = 1), 1 <= tq <= max(1, max_chunk) (calls of more than 16 / G tokens run on a kernel that
 * reads the keys twice instead of keeping 16 x slots scores on chip) and
 * 0 <= first, first + tq <= T0 (CONF_KV_ERR_INVALID_ARG). */
int conf_kv_observe(conf_kv_handle *h, int32_t layer, int32_t first, int32_t tq, const void *dev_q16,
                    void *dev_out16, conf_kv_stream stream);

/* The prompt-phase importance in full (the step before the decode loop; "Related work" names
 * prompt-phase observation as the neighbouring idea, the paper's own update is "using A" per
 * decode step): every prompt query observes the prompt causally, as conf_kv_observe over the
 * consecutive windows first = 0, max_chunk, 2 max_chunk, .. covering all T0 cached tokens would
 * leave it, in one to five launches.  dev_q16: fp16 [B][T0][Hq][D], the queries of all prompt
 * tokens.  The result is what T0 single-token decode steps over the stored prompt would have left
 * (see conf_kv_attend_chunk for the telescoped update), rounded to fp32 once; normalisers and the
 * sums over heads and tokens are float64 (queries so far back that all of them together add less than
 * half of the smallest fp32 number to any slot are left out; one that is NaN or infinite still makes the
 * importance of every slot its token sees NaN).  (A prompt that fits one conf_kv_observe call may run as
 * one, with that kernel's sums.)  Same call order rules and errors as conf_kv_observe; needs
 * max_chunk >= 2 (or a group of more than 8 heads). */
int conf_kv_observe_prompt(conf_kv_handle *h, int32_t layer, const void *dev_q16, conf_kv_stream stream);

/*
 * Confidence estimator and budget selector (Eq. 1; "Budget and ranker"; Algorithm 1,
 * lines softmax / c / N).  For every sequence b: p = softmax(logits[b]),
 * c = w_entropy (1 - H(p)/log V) + w_margin sigmoid(log p_(1) - log p_(2)) + w_top p_(1);
 * tight = (c >= tau); the per-layer budget N[l][b] = tight ? n_tight[l] : n_loose[l]
 * stays on the device for the next conf_kv_evict_compact.
 * dev_logits: fp32 [B][V] (-inf entries allowed).  dev_conf: fp32 [B] written.
 * dev_sel: uint8 [B] written, 1 = tight.  Either output may be NULL.
 */
int conf_kv_step(conf_kv_handle *h, const float *dev_logits, float *dev_conf, uint8_t *dev_sel,
                 conf_kv_stream stream);

/*
 * conf_kv_step for callers that cannot allocate or hand over a workspace at the time of the call
 * (code under HIP graph capture, tight serving loops, harnesses that forbid allocation): same
 * arguments, same results, but the per-chunk partial sums of the reduction live in a device
 * array of the library itself (1 MiB per GPU, resident from the library's load until the
 * process ends) instead of the handle's dev_scratch.  The call allocates and frees nothing.
 * Limit: batch * ceil(vocab / 4096) * 64 bytes must fit that array, i.e. batch * ceil(vocab /
 * 4096) <= 16384 (CONF_KV_ERR_CAPACITY otherwise, before anything is launched).  Every call on
 * one GPU, from any handle, uses that GPU's one array: calls that overlap in time on one GPU
 * (different streams or host threads) race and give undefined results; calls in stream order
 * are safe, whatever their sizes.
 */
int conf_kv_step_static(conf_kv_handle *h, const float *dev_logits, float *dev_conf, uint8_t *dev_sel,
                        conf_kv_stream stream);

/*
 * Ranker, eviction, in-place compaction and demotion for every layer (Algorithm 1's
 * per-layer tail; "Budget and ranker"; "Cache manager").  For each unit with
 * n > N[l][b]: the newest min(P, n) slots are protected; over the other slots
 * s_i = alpha * minmax(ema_i) + (1 - alpha) * minmax(pos_i) (min-max over those
 * candidates, 0 when degenerate), the min(n - N, n - P) lowest are evicted (equal
 * scores: oldest first), survivors are gathered in place keeping position order, and
 * then the oldest FP16 slots are quantised until at most W stay FP16.
 * Uses the budgets of the last conf_kv_step (the loose ones before any).  Commits the
 * appends made by conf_kv_attend since the previous call.
 */
int conf_kv_evict_compact(conf_kv_handle *h, conf_kv_stream stream);

/* Type of the values a model hands over. */
typedef enum conf_kv_type {
  CONF_KV_TYPE_FP32 = 0,     /* IEEE binary32 */
  CONF_KV_TYPE_FP16 = 1,     /* IEEE binary16 */
  CONF_KV_TYPE_BF16 = 2      /* the upper half of a binary32 */
} conf_kv_type;

/* Arguments of conf_kv_prepare_qkv.  Strides count values, are not negative and may be anything the alignment allows (a
 * projection's fused row [Hq + 2 Hkv][D] is read where it is); the heads of a token are dense. */
typedef struct conf_kv_qkv {
  int32_t tokens;            /* T >= 0 per sequence; 0: nothing is done                                     */
  int32_t type;              /* conf_kv_type of dev_q, dev_k, dev_v                                         */
  const void *dev_q;         /* [B][T][Hq][D]                                                               */
  const void *dev_k;         /* [B][T][Hkv][D]                                                              */
  const void *dev_v;         /* [B][T][Hkv][D]                                                              */
  int64_t q_batch_stride, q_token_stride;
  int64_t k_batch_stride, k_token_stride;
  int64_t v_batch_stride, v_token_stride;
  const float *dev_q_weight; /* fp32 [D], or NULL: queries are not normalised                               */
  const float *dev_k_weight; /* fp32 [D], or NULL: keys are not normalised                                  */
  const float *dev_freq;     /* fp32 [rotated / 2]: angle per position of each pair                         */
  const int32_t *dev_pos;    /* int32 [B][T] positions, or NULL: token t has the position that the next
                                token appended to the layer gets, plus t, for every sequence                */
  int32_t first;             /* added to every position (a shared prefix's tokens, say)                     */
  int32_t rotated;           /* leading channels that turn: 0 .. D, a multiple of 16                        */
  int32_t interleaved;       /* 0: pair p is channels (p, p + rotated / 2); 1: channels (2 p, 2 p + 1)      */
  int32_t prompt_layout;     /* 0: keys and values [B][T][Hkv][D]; 1: [B][Hkv][T][D] (conf_kv_load_prefill) */
  float eps;                 /* of the norm; finite, >= 0                                                   */
  void *dev_q16;             /* fp16 [B][T][Hq][D], written                                                 */
  void *dev_k16;             /* fp16, written                                                               */
  void *dev_v16;             /* fp16, written                                                               */
} conf_kv_qkv;

/*
 * Queries, keys and values as a projection leaves them, made into what conf_kv_attend, conf_kv_attend_chunk,
 * conf_kv_attend_shared, conf_kv_observe* (queries; keys and values in decode layout) and conf_kv_load_prefill (prompt
 * layout) take, in one pass.  Each query and key head x of a token becomes
 *     y = x / sqrt(mean(x^2) + eps) * weight           (where a weight is given, else y = x)
 *     (a, b) <- (a cos t - b sin t, b cos t + a sin t) for the pairs of its first `rotated` channels, t = position * freq
 * and is rounded to fp16 once; values are rounded to fp16.  Angles are formed in float64, norms (of rows of any size) and products
 * in float32.  What is beyond fp16's range becomes infinite.  Each of q, k and v may be left out (source and destination NULL), not all.
 * The handle gives B, Hq, Hkv, D and, with dev_pos NULL, the positions, which live on the device: a recorded call moves on
 * with the cache.  Nothing of the cache changes.  Tensors are 16-byte aligned and so are the strides in bytes; destinations lie
 * apart from each other and from the sources (what is between a source's first and last value).  B * T at most 2^30. */
int conf_kv_prepare_qkv(conf_kv_handle *h, int32_t layer, const conf_kv_qkv *args, conf_kv_stream stream);

/* Arguments of conf_kv_constrain.  NULL leaves a part out. */
typedef struct conf_kv_constraints {
  int32_t type;                     /* conf_kv_type of dev_logits                                              */
  int32_t max_tokens;               /* most tokens of a row of dev_tokens that are read, up to 2^30             */
  const void *dev_logits;           /* [B][V], rows logits_stride values apart                                 */
  int64_t logits_stride;            /* >= V                                                                    */
  float *dev_out;                   /* fp32 [B][V], written; may be dev_logits itself (fp32, stride V)         */
  const int32_t *dev_tokens;        /* int32 [B][..]: every row's history, prompt first, then what was
                                       generated; ids outside [0, V) count for nothing                         */
  int64_t tokens_stride;            /* >= max_tokens                                                           */
  const int32_t *dev_lengths;       /* int32 [B]: tokens of the row's history (0 .. max_tokens; taken as such)  */
  const int32_t *dev_prompt_lengths;/* int32 [B]: how many of them are the prompt; NULL: none                  */
  const float *dev_repetition;      /* fp32 [B], r > 0: logits of tokens in the history: x > 0 ? x / r : x * r  */
  const float *dev_presence;        /* fp32 [B]: subtracted where the token was generated                      */
  const float *dev_frequency;       /* fp32 [B]: subtracted as often as the token was generated                */
  const int32_t *dev_bias_offsets;  /* int32 [B + 1]: row b's biases are entries offsets[b] .. offsets[b + 1]-1 */
  const int32_t *dev_bias_tokens;   /* int32 [n_bias]                                                          */
  const float *dev_bias_values;     /* fp32 [n_bias]: added (-inf bans a token); of several entries of one row
                                       for one token the last one counts                                       */
  int32_t n_bias;                   /* entries there are, up to 2^30; offsets are held within 0 .. n_bias       */
  int32_t n_masks;                  /* rows of dev_allowed                                                     */
  const uint32_t *dev_allowed;      /* uint32 [n_masks][ceil(V / 32)]: bit v & 31 of word v / 32 set = allowed  */
  const int32_t *dev_allowed_rows;  /* int32 [B]: the mask row of each sequence, one outside 0 .. n_masks - 1
                                       (-1): no mask; NULL: row b, n_masks >= B                                */
} conf_kv_constraints;

/*
 * Logits made into what conf_kv_step takes: penalties for repeated tokens, then biases, then a grammar's mask, which puts
 * -inf wherever it forbids (whatever was there, NaN included).  Each row's steps in this order:
 *     x <- x > 0 ? x / repetition : x * repetition       where the token is in the history
 *     x <- x - frequency * count - presence               where it was generated, count times
 *     x <- x + bias;   x <- -inf where it is forbidden
 * in float32.  A row that forbids everything is all -inf; conf_kv_step then gives a confidence that is NaN and the loose
 * budget.  Penalties need dev_tokens and dev_lengths (with max_tokens 0 neither, and they do nothing); lengths, offsets, ids and
 * mask rows are held within the arrays' bounds on the device.  At most 2^27 logits a row (CONF_KV_ERR_BAD_SHAPE).  The result
 * does not depend on the order in which workgroups run. */
int conf_kv_constrain(conf_kv_handle *h, const conf_kv_constraints *args, conf_kv_stream stream);

/*
 * Launch shapes for replayed steps (for callers that record a decode step into a HIP graph).
 * on != 0: from now on the split counts and kernel variants of conf_kv_attend* and
 * conf_kv_evict_compact are derived from the loose budgets n_loose[l] (the longest a committed
 * unit can be once the first conf_kv_evict_compact has run) instead of the lengths seen so far,
 * so a step recorded now stays valid however the caches grow or shrink later.  A prompt longer
 * than n_loose[l] is still covered while it lasts.  Results do not depend on the setting; short
 * caches run a little slower with it.  on == 0: back to the default.  Host-side only.
 */
int conf_kv_static_plan(conf_kv_handle *h, int32_t on);

/* ---- inspection: these synchronise the device; meant for tests and monitoring ---- */

/* host_len: int32 [L][B] current cache length (appends included); host_n16: int32
 * [L][B][Hkv] FP16 slots per unit, or NULL. */
int conf_kv_lengths(conf_kv_handle *h, int32_t *host_len, int32_t *host_n16);

/* Position-sorted view of one unit into host buffers sized for `capacity` slots; any
 * output pointer may be NULL.  pos int32 [n]; ema fp32 [n]; is_fp16 uint8 [n];
 * k16 / v16: fp16 bits [n][D] (zeros on INT8 slots); k8 / v8: int8 [n][D] (zeros on FP16
 * slots); k_scale / v_scale: fp16 bits [n] (zero on FP16 slots), or the unit's channel scales
 * [D] under CONF_KV_SCALES_CHANNEL (give room for max(capacity, D) values); *n_out = n. */
int conf_kv_export(conf_kv_handle *h, int32_t layer, int32_t b, int32_t kv_head, int32_t *pos,
                   float *ema, uint8_t *is_fp16, uint16_t *k16, uint16_t *v16, int8_t *k8,
                   int8_t *v8, uint16_t *k_scale, uint16_t *v_scale, int32_t *n_out);

/* The inverse of conf_kv_export: replaces the cache of one unit by n slots given in the same
 * position-sorted view (harness re-synchronisation, cache hand-over between handles).
 * pos int32 [n] strictly increasing; ema fp32 [n]; is_fp16 uint8 [n]: zeros (INT8 slots) then
 * ones (FP16 slots), at most fp16_window ones, all ones for an FP16-only cache; k16 / v16 fp16
 * bits [n][D], read on FP16 slots; k8 / v8 int8 [n][D] and k_scale / v_scale fp16 bits [n], read
 * on INT8 slots (a plane no slot reads may be NULL); under CONF_KV_SCALES_CHANNEL k_scale /
 * v_scale are the unit's channel scales [D], always read, finite and >= 0.  0 <= n <= capacity - 1
 * (CONF_KV_ERR_CAPACITY); malformed views give CONF_KV_ERR_INVALID_ARG and leave the unit
 * unchanged.  Not allowed between conf_kv_attend of that layer and the next
 * conf_kv_evict_compact (CONF_KV_ERR_BAD_STATE).  The next token appended to the layer gets a
 * position above every imported one.  Budgets are per (layer, sequence): the caller keeps the
 * kv-heads of one sequence at equal length. */
int conf_kv_import(conf_kv_handle *h, int32_t layer, int32_t b, int32_t kv_head, int32_t n,
                   const int32_t *pos, const float *ema, const uint8_t *is_fp16, const uint16_t *k16,
                   const uint16_t *v16, const int8_t *k8, const int8_t *v8, const uint16_t *k_scale,
                   const uint16_t *v_scale);

/* The tags of the words through which the workgroups of a launch exchange partial results:
 * a launch's tag is a device-side base plus the launch's number since the last
 * conf_kv_evict_compact, which moves the base past them.  Once a base exceeds 0xFF000000 the
 * next conf_kv_evict_compact first clears every exchange word and then starts both bases over
 * at 0 (*clear_pending is 1 in between), so no word ever carries a tag a later launch uses.
 * Outputs (host, each may be NULL): the attention and confidence bases and the pending flag. */
int conf_kv_tag_state(conf_kv_handle *h, uint32_t *attend_base, uint32_t *conf_base, int32_t *clear_pending);

/* Device-side counters since conf_kv_create.  Returns CONF_KV_ERR_DEVICE if any kernel
 * reported an internal error (the counters are still filled in). */
int conf_kv_counters(conf_kv_handle *h, conf_kv_stats *host_stats);

/* Split count conf_kv_attend would use for `layer` now (diagnostics / benchmarks); 1000 + the
 * count when the layer's shape needs the two-launch form (the splits of a unit cannot all be
 * resident at once, or a split's scores do not fit on chip: partial results and raw scores then
 * go through the scratch buffer and a second kernel finishes the attention). */
int conf_kv_attend_splits(conf_kv_handle *h, int32_t layer);

const char *conf_kv_strerror(int status);
/* The hipError_t (as int) of the last failed HIP call on this handle, 0 if none. */
int conf_kv_last_hip_error(conf_kv_handle *h);

/* Measurement aid, not part of the decode path: one launch that reads dev_src[0 .. bytes) once
 * (plain 16-byte loads, `workgroups` workgroups of 256 threads over equal contiguous shares)
 * and folds it into dev_out, uint32 [workgroups], which the caller has zeroed.  What this
 * reaches is the practical ceiling of a streaming read on the device, to set next to the
 * published peak.  bytes a positive multiple of 16, dev_src 16-byte aligned, 1 <= workgroups
 * <= 65536; CONF_KV_ERR_INVALID_ARG otherwise, CONF_KV_ERR_HIP if the launch fails. */
int conf_kv_probe_read(const void *dev_src, size_t bytes, uint32_t *dev_out, int32_t workgroups,
                       conf_kv_stream stream);

#ifdef __cplusplus
}
#endif
#endif /* CONF_KV_H */
