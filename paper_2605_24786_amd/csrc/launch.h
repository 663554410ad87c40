// Host-side launchers of the kernels, one per source file.  Internal to the library.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "confkv_dev.h"

namespace confkv {

// ---- conf_reduce.hip ----
size_t conf_reduce_scratch_bytes(int B, int V);   // epoch-tagged chunk partials: zero before the first call
hipError_t launch_conf_reduce(const CacheView &cv, const float *logits, int V, unsigned long long *partial,
                              unsigned launch_no /* the words' tag; never 0, never reused */,
                              int device_base /* 1: the tag is launch_no + cv.ctl[kCtlConfTag] */, int spin_limit,
                              int withhold /* test hook: chunk 0 does not publish, so the bounded wait expires */,
                              float *conf, uint8_t *sel, double tau, double wH, double wm, double wp,
                              hipStream_t stream);
// words [0, bytes / 8) <- 0 on the stream (a kernel, not a memset node)
hipError_t launch_zero_words(void *p, size_t bytes, hipStream_t stream);
// The same launch with the chunk partials in a file-scope device array of the library (one copy
// per device, shared by every call on that device; kConfStaticBytes of it).  setup resolves the
// array's address on the current device once; the launch does it too if nobody has.
constexpr size_t kConfStaticBytes = (size_t)1 << 20;
hipError_t conf_reduce_static_setup();
hipError_t launch_conf_reduce_static(const CacheView &cv, const float *logits, int V, int spin_limit, int withhold,
                                     float *conf, uint8_t *sel, double tau, double wH, double wm, double wp,
                                     hipStream_t stream);
constexpr int kSpinLimitDefault = 400000;   // polls (about a microsecond each) before a bounded wait gives up

// ---- probe.hip ----
hipError_t launch_probe_read(const void *src, size_t bytes, unsigned *out, int workgroups, hipStream_t stream);

// types of the rows a model hands over (conf_kv_type)
constexpr int kTypeFp32 = 0, kTypeFp16 = 1, kTypeBf16 = 2;

// ---- prepare.hip ----
struct PrepareLaunch {
  const void *q, *k, *v;                 // [B][tokens][heads][D], each may be null
  long long q_batch, q_token, k_batch, k_token, v_batch, v_token;   // strides in values
  const float *wq, *wk, *freq;           // norm weights (null: no norm), angles per position
  const int32_t *pos;                    // [B][tokens], or null: *next + token
  const unsigned *next;
  long long first;                       // added to every position (and, without pos, what a call has appended since the last eviction)
  __half *q16, *k16, *v16;
  int B, tokens, Hq, Hkv;
  int rotated, interleaved, prompt;
  float eps;
};
hipError_t launch_prepare(const PrepareLaunch &a, int D, int type, hipStream_t stream);

// ---- constrain.hip ----
struct ConstrainLaunch {
  const void *logits;
  long long row_stride;
  float *out;                            // [B][V]
  const int32_t *tokens, *lengths, *prompt_lengths;
  long long token_stride;
  const float *repetition, *presence, *frequency;
  const int32_t *bias_offsets, *bias_tokens;
  const float *bias_values;
  const uint32_t *allowed;
  const int32_t *allowed_rows;
  int B, V, max_tokens, n_bias, n_masks;
};
hipError_t launch_constrain(const ConstrainLaunch &a, int type, hipStream_t stream);

// ---- attend.hip ----
struct AttendPlan {
  int splits;        // workgroups per unit
  int stash_tokens;  // score slots per workgroup held in LDS
  size_t lds_bytes;  // dynamic LDS per workgroup
  bool mfma;         // matrix-core body for the INT8 slots
  bool two_launch;   // stream + publish, then merge + EMA in a second launch (scores in scratch)
  int wide_groups;   // > 0: the many-rows kernel with that many groups of 32 query rows per unit
  bool wide_kept;    // its form that keeps the probabilities in registers
};
struct AttendLaunch {
  int layer;
  const __half *q, *knew, *vnew;
  __half *out;
  unsigned long long *part_ml;   // [units per layer][max splits][G][2] words: (epoch << 32) | float bits of m, of l
  unsigned long long *part_o;    // [units per layer][max splits][G][D] words: (epoch << 32) | float bits of a partial output
  unsigned epoch;          // number of the launch since the last commit, from 1; the kernels add the base in
                           // cv.ctl: the sum tags the words the launch publishes (never 0, never reused)
  int spin_limit;          // polls before a wait for the other splits gives up (device error)
  int max_splits;
  unsigned ns_magic;       // the kernels' division by the split count (split_divisor), 0 for one split
  int ns_shift;
  float sm_scale, ema_decay;
  double mass_gain;        // weight of the step's mass in the EMA update
  unsigned tag_base;       // filled in by the kernels from cv.ctl
  int pos_new;             // position of the first appended token (the kernels read it from cv.ctl)
  int tq;                  // tokens appended (and queries per head) in this call
  int gq;                  // query heads per kv-head; the kernels' row r is (token r / gq, head r % gq)
  int gq_mul;              // 65536 / gq + 1: the single-tile kernels' division of a row number by gq
  int observe_first;       // >= 0: the queries belong to the cached slots observe_first .. observe_first + tq - 1;
                           // nothing is appended and slots from observe_first + tq on are left alone
  int withhold;            // test hook: split 0 of every unit does not publish its statistics, so the
                           // other splits' bounded waits expire (the kernel still ends normally)
  int kv_major;            // grid is (kv-heads, splits, sequences) instead of (splits, kv-heads, sequences)
  float *spill;            // [units per layer][splits][G][stash_tokens] raw scores (two-launch form)
  unsigned long long *dbg; // phase-trace buffer (CONFKV_TRACE builds), else null
  int tab_off;             // paged layout: byte offset of the unit's block table in dynamic LDS
  int trace_off;           // byte offset of the time stamps in dynamic LDS (CONFKV_TRACE builds)
  // partial results of a shared prefix, which the wavefronts of a unit take in with their own (none: shared_parts = 0)
  const float2 *shared_ml; // [units per layer][parts][rows] maximum and normaliser
  const float *shared_o;   // [units per layer][parts][rows][D]
  int shared_parts, shared_rows;
};
constexpr int kAttendMaxSplits = 64;
constexpr int kChunkRows = 16;     // query rows per unit of a multi-token call (one matrix-core tile)
// Multiplier and shift of a division by ns (2 .. 64): x / ns = (high word of x * multiplier) >> shift for all 0 <= x < 2^31.
unsigned split_divisor(int ns, int *shift);
bool attend_supported(int D, int G);
size_t attend_spill_floats(int units_per_layer, int G, int cap);   // scratch the two-launch form needs
// Largest split count and LDS plan for a unit of at most n_ub tokens (after the append)
// of which at most n16_ub are FP16.  G = query rows per unit (the group size, or kChunkRows for
// a multi-token call, which only has the single-launch matrix-core form).  Returns false when no plan fits the device.
// extra_lds: bytes the launch needs behind the kernel's own dynamic LDS (the block table of the paged layout).
bool attend_plan(int D, int G, bool chan, bool paged, bool chunk, int units_per_layer, int n_ub, int n16_ub, int forced_splits,
                 bool force_two_launch, size_t extra_lds, bool shared /* a shared prefix is taken in */, AttendPlan *plan);
// Plan of a call with more than kChunkRows query rows per unit (at most kWideRowsMax); false when
// the shape cannot be served.  major_kv: kv-heads of the kv-head-first grid, 0 for the other.
// n_ub: the most slots of a unit; n16_least, n16_ub: the fewest and the most FP16 ones.
constexpr int kWideRowsMax = 128;
int attend_wide_splits(int units_per_layer, int major_kv, int n_ub, int most, int cus);
bool attend_wide_plan(int rows, int units_per_layer, int major_kv, int n_ub, int n16_least, int n16_ub, int forced_splits, AttendPlan *plan);
hipError_t launch_attend(const CacheView &cv, const AttendLaunch &a, const AttendPlan &plan,
                         hipStream_t stream);
// ---- attend_shared.hip ----
constexpr int kSharedMaxParts = 64;
struct SharedPlan {
  int row_waves;           // wavefronts of a workgroup side by side along the rows: 1, 2 or 4
  int blocks;              // workgroups along the rows of a kv-head
  int parts, part_keys;    // parts of the prefix and the keys of one
};
struct SharedLaunch {
  const __half *k, *v;     // [Hkv][T][D], heads head_stride values apart
  const __half *q;         // [B][tq][Hkv * G][D]
  const int32_t *seen;     // [B] keys each sequence sees, or null: all
  float2 *ml;              // [B * Hkv][parts][unit_rows]
  float *o;                // [B * Hkv][parts][unit_rows][D]
  long long head_stride;
  int T, B, Hkv, G, tq, unit_rows /* tq * G */, parts, part_keys;
  float sm_scale;
};
size_t shared_parts_most(int tokens);      // parts a prefix of up to that many tokens can be cut into
// rows of a kv-head; forced_row_waves: 1, 2 or 4, else the plan's own choice
void shared_plan(int rows, int Hkv, int D, int T, int cus, int forced_row_waves, SharedPlan *plan);
int device_cu_count();
hipError_t launch_shared_prefix(const SharedLaunch &a, const SharedPlan &p, int D, hipStream_t stream);
// Importance of a freshly loaded prompt of T tokens from all its queries q [B][T][Hq][D] (D = 128,
// contiguous layout).  scratch: scratch_floats floats, at least observe_scratch_floats(B * Hkv, G, T); with more the
// work is cut into parts, observe_plan_floats(B * Hkv, G, T, first block of rows, INT8 slots, chan, scratch_floats, CUs) of them are used.
size_t observe_scratch_floats(int units_per_layer, int G, int cap);
int observe_first_block(int G, int T, double decay, double gain);
size_t observe_plan_floats(int units_per_layer, int G, int T, int b0, int n8, int chan, size_t have, int cus);
hipError_t launch_observe_prompt(const CacheView &cv, int layer, const __half *q, int T, float sm, double decay, double gain,
                                 float *scratch, size_t scratch_floats, hipStream_t stream);

// ---- evict.hip ----
// Per unit, written by rank_select: [0] new length, [1] new INT8 count, [2] first evicted slot,
// [3] evicted slots, [4] last evicted INT8 slot (-1: none), [5] 1 = the INT8 rows in front of
// that slot shift right (the ring head advances), 0 = the rows behind the first hole shift
// left, [6] INT8 ring head after the compaction, [7] 1 = the entries above are final for this
// call (0 after the first ranking kernel: the unit waits for the general one).
constexpr int kSelInts = 8;
hipError_t launch_load_prefill(const CacheView &cv, int layer, const __half *k16, const __half *v16,
                               int T0, const float *ema0, hipStream_t stream);
// Ranker variants; all zero = the composite ranker per (layer, kv-head).
struct RankOptions {
  int random;                  // 1: rank by counter-based uniform draws instead of the composite score
  unsigned long long seed;
  double *shared;              // non-null: layer scope; [L * B][cap] scratch for the summed mass
  int page;                    // > 1: whole pages of that many original positions are evicted
  int separate;                // test hook: never one launch for the whole call
};
hipError_t launch_evict_compact(const CacheView &cv, const LayerMask &appended, double alpha,
                                const RankOptions &opt, double *score, int32_t *src, int32_t *sel,
                                int n_max /* longest unit */,
                                unsigned attend_launches, unsigned conf_launches /* since the last commit */,
                                int after_prompt /* a layer's prompt was loaded since the last commit: long moves */,
                                hipStream_t stream);

}  // namespace confkv
