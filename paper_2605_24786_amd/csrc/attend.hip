// Decode attention over the mixed INT8 / FP16 cache with the attention-mass EMA fused in
// (paper: "Tiled attention and mixed precision" -- blockwise read, running max and
// normaliser, dequantisation fused into the read; "Budget and ranker" -- EMA of attention
// mass; Algorithm 1 -- append in FP16, update EMA metadata).
//
// One launch per layer, grid (splits, kv-heads, sequences) -- or (kv-heads, splits, sequences)
// when the number of kv-heads is a multiple of eight, which puts all splits of a unit on one
// XCD -- of 512 threads.  The `splits` workgroups of a unit (b, kv-head) each stream a
// contiguous, byte-balanced slice of the unit's slots once and serve all G query heads of
// the group from that single read:
//
//   stream   running (max, normaliser, output) per head (online softmax); the raw scores
//            s[h][i] of the slice stay in LDS
//   publish  the workgroup's (m, l) per head go out first, then its merged output partial;
//            every published 8-byte word carries the launch's tag (its number since the last
//            commit plus a base kept on the device), so nothing waits for stores to land, no
//            counter is shared, and a recorded launch can be replayed
//   mass     gather the (m, l) words of every split of the unit (a bounded poll on their
//            tags: they all publish at about the same time), form the exact global (M, L),
//            then per slot A_i = sum_h e^{s[h][i]-M[h]} / L[h] and
//            ema_i <- lambda ema_i + (1-lambda) A_i; every split also normalises its share of
//            the unit's output row from the splits' tagged output partials.
//
// Every K/V byte is read once; the scores never leave the chip.  The wait is between
// workgroups of one launch, so the host only launches grids that are co-resident
// (splits * units <= occupancy * CUs) and the wait itself is bounded.
//
// Two streaming bodies share the prologue and the epilogue:
//   * vector-ALU body (any G, any D): lane c of a group of D/16 lanes owns channels
//     [16c, 16c+16) of a slot row, so a wavefront load covers whole rows, contiguous in
//     memory; each lane-group keeps its own running softmax state.
//   * matrix-core body (2 <= G <= 8, D = 128) for the INT8 slots: the G query heads against a
//     32-slot tile are two small contractions (scores: [G x 128] x [128 x 32]; output, transposed:
//     [128 x 32] x [32 x G]) issued as v_mfma_f32_16x16x32_f16 with the head dimension
//     padded to 16.  The vector ALU then only converts int8 -> fp16 and keeps the softmax
//     state, which is what lets the kernel stay memory-bound for grouped-query shapes.
//     FP16 slots go through the same contractions in 16-slot tiles, no conversion needed.
//     The same body with all 16 tile rows as query rows serves calls that carry several
//     tokens per sequence (conf_kv_attend_chunk), and a variant of it folds per-channel INT8
//     scales into the query and the output.
// When the splits of a unit cannot all be resident, or a slice's scores do not fit LDS, the
// launch is replaced by two (stream + publish with the scores in device scratch; merge + mass),
// which need no wait inside a kernel.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <map>
#include <set>
#include <mutex>
#include <tuple>

#include "attend_body.h"

namespace confkv {

#include "attend_wide.h"
#include "attend_rows.h"
#include "attend_observe.h"

// ---------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------

static std::atomic<bool> g_use_mfma{true};

static AttendFn attend_fn(AttendForm form, int D, int G, bool chan, AttendKind kind) {
  return kind == kAttendShared ? attend_shared_instance(form, D, G, chan) : kind == kAttendDiff ? attend_diff_instance(form, D, G, chan)
                                                                                                : attend_instance<false>(form, D, G, chan);
}
static AttendKind attend_kind(const AttendLaunch &a) { return a.lambda ? kAttendDiff : a.shared_parts > 0 ? kAttendShared : kAttendPlain; }

// Second launch of the two-launch form.
static AttendFn attend_fn_finish(int D, int G) {
#define CONFKV_CASE(d, g) \
  if (D == d && G == g) return (AttendFn)attend_finish_kernel<d, g>;
  CONFKV_CASE(64, 1) CONFKV_CASE(64, 2) CONFKV_CASE(64, 3) CONFKV_CASE(64, 4) CONFKV_CASE(64, 5)
  CONFKV_CASE(64, 6) CONFKV_CASE(64, 7) CONFKV_CASE(64, 8)
  CONFKV_CASE(128, 1) CONFKV_CASE(128, 2) CONFKV_CASE(128, 3) CONFKV_CASE(128, 4) CONFKV_CASE(128, 5)
  CONFKV_CASE(128, 6) CONFKV_CASE(128, 7) CONFKV_CASE(128, 8)
#undef CONFKV_CASE
  // (multi-token calls: the first launch is the matrix-core body)
  if (D == 128 && G == kChunkRows) return (AttendFn)attend_finish_kernel<128, kChunkRows>;
  return nullptr;
}

// Second launch behind the matrix-core body at D = 64: the partials are 128 channels wide.
static AttendFn attend_fn_finish_padded(int G) {
#define CONFKV_CASE(g) \
  case g: return (AttendFn)attend_finish_kernel<128, g, 64>;
  switch (G) {
    CONFKV_CASE(2) CONFKV_CASE(3) CONFKV_CASE(4) CONFKV_CASE(5) CONFKV_CASE(6) CONFKV_CASE(7) CONFKV_CASE(8)
    default: return nullptr;
  }
#undef CONFKV_CASE
}

// The matrix-core kernel serves every grouped-query shape, FP16-only caches included (at G >= 4
// the vector-ALU body runs out of registers); at D = 64 it pads the head to its 128-channel tiles.
static bool wants_mfma(int D, int G, bool /*has_int8*/) {
  return g_use_mfma && attend_instance<false>(kFormMfma, D, G, false) != nullptr;
}

// Groups of 9 to 16 query heads run as a one-token call of the 16-row matrix-core kernel (D = 128).
bool attend_supported(int D, int G) {
  return attend_instance<false>(kFormValu, D, G, false) != nullptr || (D == 128 && G > 8 && G <= kChunkRows);
}

static size_t attend_lds_bytes(int D, int G, int S, bool mfma) {
  if (mfma) {
    const int NP = kAttWaves;
    size_t floats = (size_t)G * (S + (G > 8 ? kStashPad : 0)) + G + 2 + 2 * NP * G;
    size_t tiles = (size_t)kAttWaves * (G > 8 ? kRowsTileBytes : kHeadTileBytes);
    return (floats * sizeof(float) + (size_t)2 * G * sizeof(double) + tiles + 32 + 15) / 16 * 16;
  }
  size_t floats = (size_t)G * S + (size_t)kAttWaves * G * D + 2 * kAttWaves * G + G + 2;
  return floats * sizeof(float) + (size_t)2 * G * sizeof(double) + 16;
}

struct DeviceLimits {
  int cus = 0;
  size_t max_lds = 0;
  bool ok = false;
};

// The two caches below are shared by every handle of the process; handles may live on
// different host threads, so both are guarded.
static std::mutex g_plan_mutex;

static const DeviceLimits &device_limits() {
  static DeviceLimits lim;
  std::lock_guard<std::mutex> lock(g_plan_mutex);
  if (!lim.ok) {
    int dev = 0;
    hipDeviceProp_t prop;
    if (hipGetDevice(&dev) == hipSuccess && hipGetDeviceProperties(&prop, dev) == hipSuccess) {
      lim.cus = prop.multiProcessorCount;
      lim.max_lds = prop.sharedMemPerBlockOptin ? prop.sharedMemPerBlockOptin
                                                : prop.sharedMemPerBlock;
      if (lim.max_lds > 160 * 1024) lim.max_lds = 160 * 1024;
      lim.ok = lim.cus > 0;
      if (const char *e = getenv("CONF_KV_NO_MFMA")) g_use_mfma = atoi(e) == 0;
    }
  }
  return lim;
}
static int device_cus() { return device_limits().cus; }
int device_cu_count() { return device_cus(); }

// Resident workgroups per CU of a kernel with `lds` bytes of dynamic LDS.
static int attend_occupancy(AttendFn fn, size_t lds) {
  static std::map<std::tuple<const void *, size_t>, int> cache;
  std::lock_guard<std::mutex> lock(g_plan_mutex);
  auto key = std::make_tuple((const void *)fn, lds);
  auto it = cache.find(key);
  if (it != cache.end()) return it->second;
  int nb = 0;
  // The dynamic-LDS ceiling of a kernel is raised once, to the most any plan can ask for: a
  // ceiling set per plan would be lowered again by a later, smaller plan of the same kernel.
  static std::set<const void *> raised;
  if (lds > 64 * 1024 && raised.insert((const void *)fn).second) {
    hipFuncAttributes fa;
    size_t fixed = 0;                            // LDS the kernel declares itself counts against the same limit
    if (hipFuncGetAttributes(&fa, (const void *)fn) == hipSuccess) fixed = fa.sharedSizeBytes;
    (void)hipFuncSetAttribute((const void *)fn, hipFuncAttributeMaxDynamicSharedMemorySize,
                              (int)(160 * 1024 - std::min<size_t>(fixed, 64 * 1024)));
  }
  if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&nb, (const void *)fn, kAttThreads, lds) !=
      hipSuccess)
    nb = 0;
  cache[key] = nb;
  return nb;
}

bool attend_plan(int D, int G, bool chan, bool paged, bool chunk, int units_per_layer, int n_ub, int n16_ub, int forced_splits,
                 bool force_two_launch, size_t extra_lds, AttendKind kind, AttendPlan *plan) {
  const DeviceLimits &lim = device_limits();
  if (!lim.ok) return false;
  if (attend_instance<false>(chunk ? kFormMfma : kFormValu, D, G, chunk && chan) == nullptr) return false;
  const bool mfma = chunk || wants_mfma(D, G, n16_ub < n_ub);
  AttendFn fn = attend_fn(!mfma ? kFormValu : paged ? kFormPaged : kFormMfma, D, G, chan, kind);
  if (!fn) return false;
  const long long nv = (long long)n_ub + n16_ub;
  // One workgroup per CU measured best: the exchange between the splits of a unit (statistics
  // and partial gather) gets slower with more participants, and a grid that is not a
  // whole number of waves over the CUs leaves a straggler round.  That holds above half of the
  // CUs too: 136 to 256 units of 700 to 9000 slots take 1.03 to 1.38 times as long on two
  // workgroups each as on one (one head, 128 channels, 192 units of 2000 slots, FP16: 41.4 against
  // 46.8 us; 64-slot window: 27.4 against 31.0).
  int want = lim.cus / units_per_layer;
  if (want < 1) want = 1;
  // Measured on 8- and 12-unit layers of 500 to 32768 slots: a unit below about 192 KB is
  // fastest on one workgroup (no exchange at all); above, splits down to about 32 KB each
  // (one 32-slot tile per wavefront) still pay.
  const long long unit_bytes = (long long)(n_ub - n16_ub) * (2 * D + 4) + (long long)n16_ub * 4 * D;
  want = unit_bytes <= 192 * 1024 ? 1 : (int)std::min<long long>(want, unit_bytes / (32 * 1024));
  if (forced_splits > 0) want = std::min<long long>(forced_splits, std::max<long long>(1, nv / 128));
  want = std::max(1, std::min(want, kAttendMaxSplits));
  // preference order: want, want-1, .., 1 (fewer, always co-resident), then want+1, .. (more
  // splits shrink the LDS stash when a long unit does not fit otherwise)
  plan->two_launch = false;
  plan->wide_groups = 0;
  for (int k = 0; k < kAttendMaxSplits && !force_two_launch; ++k) {
    const int ns = k < want ? want - k : k + 1;
    // LDS is sized in steps of 256 slots so the occupancy query is cached across calls
    const int need = (n_ub + ns - 1) / ns + (n16_ub + ns - 1) / ns + 34;
    int S = (need + 255) / 256 * 256;
    size_t lds = attend_lds_bytes(D, G, S, mfma) + extra_lds;
    if (lds > lim.max_lds) {                    // a tight fit: give the rounding up
      S = (need + 31) / 32 * 32;
      lds = attend_lds_bytes(D, G, S, mfma) + extra_lds;
    }
    if (lds > lim.max_lds) continue;
    if (ns > 1) {
      int occ = attend_occupancy(fn, lds);
      if ((long long)occ * lim.cus < (long long)ns * units_per_layer) continue;
    } else if (lds > 64 * 1024) {
      (void)attend_occupancy(fn, lds);          // raises the dynamic-LDS limit
    }
    plan->splits = ns;
    plan->stash_tokens = S;
    plan->lds_bytes = lds;
    plan->mfma = mfma;
    return true;
  }
  // No single-kernel plan: the splits of a unit cannot all be resident (many long units), or
  // the slice's scores do not fit LDS.  Two launches then: the first streams and publishes
  // partials, keeping the raw scores in device scratch; the second merges and updates the EMA.
  // Nothing waits inside a kernel, so any split count works.
  {
    // same split count as the single-kernel plan would like (measured on 64 units of 4096
    // slots: 4 splits 40 us, 16 splits 80 us -- the second launch grows with the split count)
    const int ns = want;
    int S = (n_ub + ns - 1) / ns + (n16_ub + ns - 1) / ns + 34;
    S = (S + 255) / 256 * 256;
    const size_t lds = attend_lds_bytes(D, G, 0, mfma) + extra_lds;
    if (lds > lim.max_lds) return false;
    if (lds > 64 * 1024) (void)attend_occupancy(attend_fn(kFormMfmaSpill, D, G, chan, kind), lds);   // raises the dynamic-LDS limit
    plan->splits = ns;
    plan->stash_tokens = S;
    plan->lds_bytes = lds;
    plan->mfma = mfma;
    plan->two_launch = true;
    return true;
  }
}

// Splits of a unit in the many-rows kernel, whose workgroups have a CU each and wait for the unit's other splits: two
// launches on two streams that together need more CUs than there are can each hold some that the other's splits wait for, until the
// polls expire.  256 slots a split, up to eight, are taken while the grid fits the chip.  Beyond that twice the splits pay while a
// split keeps 96 slots, 160 from eight to sixteen, and are taken where two such launches cannot stop each other: a grid of at
// most half of the CUs, or eight kv-heads or a multiple in the kv-head-first grid (major_kv; 0: the other grid).  An XCD then gets
// the splits of kv/8 units in order, so that of a launch that is not all there at most kv/8 * (splits - 1) workgroups per XCD
// wait -- all earlier units are complete and end -- and two launches leave a CU free if that is less than half of its CUs.
// us per launch, eight kv-heads with four heads, 16 tokens: 64 units of 500 slots in 1, 2, 4 splits 31, 24.8, 20.2, of 1000
// in 2, 4 32.1, 26.5; 32 of 1200 in 4, 8 25.8, 22.8; 16 of 5000 in 8, 16 37.3, 33.8, of 9000 52.0, 42.8; 8 of 2000 26.8, 28.3, of
// 3000 30.7, 29.8; of 300 slots, 8 tokens in 1, 2, 4 19.2, 16.8, 16.4; of 600 in 2, 4, 8 20.1, 17.6, 18.5.
int attend_wide_splits(int units_per_layer, int major_kv, int n_ub, int most, int cus) {
  int ns = 1;
  while (ns * 2 <= std::min(most, 8) && ns * 2 * units_per_layer <= cus && n_ub / (ns * 2) >= 256) ns *= 2;
  auto beside = [&](int n) {
    return 2 * n * units_per_layer <= cus ||
           (n * units_per_layer <= cus && major_kv > 0 && major_kv % 8 == 0 && 2 * (major_kv / 8) * (n - 1) < cus / 8);
  };
  while (ns * 2 <= most && beside(ns * 2) && n_ub / (ns * 2) >= (ns * 2 > 8 ? 160 : 96)) ns *= 2;
  return ns;
}

// Calls with more than 16 query rows per unit: row groups (a power of two) and split count.  The
// splits of a unit exchange partials inside the launch, so with more than one split the whole grid
// must be resident (one workgroup per CU: the tile buffers take most of the LDS).
static AttendFn attend_fn_wide(int rg, bool kept) {
  if (kept) return rg == 1 ? (AttendFn)attend_rows_kernel<1> : (AttendFn)attend_rows_kernel<2>;
  return rg == 1 ? (AttendFn)attend_wide_kernel<1> : rg == 2 ? (AttendFn)attend_wide_kernel<2> : (AttendFn)attend_wide_kernel<4>;
}
bool attend_wide_plan(int rows, int units_per_layer, int major_kv, int n_ub, int n16_least, int n16_ub, int forced_splits, AttendPlan *plan) {
  const DeviceLimits &lim = device_limits();
  if (!lim.ok || rows <= kChunkRows || rows > kWideMaxRows) return false;
  int rg = 1;
  while (rg * kWideRows < rows) rg *= 2;
  int ns = attend_wide_splits(units_per_layer, major_kv, n_ub, wide_max_splits(rg * kWideRows), lim.cus);
  if (forced_splits > 0) {
    ns = 1;
    while (ns * 2 <= std::min(forced_splits, wide_max_splits(rg * kWideRows)) && ns * 2 * units_per_layer <= lim.cus && n_ub / (ns * 2) >= 64) ns *= 2;
  }
  // (wherever they fit: 1.00 to 1.15 times as fast over 23 shapes, of one tile to all 48 / rg)
  plan->wide_kept = rg <= 2 && rows_tiles(n_ub, n16_least, n16_ub, ns) <= rows_rounds(rg) * kAttWaves;
  const size_t lds = plan->wide_kept ? attend_rows_lds_bytes(rg, ns) : attend_wide_lds_bytes(rg * kWideRows, ns);
  if (lds > lim.max_lds || attend_occupancy(attend_fn_wide(rg, plan->wide_kept), lds) < 1) return false;
  plan->splits = ns;
  plan->stash_tokens = 0;
  plan->lds_bytes = lds;
  plan->mfma = true;
  plan->two_launch = false;
  plan->wide_groups = rg;
  return true;
}

size_t attend_spill_floats(int units_per_layer, int G, int cap) {
  // splits * S <= n + n16 + splits * (2 + 34 + 255) with n, n16 <= cap
  return (size_t)units_per_layer * G * (2 * (size_t)cap + (size_t)kAttendMaxSplits * 291);
}

// With k = ceil(log2 ns) and the multiplier (2^(31 + k) + e) / ns, e < ns <= 2^k, the quotient before rounding down is x / ns plus
// x e / (ns 2^(31 + k)), which is below 1 / ns for x < 2^31.
unsigned split_divisor(int ns, int *shift) {
  int k = 1;
  while ((1 << k) < ns) ++k;
  *shift = k - 1;
  return (unsigned)((((unsigned long long)1 << (31 + k)) + ns - 1) / ns);
}

hipError_t launch_attend(const CacheView &cv, const AttendLaunch &a_in, const AttendPlan &plan,
                         hipStream_t stream) {
  AttendLaunch a = a_in;
  a.gq_mul = 65536 / std::max(1, a.gq) + 1;
  a.ns_magic = plan.splits > 1 ? split_divisor(plan.splits, &a.ns_shift) : 0u;
  if (plan.two_launch || !plan.mfma) a.dbg = nullptr;      // only the single matrix-core kernel is traced
  const dim3 grid = a.kv_major ? dim3(cv.Hkv, plan.splits, cv.B) : dim3(plan.splits, cv.Hkv, cv.B);
  if (plan.two_launch) {
    const bool rows16 = a.tq > 1 || a.observe_first >= 0 || cv.G > 8;
    const int rows2 = rows16 ? kChunkRows : cv.G;                   // query rows per unit
    if (rows16 && !plan.mfma) return hipErrorInvalidValue;
    AttendFn first = attend_fn(plan.mfma ? kFormMfmaSpill : kFormValuSpill, cv.D, plan.mfma ? rows2 : cv.G, cv.chan != 0, attend_kind(a));
    AttendFn second = a.lambda ? attend_diff_finish(cv.D, rows2) : plan.mfma && cv.D == 64 ? attend_fn_finish_padded(rows2) : attend_fn_finish(cv.D, rows2);
    if (!first || !second || !a.spill) return hipErrorInvalidValue;
    hipLaunchKernelGGL(first, grid, dim3(kAttThreads), plan.lds_bytes, stream, cv.len, cv.n8, cv.head16, cv.head8, a.layer * cv.B * cv.Hkv, cv.Hkv, a.kv_major, cv, a, plan.splits,
                       plan.stash_tokens);
    const size_t lds2 = ((size_t)plan.splits * rows2 * 2 + rows2 + 2) * sizeof(float) + 2 * rows2 * sizeof(double);
    hipLaunchKernelGGL(second, grid, dim3(kAttThreads), lds2, stream, cv.len, cv.n8, cv.head16, cv.head8, a.layer * cv.B * cv.Hkv, cv.Hkv, a.kv_major, cv, a, plan.splits,
                       plan.stash_tokens);
    return hipGetLastError();
  }
  if (plan.wide_groups) {
    if (attend_kind(a) != kAttendPlain) return hipErrorInvalidValue;      // (the caller has refused it)
    a.dbg = nullptr;
    a.max_splits = wide_max_splits(plan.wide_groups * kWideRows);
    hipLaunchKernelGGL(attend_fn_wide(plan.wide_groups, plan.wide_kept), grid, dim3(kAttThreads), plan.lds_bytes, stream, cv.len, cv.n8, cv.head16, cv.head8, a.layer * cv.B * cv.Hkv, cv.Hkv, a.kv_major, cv, a, plan.splits, 0);
    return hipGetLastError();
  }
  const bool rows16 = a.tq > 1 || a.observe_first >= 0 || cv.G > 8;
  const int rows = rows16 ? kChunkRows : cv.G;
  if (rows16 && !plan.mfma) return hipErrorInvalidValue;
  AttendFn fn = attend_fn(!plan.mfma ? kFormValu : cv.page_lg ? kFormPaged : kFormMfma, cv.D, plan.mfma ? rows : cv.G, cv.chan != 0, attend_kind(a));
  if (!fn) return hipErrorInvalidValue;
#ifdef CONFKV_TRACE
  if (a.dbg && plan.mfma) {             // time stamps live in LDS behind the kernel's own
    AttendLaunch at = a;
    at.trace_off = (int)((plan.lds_bytes + 15) / 16 * 16);
    const size_t lds = at.trace_off + kAttWaves * 32 * 8;
    (void)hipFuncSetAttribute((const void *)fn, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    hipLaunchKernelGGL(fn, grid, dim3(kAttThreads), lds, stream, cv.len, cv.n8, cv.head16, cv.head8, a.layer * cv.B * cv.Hkv, cv.Hkv, a.kv_major, cv, at, plan.splits, plan.stash_tokens);
    return hipGetLastError();
  }
#endif
  hipLaunchKernelGGL(fn, grid, dim3(kAttThreads), plan.lds_bytes, stream, cv.len, cv.n8, cv.head16, cv.head8, a.layer * cv.B * cv.Hkv, cv.Hkv, a.kv_major, cv, a, plan.splits,
                     plan.stash_tokens);
  return hipGetLastError();
}

}  // namespace confkv
