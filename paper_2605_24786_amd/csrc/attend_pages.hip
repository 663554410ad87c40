// Attention of a chunk of new tokens over a paged FP16 cache of the caller's (conf_kv_attend_pages).
//
// Rows of a kv-head are (token, head of the group), token first, so that all heads of the group share the tiles.  A workgroup takes
// a block of rows of one (sequence, kv-head) against the keys those rows see, or against a part of them where there are fewer
// blocks than compute units; parts leave float32 partial results,
//   ml[slot][row] = (m, l),  o[slot][row][D] = sum over the part's keys of 2^(s - m) v,   s: scores times log2(e)
// which are merged in the order of the parts, whichever was there first.
// Products are formed transposed, scores [32 keys x 32 rows] and output [D x 32 rows] (v_mfma_f32_32x32x16_f16): a lane then holds
// values of one row only, its probabilities are the operand of the second product as they stand, and the row's statistics
// need one exchange between two lanes.
// The call's own keys and values are read from its arguments, never from the pages, so their way into the pages needs no wait.
#include <algorithm>

#include "confkv_dev.h"
#include "launch.h"

namespace confkv {

typedef _Float16 pg_h8 __attribute__((ext_vector_type(8)));
typedef _Float16 pg_h4 __attribute__((ext_vector_type(4)));
typedef short pg_s4 __attribute__((ext_vector_type(4)));
typedef float pg_f16 __attribute__((ext_vector_type(16)));

constexpr int kPgKeys = 32;                            // keys of a wavefront's tile
constexpr int kPgRows = 32;                            // rows of a matrix instruction's tile
constexpr int kNoSplit = 0x7fffffff;
constexpr int kFewWaves = 4, kFewQuantum = kFewWaves * kPgKeys;   // few rows: wavefronts, and keys that a part has at least
static_assert(kFewQuantum == kPagesLeastPart);

// Per group of sixteen lanes: lane l reads four halfs of row l / 4, columns 4 (l & 3) + [0, 4), and gets half l of each row.
__device__ __forceinline__ pg_h4 pg_read_tr(const uint8_t *p) {
  return __builtin_bit_cast(pg_h4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) pg_s4 *)p));
}
__device__ __forceinline__ float pg_other_half(float v) { return __shfl_xor(v, 32, kWave); }
// Of lanes 2 i and 2 i + 1, the other's.
__device__ __forceinline__ float pg_neighbour(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0xb1, 0xf, 0xf, false));   // quad_perm:[1,0,3,2]
}
// The signs of the result: which of two halfs are infinite or NaN (their magnitude, 0x7c00 or more, carries into the sign).
typedef unsigned pg_u4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ pg_u4 pg_odd_halfs(pg_u4 d) { return ((d & 0x7fff7fffu) + 0x04000400u) & 0x80008000u; }
__device__ __forceinline__ bool pg_odd_piece(pg_u4 v) {
  const pg_u4 o = pg_odd_halfs(v);
  return (o.x | o.y | o.z | o.w) != 0u;
}
__device__ __forceinline__ pg_u4 pg_without_odd(pg_u4 v) { return v & ~((pg_odd_halfs(v) >> 15) * 0xffffu); }
// LDS operations of a wavefront execute in order: between lanes that exchange data only the compiler has to keep it.
__device__ __forceinline__ void pg_wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// ---------------------------------------------------------------------------------------
// Which sequence, block of rows and part a workgroup has.  The lengths live on the device, so every workgroup works it out for
// itself: a lane per sequence, a scan over the wavefront.
// ---------------------------------------------------------------------------------------
struct PgSequence {
  int n, c, s;                                         // new tokens, tokens before them, first row of the call's tensors
};
__device__ __forceinline__ PgSequence pg_sequence(const PagesLaunch &a, int b) {
  PgSequence q;
  const int room = (int)min((long long)a.pages.max_pages << a.pages.lg, 1ll << 30);
  q.c = min(max(a.context[b], 0), room);
  q.n = a.count ? min(max(a.count[b], 0), a.tokens) : a.tokens;
  q.n = min(q.n, room - q.c);
  const int s = a.starts ? a.starts[b] : b * a.tokens;
  q.s = min(max(s, 0), a.rows);
  q.n = s == q.s ? min(q.n, a.rows - q.s) : 0;
  return q;
}

// Token of a sequence's row (a division by the group size; a multiplier of 0: groups of one).
__device__ __forceinline__ int pg_token(const PagesLaunch &a, int row) { return a.g_magic ? (int)(__umulhi((unsigned)row, a.g_magic) >> a.g_shift) : row; }

struct PgJob {
  int b, g, block, part, parts, part_keys;
  PgSequence q;
};
// The least quanta that a part has.  Few rows: a part takes 10 ns for each of its keys, and the workgroup that merges the parts, alone,
// some 19 ns for each row of each; the sum is least with parts of sqrt(1.9 keys rows).
// Many rows: 256 keys, of caches of 512 and more (us with parts of 256, 512, 1024: 64 rows behind 2000 tokens 19.5, 25.0, 37.9, 256 behind
// 500 22.6, 30.1, 27.2, 1024 behind 2000 32.7, 35.2, 47.4; four sequences of 333 tokens, uncut 14.5, in halves 23.5).
constexpr int kManyLeastPart = 256;
template <int R, int QUANTUM>
__device__ __forceinline__ unsigned pg_least_part(const PagesLaunch &a, unsigned longest) {
  if constexpr (R != kPgRows) return longest * QUANTUM < 2 * kManyLeastPart ? longest : kManyLeastPart / QUANTUM;
  const float rows = (float)min((long long)a.tokens * a.G, (long long)R);
  return max(1u, (unsigned)(__builtin_sqrtf((float)longest * QUANTUM * rows * 1.9f) * (1.f / QUANTUM) + 0.5f));
}
// Inclusive prefix sums over the wavefront by lane moves (an exchange through LDS takes ten times as long).
__device__ __forceinline__ int pg_scan(int v) {
#define CONFKV_DPP(ctrl, rows) v += __builtin_amdgcn_update_dpp(0, v, ctrl, rows, 0xf, false)
  CONFKV_DPP(0x111, 0xf);                              // row_shr:1
  CONFKV_DPP(0x112, 0xf);                              // row_shr:2
  CONFKV_DPP(0x114, 0xf);                              // row_shr:4
  CONFKV_DPP(0x118, 0xf);                              // row_shr:8
  CONFKV_DPP(0x142, 0xa);                              // row_bcast:15, rows 1 and 3
  CONFKV_DPP(0x143, 0xc);                              // row_bcast:31, rows 2 and 3
#undef CONFKV_DPP
  return v;
}
__device__ __forceinline__ int pg_last(int v) { return __builtin_amdgcn_readlane(v, 63); }
// The largest of values that are not negative.
__device__ __forceinline__ int pg_max(int v) {
#define CONFKV_DPP(ctrl, rows) v = max(v, __builtin_amdgcn_update_dpp(0, v, ctrl, rows, 0xf, false))
  CONFKV_DPP(0x111, 0xf);
  CONFKV_DPP(0x112, 0xf);
  CONFKV_DPP(0x114, 0xf);
  CONFKV_DPP(0x118, 0xf);
  CONFKV_DPP(0x142, 0xa);
  CONFKV_DPP(0x143, 0xc);
#undef CONFKV_DPP
  return pg_last(v);
}

// Parts of equal length for all sequences, the shortest for which every (block, part) has a slot; the blocks of a
// sequence from the last one on, whose rows see the most keys.  False: the workgroup has nothing to do.
// (R rows a block; parts in whole quanta of keys, and no shorter than is worth their merge, see pg_least_part.)
template <int R, int QUANTUM>
__device__ __forceinline__ bool pg_job(const PagesLaunch &a, unsigned x, PgJob &j) {
  const int lane = threadIdx.x & 63;
  const PgSequence mine = lane < a.B ? pg_sequence(a, lane) : PgSequence{0, 0, 0};
  auto sequence = [&](int b0) { return b0 == 0 ? mine : b0 + lane < a.B ? pg_sequence(a, b0 + lane) : PgSequence{0, 0, 0}; };
  // (n * G is below 2^30, lengths below 2^30 + 2^30)
  auto blocks_of = [&](const PgSequence &q) { return (int)(((unsigned)q.n * (unsigned)a.G + (R - 1)) / R); };
  auto length = [](const PgSequence &q) { return (unsigned)(q.c + q.n + (QUANTUM - 1)) / QUANTUM; };   // in quanta
  unsigned part = 0;                                   // quanta of a part; 0: none is cut
  if (a.slots > 0) {
    const unsigned most = (unsigned)a.slots_per_head;    // (block, part) pairs per kv-head
    unsigned blocks = 0, longest = 0;
    for (int b0 = 0; b0 < a.B; b0 += kWave) {
      const PgSequence q = sequence(b0);
      blocks += (unsigned)pg_last(pg_scan(blocks_of(q)));
      longest = max(longest, (unsigned)pg_max((int)length(q)));
    }
    const unsigned least = pg_least_part<R, QUANTUM>(a, longest);
    if (blocks > 0 && blocks <= most && least < longest) {
      float work = 0.f;                                  // (an estimate to begin with)
      for (int b0 = 0; b0 < a.B; b0 += kWave) {
        const PgSequence q = sequence(b0);
        work += (float)pg_last(pg_scan((int)fminf((float)blocks_of(q) * (float)length(q), 0x1p24f)));
      }
      part = max(least, (unsigned)(work / (float)most));
      for (;;) {
        unsigned jobs = 0;
        for (int b0 = 0; b0 < a.B; b0 += kWave) {
          const PgSequence q = sequence(b0);
          jobs += (unsigned)pg_last(pg_scan((int)min((unsigned long long)blocks_of(q) * ((length(q) + part - 1) / part), 1ull << 24)));
        }
        if (jobs <= most) break;
        part += (part + 15) / 16;
      }
    }
  }
  int at = a.h_magic ? (int)(__umulhi(x, a.h_magic) >> a.h_shift) : (int)x;   // x / Hkv
  j.g = (int)(x - (unsigned)at * (unsigned)a.Hkv);
  for (int b0 = 0; b0 < a.B; b0 += kWave) {
    const PgSequence q = sequence(b0);
    const int blocks = blocks_of(q), parts = part ? (int)((length(q) + part - 1) / part) : 1;
    const int jobs = blocks * parts;
    int end = pg_scan(jobs);
    const int all = pg_last(end);
    const int len = q.c + q.n;
    if (R != kPgRows && a.B <= kWave && __builtin_amdgcn_ballot_w64(lane < a.B && len != __builtin_amdgcn_readlane(len, 0))) {
      // long sequences first: the workgroups that come last shall have little to do (16 sequences of 0 to 700 tokens behind up
      // to 5000: 416 -> 393 us)
      end = jobs;
      for (int i = 0; i < a.B; ++i) {
        const int other = __builtin_amdgcn_readlane(len, i);
        end += other > len || (other == len && i < lane) ? __builtin_amdgcn_readlane(jobs, i) : 0;
      }
    }
    const unsigned long long hit = __builtin_amdgcn_ballot_w64(at < end && at >= end - jobs);
    if (hit) {
      const int l = __builtin_ctzll(hit);
      at -= __builtin_amdgcn_readlane(end, l) - __builtin_amdgcn_readlane(jobs, l);
      j.b = b0 + l;
      j.parts = __builtin_amdgcn_readlane(parts, l);
      const int back = j.parts > 1 ? at / j.parts : at;
      j.part = at - back * j.parts;
      j.block = __builtin_amdgcn_readlane(blocks, l) - 1 - back;
      j.part_keys = j.parts > 1 ? (int)(part * QUANTUM) : kNoSplit;
      j.q.n = __builtin_amdgcn_readlane(q.n, l);
      j.q.c = __builtin_amdgcn_readlane(q.c, l);
      j.q.s = __builtin_amdgcn_readlane(q.s, l);
      return true;
    }
    at -= all;
  }
  return false;
}

// ---------------------------------------------------------------------------------------
// Rows of K and V of one kv-head, wherever they are.
// ---------------------------------------------------------------------------------------
template <int D>
struct PgSource {
  static constexpr int PR = D / 8, RWI = kWave / PR;   // 16-byte pieces of a row; rows that a wavefront's load covers
  const __half *k, *v, *knew, *vnew;                   // of the kv-head
  const int32_t *table;                                // of the sequence
  long long page_stride, token_stride, new_stride, lane_off;
  int lg, max_pages, n_pages, c, n;                    // tokens in front (0x7fffffff: all come from the pages), tokens in all

  __device__ __forceinline__ void init(const PagesLaunch &a, const PgJob &j) {
    const int lane = threadIdx.x & 63;
    k = a.pages.k + j.g * a.pages.head_stride;
    v = a.pages.v + j.g * a.pages.head_stride;
    new_stride = (long long)a.Hkv * D;
    knew = a.knew ? a.knew + (j.q.s * (long long)a.Hkv + j.g) * D : nullptr;
    vnew = a.knew ? a.vnew + (j.q.s * (long long)a.Hkv + j.g) * D : nullptr;
    table = a.pages.table + j.b * a.pages.table_stride;
    page_stride = a.pages.page_stride;
    token_stride = a.pages.token_stride;
    lane_off = (lane / PR) * token_stride + (lane % PR) * 8;
    lg = a.pages.lg;
    max_pages = a.pages.max_pages;
    n_pages = a.pages.n_pages;
    c = a.knew ? j.q.c : 0x7fffffff;
    n = j.q.c + j.q.n;
  }
  // the table's entry for a token (a place behind the table: its last entry; nothing read from there counts)
  __device__ __forceinline__ int entry(int token) const { return table[min(token >> lg, max_pages - 1)]; }
  // Offset of token r0's row (a multiple of RWI, as are the pages' lengths: the next RWI lie in one page, whose entry is e).
  __device__ __forceinline__ long long page_offset(int r0, int e) const {
    e = min(max(e, 0), n_pages - 1);
    return e * page_stride + (r0 & ((1 << lg) - 1)) * token_stride;
  }
  __device__ __forceinline__ void load(int r0, int e, pg_u4 &kr, pg_u4 &vr) const {
    const long long o = page_offset(r0, e) + lane_off;
    const __half *kp = k + o, *vp = v + o;
    if (r0 + RWI > c) {                                // (tokens of the call among them; behind the last one its row again)
      const int lane = threadIdx.x & 63, t = min(r0 + lane / PR, n - 1);
      if (t >= c) {
        const long long m = (t - c) * new_stride + (lane % PR) * 8;
        kp = knew + m;
        vp = vnew + m;
      }
    }
    kr = *(const pg_u4 *)kp;
    vr = *(const pg_u4 *)vp;
  }
  __device__ __forceinline__ const __half *value_row(int t) const {
    if (t >= c) return vnew + (t - c) * new_stride;
    const int e = min(max(entry(t), 0), n_pages - 1);
    return v + e * page_stride + (t & ((1 << lg) - 1)) * token_stride;
  }
};

// ---------------------------------------------------------------------------------------
// Thirty-two rows of a wavefront: queries, running reference, sum and output, and how many keys they see.
// ---------------------------------------------------------------------------------------
template <int D>
struct PgRows {
  pg_h8 qf[D / 16];
  pg_f16 O[D / 32];
  // Probabilities are 2^((score - ref) * c + off): off follows the row's maximum, and lifts it to 2^10, so that as fp16 operands they keep
  // eleven bits down to 2^-24 of the largest (unlifted 2^-14).  One fused operation per score, whose product is not rounded;
  // what off is rounded to is off for all keys alike.  Up to kFar ref is 0.  Beyond, off's steps come near the slack that fp16
  // leaves (2^27: 16 powers of two), so there the maximum is ref, taken away before the score is scaled, in a pass of its own
  // that only wavefronts with such a row run (`far`).
  float off, ref, limit, l;                            // limit: the score beyond which the reference moves
  bool far;
  int lim, least, most;                                // keys the lane's row sees; the fewest and the most

  static constexpr float kLift = 10.f, kSlack = 5.5f;  // 2^15.5 is 46341 of fp16's 65504
  static constexpr float kFar = 0x1p20f;               // off within 2^-3 of what it is meant to be

  __device__ __forceinline__ void reset() {
#pragma unroll
    for (int nt = 0; nt < D / 32; ++nt)
#pragma unroll
      for (int i = 0; i < 16; ++i) O[nt][i] = 0.f;
    off = INFINITY;
    ref = 0.f;
    limit = -INFINITY;
    far = false;
    l = 0.f;
  }
  // rows first .. first + 31 of the sequence's n * G
  __device__ __forceinline__ void init(const PagesLaunch &a, const PgJob &j, int first) {
    const int lane = threadIdx.x & 63, h = lane >> 5, all = j.q.n * a.G;
    const int r = min(first + (lane & 31), all - 1), t = pg_token(a, r), hq = r - t * a.G;
    const __half *q = a.q + ((long long)(j.q.s + t) * a.Hkv * a.G + j.g * a.G + hq) * D;
#pragma unroll
    for (int s = 0; s < D / 16; ++s) qf[s] = __builtin_bit_cast(pg_h8, *(const int4 *)(q + 16 * s + 8 * h));
    lim = j.q.c + t + 1;
    least = __builtin_amdgcn_readfirstlane(lim);       // (rows in order: the first sees least)
    most = first < all ? __builtin_amdgcn_readlane(lim, 31) : 0;
    reset();
  }
  template <int KROW>
  __device__ __forceinline__ void scores(const uint8_t *Kt, pg_f16 &sc) const {
    const int lane = threadIdx.x & 63, l32 = lane & 31, h = lane >> 5;
#pragma unroll
    for (int i = 0; i < 16; ++i) sc[i] = 0.f;
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      const pg_h8 kf = *(const pg_h8 *)(Kt + l32 * KROW + 32 * s + 16 * h);
      sc = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf, qf[s], sc, 0, 0, 0);
    }
  }
  // The lane's largest score of keys key0 .. key0 + 31; element i: key key0 + 8 (i / 4) + 4 h + i % 4 (kMask: some may be behind what
  // a row sees, and leave).
  template <bool kMask>
  __device__ __forceinline__ float peak(pg_f16 &sc, int key0) const {
    const int h = (threadIdx.x & 63) >> 5;
    if (kMask && key0 + kPgKeys > least) {
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[i] = 8 * (i / 4) + (i & 3) < lim - key0 - 4 * h ? sc[i] : -INFINITY;
    }
    float mx = sc[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, sc[i]);
    return mx;
  }
  // The reference only has to stay near the maximum (the merges are exact for any), so the exchange and the rescaling run
  // where a score passes it by more than kSlack (a far one at all: its steps are as long).
  __device__ __forceinline__ bool passes(float mx) const { return mx > limit; }
  __device__ __forceinline__ void raise(float mx, float c) {
    const float top = fmaxf(mx, pg_other_half(mx)), scaled = top * c;
    const bool higher = fmaf(top - ref, c, off) > kLift, distant = !(fabsf(scaled) < kFar);   // (no score yet: top is -inf, nothing is higher)
    const float now_ref = !higher ? ref : distant ? top : 0.f, now = !higher ? off : distant ? kLift : kLift - scaled;
    const float corr = higher ? __builtin_amdgcn_exp2f(fmaf(ref - now_ref, c, now - off)) : 1.f;
    off = now;
    ref = now_ref;
    limit = !higher ? limit : distant ? top : top + kSlack / c;
    far = __builtin_amdgcn_ballot_w64(ref != 0.f) != 0ull;
    l *= corr;
#pragma unroll
    for (int nt = 0; nt < D / 32; ++nt) O[nt] *= corr;
  }
  __device__ __forceinline__ void follow(float mx, float c, pg_f16 &sc) {
    if (__builtin_amdgcn_ballot_w64(passes(mx))) raise(mx, c);
    if (__builtin_expect(far, 0)) {
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[i] -= ref;
    }
  }
  // scores, behind follow() -> probabilities
  __device__ __forceinline__ void weights(const pg_f16 &sc, float c, pg_h8 (&pb)[2]) {
    const float at = off == INFINITY ? 0.f : off;
    float sum[4];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float p = __builtin_amdgcn_exp2f(fmaf(sc[i], c, at));
      sum[i & 3] = i < 4 ? p : sum[i & 3] + p;
      // (fp16 operands: half a step, 2^-11 of each probability)
      pb[i / 8][i & 7] = (_Float16)p;
    }
    l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
  }
  template <bool kMask>
  __device__ __forceinline__ void weigh(pg_f16 &sc, int key0, float c, pg_h8 (&pb)[2]) {
    const float mx = peak<kMask>(sc, key0);
    follow(mx, c, sc);
    weights(sc, c, pb);
  }
  template <int VROW>
  __device__ __forceinline__ void add(const uint8_t *Vt, const pg_h8 (&pb)[2]) {
    const int lane = threadIdx.x & 63, h = lane >> 5, t16 = lane & 15, c2 = (lane >> 4) & 1;
    const uint8_t *vp = Vt + (4 * h + (t16 >> 2)) * VROW + 32 * c2 + 8 * (t16 & 3);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
#pragma unroll
      for (int nt = 0; nt < D / 32; ++nt) {
        const pg_h4 v0 = pg_read_tr(vp + 16 * s * VROW + 64 * nt), v1 = pg_read_tr(vp + (16 * s + 8) * VROW + 64 * nt);
        O[nt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7), pb[s], O[nt], 0, 0, 0);
      }
    }
  }
  // Whether some channel is no number although the row's sum, of both halves, is one.
  __device__ __forceinline__ bool odd(float sum) const {
    float z[8] = {};
#pragma unroll
    for (int nt = 0; nt < D / 32; ++nt)
#pragma unroll
      for (int i = 0; i < 16; ++i) z[i & 7] = fmaf(O[nt][i], 0.f, z[i & 7]);
    const float all = ((z[0] + z[1]) + (z[2] + z[3])) + ((z[4] + z[5]) + (z[6] + z[7]));
    return all != all && sum == sum;
  }
  // The row's sum over both halves, with what the tiles left out put right.
  __device__ __forceinline__ float finish(const PgSource<D> &src, int lo, int hi, bool dropped) {
    const float sum = l + pg_other_half(l);
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(dropped || odd(sum)) != 0ull, 0)) show_odd_values(src, lo, hi);
    return sum;
  }
  // Its maximum for the merges.  (No key: -inf.  A sum that is NaN, from a score that is none, outweighs the others: a merge shall not
  // lose it.)
  __device__ __forceinline__ float maximum(float sum, float c) const { return sum == sum ? fmaf(ref, c, -off) : INFINITY; }
  template <int OROW>
  __device__ __forceinline__ void store_partial(float *to) const {
    const int h = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int nt = 0; nt < D / 32; ++nt)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *(float4 *)(to + 32 * nt + 8 * i + 4 * h) = make_float4(O[nt][4 * i], O[nt][4 * i + 1], O[nt][4 * i + 2], O[nt][4 * i + 3]);
  }
  // Values that are infinite or NaN, of the keys [lo, hi) that the lane's row sees: each makes its channel what they add up to, since a
  // probability is positive however far the products above rounded it (where to zero, they made NaN of an infinite value, and
  // where the values left the tile they were never met).  The first pass empties these channels, the second adds.
  __device__ __forceinline__ void show_odd_values(const PgSource<D> &src, int lo, int hi) {
    constexpr int PR = D / 8, RWI = kWave / PR;
    const int lane = threadIdx.x & 63, h = lane >> 5;
    hi = min(hi, most);
#pragma unroll 1
    for (int pass = 0; pass < 2; ++pass) {
#pragma unroll 1
      for (int r0 = lo; r0 < hi; r0 += RWI) {
        const int t = min(r0 + lane / PR, hi - 1);
        const pg_u4 v = *(const pg_u4 *)(src.value_row(t) + lane % PR * 8);
        if (__builtin_amdgcn_ballot_w64(pg_odd_piece(v)) == 0ull) continue;
#pragma unroll 1
        for (int key = r0; key < min(r0 + RWI, hi); ++key) {
          const __half *vr = src.value_row(key);
#pragma unroll
          for (int nt = 0; nt < D / 32; ++nt)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const pg_h4 x4 = *(const pg_h4 *)(vr + 32 * nt + 8 * k + 4 * h);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float x = (float)x4[e];
                const int i = 4 * k + e;
                if (key < lim && !(fabsf(x) < INFINITY)) O[nt][i] = pass ? O[nt][i] + x : 0.f;
              }
            }
        }
      }
    }
  }
};

// Weight of a partial result with maximum m beside one of maximum M.
__device__ __forceinline__ float pg_weight(float m, float M) {
  return m == -INFINITY ? 0.f : fmaxf(__builtin_amdgcn_exp2f(m - M), kLeastWeight);
}
// y += f x (f zero, of a result without keys: whatever x holds)
__device__ __forceinline__ void pg_add4(float4 &y, float f, const float4 &x) {
  const bool some = f != 0.f;
  y.x = some ? fmaf(f, x.x, y.x) : y.x;
  y.y = some ? fmaf(f, x.y, y.y) : y.y;
  y.z = some ? fmaf(f, x.z, y.z) : y.z;
  y.w = some ? fmaf(f, x.w, y.w) : y.w;
}
// Where row `row` of the sequence goes, [rows][heads][D]: nowhere behind the last one, and where heads are subtracted in pairs, odd
// rows into their pair's with the weight f.
struct PgOut {
  __half *at;
  float f;
};
template <int D>
__device__ __forceinline__ PgOut pg_out(const PagesLaunch &a, const PgJob &j, int row) {
  const int r = min(row, j.q.n * a.G - 1), t = pg_token(a, r), hq = r - t * a.G;
  const long long token = j.q.s + t;
  if (!a.lambda) return {row == r ? a.out + ((token * a.Hkv + j.g) * a.G + hq) * D : nullptr, 0.f};
  const int half = a.G >> 1, pair = hq >> 1;
  return {row == r && (hq & 1) == 0 ? a.out + ((token * a.Hkv + j.g) * half + pair) * D : nullptr, a.lambda[token * a.lambda_stride + j.g * half + pair]};
}
// Channels d .. d + 3 of a row, sums y over its normaliser; sixteen neighbouring lanes hold a row, the next sixteen the next one.
// (All lanes call it.)
__device__ __forceinline__ void pg_write_out(const PagesLaunch &a, const PgOut &to, int d, float4 y, float inv) {
  y.x *= inv;
  y.y *= inv;
  y.z *= inv;
  y.w *= inv;
  if (a.lambda) {
    const float4 z = make_float4(__shfl_xor(y.x, 16, kWave), __shfl_xor(y.y, 16, kWave), __shfl_xor(y.z, 16, kWave), __shfl_xor(y.w, 16, kWave));
    y = make_float4(fmaf(-to.f, z.x, y.x), fmaf(-to.f, z.y, y.y), fmaf(-to.f, z.z, y.z), fmaf(-to.f, z.w, y.w));
  }
  if (to.at) *(pg_h4 *)(to.at + d) = pg_h4{(_Float16)y.x, (_Float16)y.y, (_Float16)y.z, (_Float16)y.w};
}

// ---------------------------------------------------------------------------------------
// The parts of a block of few rows: partial results go to scratch, and the workgroup that is last there merges them.  They go and
// come at device scope, past the L2 of the workgroup's XCD, so that no cache is written back or emptied; a part is counted once its
// stores have been acknowledged.  The counter goes back to zero for the next call.  (A merge in a launch of its own took 6 to 20 us.)
// ---------------------------------------------------------------------------------------
__device__ __forceinline__ void pg_store8(float *to, float x, float y) {
  __hip_atomic_store((unsigned long long *)to, (unsigned long long)__float_as_uint(y) << 32 | __float_as_uint(x), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 pg_load8(const float *from) {
  const unsigned long long v = __hip_atomic_load((const unsigned long long *)from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return make_float2(__uint_as_float((unsigned)v), __uint_as_float((unsigned)(v >> 32)));
}
template <int D>
struct PgParts {
  static constexpr int R = kPgRows;
  static __device__ __forceinline__ long long at(int row) { return (long long)blockIdx.x * R + row; }
  static __device__ __forceinline__ void store(const PagesLaunch &a, int row, int d, const float4 &y) {
    float *to = a.o + at(row) * D + d;
    pg_store8(to, y.x, y.y);
    pg_store8(to + 2, y.z, y.w);
  }
  static __device__ __forceinline__ void store_sums(const PagesLaunch &a, int row, float m, float l) { pg_store8((float *)(a.ml + at(row)), m, l); }
  // Behind the stores, all threads of the workgroup; `room` is kRoom floats of LDS that nobody uses any more.
  static constexpr int kGroups = kFewWaves * kWave / 16, kSlot = D + 4, kRoom = R * kSlot;
  static __device__ __forceinline__ void merge(const PagesLaunch &a, const PgJob &j, float *room) {
    __shared__ int s_last;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    const unsigned first = blockIdx.x - j.part * a.Hkv;  // the slot of part 0, whose counter is the block's
    if (threadIdx.x == 0) {
      const unsigned before = __hip_atomic_fetch_add(a.arrived + first, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      s_last = before == (unsigned)j.parts - 1u;
      if (s_last) __hip_atomic_store(a.arrived + first, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (!s_last) return;
    // Groups of sixteen threads.  Where there are fewer rows than groups, 2^lg of them share a row, each with parts of its own.
    const int first_row = j.block * R, rows = min(R, j.q.n * a.G - first_row), d = (threadIdx.x & 15) * 4, group = threadIdx.x >> 4;
    int lg = 0;
    while ((2 << lg) * rows <= kGroups) ++lg;
    const int mate = group & ((1 << lg) - 1), each = kGroups >> lg;
    const long long apart = (long long)a.Hkv * R;
    auto clear = [](float4 (&y)[D / 64], float &l) {
#pragma unroll
      for (int q = 0; q < D / 64; ++q) y[q] = make_float4(0.f, 0.f, 0.f, 0.f);
      l = 0.f;
    };
    for (int r0 = 0, slot = group; r0 < rows; r0 += each, slot += kGroups) {
      const int r = min(r0 + (group >> lg), rows - 1);
      const float *ml = (const float *)(a.ml + (long long)first * R + r);
      const float *o = a.o + ((long long)first * R + r) * D + d;
      float M = -INFINITY, l;
      float4 y[D / 64];
      clear(y, l);
      constexpr int kAhead = 8;                          // parts whose words are requested together
      for (int p0 = mate; p0 < j.parts; p0 += kAhead << lg) {
        float2 s[kAhead], x[kAhead][D / 64][2];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          const long long p = min(p0 + (k << lg), j.parts - 1) * apart;
          s[k] = pg_load8(ml + 2 * p);
#pragma unroll
          for (int q = 0; q < D / 64; ++q) {
            x[k][q][0] = pg_load8(o + p * D + 64 * q);
            x[k][q][1] = pg_load8(o + p * D + 64 * q + 2);
          }
        }
        float now = M;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) now = fmaxf(now, s[k].x);
        const float f0 = pg_weight(M, now), was = l;
        float4 old[D / 64];
#pragma unroll
        for (int q = 0; q < D / 64; ++q) old[q] = y[q];
        clear(y, l);
        l = f0 == 0.f ? l : was * f0;
#pragma unroll
        for (int q = 0; q < D / 64; ++q) pg_add4(y[q], f0, old[q]);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          const float f = p0 + (k << lg) < j.parts ? pg_weight(s[k].x, now) : 0.f;
          l = f == 0.f ? l : fmaf(f, s[k].y, l);
#pragma unroll
          for (int q = 0; q < D / 64; ++q) pg_add4(y[q], f, make_float4(x[k][q][0].x, x[k][q][0].y, x[k][q][1].x, x[k][q][1].y));
        }
        M = now;
      }
      if (slot < R) {
#pragma unroll
        for (int q = 0; q < D / 64; ++q) *(float4 *)(room + slot * kSlot + d + 64 * q) = y[q];
        if (d == 0) *(float2 *)(room + slot * kSlot + D) = make_float2(M, l);
      }
    }
    __syncthreads();
    for (int r0 = 0; r0 < rows; r0 += kGroups) {
      const int row = r0 + group, r = min(row, rows - 1);
      const float *mine = room + (r / each * kGroups + ((r & (each - 1)) << lg)) * kSlot;
      float M = -INFINITY, l;
      float4 y[D / 64];
      clear(y, l);
      for (int k = 0; k < 1 << lg; ++k) M = fmaxf(M, mine[k * kSlot + D]);
      for (int k = 0; k < 1 << lg; ++k) {
        const float2 s = *(const float2 *)(mine + k * kSlot + D);
        const float f = pg_weight(s.x, M);
        l = f == 0.f ? l : fmaf(f, s.y, l);
#pragma unroll
        for (int q = 0; q < D / 64; ++q) pg_add4(y[q], f, *(const float4 *)(mine + k * kSlot + d + 64 * q));
      }
      const PgOut to = pg_out<D>(a, j, first_row + row);
#pragma unroll
      for (int q = 0; q < D / 64; ++q) pg_write_out(a, to, d + 64 * q, y[q], 1.f / l);
    }
  }
};

// The new tokens whose first row lies in rows [lo, hi) of the sequence go to their pages (an entry that is no page: nowhere).
template <int D>
__device__ __forceinline__ void pg_append(const PagesLaunch &a, const PgJob &j, int lo, int hi, int threads) {
  if (!a.knew || j.part != j.parts - 1) return;          // (the last part is the shortest)
  constexpr int PR = D / 8, kAhead = 4;                  // pieces of a thread whose rows are requested together
  const int t0 = pg_token(a, lo + a.G - 1), t1 = min(j.q.n, pg_token(a, hi + a.G - 1));
  const int32_t *table = a.pages.table + j.b * a.pages.table_stride;
  for (int i0 = threadIdx.x; i0 < (t1 - t0) * PR; i0 += kAhead * threads) {
    pg_u4 k[kAhead], v[kAhead];
    long long to[kAhead];
#pragma unroll
    for (int n = 0; n < kAhead; ++n) {
      to[n] = -1;
      if (__builtin_amdgcn_readfirstlane(i0) + n * threads >= (t1 - t0) * PR) continue;
      const int i = i0 + n * threads, t = min(t0 + i / PR, t1 - 1), at = j.q.c + t, e = table[at >> a.pages.lg];
      const long long from = ((j.q.s + t) * (long long)a.Hkv + j.g) * D + i % PR * 8;
      k[n] = *(const pg_u4 *)(a.knew + from);
      v[n] = *(const pg_u4 *)(a.vnew + from);
      to[n] = i < (t1 - t0) * PR && (unsigned)e < (unsigned)a.pages.n_pages ? a.pages.offset(e, at, j.g) + i % PR * 8 : -1;
    }
#pragma unroll
    for (int n = 0; n < kAhead; ++n) {
      if (to[n] < 0) continue;
      *(pg_u4 *)(a.pages.k + to[n]) = k[n];
      *(pg_u4 *)(a.pages.v + to[n]) = v[n];
    }
  }
}

// Tiles in LDS, rows of these strides (bytes): 16-byte pieces of eight K rows on different banks, 64-byte pieces of four V rows
// likewise.
template <int D>
struct PgTile {
  static constexpr int KROW = 2 * D + 16, VROW = 2 * D + 64;
  static constexpr int kBytes = kPgKeys * (KROW + VROW);
  static constexpr int OROW = D + 4;                   // floats of a partial's row where wavefronts merge
};

// ---------------------------------------------------------------------------------------
// Up to 32 rows of a (sequence, kv-head), single tokens above all: bound by the bytes of K and V.  Four wavefronts take the
// part's tiles of 32 keys in turn; a wavefront waits for nobody before the merge: it loads and multiplies tiles of its own, the
// next one in flight in registers while this one is used.  Two workgroups share a compute unit, so that one's first and last trips
// to memory run beside the other's rows: 32 single tokens behind up to 8192 tokens, 437 MB in 96 us (4.6 TB/s; a large copy reaches
// 5.1), 167 with eight wavefronts in one workgroup per unit.  One token behind 1000: 10.4 us, a chain of lengths, table entry, rows,
// the tile, the partial results' way out, the counter and their way back.
// ---------------------------------------------------------------------------------------
constexpr int kManyQuantum = 64;

template <int D>
__global__ __launch_bounds__(kFewWaves *kWave) __attribute__((amdgpu_waves_per_eu(2, 2))) void pages_few_kernel(PagesLaunch a) {
  using L = PgTile<D>;
  constexpr int PR = D / 8, RWI = kWave / PR, NP = kPgKeys / RWI;
  __shared__ __align__(16) uint8_t s_tile[kFewWaves * L::kBytes];
  __shared__ float s_m[kFewWaves][kPgRows], s_l[kFewWaves][kPgRows];
  static_assert(kPgRows * L::OROW * 4 <= L::kBytes, "a wavefront's partial fits its tile");
  PgJob j;
  if (!pg_job<kPgRows, kFewQuantum>(a, blockIdx.x, j)) return;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, h = lane >> 5;
  PgSource<D> src;
  src.init(a, j);
  const int first_row = j.block * kPgRows;
  const int lo = j.parts > 1 ? j.part * j.part_keys : 0;
  const int hi = (int)min((long long)lo + j.part_keys, (long long)(j.q.c + j.q.n));
  PgRows<D> st;
  struct Turn { pg_u4 k[NP], v[NP]; } x;
  auto load = [&](int base, int ent) {
#pragma unroll
    for (int i = 0; i < NP; ++i) src.load(base + RWI * i, __builtin_amdgcn_readlane(ent, RWI * i), x.k[i], x.v[i]);
  };
  int key0 = lo + w * kPgKeys;
  int ent = 0;
  if (key0 < hi) {
    ent = src.entry(key0 + l32);
    load(key0, ent);
    ent = src.entry(key0 + kFewQuantum + l32);
  }
  st.init(a, j, first_row);
  pg_append<D>(a, j, first_row, first_row + kPgRows, kFewWaves * kWave);
  const int end = min(hi, st.most);
  const float c = a.sm_scale * 1.44269504088896341f;
  uint8_t *Kt = s_tile + w * L::kBytes, *Vt = Kt + kPgKeys * L::KROW;
  bool dropped = false;
  for (; key0 < end; key0 += kFewQuantum) {
    // Keys that some row does not see meet it with probability 0, which does not silence an infinite or NaN value: where there
    // are such rows these values leave the tile here and reach the rows that do see them at the end.
    if (key0 + kPgKeys > st.least) {
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        dropped |= pg_odd_piece(x.v[i]);
        x.v[i] = pg_without_odd(x.v[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int row = RWI * i + lane / PR;
      *(pg_u4 *)(Kt + row * L::KROW + lane % PR * 16) = x.k[i];
      *(pg_u4 *)(Vt + row * L::VROW + lane % PR * 16) = x.v[i];
    }
    pg_wave_sync();
    if (key0 + kFewQuantum < end) {
      load(key0 + kFewQuantum, ent);
      ent = src.entry(key0 + 2 * kFewQuantum + l32);
    }
    pg_f16 sc;
    pg_h8 pb[2];
    st.template scores<L::KROW>(Kt, sc);
    st.template weigh<true>(sc, key0, c, pb);
    st.template add<L::VROW>(Vt, pb);
    pg_wave_sync();
  }
  const float sum = st.finish(src, lo, hi, dropped);
  // (no key: -inf stays; a sum that is NaN, from a score that is none, outweighs the others: a merge shall not lose it)
  if (h == 0) {
    s_m[w][l32] = st.maximum(sum, c);
    s_l[w][l32] = sum;
  }
  st.template store_partial<L::OROW>((float *)(s_tile + w * L::kBytes) + l32 * L::OROW);
  __syncthreads();
  // sixteen threads per row merge the wavefronts' partials
  const int rows = min(kPgRows, j.q.n * a.G - first_row);
  for (int r0 = 0; r0 < rows; r0 += kFewWaves * 4) {
    const int row = r0 + (tid >> 4);
    const PgOut to = pg_out<D>(a, j, first_row + row);
    float m[kFewWaves], M = -INFINITY, l = 0.f;
#pragma unroll
    for (int k = 0; k < kFewWaves; ++k) {
      m[k] = s_m[k][row];
      M = fmaxf(M, m[k]);
    }
#pragma unroll
    for (int k = 0; k < kFewWaves; ++k) {
      m[k] = pg_weight(m[k], M);
      l = m[k] == 0.f ? l : fmaf(m[k], s_l[k][row], l);
    }
#pragma unroll
    for (int p = 0; p < D / 64; ++p) {
      const int d = (tid & 15) * 4 + 64 * p;
      float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < kFewWaves; ++k) pg_add4(y, m[k], *(const float4 *)((const float *)(s_tile + k * L::kBytes) + row * L::OROW + d));
      if (j.parts == 1) pg_write_out(a, to, d, y, 1.f / l);
      else if (row < rows) PgParts<D>::store(a, row, d, y);
    }
    if (j.parts > 1 && row < rows && (tid & 15) == 0) PgParts<D>::store_sums(a, row, M, l);
  }
  if (j.parts > 1) PgParts<D>::merge(a, j, (float *)s_tile);
  static_assert(PgParts<D>::kRoom * 4 <= sizeof(s_tile));
}

// ---------------------------------------------------------------------------------------
// More rows: bound by the matrix products and the exponentials, and in the end by power.  Eight wavefronts of 32 rows each share tiles
// of 64 keys in three buffers, one barrier per tile; the tile after the next is on its way.
// Four prompts of 8192 tokens (32 heads, 8 kv-heads, 128 channels): 2.20 ms, 1000 TFLOP/s where a large library product reaches 1136 (other
// cards take up to 2.46: the clock that their power leaves).  The
// matrix units are busy in 48 % of the cycles and the vector units in 47 %, at 1.68 of 2.4 GHz.  On the way: tiles through registers
// with padded rows 3.75 ms; straight into LDS 2.57; addresses of whole tiles from scalars 2.51; scores a step ahead 2.46 (before: four
// wavefronts and two buffers, two workgroups to a unit).  64 rows a wavefront, which halves the reads of the tiles, leave one wavefront
// to a SIMD: 2.9 to 3.0, with their halves half a step apart 2.47.
//
// Rows come straight into LDS (16 bytes a lane, no registers on the way), so a tile's rows lie as they are, 2 D bytes apart, and the
// pieces of a row are permuted instead: piece p of row r lies at slot p ^ f(r), with an f that puts what the reads below take
// together on different banks -- eight lanes' pieces of K at one place of their rows, the pieces of four neighbouring V rows.
// ---------------------------------------------------------------------------------------
constexpr int kManyWaves = 8, kManyKeys = 64, kManyBuffers = 3, kManyThreads = kManyWaves * kWave, kManyRows = kManyWaves * kPgRows;

template <int D>
__device__ __forceinline__ constexpr int pg_swizzle(int r) {
  return D == 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
}
// Sixteen bytes per lane from the lane's address to LDS bytes [to, to + 1024), lane by lane.  (m0, which holds `to`, is an operand that the
// compiler writes, so that it knows what became of its own; the load may follow that write by one wait state at the least.)
__device__ __forceinline__ void pg_load_lds(const void *from, unsigned to) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"{m0}"(__builtin_amdgcn_readfirstlane(to)), "v"(from) : "memory");
}
// The same from `from`, alike in all lanes, plus the lane's offset in bytes.
__device__ __forceinline__ void pg_load_lds(const void *from, unsigned offset, unsigned to) {
  const unsigned long long p = (unsigned long long)from;
  const unsigned long long at = (unsigned long long)__builtin_amdgcn_readfirstlane((int)(p >> 32)) << 32 | (unsigned)__builtin_amdgcn_readfirstlane((int)p);
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"{m0}"(__builtin_amdgcn_readfirstlane(to)), "v"(offset), "s"(at) : "memory");
}
__device__ __forceinline__ unsigned pg_lds_at(const void *p) {
  return (unsigned)(uintptr_t)(__attribute__((address_space(3))) const char *)p;
}
// Everything the wavefront has requested is there, and then everybody's.
__device__ __forceinline__ void pg_arrive() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void pg_barrier() { asm volatile("s_barrier" ::: "memory"); }

template <int D>
struct PgMany {
  static constexpr int PR = D / 8, RWI = kWave / PR, RPP = kManyThreads / PR, NP = kManyKeys / RPP, ROW = 2 * D;
  static constexpr int kPlane = kManyKeys * ROW, kBuffer = 2 * kPlane, kSub = kPgKeys * ROW;

  PgRows<D> rows;
  float c;
  int k_off, v_off;                                    // the lane's places in a tile: K fragment 0, V fragment 0

  __device__ __forceinline__ void init(const PagesLaunch &a, const PgJob &j, int first_row) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, l32 = lane & 31, h = lane >> 5, t16 = lane & 15, c2 = (lane >> 4) & 1;
    rows.init(a, j, first_row + w * kPgRows);
    c = a.sm_scale * 1.44269504088896341f;
    k_off = l32 * ROW + ((h ^ pg_swizzle<D>(l32)) << 4);
    const int vr = 4 * h + (t16 >> 2);
    v_off = kPlane + vr * ROW + (((2 * c2 + ((t16 & 3) >> 1)) ^ pg_swizzle<D>(vr)) << 4) + 8 * (t16 & 1);
  }
  // scores of the 32 keys at byte offset `at`
  __device__ __forceinline__ void scores(const uint8_t *lds, int at, pg_f16 &sc) const {
#pragma unroll
    for (int i = 0; i < 16; ++i) sc[i] = 0.f;
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
      sc = __builtin_amdgcn_mfma_f32_32x32x16_f16(*(const pg_h8 *)(lds + at + (k_off ^ (s << 5))), rows.qf[s], sc, 0, 0, 0);
  }
  __device__ __forceinline__ void add(const uint8_t *lds, int at, const pg_h8 (&pb)[2]) {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int nt = 0; nt < D / 32; ++nt) {
        const uint8_t *vp = lds + at + 16 * s * ROW;
        const pg_h4 v0 = pg_read_tr(vp + (v_off ^ (nt << 6))), v1 = pg_read_tr(vp + 8 * ROW + (v_off ^ (nt << 6) ^ 32));
        rows.O[nt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7), pb[s], rows.O[nt], 0, 0, 0);
      }
  }
};

template <int D>
__global__ __launch_bounds__(kManyThreads) __attribute__((amdgpu_waves_per_eu(D == 64 ? 4 : 2, D == 64 ? 4 : 2))) void pages_many_kernel(PagesLaunch a) {
  using M = PgMany<D>;
  constexpr int PR = M::PR, RWI = M::RWI, RPP = M::RPP, NP = M::NP, R = kManyRows, ROW = M::ROW;
  constexpr int kRoom = std::max(kManyBuffers * M::kBuffer, kManyWaves * kPgRows * 256);   // the tiles, later the rows
  __shared__ __align__(16) uint8_t s_tile[kRoom];
  __shared__ int s_bad[kManyBuffers];
  PgJob j;
  if (!pg_job<R, kManyQuantum>(a, blockIdx.x, j)) return;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  PgSource<D> src;
  src.init(a, j);
  const int first_row = j.block * R, last_row = min(first_row + R, j.q.n * a.G) - 1;
  const int lo = j.parts > 1 ? j.part * j.part_keys : 0;
  const int seen = j.q.c + pg_token(a, last_row) + 1;    // keys that the block's last row sees
  const int hi = (int)min((long long)lo + j.part_keys, (long long)seen);
  const int all_least = j.q.c + pg_token(a, first_row) + 1;   // and its first one
  const int tiles = hi > lo ? (hi - lo + kManyKeys - 1) / kManyKeys : 0;
  const int full = max(0, (min(all_least, hi) - lo) / kManyKeys);   // tiles that every row sees to the end
  // The lane's row and piece of a wavefront's load; f does not depend on which of a tile's loads it is.
  const int lrow = RWI * w + lane / PR, lpiece = (lane % PR) ^ pg_swizzle<D>(lrow);
  const long long lane_off = (lane / PR) * src.token_stride + lpiece * 8;
  const unsigned page_lane = (unsigned)(2 * lane_off), new_lane = (unsigned)(2 * ((lane / PR) * src.new_stride + lpiece * 8));
  const bool near = src.token_stride < 1 << 26 && src.new_stride < 1 << 26;   // (a wavefront's rows less than 2^32 bytes apart)
  const unsigned lds0 = pg_lds_at(s_tile);
  int ent = src.entry(lo + lane);
  auto issue = [&](int t, int buffer) {                  // (every tile's entries were requested with the tile before)
    if (t >= tiles) return;
    const int base = lo + t * kManyKeys;
    const unsigned to = lds0 + buffer * M::kBuffer + RWI * w * ROW;
    if (base >= src.c && base + kManyKeys <= src.n && near) {   // nothing but tokens of the call
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const long long m = (base + RPP * i + RWI * w - src.c) * src.new_stride;
        pg_load_lds(src.knew + m, new_lane, to + RPP * i * ROW);
        pg_load_lds(src.vnew + m, new_lane, to + M::kPlane + RPP * i * ROW);
      }
    } else if (base + kManyKeys <= src.c && near) {      // nothing but tokens in pages
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const int r = RPP * i + RWI * w;
        const long long o = src.page_offset(base + r, __builtin_amdgcn_readlane(ent, r));
        pg_load_lds(src.k + o, page_lane, to + RPP * i * ROW);
        pg_load_lds(src.v + o, page_lane, to + M::kPlane + RPP * i * ROW);
      }
    } else {
#pragma unroll 1
      for (int i = 0; i < NP; ++i) {
        const int r = RPP * i + RWI * w, token = min(base + RPP * i + lrow, src.n - 1);
        const long long o = src.page_offset(base + r, __builtin_amdgcn_readlane(ent, r)) + lane_off;
        const bool fresh = base + RPP * i + lrow >= src.c;
        const long long m = (token - src.c) * src.new_stride + lpiece * 8;
        const __half *kp = src.k + o, *vp = src.v + o;
        if (fresh) {
          kp = src.knew + m;
          vp = src.vnew + m;
        }
        pg_load_lds(kp, to + RPP * i * ROW);
        pg_load_lds(vp, to + M::kPlane + RPP * i * ROW);
      }
    }
    if (t + 1 < tiles) ent = src.entry(base + kManyKeys + lane);
  };
  if (tid < kManyBuffers) s_bad[tid] = -1;
  issue(0, 0);
  M st;
  st.init(a, j, first_row);
  issue(1, 1);
  pg_append<D>(a, j, first_row, first_row + R, kManyThreads);   // (its trip to memory beside that of the first tiles)
  __syncthreads();
  bool dropped = false;
  // Values of keys that some row does not see meet it with probability 0, which does not silence an infinite or NaN one: where
  // there are such rows these values leave the tile, by the hand of the lane that brought them, and reach the rows that do see
  // them at the end.
  auto scrub = [&](int t, int buffer) {
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      pg_u4 *p = (pg_u4 *)(s_tile + buffer * M::kBuffer + M::kPlane + (RPP * i + RWI * w) * ROW + lane * 16);
      const pg_u4 v = *p;
      if (__builtin_expect(pg_odd_piece(v), 0)) {
        s_bad[buffer] = t;
        *p = pg_without_odd(v);
      }
    }
  };
  int buffer = 0;
  auto next_buffer = [&](int b) { return b + 1 == kManyBuffers ? 0 : b + 1; };
  auto turn = [&](int t, bool tail) {                    // tiles t and t + 1 are there, t + 2 is requested
    pg_arrive();
    // The entries among it, which the compiler learns here: it waited for them in front of the next ones' request otherwise, and so for
    // the tile just requested (15 % of the loop, where registers happened to fall that way).
    asm volatile("" : "+v"(ent));
    if (tail) {
      scrub(t, buffer);
      pg_arrive();
    }
    pg_barrier();
    issue(t + kManyBuffers - 1, buffer == 0 ? kManyBuffers - 1 : buffer - 1);
  };
  int t = 0;
  // Keys that all rows see.  The scores of the next 32 keys are formed while the exponentials of these are, their maximum while
  // these meet the values: matrix products beside vector arithmetic in either half of a step.
  pg_f16 sc[2];
  float mx = 0.f;
  auto step = [&](int at, int next, pg_f16 &now, pg_f16 &then) {
    pg_h8 pb[2];
    st.rows.follow(mx, st.c, now);
    __builtin_amdgcn_sched_barrier(0);
    st.scores(s_tile, next, then);
    st.rows.weights(now, st.c, pb);
    __builtin_amdgcn_sched_barrier(0);
    st.add(s_tile, at, pb);
    mx = st.rows.template peak<false>(then, 0);
    __builtin_amdgcn_sched_barrier(0);
  };
  for (; t < full; ++t, buffer = next_buffer(buffer)) {
    turn(t, false);
    const int at = buffer * M::kBuffer;
    if (t == 0) {
      st.scores(s_tile, at, sc[0]);
      mx = st.rows.template peak<false>(sc[0], 0);
    }
    step(at, at + M::kSub, sc[0], sc[1]);
    // (behind the last of them: scores that are not used, of the next tile or of whatever lies there)
    step(at + M::kSub, next_buffer(buffer) * M::kBuffer, sc[1], sc[0]);
  }
  for (; t < tiles; ++t, buffer = next_buffer(buffer)) {
    turn(t, true);
    dropped |= s_bad[buffer] == t;
#pragma unroll 1
    for (int sub = 0; sub < 2; ++sub) {
      const int key0 = lo + t * kManyKeys + sub * kPgKeys, at = buffer * M::kBuffer + sub * M::kSub;
      if (key0 >= st.rows.most) break;
      pg_h8 pb[2];
      st.scores(s_tile, at, sc[0]);
      st.rows.template weigh<true>(sc[0], key0, st.c, pb);
      st.add(s_tile, at, pb);
    }
  }
  __syncthreads();
  const float l = st.rows.finish(src, lo, hi, dropped), m = st.rows.maximum(l, st.c);
  const int l32 = lane & 31, h = lane >> 5, row0 = w * kPgRows;
  if (j.parts > 1) {
    // the wavefront's rows through LDS, 64 channels at a time in its own share of the tiles' room, so that they leave as whole lines
    float *wo = (float *)s_tile + row0 * 64;
#pragma unroll
    for (int q = 0; q < D / 64; ++q) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {                      // (sixteen bytes to the place that keeps rows on different banks)
        const pg_f16 &o = st.rows.O[2 * q + i / 4];
        const int e = i % 4 * 4;
        *(float4 *)(wo + l32 * 64 + (((2 * i + h) ^ (l32 & 15)) << 2)) = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
      }
      pg_wave_sync();
#pragma unroll
      for (int p = 0; p < kPgRows / 4; ++p) {
        const int r = 4 * p + (lane >> 4), piece = lane & 15;
        const float4 y = *(const float4 *)(wo + r * 64 + ((piece ^ (r & 15)) << 2));
        if (first_row + row0 + r <= last_row) *(float4 *)(a.o + ((long long)blockIdx.x * R + row0 + r) * D + 64 * q + 4 * piece) = y;
      }
      pg_wave_sync();
    }
    if (lane < kPgRows) a.ml[(long long)blockIdx.x * R + row0 + lane] = make_float2(m, l);
    return;
  }
  // The same in fp16.  Instructions count here, and a division or a wide product per row costs four to ten: rows are counted from the
  // block's first token (fewer than 256 + G; G is at most 16, so that the product with 65536 / G + 1 divides exactly).
  const int first_token = pg_token(a, first_row), ahead = first_row - first_token * a.G;
  auto token = [&](int rel) { return (int)(__umul24(rel, a.g_mul) >> 16); };
  const int heads = a.lambda ? a.G >> 1 : a.G;           // of the output
  float f = 0.f;
  if (a.lambda) {
    const int rel = ahead + min(row0 + l32, last_row - first_row), t = token(rel);
    f = a.lambda[(long long)(j.q.s + first_token + t) * a.lambda_stride + j.g * heads + ((rel - t * a.G) >> 1)];
  }
  const float inv = 1.f / l;
  uint8_t *wo = s_tile + row0 * 2 * D;
#pragma unroll
  for (int i = 0; i < D / 8; ++i) {
    const pg_f16 &o = st.rows.O[i / 4];
    pg_h4 out;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float y = o[i % 4 * 4 + e] * inv;
      if (a.lambda) y = fmaf(-f, pg_neighbour(y), y);    // (the pair's other row)
      out[e] = (_Float16)y;
    }
    *(pg_h4 *)(wo + l32 * 2 * D + ((i ^ (l32 % PR)) << 4) + 8 * h) = out;
  }
  pg_wave_sync();
  __half *base = a.out + ((long long)(j.q.s + first_token) * a.Hkv + j.g) * heads * D;
#pragma unroll
  for (int p = 0; p < kPgRows / 8; ++p) {                // eight rows, 64 channels of them at a time
    const int r = 8 * p + (lane >> 3), rel = ahead + row0 + r, t = token(rel), hq = rel - t * a.G;
    __half *to = base + ((long long)t * (a.Hkv * heads) + (a.lambda ? hq >> 1 : hq)) * D + (lane & 7) * 8;
    const bool leaves = first_row + row0 + r <= last_row && !(a.lambda && (hq & 1));
#pragma unroll
    for (int q = 0; q < D / 64; ++q) {
      const pg_h8 out = *(const pg_h8 *)(wo + r * 2 * D + (((8 * q + (lane & 7)) ^ (r % PR)) << 4));
      if (leaves) *(pg_h8 *)(to + 64 * q) = out;
    }
  }
}

// Many rows: their parts' partial results are merged in a launch of its own, by as many workgroups as there are parts: alone, a
// compute unit would read the 540 KB of four parts in 28 us.
template <int D>
__global__ __launch_bounds__(kManyThreads) void pages_merge_kernel(PagesLaunch a) {
  constexpr int R = kManyRows, kEach = kManyThreads / 16;   // sixteen threads per row
  PgJob j;
  if (!pg_job<R, kManyQuantum>(a, blockIdx.x, j) || j.parts == 1) return;
  const int first_row = j.block * R, rows = min(R, j.q.n * a.G - first_row), d = (threadIdx.x & 15) * 4;
  const int share = ((rows + j.parts - 1) / j.parts + 1) & ~1, from = j.part * share, to = min(rows, from + share);   // (pairs stay together)
  const long long apart = (long long)a.Hkv * R, slot = (long long)(blockIdx.x - j.part * a.Hkv) * R;
  for (int r0 = from; r0 < to; r0 += kEach) {
    const int at = r0 + (threadIdx.x >> 4), r = min(at, to - 1);
    const float2 *ml = a.ml + slot + r;
    const float *o = a.o + (slot + r) * D + d;
    float M = -INFINITY, l = 0.f;
    for (int p = 0; p < j.parts; ++p) M = fmaxf(M, ml[p * apart].x);
    float4 y[D / 64];
#pragma unroll
    for (int q = 0; q < D / 64; ++q) y[q] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int p = 0; p < j.parts; ++p) {
      const float2 s = ml[p * apart];
      const float f = pg_weight(s.x, M);
      l = f == 0.f ? l : fmaf(f, s.y, l);
#pragma unroll
      for (int q = 0; q < D / 64; ++q) {
        const float4 x = *(const float4 *)(o + p * apart * D + 64 * q);
        pg_add4(y[q], f, x);
      }
    }
    const PgOut place = pg_out<D>(a, j, at < to ? first_row + at : kNoSplit);
#pragma unroll
    for (int q = 0; q < D / 64; ++q) pg_write_out(a, place, d + 64 * q, y[q], 1.f / l);
  }
}

// ---------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------
// Slots of a split call: as many as there are workgroups on the chip (256 compute units) at a time, one of many rows to a unit or two of few (with
// twice as many 8 tokens behind 2000 took 25.8 us instead of 20.9, 32 behind 600 27.3 instead of 24.0).
constexpr int kManySlots = 256, kFewSlots = 512;
static_assert(kFewSlots <= kPagesCounters, "a block's counter is that of its first part's slot");
constexpr size_t kSlotRows = std::max(kManySlots * kManyRows, kFewSlots * kPgRows);
size_t pages_scratch_floats(int D) { return kSlotRows * (D + 2); }

// The launch's slots, and the workgroups it has: no more than there can be blocks, a sequence's last one apart (rows belong to one
// sequence), and one per slot where the call may be split.  Without counts of their own all sequences have `tokens` each: the blocks
// are known, and where they fill the slots none is cut.  0: too many for a launch.
template <int R>
static unsigned plan_blocks(PagesLaunch &a, int slots, int least_part, int threads, float *scratch) {
  const long long each = ((long long)a.tokens * a.G + R - 1) / R;
  const long long most = a.Hkv * std::min(a.B * each, (long long)a.rows * a.G / R + a.B);
  const bool may_split = scratch && (long long)a.pages.max_pages << a.pages.lg > least_part && (a.count || a.B * each * a.Hkv <= slots);
  a.slots = may_split ? slots : 0;
  a.slots_per_head = a.slots / a.Hkv;
  a.ml = (float2 *)scratch;
  a.o = scratch + kSlotRows * 2;
  const long long grid = std::max<long long>(most, a.slots);
  return grid * threads < 1ll << 32 ? (unsigned)grid : 0u;
}
template <int D>
static hipError_t launch_pages_of(PagesLaunch a, float *scratch, hipStream_t stream) {
  const bool few = (long long)a.tokens * a.G <= kPgRows;
  a.g_mul = 65536 / a.G + 1;
  a.g_magic = a.G > 1 ? split_divisor(a.G, &a.g_shift) : 0u;
  a.h_magic = a.Hkv > 1 ? split_divisor(a.Hkv, &a.h_shift) : 0u;
  const unsigned grid = few ? plan_blocks<kPgRows>(a, kFewSlots, kFewQuantum, kFewWaves * kWave, scratch)
                            : plan_blocks<kManyRows>(a, kManySlots, 2 * kManyLeastPart - kManyKeys, kManyThreads, scratch);
  if (grid == 0) return hipErrorInvalidValue;
  if (few) {
    hipLaunchKernelGGL(pages_few_kernel<D>, dim3(grid), dim3(kFewWaves * kWave), 0, stream, a);
  } else {
    hipLaunchKernelGGL(pages_many_kernel<D>, dim3(grid), dim3(kManyThreads), 0, stream, a);
    if (a.slots) hipLaunchKernelGGL(pages_merge_kernel<D>, dim3(a.slots), dim3(kManyThreads), 0, stream, a);
  }
  return hipGetLastError();
}
hipError_t launch_pages(const PagesLaunch &a, int D, float *scratch, hipStream_t stream) {
  return D == 64 ? launch_pages_of<64>(a, scratch, stream) : launch_pages_of<128>(a, scratch, stream);
}

}  // namespace confkv
