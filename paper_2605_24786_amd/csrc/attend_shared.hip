// Attention over a prefix that the sequences of a batch share, stored once: the partial results that conf_kv_attend_shared's
// second launch (attend.hip) takes in with the partials of its own wavefronts.
//
// All rows (sequence, token, head of the group) of a kv-head meet every prefix key, so this is a product of [rows x D] with
// [D x T] and, behind the softmax, of [rows x T] with [T x D]: matrix instructions on tiles that the whole batch shares.  The
// prefix is cut into `parts`; a workgroup takes one part for 32, 64 or 128 rows of a kv-head, and its eight wavefronts take the
// part's tiles of 32 keys in turn, each keeping the running maximum, sum and output of 32 rows (online softmax).  They merge at the
// end and leave float32:
//   ml[unit][part][row] = (m, l),  o[unit][part][row][D] = sum over the part's keys of e^(s - m) v
// The products are formed transposed, scores [32 keys x 32 rows] and output [D x 32 rows]: a lane then holds values of one row
// only, its probabilities are the operand of the second product as they stand, and the row's statistics need one exchange
// between two lanes.
#include <algorithm>

#include "confkv_dev.h"
#include "launch.h"

namespace confkv {

constexpr int kShWaves = 8, kShThreads = kShWaves * kWave;
constexpr int kShKeys = 32;                            // keys of a wavefront's tile
constexpr int kShRows = 32;

typedef _Float16 sh_h8 __attribute__((ext_vector_type(8)));
typedef _Float16 sh_h4 __attribute__((ext_vector_type(4)));
typedef short sh_s4 __attribute__((ext_vector_type(4)));
typedef float sh_f16 __attribute__((ext_vector_type(16)));

// Per group of sixteen lanes: lane l reads four halfs of row l / 4, columns 4 (l & 3) + [0, 4), and gets half l of each row.
__device__ __forceinline__ sh_h4 sh_read_tr(const uint8_t *p) {
  return __builtin_bit_cast(sh_h4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) sh_s4 *)p));
}
__device__ __forceinline__ float other_half(float v) { return __shfl_xor(v, 32, kWave); }

// The signs of the result: which of two halfs are infinite or NaN (their magnitude, 0x7c00 or more, carries into the sign).
__device__ __forceinline__ unsigned nonfinite_halfs(int d) { return ((unsigned)d & 0x7fff7fffu) + 0x04000400u; }
// Sets halfs that are infinite or NaN to zero.
__device__ __forceinline__ void drop_nonfinite(int4 &v) {
  int *d = &v.x;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const unsigned odd = nonfinite_halfs(d[k]) & 0x80008000u;
    d[k] &= (int)~((odd >> 15) * 0xffffu);
  }
}

// A workgroup's wavefronts: RW side by side along the rows, KW = 8 / RW along the keys.  A turn is one tile for each of the KW
// (RW = 4: two), in LDS in rows of these strides (bytes): 16-byte pieces of eight K rows on different banks, 64-byte pieces of
// four V rows likewise.
template <int D, int RW>
struct SharedTile {
  static constexpr int KW = kShWaves / RW, SUB = RW == 4 ? 2 : 1;
  static constexpr int TK = kShKeys * KW * SUB;        // keys of a turn
  static constexpr int KROW = 2 * D + 16, VROW = 2 * D + 64;
  static constexpr int kTurnBytes = TK * (KROW + VROW);
  static constexpr int kBuffers = RW == 1 ? 1 : 2;
  static constexpr int OROW = D + 4;                   // floats of a partial's row where the wavefronts merge
  static constexpr int kPartBytes = kShRows * OROW * 4;
  static constexpr int kBytes = kBuffers * kTurnBytes;
  static_assert(kShWaves * kPartBytes <= kBytes, "the wavefronts' partials fit the tiles' room");
  static_assert(kPartBytes <= kShKeys * (KROW + VROW), "and one of them a wavefront's own tile's");
};

// LDS operations of a wavefront execute in order: between lanes that exchange data only the compiler has to keep it.
__device__ __forceinline__ void sh_wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// A wavefront's 32 rows: queries, running reference, sum and output, and how much of the prefix they see.
template <int D>
struct SharedRowsState {
  sh_h8 qf[D / 16];
  sh_f16 O[D / 32];
  float mref, l;                                       // reference in units of the raw score; per-lane partial sum (lifted, as O)
  int lim, least, most;                                // keys the lane's row sees; the fewest and the most of the 32 rows

  __device__ __forceinline__ void reset() {
#pragma unroll
    for (int nt = 0; nt < D / 32; ++nt)
#pragma unroll
      for (int i = 0; i < 16; ++i) O[nt][i] = 0.f;
    mref = -INFINITY;
    l = 0.f;
  }

  // The tile of keys key0 .. key0 + 31 at Kt, Vt.
  template <int KROW, int VROW>
  __device__ __forceinline__ void take(const uint8_t *Kt, const uint8_t *Vt, int key0, float sm) {
    const int lane = threadIdx.x & 63, l32 = lane & 31, h = lane >> 5, t16 = lane & 15, c2 = (lane >> 4) & 1;
    const float NEG = -INFINITY, c = sm * 1.44269504088896341f;
    constexpr float kSlack = 4.0f, kLift = 10.0f;
    sh_f16 sc;
#pragma unroll
    for (int i = 0; i < 16; ++i) sc[i] = 0.f;
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      const sh_h8 kf = *(const sh_h8 *)(Kt + l32 * KROW + 32 * s + 16 * h);
      sc = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf, qf[s], sc, 0, 0, 0);
    }
    // element i: key key0 + 8 (i / 4) + 4 h + i % 4 of row l32
    if (key0 + kShKeys > least) {
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[i] = 8 * (i / 4) + (i & 3) < lim - key0 - 4 * h ? sc[i] : NEG;
    }
    float mx = sc[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, sc[i]);
    // The reference only has to stay near the maximum (the merge is exact for any), so the exchange and the rescaling run
    // where a score passes it by more than kSlack.
    if (__builtin_amdgcn_ballot_w64((mx - mref) * sm > kSlack)) {
      const float mn = fmaxf(mref, fmaxf(mx, other_half(mx)));
      const float corr = mn == NEG ? 1.f : __builtin_amdgcn_exp2f((mref - mn) * c);
      mref = mn;
      l *= corr;
#pragma unroll
      for (int nt = 0; nt < D / 32; ++nt) O[nt] *= corr;
    }
    // Probabilities are held 2^10 times as large, at most 55910 of fp16's 65504: as fp16 operands they keep eleven bits down to
    // 6e-8 (unscaled 6e-5, which the tail of a long prefix is below).  (The difference comes first: a rounded mref * c is off by
    // more than fp16's exponents from scores of 10^7 on.)
    const float ref = mref == NEG ? 0.f : mref;
    sh_h8 pb[2];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float p = __builtin_amdgcn_exp2f(fmaf(sc[i] - ref, c, kLift));
      l += p;
      // (fp16 operands: half a step, 2^-11 of each probability.  32 sequences behind 4096 tokens are 2.3e-4 from a float64
      // evaluation, relative, against 2.1e-4 of one that keeps float32 until it rounds the result; a second operand for what the
      // rounding leaves would double the products.)
      pb[i / 8][i & 7] = (_Float16)p;
    }
    const uint8_t *vp = Vt + (4 * h + (t16 >> 2)) * VROW + 32 * c2 + 8 * (t16 & 3);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
#pragma unroll
      for (int nt = 0; nt < D / 32; ++nt) {
        const sh_h4 v0 = sh_read_tr(vp + 16 * s * VROW + 64 * nt), v1 = sh_read_tr(vp + (16 * s + 8) * VROW + 64 * nt);
        O[nt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7), pb[s], O[nt], 0, 0, 0);
      }
    }
  }

  // Whether some channel is no number although the row's sum l, of both halves, is one.
  __device__ __forceinline__ bool odd() const {
    float z[8] = {};
#pragma unroll
    for (int nt = 0; nt < D / 32; ++nt)
#pragma unroll
      for (int i = 0; i < 16; ++i) z[i & 7] = fmaf(O[nt][i], 0.f, z[i & 7]);
    const float all = ((z[0] + z[1]) + (z[2] + z[3])) + ((z[4] + z[5]) + (z[6] + z[7]));
    return all != all && l == l;
  }

  // Values that are infinite or NaN, of the keys of `tiles` (which calls its argument with the first key of each) that the lane's row
  // sees: each makes its channel what they add up to, since a probability is positive however far the products above rounded it
  // (where to zero, they made NaN of an infinite value, and where the values left the tile they were never met).  The first
  // pass empties these channels, the second adds; tiles without such a value cost a read.
  template <typename Tiles>
  __device__ __forceinline__ void show_odd_values(const __half *V, int T, Tiles tiles) {
    constexpr int PR = D / 8;
    const int lane = threadIdx.x & 63, h = lane >> 5;
#pragma unroll 1
    for (int pass = 0; pass < 2; ++pass) {
      tiles([&](int key0) {
        const int end = min(key0 + kShKeys, T);
        unsigned any = 0u;
#pragma unroll
        for (int j = 0; j < kShKeys * PR / kWave; ++j) {
          const int4 v = *(const int4 *)(V + (size_t)min(key0 + (lane + j * kWave) / PR, T - 1) * D + lane % PR * 8);
          any |= nonfinite_halfs(v.x) | nonfinite_halfs(v.y) | nonfinite_halfs(v.z) | nonfinite_halfs(v.w);
        }
        if (__builtin_amdgcn_ballot_w64((any & 0x80008000u) != 0u) == 0ull) return;
#pragma unroll 1
        for (int key = key0; key < end; ++key) {
          sh_h4 v[D / 32][4];
#pragma unroll
          for (int nt = 0; nt < D / 32; ++nt)
#pragma unroll
            for (int k = 0; k < 4; ++k) v[nt][k] = *(const sh_h4 *)(V + (size_t)key * D + 32 * nt + 8 * k + 4 * h);
#pragma unroll
          for (int nt = 0; nt < D / 32; ++nt)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const float x = (float)v[nt][i / 4][i & 3];
              if (key < lim && !(fabsf(x) < INFINITY)) O[nt][i] = pass ? O[nt][i] + x : 0.f;
            }
        }
      });
    }
  }
};

// Workgroups of one (kv-head, part) read the same keys for different rows, so they shall share an L2: workgroups go to the eight
// XCDs in turn, and XCD x takes the logical ones x * each .. x * each + each - 1 (rows fastest, then parts, then kv-heads).
//
// What bounds it: the prefix's bytes for some forty rows per kv-head; with more of them what every row adds, products, exponentials and
// reads of the tiles in LDS (80 rows behind 32001 tokens: 40 us, where the bytes take 25; at the rates of a large copy and a large
// product bytes and operations meet at 220 rows); a short prefix the chain of a workgroup (first rows, a tile or two, the merge).  With up to 32 rows (RW = 1) a wavefront waits for nobody before the merge: it loads and multiplies
// tiles of its own, the next one in flight in registers while this one is used.  More rows share a turn's tiles through LDS, two
// buffers, one barrier per turn, the two turns after the next in flight.
// Its loads are streaming ones although several workgroups may read a line: plain loads took 17.9 us instead of 12.7 (8192 tokens, 32
// rows), 21.1 instead of 13.4 (4096, 128) and 61.5 instead of 40.1 (32001, 80).
template <int D, int RW>
__global__ __launch_bounds__(kShThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void shared_prefix_kernel(SharedLaunch a, int blocks, int each) {
  using L = SharedTile<D, RW>;
  constexpr int PR = D / 8;                              // 16-byte pieces of a row
  constexpr int TK = L::TK;
  constexpr int kLoaders = RW == 1 ? kWave : kShThreads; // lanes that share the loads of kRowsLoaded keys
  constexpr float kUnlift = 0x1p-10f;                    // see SharedRowsState::take
  constexpr int kRowsLoaded = RW == 1 ? kShKeys : TK, NP = kRowsLoaded * PR / kLoaders, kStep = kLoaders / PR;
  __shared__ __align__(16) uint8_t s_tile[L::kBytes];
  __shared__ float s_m[kShWaves][kShRows], s_l[kShWaves][kShRows];
  __shared__ int s_bad[2];
  const int job = (blockIdx.x & 7) * each + (blockIdx.x >> 3);
  if (job >= blocks * a.parts * a.Hkv) return;
  const int block = job % blocks, part = (job / blocks) % a.parts, g = job / (blocks * a.parts);
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, h = lane >> 5;
  const int rw = w % RW, kw = w / RW;
  const float NEG = -INFINITY;
  const __half *K = a.k + g * a.head_stride, *V = a.v + g * a.head_stride;
  const int lo = part * a.part_keys, hi = min(lo + a.part_keys, a.T);
  const int lrow = RW == 1 ? lane / PR : tid / PR, lcol = lane % PR;   // of the first piece that the lane loads
  struct Turn { int4 k[NP], v[NP]; };                   // pieces in flight
  auto load = [&](Turn &x, int base) {
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      const size_t at = (size_t)min(base + lrow + j * kStep, a.T - 1) * D + lcol * 8;
      x.k[j] = ld_stream16(K + at);
      x.v[j] = ld_stream16(V + at);
    }
  };
  Turn x, y;
  const int first = RW == 1 ? lo + w * kShKeys : lo;
  if (first < hi) load(x, first);
  if (RW > 1 && lo + TK < hi) load(y, lo + TK);
  const int rows = a.B * a.unit_rows;
  const int n = (block * RW + rw) * kShRows + l32;       // this lane's row of the kv-head
  const bool real = n < rows;
  const int b = real ? n / a.unit_rows : 0, r = real ? n - b * a.unit_rows : 0;
  SharedRowsState<D> st;
  {
    const int t = r / a.G, hq = r - t * a.G;
    const __half *q = a.q + (((size_t)b * a.tq + t) * a.Hkv * a.G + (size_t)g * a.G + hq) * D;
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      int4 raw = *(const int4 *)(q + 16 * s + 8 * h);
      if (!real) raw = make_int4(0, 0, 0, 0);
      st.qf[s] = __builtin_bit_cast(sh_h8, raw);
    }
  }
  // The fewest and the most keys that the wavefront's rows see, and the fewest of the workgroup's.
  st.lim = st.least = st.most = a.T;
  int all_least = a.T;
  if (a.seen) {
    if (real) st.lim = min(max(a.seen[b], 0), a.T);
    st.least = st.lim;
    st.most = real ? st.lim : 0;
    if constexpr (RW > 1) {
      for (int k = lane; k < RW * kShRows; k += kWave) {
        const int nn = block * RW * kShRows + k;
        if (nn < rows) all_least = min(all_least, min(max(a.seen[nn / a.unit_rows], 0), a.T));
      }
    }
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) {
      st.least = min(st.least, __shfl_xor(st.least, m, kWave));
      st.most = max(st.most, __shfl_xor(st.most, m, kWave));
      if constexpr (RW > 1) all_least = min(all_least, __shfl_xor(all_least, m, kWave));
    }
    st.least = __builtin_amdgcn_readfirstlane(st.least);
    st.most = __builtin_amdgcn_readfirstlane(st.most);
    all_least = __builtin_amdgcn_readfirstlane(all_least);
  } else if (RW > 1 && (block * RW + rw) * kShRows >= rows) {
    st.most = 0;                                         // (a wavefront without rows)
  }
  if constexpr (RW == 1) all_least = st.least;
  st.reset();
  // Registers -> LDS.  Keys that some row does not see meet it with probability 0, which does not silence an infinite or NaN
  // value: where there are such rows these values leave the tile here and reach the rows that do see them at the end.
  auto store = [&](Turn &x, uint8_t *Kt, uint8_t *Vt, int base) {
    bool bad = false;
    if (base + kRowsLoaded > all_least) {
      unsigned odd = 0u;
#pragma unroll
      for (int j = 0; j < NP; ++j) {
        if (base + lrow + j * kStep >= a.T) x.v[j] = make_int4(0, 0, 0, 0);
        odd |= nonfinite_halfs(x.v[j].x) | nonfinite_halfs(x.v[j].y) | nonfinite_halfs(x.v[j].z) | nonfinite_halfs(x.v[j].w);
      }
      bad = (odd & 0x80008000u) != 0u;
      if (__builtin_expect(bad, 0)) {
#pragma unroll
        for (int j = 0; j < NP; ++j) drop_nonfinite(x.v[j]);
      }
    }
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      const int row = lrow + j * kStep;
      *(int4 *)(Kt + row * L::KROW + lcol * 16) = x.k[j];
      *(int4 *)(Vt + row * L::VROW + lcol * 16) = x.v[j];
    }
    return bad;
  };
  // where the thread's rows of the merge go (a division, worked out while the first rows are on their way)
  int out_at[RW];
#pragma unroll
  for (int p = 0; p < RW; ++p) {
    const int nn = (block * RW + p) * kShRows + (tid >> 4), bb = nn / a.unit_rows;
    out_at[p] = nn < rows ? ((bb * a.Hkv + g) * a.parts + part) * a.unit_rows + (nn - bb * a.unit_rows) : -1;
  }
  bool dropped = false;                                  // values left a tile that was taken
  if constexpr (RW == 1) {
    uint8_t *Kt = s_tile + w * kShKeys * (L::KROW + L::VROW), *Vt = Kt + kShKeys * L::KROW;
    for (int key0 = first; key0 < min(hi, st.most); key0 += TK) {
      dropped |= store(x, Kt, Vt, key0);
      sh_wave_sync();
      if (key0 + TK < hi) load(x, key0 + TK);
      st.template take<L::KROW, L::VROW>(Kt, Vt, key0, a.sm_scale);
      sh_wave_sync();
    }
  } else {
    if (tid < 2) s_bad[tid] = -1;
    __syncthreads();
    auto buffer = [&](int turn) { return s_tile + (turn & 1) * L::kTurnBytes; };
    auto fill = [&](Turn &x, int turn, int base) {
      uint8_t *Kt = buffer(turn);
      if (store(x, Kt, Kt + TK * L::KROW, base)) s_bad[turn & 1] = turn;
    };
    // A turn: the next one's rows, which came in `next`, go to the other buffer, the one but two is requested in their place.
    auto take_turn = [&](Turn &next, int turn, int base) {
      if (base + TK < hi) fill(next, turn + 1, base + TK);
      if (base + 3 * TK < hi) load(next, base + 3 * TK);
      const uint8_t *Kt = buffer(turn), *Vt = Kt + TK * L::KROW;
      dropped |= s_bad[turn & 1] == turn;
#pragma unroll
      for (int sub = 0; sub < L::SUB; ++sub) {
        const int ks = (kw + L::KW * sub) * kShKeys;
        if (base + ks < min(hi, st.most))
          st.template take<L::KROW, L::VROW>(Kt + ks * L::KROW, Vt + ks * L::VROW, base + ks, a.sm_scale);
      }
      __syncthreads();
    };
    fill(x, 0, lo);
    if (lo + 2 * TK < hi) load(x, lo + 2 * TK);
    __syncthreads();
    int turn = 0;
    for (int base = lo; base < hi; base += 2 * TK, turn += 2) {
      take_turn(y, turn, base);
      if (base + TK < hi) take_turn(x, turn + 1, base + TK);
    }
  }
  st.l = (st.l + other_half(st.l)) * kUnlift;
  if (__builtin_expect(__builtin_amdgcn_ballot_w64(dropped || st.odd()) != 0ull, 0)) {
    st.show_odd_values(V, a.T, [&](auto take) {          // the wavefront's tiles, as above
      const int end = min(hi, st.most);
      if constexpr (RW == 1) {
        for (int key0 = first; key0 < end; key0 += TK) take(key0);
      } else {
        for (int base = lo; base < hi; base += TK)
          for (int sub = 0; sub < L::SUB; ++sub)
            if (base + (kw + L::KW * sub) * kShKeys < end) take(base + (kw + L::KW * sub) * kShKeys);
      }
    });
  }
  // (-inf stays; a sum that is NaN, from a score that is none, outweighs the others: a merge shall not lose it to larger scores)
  if (h == 0) {
    s_m[w][l32] = st.l == st.l ? st.mref * a.sm_scale : INFINITY;
    s_l[w][l32] = st.l;
  }
  // The partials take the tiles' room: with RW = 1 a wavefront's own tile, which nobody else reads, else any.
  constexpr int kPartStride = RW == 1 ? kShKeys * (L::KROW + L::VROW) : L::kPartBytes;
  float *wo = (float *)(s_tile + w * kPartStride);
#pragma unroll
  for (int nt = 0; nt < D / 32; ++nt)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *(float4 *)(wo + l32 * L::OROW + 32 * nt + 8 * i + 4 * h) =
          make_float4(st.O[nt][4 * i] * kUnlift, st.O[nt][4 * i + 1] * kUnlift, st.O[nt][4 * i + 2] * kUnlift, st.O[nt][4 * i + 3] * kUnlift);
  __syncthreads();
  // sixteen threads per row merge the partials of the wavefronts along the keys
  const int row = tid >> 4;
#pragma unroll
  for (int p = 0; p < RW; ++p) {
    if (out_at[p] < 0) continue;
    float m[L::KW], M = NEG, sum = 0.f;
#pragma unroll
    for (int k = 0; k < L::KW; ++k) {
      m[k] = s_m[p + k * RW][row];
      M = fmaxf(M, m[k]);
    }
#pragma unroll
    for (int k = 0; k < L::KW; ++k) {
      m[k] = m[k] == NEG ? 0.f : fmaxf(__expf(m[k] - M), kLeastWeight);   // (a wavefront that saw no key of the row: its partial is zero)
      sum = fmaf(m[k], s_l[p + k * RW][row], sum);
    }
    if ((tid & 15) == 0) a.ml[out_at[p]] = make_float2(M, sum);
#pragma unroll
    for (int q = 0; q < D / 64; ++q) {
      const int d = (tid & 15) * 4 + 64 * q;
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < L::KW; ++k) {
        const float4 y = *(const float4 *)((const float *)(s_tile + (p + k * RW) * kPartStride) + row * L::OROW + d);
        x.x = fmaf(m[k], y.x, x.x);
        x.y = fmaf(m[k], y.y, x.y);
        x.z = fmaf(m[k], y.z, x.z);
        x.w = fmaf(m[k], y.w, x.w);
      }
      *(float4 *)(a.o + (size_t)out_at[p] * D + d) = x;
    }
  }
}

size_t shared_parts_most(int tokens) { return (size_t)std::min(kSharedMaxParts, (tokens + 4 * kShKeys - 1) / (4 * kShKeys)); }

// One workgroup per CU (its tiles take the LDS), and no part shorter than a turn.  More parts than CUs were slower everywhere, half
// as many too but where the partial results outweigh the prefix.
// Rows side by side: `blocks` workgroups read the same keys, some 18 TB/s all together where an L2 serves most of them, so fewer
// blocks save loads; each doubling of RW costs the barriers and a longer way to the first product and from the last, about 7 us'
// worth of loads.  us per layer (prefix and cache of 256 tokens, 128 channels, 8 kv-heads) with RW = 1, 2, 4: 40 rows behind 12000
// tokens 27.5, 29.4, 30.9, 32768 45.5, 41.0, 43.0; 128 rows, 4096 25.2, 26.0, 29.4, 12000 35.8, 35.0, 38.1, 32768 65.3, 52.7, 56.1; 256 rows,
// 4096 30.6, 29.9, 31.5, 12000 48.5, 43.5, 45.0, 32768 98.0, 77.3, 73.0.  (So the rule is off by up to 6 %: it takes 4 for 128 rows behind
// 32768.)
void shared_plan(int rows, int Hkv, int D, int T, int cus, int forced_row_waves, SharedPlan *p) {
  constexpr double kStep = 7e-6 * 18e12;
  double least = 0.0;
  p->row_waves = 0;
  for (int rw = 1, step = 0; rw <= 4; rw *= 2, ++step) {
    const int blocks = (rows + rw * kShRows - 1) / (rw * kShRows);
    const double cost = (double)blocks * Hkv * T * 4.0 * D + step * kStep;
    if (p->row_waves && cost >= least && rw != forced_row_waves) continue;
    least = cost;
    p->row_waves = rw;
    p->blocks = blocks;
    if (rw == forced_row_waves) break;
  }
  const int turn = p->row_waves == 1 ? kShWaves * kShKeys : 4 * kShKeys, turns = (T + turn - 1) / turn;
  int want = (int)std::max<long long>(1, cus / ((long long)Hkv * p->blocks));
  want = std::min(want, std::min(turns, kSharedMaxParts));
  // equal parts in whole tiles: a part's last turn need not be full
  const int tiles = (T + kShKeys - 1) / kShKeys, per = (tiles + want - 1) / want;
  p->parts = (tiles + per - 1) / per;
  p->part_keys = per * kShKeys;
}

hipError_t launch_shared_prefix(const SharedLaunch &a, const SharedPlan &p, int D, hipStream_t stream) {
  const long long jobs = (long long)a.Hkv * p.blocks * p.parts, each = (jobs + 7) / 8;
  if (jobs > 0x7ffffff0ll) return hipErrorInvalidValue;
#define CONFKV_CASE(d, rw) \
  if (D == d && p.row_waves == rw) \
    hipLaunchKernelGGL((shared_prefix_kernel<d, rw>), dim3((unsigned)(each * 8)), dim3(kShThreads), 0, stream, a, p.blocks, (int)each);
  CONFKV_CASE(64, 1) CONFKV_CASE(64, 2) CONFKV_CASE(64, 4) CONFKV_CASE(128, 1) CONFKV_CASE(128, 2) CONFKV_CASE(128, 4)
#undef CONFKV_CASE
  return hipGetLastError();
}

}  // namespace confkv
