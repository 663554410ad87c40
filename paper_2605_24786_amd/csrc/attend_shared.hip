// Attention over a prefix that the sequences of a batch share, stored once: the partial results that conf_kv_attend_shared's
// second launch (attend.hip) takes in with the partials of its own wavefronts.
//
// All rows (sequence, token, head of the group) of a kv-head meet every prefix key, so this is a product of [rows x D] with
// [D x T] and, behind the softmax, of [rows x T] with [T x D]: matrix instructions on tiles that the whole batch shares.  The
// prefix is cut into `parts`, and a workgroup takes one part for up to 128 rows of a kv-head, keeps the running maximum, sum
// and output of each row (online softmax) and writes them as float32:
//   ml[unit][part][row] = (m, l),  o[unit][part][row][D] = sum over the part's keys of e^(s - m) v
// A wavefront owns 32 rows and forms the transposed products, scores [32 keys x 32 rows] and output [D x 32 rows]: a lane
// then holds values of one row only, its probabilities are the operand of the second product as they stand, and the row's
// statistics need one exchange between two lanes.
#include <algorithm>

#include "confkv_dev.h"
#include "launch.h"

namespace confkv {

constexpr int kShThreads = 256;

typedef _Float16 sh_h8 __attribute__((ext_vector_type(8)));
typedef _Float16 sh_h4 __attribute__((ext_vector_type(4)));
typedef short sh_s4 __attribute__((ext_vector_type(4)));
typedef float sh_f16 __attribute__((ext_vector_type(16)));

// Per group of sixteen lanes: lane l reads four halfs of row l / 4, columns 4 (l & 3) + [0, 4), and gets half l of each row.
__device__ __forceinline__ sh_h4 sh_read_tr(const uint8_t *p) {
  return __builtin_bit_cast(sh_h4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) sh_s4 *)p));
}
__device__ __forceinline__ float other_half(float v) { return __shfl_xor(v, 32, kWave); }

// Whether any of eight halfs is infinite or NaN; if so they are set to zero.
__device__ __forceinline__ bool drop_nonfinite(int4 &v) {
  bool bad = false;
  int *d = &v.x;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if ((d[k] & 0x7c00) == 0x7c00) { d[k] &= (int)0xffff0000; bad = true; }
    if ((d[k] & 0x7c000000) == 0x7c000000) { d[k] &= 0xffff; bad = true; }
  }
  return bad;
}

// RW wavefronts side by side along the rows, 4 / RW along the keys.
template <int D, int RW>
struct SharedTile {
  static constexpr int KW = 4 / RW;
  static constexpr int SUB = RW == 4 ? 2 : 1;              // 32-key subtiles per wavefront
  static constexpr int TK = 32 * KW * SUB;                 // keys of a tile
  // row strides in LDS (bytes): eight rows' 16-byte pieces on different banks; four rows' 64-byte pieces likewise
  static constexpr int KROW = 2 * D + 16, VROW = 2 * D + 64;
  static constexpr int OROW = D + 4;                       // floats of a partial's row where wavefronts merge
  static constexpr int kTileBytes = TK * (KROW + VROW);
  static constexpr int kMergeBytes = KW > 1 ? 4 * 32 * OROW * 4 : 0;
  static constexpr int kBytes = kTileBytes > kMergeBytes ? kTileBytes : kMergeBytes;
};

template <int D, int RW>
__global__ __launch_bounds__(kShThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void shared_prefix_kernel(SharedLaunch a) {
  using L = SharedTile<D, RW>;
  constexpr int TK = L::TK, PR = D / 8, NP = TK * PR / kShThreads;
  __shared__ __align__(16) uint8_t s_tile[L::kBytes];
  __shared__ float s_m[4][32], s_l[4][32];
  __shared__ int s_least;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, h = lane >> 5, t16 = lane & 15, c2 = (lane >> 4) & 1;
  const int rw = w % RW, kw = w / RW;
  const int g = blockIdx.x, part = blockIdx.z;
  const int rows = a.B * a.unit_rows;
  const int n = (blockIdx.y * RW + rw) * 32 + l32;          // this lane's row of the kv-head
  const bool real = n < rows;
  const int b = real ? n / a.unit_rows : 0, r = real ? n - b * a.unit_rows : 0;
  const int t = r / a.G, hq = r - t * a.G;
  const float NEG = -INFINITY;
  const int lo = part * a.part_keys, hi = min(lo + a.part_keys, a.T);
  // prefix keys the row sees
  const int lim = real && a.seen ? min(max(a.seen[b], 0), a.T) : a.T;
  int least = lim, most = real ? lim : 0;
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) {
    least = min(least, __shfl_xor(least, m, kWave));
    most = max(most, __shfl_xor(most, m, kWave));
  }
  least = __builtin_amdgcn_readfirstlane(least);
  most = __builtin_amdgcn_readfirstlane(most);
  if (tid == 0) s_least = a.T;
  __syncthreads();
  if (lane == 0) atomicMin(&s_least, least);
  const __half *K = a.k + g * a.head_stride, *V = a.v + g * a.head_stride;
  sh_h8 qf[D / 16];
  {
    const __half *q = a.q + (((size_t)b * a.tq + t) * a.Hkv * a.G + (size_t)g * a.G + hq) * D;
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      int4 raw = *(const int4 *)(q + 16 * s + 8 * h);
      if (!real) raw = make_int4(0, 0, 0, 0);
      qf[s] = __builtin_bit_cast(sh_h8, raw);
    }
  }
  int4 kr[NP], vr[NP];
  auto load = [&](int base) {
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      const int i = tid + j * kShThreads;
      const size_t at = (size_t)min(base + i / PR, a.T - 1) * D + (i % PR) * 8;
      kr[j] = ld_stream16(K + at);
      vr[j] = ld_stream16(V + at);
    }
  };
  load(lo);
  __syncthreads();
  const int wg_least = s_least;
  uint8_t *Kt = s_tile, *Vt = s_tile + TK * L::KROW;
  sh_f16 O[D / 32];
#pragma unroll
  for (int nt = 0; nt < D / 32; ++nt)
#pragma unroll
    for (int i = 0; i < 16; ++i) O[nt][i] = 0.f;
  float mref = NEG, l = 0.f;                                // reference in units of the raw score; per-lane partial sum
  const float c = a.sm_scale * 1.44269504088896341f;
  constexpr float kSlack = 4.0f;
  for (int base = lo; base < hi; base += TK) {
    // Keys that some row does not see meet it with probability 0, which does not silence an infinite or NaN value: such
    // values leave the tile here and reach the rows that do see them below.
    bool bad = false;
    if (base + TK > wg_least) {
#pragma unroll
      for (int j = 0; j < NP; ++j) {
        if (base + (tid + j * kShThreads) / PR >= a.T) vr[j] = make_int4(0, 0, 0, 0);
        bad |= drop_nonfinite(vr[j]);
      }
    }
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      const int i = tid + j * kShThreads;
      *(int4 *)(Kt + (i / PR) * L::KROW + (i % PR) * 16) = kr[j];
      *(int4 *)(Vt + (i / PR) * L::VROW + (i % PR) * 16) = vr[j];
    }
    bool any_bad = false;
    if (base + TK > wg_least) any_bad = __syncthreads_or(bad);
    else __syncthreads();
    if (base + TK < hi) load(base + TK);
#pragma unroll
    for (int sub = 0; sub < L::SUB; ++sub) {
      const int ks = (kw + L::KW * sub) * 32, key0 = base + ks;
      if (key0 >= most) continue;
      sh_f16 sc;
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[i] = 0.f;
#pragma unroll
      for (int s = 0; s < D / 16; ++s) {
        const sh_h8 kf = *(const sh_h8 *)(Kt + (ks + l32) * L::KROW + 32 * s + 16 * h);
        sc = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf, qf[s], sc, 0, 0, 0);
      }
      // element i: key key0 + 8 (i / 4) + 4 h + i % 4 of row l32
      if (key0 + 32 > least) {
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[i] = key0 + 8 * (i / 4) + 4 * h + (i & 3) < lim ? sc[i] : NEG;
      }
      float mx = sc[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) mx = fmaxf(mx, sc[i]);
      // The reference only has to stay near the maximum (the merge is exact for any), so the exchange and the rescaling run
      // where a score passes it by more than kSlack; e^kSlack times the largest fp16 value is far inside float32.
      if (__builtin_amdgcn_ballot_w64((mx - mref) * a.sm_scale > kSlack)) {
        const float mn = fmaxf(mref, fmaxf(mx, other_half(mx)));
        const float corr = mn == NEG ? 1.f : __builtin_amdgcn_exp2f((mref - mn) * c);
        mref = mn;
        l *= corr;
#pragma unroll
        for (int nt = 0; nt < D / 32; ++nt) O[nt] *= corr;
      }
      const float ref = mref == NEG ? 0.f : mref;
      sh_h8 pb[2];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float p = __builtin_amdgcn_exp2f((sc[i] - ref) * c);
        l += p;
        pb[i / 8][i & 7] = (_Float16)p;                     // (fp16 operands: half a step, 2^-11 of each probability)
      }
      const uint8_t *vp = Vt + (ks + 4 * h + (t16 >> 2)) * L::VROW + 32 * c2 + 8 * (t16 & 3);
#pragma unroll
      for (int s = 0; s < 2; ++s) {
#pragma unroll
        for (int nt = 0; nt < D / 32; ++nt) {
          const sh_h4 v0 = sh_read_tr(vp + 16 * s * L::VROW + 64 * nt), v1 = sh_read_tr(vp + (16 * s + 8) * L::VROW + 64 * nt);
          O[nt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7), pb[s], O[nt], 0, 0, 0);
        }
      }
      if (__builtin_expect(any_bad, 0)) {
#pragma unroll 1
        for (int key = key0; key < min(key0 + 32, a.T); ++key) {
#pragma unroll
          for (int nt = 0; nt < D / 32; ++nt)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const float v = __half2float(V[(size_t)key * D + 32 * nt + 8 * (i / 4) + 4 * h + (i & 3)]);
              if (key < lim && !(fabsf(v) < INFINITY)) O[nt][i] += v;
            }
        }
      }
    }
    __syncthreads();
  }
  l += other_half(l);
  const size_t at = ((size_t)(b * a.Hkv + g) * a.parts + part) * a.unit_rows + r;
  // (-inf stays; where every score was NaN the maximum saw none: +inf lets the merges give NaN)
  const float m = mref == NEG && l != l ? INFINITY : mref * a.sm_scale;
  if constexpr (L::KW == 1) {
    if (!real) return;
    if (h == 0) a.ml[at] = make_float2(m, l);
    float *o = a.o + at * D + 4 * h;
#pragma unroll
    for (int nt = 0; nt < D / 32; ++nt)
#pragma unroll
      for (int i = 0; i < 4; ++i) *(float4 *)(o + 32 * nt + 8 * i) = make_float4(O[nt][4 * i], O[nt][4 * i + 1], O[nt][4 * i + 2], O[nt][4 * i + 3]);
  } else {
    // the wavefronts along the keys merge (the tiles are idle behind the loop's last barrier)
    if (h == 0) { s_m[w][l32] = m; s_l[w][l32] = l; }
    __syncthreads();
    float M = NEG, sum = 0.f;
#pragma unroll
    for (int k = 0; k < L::KW; ++k) M = fmaxf(M, s_m[rw + k * RW][l32]);
#pragma unroll
    for (int k = 0; k < L::KW; ++k) {
      const float mk = s_m[rw + k * RW][l32];
      sum += mk > NEG ? __expf(mk - M) * s_l[rw + k * RW][l32] : 0.f;
    }
    const float f = m > NEG ? __expf(m - M) : 0.f;
    float *wo = (float *)s_tile + (size_t)w * 32 * L::OROW;
#pragma unroll
    for (int nt = 0; nt < D / 32; ++nt)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *(float4 *)(wo + l32 * L::OROW + 32 * nt + 8 * i + 4 * h) =
            make_float4(O[nt][4 * i] * f, O[nt][4 * i + 1] * f, O[nt][4 * i + 2] * f, O[nt][4 * i + 3] * f);
    if (kw == 0 && h == 0 && real) a.ml[at] = make_float2(M, sum);
    __syncthreads();
    for (int i = tid; i < RW * 32 * (D / 4); i += kShThreads) {
      const int row = i / (D / 4), d = (i % (D / 4)) * 4, nn = blockIdx.y * RW * 32 + row;
      if (nn >= rows) continue;
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < L::KW; ++k) {
        const float4 y = *(const float4 *)((const float *)s_tile + (size_t)((row >> 5) + k * RW) * 32 * L::OROW + (row & 31) * L::OROW + d);
        x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
      }
      const int bb = nn / a.unit_rows, rr = nn - bb * a.unit_rows;
      *(float4 *)(a.o + (((size_t)(bb * a.Hkv + g) * a.parts + part) * a.unit_rows + rr) * D + d) = x;
    }
  }
}

size_t shared_parts_most(int tokens) { return (size_t)std::min(kSharedMaxParts, (tokens + 63) / 64); }

void shared_plan(int rows, int Hkv, int T, int cus, SharedPlan *p) {
  p->row_waves = rows <= 32 ? 1 : rows <= 64 ? 2 : 4;
  p->blocks = (rows + 32 * p->row_waves - 1) / (32 * p->row_waves);
  const int tk = p->row_waves == 1 ? 128 : 64;
  const int tiles = (T + tk - 1) / tk;
  int want = std::max(1, 2 * cus / (Hkv * p->blocks));
  want = std::min(want, std::min(tiles, kSharedMaxParts));
  const int per = (tiles + want - 1) / want;
  p->parts = (tiles + per - 1) / per;
  p->part_keys = per * tk;
}

hipError_t launch_shared_prefix(const SharedLaunch &a, const SharedPlan &p, int D, hipStream_t stream) {
  const dim3 grid(a.Hkv, p.blocks, p.parts);
#define CONFKV_CASE(d, rw) \
  if (D == d && p.row_waves == rw) hipLaunchKernelGGL((shared_prefix_kernel<d, rw>), grid, dim3(kShThreads), 0, stream, a);
  CONFKV_CASE(64, 1) CONFKV_CASE(64, 2) CONFKV_CASE(64, 4) CONFKV_CASE(128, 1) CONFKV_CASE(128, 2) CONFKV_CASE(128, 4)
#undef CONFKV_CASE
  return hipGetLastError();
}

}  // namespace confkv
