// Queries, keys and values as a projection leaves them -> what the cache manager takes: RMS norm of every query and key
// head, position rotation, one rounding to FP16, the decode layout [B][T][heads][D] or the prompt layout [B][Hkv][T][D].
//
//   y_d = x_d * w_d / sqrt(mean(x^2) + eps)                        (w given; else y = x)
//   (a, b) -> (a cos t - b sin t, b cos t + a sin t),  t = position * freq[p]   for the pairs p of the first `rotated`
//   channels: (y_p, y_(p + rotated/2)), or (y_2p, y_(2p+1)) when interleaved; the channels behind them stay y.
//
// A wavefront takes one token.  A row (one head of one token) is D / 16 lanes of sixteen channels, arranged as two runs of
// eight such that a lane holds both halves of its eight pairs: no exchange between lanes but the sum of squares.  The angle
// of pair `lane` is computed once per token by that lane, the product in float64 (at position 10^6 a float32 angle is off by
// 0.03) and reduced to turns there, and shared through LDS.
#include "confkv_dev.h"
#include "launch.h"

namespace confkv {

constexpr int kPrepWaves = 4;

typedef float prep_f8 __attribute__((ext_vector_type(8)));
typedef _Float16 prep_h8 __attribute__((ext_vector_type(8)));

// eight neighbouring values as stored, and as float32
template <int kType> struct Run8 { int4 a; };
template <> struct Run8<kTypeFp32> { int4 a, b; };

template <int kType>
__device__ __forceinline__ Run8<kType> load_run(const void *base, long long at) {
  Run8<kType> r;
  const char *p = (const char *)base + at * (kType == kTypeFp32 ? 4 : 2);
  r.a = ld_stream16(p);
  if constexpr (kType == kTypeFp32) r.b = ld_stream16(p + 16);
  return r;
}
template <int kType>
__device__ __forceinline__ void unpack_run(const Run8<kType> &r, float (&f)[16], int at) {
  if constexpr (kType == kTypeFp32) {
    const int v[8] = {r.a.x, r.a.y, r.a.z, r.a.w, r.b.x, r.b.y, r.b.z, r.b.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) f[at + e] = __int_as_float(v[e]);
  } else if constexpr (kType == kTypeFp16) {
    const prep_h8 h = __builtin_bit_cast(prep_h8, r.a);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[at + e] = (float)h[e];
  } else {
    const unsigned v[4] = {(unsigned)r.a.x, (unsigned)r.a.y, (unsigned)r.a.z, (unsigned)r.a.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      f[at + 2 * e] = __uint_as_float(v[e] << 16);
      f[at + 2 * e + 1] = __uint_as_float(v[e] & 0xffff0000u);
    }
  }
}
__device__ __forceinline__ void store_run(__half *dst, const float (&f)[16], int at) {
  prep_h8 h;
#pragma unroll
  for (int e = 0; e < 8; ++e) h[e] = (_Float16)f[at + e];
  *(int4 *)dst = __builtin_bit_cast(int4, h);
}

// Rows of a token in the order q, k, v, in passes of 64 / (D / 16) rows of one kind each; `per` passes per wavefront.
template <int kType, int D>
__global__ __launch_bounds__(kPrepWaves * kWave) void prepare_kernel(PrepareLaunch a, int parts, int per) {
  constexpr int LPR = D / 16, RPP = kWave / LPR;
  __shared__ float2 s_turn[kPrepWaves][64];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long long task = (long long)blockIdx.x * kPrepWaves + w;
  const long long tok = task / parts;
  if (tok >= (long long)a.B * a.tokens) return;
  const int part = (int)(task - tok * parts);
  const int b = (int)(tok / a.tokens), t = (int)(tok - (long long)b * a.tokens);
  const int nq = a.q ? (a.Hq + RPP - 1) / RPP : 0, nk = a.k ? (a.Hkv + RPP - 1) / RPP : 0;
  const int nv = a.v ? (a.Hkv + RPP - 1) / RPP : 0;
  const int p0 = part * per, p1 = min(p0 + per, nq + nk + nv);
  const int c = lane % LPR, r = lane / LPR;
  const int half = a.rotated >> 1;
  const bool turns = a.interleaved ? 16 * c < a.rotated : 8 * c < half;
  // channels of the lane's two runs
  const int oa = turns && !a.interleaved ? 8 * c : 16 * c, ob = turns && !a.interleaved ? half + 8 * c : 16 * c + 8;
  if (p0 < nq + nk) {
    if (lane < half) {
      const long long pos = a.pos ? (long long)a.pos[tok] : (long long)*a.next + t;
      const double turn = (double)(pos + a.first) * (double)a.freq[lane] * 0.15915494309189533577;   // 1 / (2 pi)
      float s, cs;
      sincospif(2.0f * (float)(turn - rint(turn)), &s, &cs);
      s_turn[w][lane] = make_float2(cs, s);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
  float cs[8], sn[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float2 v = turns ? s_turn[w][8 * c + e] : make_float2(1.f, 0.f);
    cs[e] = v.x;
    sn[e] = v.y;
  }
  for (int p = p0; p < p1; ++p) {
    const int kind = p < nq ? 0 : p < nq + nk ? 1 : 2;
    const int head = (p - (kind == 0 ? 0 : kind == 1 ? nq : nq + nk)) * RPP + r;
    const int heads = kind == 0 ? a.Hq : a.Hkv;
    if (head >= heads) continue;
    const void *src = kind == 0 ? a.q : kind == 1 ? a.k : a.v;
    const long long row = (kind == 0 ? b * a.q_batch + t * a.q_token
                                     : kind == 1 ? b * a.k_batch + t * a.k_token : b * a.v_batch + t * a.v_token) + head * D;
    const int xa = kind == 2 ? 16 * c : oa, xb = kind == 2 ? 16 * c + 8 : ob;
    float f[16];
    unpack_run<kType>(load_run<kType>(src, row + xa), f, 0);
    unpack_run<kType>(load_run<kType>(src, row + xb), f, 8);
    const float *wt = kind == 0 ? a.wq : kind == 1 ? a.wk : nullptr;
    if (wt) {
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e) ss = fmaf(f[e], f[e], ss);
#pragma unroll
      for (int m = LPR / 2; m >= 1; m >>= 1) ss += __shfl_xor(ss, m, kWave);
      const float inv = 1.0f / sqrtf(ss * (1.0f / D) + a.eps);
#pragma unroll
      for (int e = 0; e < 16; ++e) f[e] *= inv * wt[e < 8 ? xa + e : xb + e - 8];
    }
    if (kind < 2 && turns) {
      if (a.interleaved) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float x = f[2 * e], y = f[2 * e + 1];
          f[2 * e] = x * cs[e] - y * sn[e];
          f[2 * e + 1] = y * cs[e] + x * sn[e];
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float x = f[e], y = f[8 + e];
          f[e] = x * cs[e] - y * sn[e];
          f[8 + e] = y * cs[e] + x * sn[e];
        }
      }
    }
    __half *dst = kind == 0 ? a.q16 : kind == 1 ? a.k16 : a.v16;
    dst += (kind != 0 && a.prompt ? ((long long)b * a.Hkv + head) * a.tokens + t : tok * heads + head) * D;
    store_run(dst + xa, f, 0);
    store_run(dst + xb, f, 8);
  }
}

hipError_t launch_prepare(const PrepareLaunch &a, int D, int type, hipStream_t stream) {
  const long long tokens = (long long)a.B * a.tokens;
  const int rpp = kWave / (D / 16);
  const int passes = (a.q ? (a.Hq + rpp - 1) / rpp : 0) + ((a.k ? 1 : 0) + (a.v ? 1 : 0)) * ((a.Hkv + rpp - 1) / rpp);
  if (tokens == 0 || passes == 0) return hipSuccess;
  int per = passes;
  while (per > 1 && tokens * ((passes + per - 1) / per) < 4096) per = (per + 1) / 2;
  const int parts = (passes + per - 1) / per;
  const long long blocks = (tokens * parts + kPrepWaves - 1) / kPrepWaves;
  if (blocks > 0x7fffffff) return hipErrorInvalidValue;
  auto fn = type == kTypeFp32 ? (D == 64 ? prepare_kernel<kTypeFp32, 64> : prepare_kernel<kTypeFp32, 128>)
          : type == kTypeFp16 ? (D == 64 ? prepare_kernel<kTypeFp16, 64> : prepare_kernel<kTypeFp16, 128>)
                              : (D == 64 ? prepare_kernel<kTypeBf16, 64> : prepare_kernel<kTypeBf16, 128>);
  hipLaunchKernelGGL(fn, dim3((unsigned)blocks), dim3(kPrepWaves * kWave), 0, stream, a, parts, per);
  return hipGetLastError();
}

}  // namespace confkv
