// Queries, keys and values as a projection leaves them -> what the cache manager takes: RMS norm of every query and key
// head, position rotation, one rounding to FP16, the decode layout [B][T][heads][D] or the prompt layout [B][Hkv][T][D].
//
//   y_d = x_d * w_d / sqrt(mean(x^2) + eps)                        (w given; else y = x)
//   (a, b) -> (a cos t - b sin t, b cos t + a sin t),  t = position * freq[p]   for the pairs p of the first `rotated`
//   channels: (y_p, y_(p + rotated/2)), or (y_2p, y_(2p+1)) when interleaved; the channels behind them stay y.
//
// A wavefront takes one token.  A row (one head of one token) is D / 16 lanes of sixteen channels, in runs of sixteen bytes as
// stored, arranged such that lanes side by side load neighbouring runs and a lane holds both halves of its pairs: no exchange
// between lanes but the sum of squares.  The angle of pair `lane` is computed once per token by that lane, the product in
// float64 (at position 10^6 a float32 angle is off by 0.03) and reduced to turns there, and shared through LDS.
// What bounds it: bytes.  Where every access of a wavefront is whole 128-byte lines (128 channels of 16 bits, none or all of
// which turn, or interleaved) streaming accesses take eight prompts of 4096 tokens, 48 heads, BF16 from 152 to 141 us (5.7 TB/s read
// and written, more than a large copy reaches); where a line is met by two accesses they cost (64 channels of float32, 32 of
// them turning, 5271 tokens: 162 and 200 us), so these, and short calls, whose result is read next, do without.
// A decode step's call is a launch (3 to 4 us on the device): its rows are spread over as many wavefronts as they make.
#include <algorithm>

#include "confkv_dev.h"
#include "launch.h"

namespace confkv {

constexpr int kPrepWaves = 4;
constexpr int kPrepGridX = 1 << 23;                    // workgroups along x: a dimension of a grid has fewer than 2^32 threads

typedef _Float16 prep_h4 __attribute__((ext_vector_type(4)));
typedef _Float16 prep_h8 __attribute__((ext_vector_type(8)));

// Sixteen bytes of values as float32: eight, or four of a float32 source.
template <int kType, bool kStream>
__device__ __forceinline__ void load_run(const void *base, long long at, int4 &raw) {
  const char *p = (const char *)base + at * (kType == kTypeFp32 ? 4 : 2);
  raw = kStream ? ld_stream16(p) : *(const int4 *)p;
}
template <int kType, int kRun>
__device__ __forceinline__ void unpack_run(const int4 &r, float (&f)[kRun]) {
  const unsigned v[4] = {(unsigned)r.x, (unsigned)r.y, (unsigned)r.z, (unsigned)r.w};
  if constexpr (kType == kTypeFp32) {
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = __uint_as_float(v[e]);
  } else if constexpr (kType == kTypeFp16) {
    const prep_h8 h = __builtin_bit_cast(prep_h8, r);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = (float)h[e];
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      f[2 * e] = __uint_as_float(v[e] << 16);
      f[2 * e + 1] = __uint_as_float(v[e] & 0xffff0000u);
    }
  }
}
template <int kRun, bool kStream>
__device__ __forceinline__ void store_run(__half *dst, const float (&f)[kRun]) {
  if constexpr (kRun == 8) {
    prep_h8 h;
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = (_Float16)f[e];
    if constexpr (kStream) st_stream16(dst, __builtin_bit_cast(int4, h));
    else *(int4 *)dst = __builtin_bit_cast(int4, h);
  } else {
    prep_h4 h;
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = (_Float16)f[e];
    *(int2 *)dst = __builtin_bit_cast(int2, h);
  }
}

// Rows of a token in the order q, k, v, in passes of 64 / (D / 16) rows of one kind each; `per` passes per wavefront.
template <int kType, int D, bool kStream>
__global__ __launch_bounds__(kPrepWaves * kWave) void prepare_kernel(PrepareLaunch a, int parts, int per) {
  constexpr int LPR = D / 16, RPP = kWave / LPR;
  constexpr int kRun = kType == kTypeFp32 ? 4 : 8, kSets = 8 / kRun;   // a lane's sets of two runs
  __shared__ float2 s_turn[kPrepWaves][64];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long long task = ((long long)blockIdx.y * kPrepGridX + blockIdx.x) * kPrepWaves + w;
  const long long tok = task / parts;
  if (tok >= (long long)a.B * a.tokens) return;
  const int part = (int)(task - tok * parts);
  const int b = (int)(tok / a.tokens), t = (int)(tok - (long long)b * a.tokens);
  const int nq = a.q ? (a.Hq + RPP - 1) / RPP : 0, nk = a.k ? (a.Hkv + RPP - 1) / RPP : 0;
  const int nv = a.v ? (a.Hkv + RPP - 1) / RPP : 0;
  const int p0 = part * per, p1 = min(p0 + per, nq + nk + nv);
  const int c = lane % LPR, r = lane / LPR;
  const int half = a.rotated >> 1;
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
  // Set s of the lane: the runs at channels at[s][0] and at[s][1], and cosine and sine of their kRun pairs.  With j = kRun (c + LPR s):
  //   halves:       (j, j + rotated / 2) while j is below rotated / 2, else two runs of the channels that do not turn
  //   interleaved:  (j, j + D / 2), each of which holds kRun / 2 pairs if it turns
  int at[kSets][2];
  bool turns[kSets][2];
  float cs[kSets][kRun], sn[kSets][kRun];
#pragma unroll
  for (int s = 0; s < kSets; ++s) {
    const int j = kRun * (c + LPR * s);
    if (a.interleaved) {
      at[s][0] = j;
      at[s][1] = j + D / 2;
    } else if (j < half) {
      at[s][0] = j;
      at[s][1] = j + half;
    } else {
      at[s][0] = half + j;
      at[s][1] = half + j + (D - a.rotated) / 2;
    }
    turns[s][0] = at[s][0] < a.rotated;
    turns[s][1] = at[s][1] < a.rotated;
#pragma unroll
    for (int e = 0; e < kRun; ++e) {
      const int which = a.interleaved && e >= kRun / 2 ? 1 : 0;
      const int pair = a.interleaved ? at[s][which] / 2 + (e & (kRun / 2 - 1)) : j + e;
      const float2 v = turns[s][which] ? s_turn[w][pair] : make_float2(1.f, 0.f);
      cs[s][e] = v.x;
      sn[s][e] = v.y;
    }
  }
  for (int p = p0; p < p1; ++p) {
    const int kind = p < nq ? 0 : p < nq + nk ? 1 : 2;
    const int head = (p - (kind == 0 ? 0 : kind == 1 ? nq : nq + nk)) * RPP + r;
    const int heads = kind == 0 ? a.Hq : a.Hkv;
    if (head >= heads) continue;
    const void *src = kind == 0 ? a.q : kind == 1 ? a.k : a.v;
    const long long row = (kind == 0 ? b * a.q_batch + t * a.q_token
                                     : kind == 1 ? b * a.k_batch + t * a.k_token : b * a.v_batch + t * a.v_token) + head * D;
    int4 raw[kSets][2];
#pragma unroll
    for (int s = 0; s < kSets; ++s)
#pragma unroll
      for (int i = 0; i < 2; ++i) load_run<kType, kStream>(src, row + at[s][i], raw[s][i]);
    float f[kSets][2][kRun];
#pragma unroll
    for (int s = 0; s < kSets; ++s)
#pragma unroll
      for (int i = 0; i < 2; ++i) unpack_run<kType, kRun>(raw[s][i], f[s][i]);
    const float *wt = kind == 0 ? a.wq : kind == 1 ? a.wk : nullptr;
    if (wt) {
      auto sum_of_squares = [&]() {
        float ss = 0.f;
#pragma unroll
        for (int s = 0; s < kSets; ++s)
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < kRun; ++e) ss = fmaf(f[s][i][e], f[s][i][e], ss);
#pragma unroll
        for (int m = LPR / 2; m >= 1; m >>= 1) ss += __shfl_xor(ss, m, kWave);
        return ss;
      };
      float ss = sum_of_squares(), eps = a.eps;
      // A row whose squares leave float32 (FP16's do not) is scaled by a power of two, its norm's eps by its square.
      if constexpr (kType != kTypeFp16) {
        const bool large = !(ss < 3e38f), small = ss < 1e-30f && eps < 1e-30f;
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(large || small) != 0ull, 0)) {
          const float by = large ? 0x1p-70f : small ? 0x1p100f : 1.f;
#pragma unroll
          for (int s = 0; s < kSets; ++s)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
              for (int e = 0; e < kRun; ++e) f[s][i][e] *= by;
          ss = sum_of_squares();
          eps = eps * by * by;
        }
      }
      const float inv = 1.0f / sqrtf(ss * (1.0f / D) + eps);
#pragma unroll
      for (int s = 0; s < kSets; ++s)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < kRun; ++e) f[s][i][e] *= inv * wt[at[s][i] + e];
    }
    if (kind < 2) {
#pragma unroll
      for (int s = 0; s < kSets; ++s) {
        if (a.interleaved) {
#pragma unroll
          for (int e = 0; e < kRun; ++e) {
            const int i = e / (kRun / 2), o = 2 * (e & (kRun / 2 - 1));
            if (turns[s][i]) {
              const float x = f[s][i][o], y = f[s][i][o + 1];
              f[s][i][o] = x * cs[s][e] - y * sn[s][e];
              f[s][i][o + 1] = y * cs[s][e] + x * sn[s][e];
            }
          }
        } else if (turns[s][0]) {
#pragma unroll
          for (int e = 0; e < kRun; ++e) {
            const float x = f[s][0][e], y = f[s][1][e];
            f[s][0][e] = x * cs[s][e] - y * sn[s][e];
            f[s][1][e] = y * cs[s][e] + x * sn[s][e];
          }
        }
      }
    }
    __half *dst = kind == 0 ? a.q16 : kind == 1 ? a.k16 : a.v16;
    dst += (kind != 0 && a.prompt ? ((long long)b * a.Hkv + head) * a.tokens + t : tok * heads + head) * D;
#pragma unroll
    for (int s = 0; s < kSets; ++s)
#pragma unroll
      for (int i = 0; i < 2; ++i) store_run<kRun, kStream>(dst + at[s][i], f[s][i]);
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
  const dim3 grid((unsigned)std::min<long long>(blocks, kPrepGridX), (unsigned)((blocks + kPrepGridX - 1) / kPrepGridX));
  // (see the top)
  const bool stream_lines = D == 128 && type != kTypeFp32 && (a.interleaved || a.rotated == 0 || a.rotated == D) && tokens >= 4096;
  auto fn = type == kTypeFp32 ? (D == 64 ? prepare_kernel<kTypeFp32, 64, false> : prepare_kernel<kTypeFp32, 128, false>)
          : type == kTypeFp16 ? (D == 64 ? prepare_kernel<kTypeFp16, 64, false> : stream_lines ? prepare_kernel<kTypeFp16, 128, true> : prepare_kernel<kTypeFp16, 128, false>)
                              : (D == 64 ? prepare_kernel<kTypeBf16, 64, false> : stream_lines ? prepare_kernel<kTypeBf16, 128, true> : prepare_kernel<kTypeBf16, 128, false>);
  hipLaunchKernelGGL(fn, grid, dim3(kPrepWaves * kWave), 0, stream, a, parts, per);
  return hipGetLastError();
}

}  // namespace confkv
