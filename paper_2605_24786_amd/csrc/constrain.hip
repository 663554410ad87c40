// Logits -> what the confidence estimator takes: penalties for repeated tokens, biases, a grammar's mask, float32.
//
// For row b and token v, with the history's counts  n(v) = times v was generated,  h(v) = v occurs in prompt or generated part:
//   x <- h(v) ? (x > 0 ? x / r_b : x r_b) : x
//   x <- x - f_b n(v) - [n(v) > 0] p_b
//   x <- x + bias_b(v)           (of several entries for one token the last one in the row's list counts)
//   x <- allowed_b(v) ? x : -inf
// A workgroup owns a range of the vocabulary of one row: it counts the row's history into LDS, keeping the tokens of its own
// range (integer atomics, so that the order of arrival changes nothing), and then passes over its logits once.
#include "confkv_dev.h"
#include "launch.h"

namespace confkv {

constexpr int kConThreads = 256;
constexpr int kConPer = 16;
constexpr int kConRange = kConThreads * kConPer;     // logits per workgroup
constexpr unsigned kConSeen = 0x80000000u;           // the token occurs in the history; the other bits count its generated part

template <int kType>
__device__ __forceinline__ float logit_at(const void *row, long long i) {
  if constexpr (kType == kTypeFp32) return ((const float *)row)[i];
  if constexpr (kType == kTypeFp16) return __half2float(((const __half *)row)[i]);
  return __uint_as_float((unsigned)((const unsigned short *)row)[i] << 16);
}

template <int kType>
__global__ __launch_bounds__(kConThreads) void constrain_kernel(ConstrainLaunch a) {
  __shared__ unsigned s_count[kConRange];
  __shared__ int s_bias[kConRange];
  const int b = blockIdx.y, tid = threadIdx.x;
  const int lo = blockIdx.x * kConRange, size = min(kConRange, a.V - lo);
  const char *row = (const char *)a.logits + (long long)b * a.row_stride * (kType == kTypeFp32 ? 4 : 2);
  float x[kConPer];
#pragma unroll
  for (int k = 0; k < kConPer; ++k) x[k] = logit_at<kType>(row, min(lo + tid + k * kConThreads, a.V - 1));
  const bool counts = a.tokens != nullptr, biases = a.bias_offsets != nullptr;
  int b0 = 0, b1 = 0;
  if (counts || biases) {
    for (int i = tid; i < kConRange; i += kConThreads) {
      s_count[i] = 0u;
      s_bias[i] = 0;
    }
    __syncthreads();
    if (counts) {
      const int32_t *ids = a.tokens + (long long)b * a.token_stride;
      const int n = min(max(a.lengths[b], 0), a.max_tokens), first = a.prompt_lengths ? a.prompt_lengths[b] : 0;
      for (int i = tid; i < n; i += kConThreads) {
        const unsigned at = (unsigned)(ids[i] - lo);
        if (at < (unsigned)size) {
          if (i < first) atomicOr(&s_count[at], kConSeen);
          else atomicAdd(&s_count[at], 1u);
        }
      }
    }
    if (biases) {
      b0 = min(max(a.bias_offsets[b], 0), a.n_bias);
      b1 = min(a.bias_offsets[b + 1], a.n_bias);
      for (int i = b0 + tid; i < b1; i += kConThreads) {
        const unsigned at = (unsigned)(a.bias_tokens[i] - lo);
        if (at < (unsigned)size) atomicMax(&s_bias[at], i - b0 + 1);
      }
    }
    __syncthreads();
  }
  const float rep = a.repetition ? a.repetition[b] : 1.f, pres = a.presence ? a.presence[b] : 0.f;
  const float freq = a.frequency ? a.frequency[b] : 0.f;
  const uint32_t *mask = nullptr;
  if (a.allowed) {
    const int m = a.allowed_rows ? a.allowed_rows[b] : b;
    if (m >= 0 && m < a.n_masks) mask = a.allowed + (long long)m * ((a.V + 31) / 32);
  }
  float *out = a.out + (long long)b * a.V;
#pragma unroll
  for (int k = 0; k < kConPer; ++k) {
    const int i = tid + k * kConThreads;
    if (i >= size) break;
    float v = x[k];
    if (counts) {
      const unsigned s = s_count[i];
      if (s != 0u) {
        v = v > 0.f ? v / rep : v * rep;
        const unsigned n = s & ~kConSeen;
        if (n != 0u) v = v - freq * (float)n - pres;
      }
    }
    if (biases && s_bias[i] != 0) v += a.bias_values[b0 + s_bias[i] - 1];
    if (mask && !((mask[(lo + i) >> 5] >> ((lo + i) & 31)) & 1u)) v = -INFINITY;
    out[lo + i] = v;
  }
}

hipError_t launch_constrain(const ConstrainLaunch &a, int type, hipStream_t stream) {
  const dim3 grid((a.V + kConRange - 1) / kConRange, a.B);
  auto fn = type == kTypeFp32 ? constrain_kernel<kTypeFp32> : type == kTypeFp16 ? constrain_kernel<kTypeFp16> : constrain_kernel<kTypeBf16>;
  hipLaunchKernelGGL(fn, grid, dim3(kConThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace confkv
