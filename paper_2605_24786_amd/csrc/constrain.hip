// Logits -> what the confidence estimator takes: penalties for repeated tokens, biases, a grammar's mask, float32.
//
// For row b and token v, with the history's counts  n(v) = times v was generated,  h(v) = v occurs in prompt or generated part:
//   x <- h(v) ? (x > 0 ? x / r_b : x r_b) : x
//   x <- x - f_b n(v) - [n(v) > 0] p_b
//   x <- x + bias_b(v)           (of several entries for one token the last one in the row's list counts)
//   x <- allowed_b(v) ? x : -inf
// A workgroup owns a range of the vocabulary of one row: it requests its logits and mask words, reads the row's whole history
// meanwhile and counts the tokens of its own range in LDS (integer atomics, so that the order of arrival changes nothing),
// applies the counts, reuses the LDS for the places of the biases, and writes its range once.
#include <algorithm>
#include <type_traits>

#include "confkv_dev.h"
#include "constrain_ranges.h"
#include "launch.h"

namespace confkv {

constexpr int kConThreads = 1024;
constexpr int kConAhead = 4;                          // groups of four tokens per thread in flight
constexpr unsigned kConSeen = 0x80000000u;            // the token occurs in the history; the other bits count its generated part

typedef unsigned con_u4 __attribute__((ext_vector_type(4)));

template <int kType>
__device__ __forceinline__ float logit_at(const void *row, int i) {
  if constexpr (kType == kTypeFp32) return ((const float *)row)[i];
  if constexpr (kType == kTypeFp16) return __half2float(((const __half *)row)[i]);
  return __uint_as_float((unsigned)((const unsigned short *)row)[i] << 16);
}
// four logits from a place aligned to them
template <int kType>
__device__ __forceinline__ void load_quad(const void *row, int i, float (&x)[4]) {
  if constexpr (kType == kTypeFp32) {
    const int4 v = ld_stream16((const float *)row + i);
    x[0] = __int_as_float(v.x); x[1] = __int_as_float(v.y); x[2] = __int_as_float(v.z); x[3] = __int_as_float(v.w);
  } else {
    const confkv_v2u v = __builtin_nontemporal_load((const confkv_v2u *)((const unsigned short *)row + i));
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const unsigned w = k ? v.y : v.x;
      if constexpr (kType == kTypeFp16) {
        x[2 * k] = __half2float(__ushort_as_half((unsigned short)w));
        x[2 * k + 1] = __half2float(__ushort_as_half((unsigned short)(w >> 16)));
      } else {
        x[2 * k] = __uint_as_float(w << 16);
        x[2 * k + 1] = __uint_as_float(w & 0xffff0000u);
      }
    }
  }
}

// A row's logits are counted from the 16-byte boundary of the result at or ahead of its first one (`off` places), so that quads
// of them are one store each, and one load where the logits lie on boundaries likewise: thread t's quad k is logits i .. i + 3
// with i = lo + 4 (t + k kThreads), lo = the range's start minus `off`.
// kWhole: every row consists of whole quads that lie on boundaries on both sides.
//
// What bounds it: a call on a few rows is a chain -- arguments, lengths, the history, two barriers, the result -- so whatever can
// be requested ahead of what it waits for is (first tokens of the history ahead of its length, biases ahead of the counts).  On
// many rows it is the bytes of the logits and, with long histories, the vector ALU: every range passes over the row's whole
// history, some seven instructions per token and wavefront.  So sixteen wavefronts share a pass, and a range is 4096 logits per
// quad of a thread, with as many quads (1, 2, 4 or 5) as make the fewest rounds of workgroups over the CUs times their length.
// us with 1, 2, 4, 5 quads (BF16 logits, 64 biases, a mask; histories of 300 and 32768 tokens): 8 rows of 128256 4.4, 4.9, 6.1, 6.6
// and 6.8, 7.5, 9.5, 10.5; 32 of 50257 6.1, 5.8, 7.0, 7.5 and 9.9, 8.8, 10.9, 12.0; 32 of 152064 12.9, 11.0, 10.1, 9.8 and 19.1, 15.6, 15.5,
// 13.6 (30 MB read and written, 3.6 more of history: 2.5 TB/s; without a history 8.3: 3.6).  Three quads, which are not among them, took
// 9.4 and 14.0 there, and 6.9 and 10.5 for 32 rows of 85000, which have four (7.5 and 11.5).  256 threads of four quads: 1 row of
// 128256 5.0 and 10.8 against 3.8 and 5.8.
// Tried and slower: a row's blocks of 64 logits dealt out among its workgroups, which spreads the frequent low token numbers but
// takes twice the instructions per token; one LDS operation for up to four tokens of a lane; more tokens in flight.
// Rows are the grid's fast axis: with a multiple of eight of them all ranges of a row run on one XCD, whose L2 then serves the
// history.
template <int kType, int kQuads, bool kWhole>
__global__ __launch_bounds__(kConThreads) void constrain_kernel(ConstrainLaunch a) {
  constexpr int kThreads = kConThreads, kRange = kThreads * 4 * kQuads;
  constexpr int kValue = kType == kTypeFp32 ? 4 : 2;
  __shared__ con_u4 s_slot[kRange / 4];
  unsigned *slot = (unsigned *)s_slot;
  const int b = blockIdx.x, tid = threadIdx.x, V = a.V;
  float *out = a.out + (long long)b * V;
  const int off = kWhole ? 0 : con_off((uintptr_t)out);
  const int lo = con_first(blockIdx.y, off, kRange);
  if (con_empty(lo, V)) return;
  const char *row = (const char *)a.logits + (long long)b * a.row_stride * kValue;
  const bool quads = kWhole || (((uintptr_t)(row - off * kValue) & (4 * kValue - 1)) == 0 && V >= 8);
  const int first_quad = (4 - off) & 3, last_quad = ((V - 4 + off) & ~3) - off;   // whole quads of the row: the first and the last
  // first logit of the thread's quad k (-3 .. -1: a quad that begins ahead of the row; V and more: none)
  auto place = [&](int k) { return lo + 4 * (tid + k * kThreads); };
  // ---- requests ----
  float x[kQuads][4];
  if (quads) {
#pragma unroll
    for (int k = 0; k < kQuads; ++k) load_quad<kType>(row, min(max(place(k), first_quad), last_quad), x[k]);
  } else {
#pragma unroll
    for (int k = 0; k < kQuads; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) x[k][e] = logit_at<kType>(row, min(max(place(k) + e, 0), V - 1));
  }
  int n = 0, first = 0;
  float rep = 1.f, pres = 0.f, freq = 0.f;
  const int32_t *ids = a.tokens + (long long)b * a.token_stride;
  const bool by_four = a.tokens && ((uintptr_t)ids & 15) == 0 && a.max_tokens >= 4;
  int4 ahead = make_int4(0, 0, 0, 0);
  if (by_four) ahead = ((const int4 *)ids)[min(tid, (a.max_tokens >> 2) - 1)];
  if (a.tokens) {
    n = a.lengths[b];
    if (a.prompt_lengths) first = a.prompt_lengths[b];
    if (a.repetition) rep = a.repetition[b];
    if (a.presence) pres = a.presence[b];
    if (a.frequency) freq = a.frequency[b];
  }
  typename std::conditional<kWhole, unsigned, unsigned long long>::type bits[kQuads];   // the quad's mask bits, and what lies behind them
#pragma unroll
  for (int k = 0; k < kQuads; ++k) bits[k] = 15u;
  if (a.allowed) {
    const int m = a.allowed_rows ? a.allowed_rows[b] : b;
    if (m >= 0 && m < a.n_masks) {
      const int words = (V + 31) / 32;
      const uint32_t *mask = a.allowed + (long long)m * words;
#pragma unroll
      for (int k = 0; k < kQuads; ++k) {
        // (a quad that starts ahead of the row takes its bits from the row's first word, moved up)
        const int i = place(k), w = min(max(i, 0) >> 5, words - 1);
        if constexpr (kWhole) {
          bits[k] = mask[w] >> (i & 31);
        } else {
          const unsigned long long two = mask[w] | (unsigned long long)mask[min(w + 1, words - 1)] << 32;
          bits[k] = i < 0 ? two << -i : two >> (i & 31);
        }
      }
    }
  }
  int b0 = 0, b1 = 0, bias_ahead = -1;
  if (a.bias_offsets) {
    b0 = min(max(a.bias_offsets[b], 0), a.n_bias);
    b1 = min(a.bias_offsets[b + 1], a.n_bias);
    if (b0 + tid < b1) bias_ahead = a.bias_tokens[b0 + tid];
  }
  // the row's first and last quad where they are no whole ones (behind the requests: what is loaded twice is waited for)
  if (!kWhole && quads) {
#pragma unroll
    for (int k = 0; k < kQuads; ++k) {
      const int i = place(k);
      if (i < 0 || (i + 4 > V && i < V)) {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[k][e] = logit_at<kType>(row, min(max(i + e, 0), V - 1));
      }
    }
  }
  // Token id's slot is id - lo.  (An id of -3 .. -1 may find a slot ahead of the row: nothing reads it.)
  const unsigned size = (unsigned)con_size(lo, V, kRange);
  n = min(max(n, 0), a.max_tokens);
  // ---- the history's counts ----
  if (n > 0) {
#pragma unroll
    for (int k = 0; k < kQuads; ++k) s_slot[tid + k * kThreads] = con_u4{0u, 0u, 0u, 0u};
    __syncthreads();
    // kind: 0 prompt, 1 generated, 2 either
    auto count = [&](int id, int i, auto kind) {
      const unsigned at = (unsigned)id - (unsigned)lo;
      if (at < size) {
        if (kind == 0 || (kind == 2 && i < first)) atomicOr(&slot[at], kConSeen);
        else atomicAdd(&slot[at], 1u);
      }
    };
    auto count4 = [&](const int4 &v, int i, auto kind) {
      count(v.x, i, kind);
      count(v.y, i + 1, kind);
      count(v.z, i + 2, kind);
      count(v.w, i + 3, kind);
    };
    int done = 0;
    if (by_four) {
      const int groups = n >> 2;
      // (a wavefront's 256 tokens are mostly of one kind)
      auto count_group = [&](const int4 &v, int g) {
        const int w0 = __builtin_amdgcn_readfirstlane(4 * g);
        if (w0 >= first) count4(v, 4 * g, std::integral_constant<int, 1>{});
        else if (w0 + 4 * kWave <= first) count4(v, 4 * g, std::integral_constant<int, 0>{});
        else count4(v, 4 * g, std::integral_constant<int, 2>{});
      };
      if (tid < groups) count_group(ahead, tid);
      for (int g0 = tid + kThreads; g0 < groups; g0 += kConAhead * kThreads) {
        int4 v[kConAhead];
#pragma unroll
        for (int u = 0; u < kConAhead; ++u) v[u] = ((const int4 *)ids)[min(g0 + u * kThreads, groups - 1)];
#pragma unroll
        for (int u = 0; u < kConAhead; ++u) {
          const int g = g0 + u * kThreads;
          if (g >= groups) break;
          count_group(v[u], g);
        }
      }
      done = groups << 2;
    }
    for (int i0 = done + tid; i0 < n; i0 += 8 * kThreads) {
      int v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] = ids[min(i0 + u * kThreads, n - 1)];
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (i0 + u * kThreads < n) count(v[u], i0 + u * kThreads, std::integral_constant<int, 2>{});
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kQuads; ++k) {
      const con_u4 s = s_slot[tid + k * kThreads];
      if ((s.x | s.y | s.z | s.w) == 0u) continue;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (s[e] == 0u) continue;
        const float v = x[k][e] > 0.f ? x[k][e] / rep : x[k][e] * rep;
        const unsigned c = s[e] & ~kConSeen;
        x[k][e] = c != 0u ? v - freq * (float)c - pres : v;
      }
    }
  }
  // ---- the row's biases ----
  if (b0 < b1) {
    // (a thread clears the slots that only it has read since the last barrier)
#pragma unroll
    for (int k = 0; k < kQuads; ++k) s_slot[tid + k * kThreads] = con_u4{0u, 0u, 0u, 0u};
    __syncthreads();
    for (int i = b0 + tid; i < b1; i += kThreads) {
      const unsigned at = (unsigned)(i == b0 + tid ? bias_ahead : a.bias_tokens[i]) - (unsigned)lo;
      if (at < size) atomicMax(&slot[at], (unsigned)(i - b0 + 1));
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kQuads; ++k) {
      const con_u4 s = s_slot[tid + k * kThreads];
      if ((s.x | s.y | s.z | s.w) == 0u) continue;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (s[e] != 0u) x[k][e] += a.bias_values[b0 + (int)s[e] - 1];
    }
  }
#pragma unroll
  for (int k = 0; k < kQuads; ++k) {
    const int i = place(k);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[k][e] = (bits[k] >> e) & 1u ? x[k][e] : -INFINITY;
    if (kWhole ? i < V : i >= 0 && i + 4 <= V) {
      *(float4 *)(out + i) = make_float4(x[k][0], x[k][1], x[k][2], x[k][3]);
    } else if (!kWhole) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (i + e >= 0 && i + e < V) out[i + e] = x[k][e];
    }
  }
}

hipError_t launch_constrain(const ConstrainLaunch &a, int type, hipStream_t stream) {
  const size_t value = type == kTypeFp32 ? 4 : 2;
  const bool whole = a.V % 4 == 0 && a.row_stride % 4 == 0 && (uintptr_t)a.logits % (4 * value) == 0 && (uintptr_t)a.out % 16 == 0;
  // quads per thread: see the kernel
  const long long cus = std::max(1, device_cu_count());
  int quads = 1;
  long long least = 0;
  for (int q : {1, 2, 4, 5}) {
    const long long groups = (long long)a.B * con_grid_ranges((uintptr_t)a.out, a.B, a.V, kConThreads * 4 * q, whole);
    const long long cost = (groups + cus - 1) / cus * (q + 1);
    if (q > 1 && cost >= least) continue;
    least = cost;
    quads = q;
  }
  const dim3 grid(a.B, con_grid_ranges((uintptr_t)a.out, a.B, a.V, kConThreads * 4 * quads, whole));
#define CONFKV_CASE(q) \
  if (quads == q) { \
    auto fn = type == kTypeFp32 ? (whole ? constrain_kernel<kTypeFp32, q, true> : constrain_kernel<kTypeFp32, q, false>) \
            : type == kTypeFp16 ? (whole ? constrain_kernel<kTypeFp16, q, true> : constrain_kernel<kTypeFp16, q, false>) \
                                : (whole ? constrain_kernel<kTypeBf16, q, true> : constrain_kernel<kTypeBf16, q, false>); \
    hipLaunchKernelGGL(fn, grid, dim3(kConThreads), 0, stream, a); \
  }
  CONFKV_CASE(1) CONFKV_CASE(2) CONFKV_CASE(4) CONFKV_CASE(5)
#undef CONFKV_CASE
  return hipGetLastError();
}

}  // namespace confkv
