// kvq_adjust_logits: penalties for repeated tokens, biases and a grammar's mask.
//
// A CTA owns a slice of one row's vocabulary.  It counts the history's tokens that lie in
// the slice in shared memory (a word a token: a bit for a prompt's, one for a bias, the times
// it was answered in the others) and finds the last bias of each token there (the largest
// place in the list, so equal ids need no order).  Whoever meets a token first puts it on a
// list.  Meanwhile the whole slice is converted and masked from registers, four logits a
// thread and step, and behind a barrier the tokens of the list, a few in a hundred, get
// their values.
#include "block8.cuh"

#include <cuda_bf16.h>

namespace kvq {

namespace {

constexpr int kThreads = 512;
constexpr unsigned kMet = 0x80000000u, kBias = 0x40000000u;  // behind them: times answered

template <typename T>
__device__ __forceinline__ float as_float(T x) {
  if constexpr (sizeof(T) == 4) return x;
  else if constexpr (std::is_same<T, __half>::value) return __half2float(x);
  else return __bfloat162float(x);
}

// [begin, end) of row b's part of a list of n entries; empty where the starts are not
// in order or outside.
__device__ __forceinline__ int2 part_of(const int32_t* starts, int b, int n) {
  const int s0 = __ldg(starts + b), s1 = __ldg(starts + b + 1);
  return s0 < 0 || s1 < s0 || s1 > n ? make_int2(0, 0) : make_int2(s0, s1);
}

// Every token of a list's part that lies in [v0, v0 + n): f(token - v0, place in the part).
// Four at a time, sixteen bytes a load, four loads on their way.
template <typename F>
__device__ __forceinline__ void each_in(const int32_t* ids, int2 part, int v0, int n, F f) {
  const auto one = [&](int id, int i) {
    const unsigned v = (unsigned)id - (unsigned)v0;
    if (v < (unsigned)n) f(v, i - part.x);
  };
  // the part's first place on a 16-byte boundary, and its last
  const int skew = (int)((16u - ((unsigned)(uintptr_t)ids & 15u)) & 15u) >> 2;
  const int a0 = min(part.y, part.x + ((skew - part.x) & 3)), a1 = a0 + ((part.y - a0) & ~3);
  const int tid = threadIdx.x;
  if (tid < a0 - part.x) one(__ldg(ids + part.x + tid), part.x + tid);
  if (tid < part.y - a1) one(__ldg(ids + a1 + tid), a1 + tid);
#pragma unroll 4
  for (int i = a0 + 4 * tid; i < a1; i += 4 * kThreads) {
    const int4 x = __ldg(reinterpret_cast<const int4*>(ids + i));
    one(x.x, i);
    one(x.y, i + 1);
    one(x.z, i + 2);
    one(x.w, i + 3);
  }
}

// Four logits from z on, of which the first `n` exist.  16-bit ones need not stand on an
// eight-byte boundary: two loads of eight bytes around them, inside [lo, hi) of the row
// extended to whole boundaries, which lie within the same pages as the row's ends.
template <typename T>
__device__ __forceinline__ void load4(const T* z, int n, float (&x)[4]) {
  if constexpr (sizeof(T) == 4) {
    if (n >= 4 && (reinterpret_cast<uintptr_t>(z) & 15u) == 0) {
      const float4 v = *reinterpret_cast<const float4*>(z);
      x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
      return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = i < n ? (float)z[i] : 0.0f;
  } else {
    const unsigned skew = (unsigned)(reinterpret_cast<uintptr_t>(z) & 7u);
    if (n >= 4) {
      const uint2* at = reinterpret_cast<const uint2*>(reinterpret_cast<uintptr_t>(z) - skew);
      const uint2 a = at[0];
      uint2 v = a;
      if (skew) {
        const uint2 c = at[1];
        const unsigned bits = 8u * (skew & 3u);
        const unsigned w0 = skew & 4u ? a.y : a.x, w1 = skew & 4u ? c.x : a.y,
                       w2 = skew & 4u ? c.y : c.x;
        v = make_uint2(__funnelshift_r(w0, w1, bits), __funnelshift_r(w1, w2, bits));
      }
      const T* h = reinterpret_cast<const T*>(&v);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = as_float(h[i]);
      return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = i < n ? as_float(z[i]) : 0.0f;
  }
}

// E logits a thread, in fours; the first of them stands `head` logits ahead of the slice, so
// that results lie on 16-byte boundaries.
template <typename T, int E, bool BIAS>
__global__ void __launch_bounds__(kThreads)
adjust_kernel(const __grid_constant__ kvq_adjust_params p) {
  constexpr int kSlice = E * kThreads, kSteps = E / 4;
  extern __shared__ unsigned sm[];
  __shared__ int n_list;
  unsigned* met = sm;
  unsigned* bias = sm + kSlice;
  uint16_t* list = reinterpret_cast<uint16_t*>(sm + (BIAS ? 2 : 1) * kSlice);
  const int tid = threadIdx.x, b = blockIdx.y;
  const T* z = static_cast<const T*>(p.logits) + b * p.logits_stride;
  float* out = p.out + b * p.out_stride;
  // slices begin at the row's results' 16-byte boundaries
  const int head = (int)((reinterpret_cast<uintptr_t>(out) >> 2) & 3u);
  const int first = (int)blockIdx.x * kSlice - head;  // may be below 0
  const int v0 = max(first, 0), n = min(first + kSlice, p.vocab) - v0;
  if (n <= 0) return;
  const int2 h = p.history_starts ? part_of(p.history_starts, b, p.n_history) : make_int2(0, 0);
  const int2 biases = BIAS ? part_of(p.bias_starts, b, p.n_bias) : make_int2(0, 0);
  const int prompt = p.prompt_lengths ? __ldg(p.prompt_lengths + b) : 0;
  const int32_t* mask = nullptr;
  if (p.mask) {
    const int m = p.mask_rows ? __ldg(p.mask_rows + b) : b;
    if (m >= 0 && m < p.n_masks) mask = p.mask + m * p.mask_stride;
  }
  const auto allowed = [&](int v) {
    return !mask || (unsigned)__ldg(mask + (v >> 5)) >> (v & 31) & 1u;
  };
  float x[kSteps][4];
  unsigned bits[kSteps];
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int v = first + 4 * (i * kThreads + tid);
    bits[i] = 0xfu;
    if (v >= v0 && v < v0 + n) {
      load4(z + v, v0 + n - v, x[i]);
      if (mask) {
        const unsigned w0 = (unsigned)__ldg(mask + (v >> 5)), s = v & 31;
        bits[i] = w0 >> s;
        if (s > 28 && v + 3 < p.vocab)
          bits[i] |= (unsigned)__ldg(mask + (v >> 5) + 1) << (32 - s);
      }
    }
  }
  const bool lists = h.y > h.x || biases.y > biases.x;
  if (lists) {
    uint4* to = reinterpret_cast<uint4*>(sm);
#pragma unroll
    for (int i = 0; i < (BIAS ? 2 : 1) * kSteps; ++i)
      to[i * kThreads + tid] = make_uint4(0u, 0u, 0u, 0u);
    if (tid == 0) n_list = 0;
    __syncthreads();
    const auto put = [&](unsigned v, unsigned was) {
      if (!was) list[atomicAdd(&n_list, 1)] = (uint16_t)v;
    };
    each_in(p.history, h, v0, n, [&](unsigned v, int place) {
      put(v, place >= prompt ? atomicAdd(&met[v], 1u) : atomicOr(&met[v], kMet));
    });
    if (BIAS)
      each_in(p.bias_ids, biases, v0, n, [&](unsigned v, int place) {
        atomicMax(&bias[v], (unsigned)place + 1u);
        put(v, atomicOr(&met[v], kBias));
      });
  }
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int v = first + 4 * (i * kThreads + tid);
    if (v >= v0 + n) continue;
    if (v >= v0 && v + 3 < v0 + n) {
      float4 y;
      y.x = bits[i] & 1u ? x[i][0] : -INFINITY;
      y.y = bits[i] & 2u ? x[i][1] : -INFINITY;
      y.z = bits[i] & 4u ? x[i][2] : -INFINITY;
      y.w = bits[i] & 8u ? x[i][3] : -INFINITY;
      *reinterpret_cast<float4*>(out + v) = y;
    } else if (v >= v0) {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (v + k < v0 + n) out[v + k] = bits[i] >> k & 1u ? x[i][k] : -INFINITY;
    } else {  // the row's first, up to three
      for (int k = max(0, -v); k < 4 && v + k < v0 + n; ++k)
        out[v + k] = allowed(v + k) ? as_float(z[v + k]) : -INFINITY;
    }
  }
  if (!lists) return;
  __syncthreads();
  const int found = n_list;
  if (tid >= found) return;
  float rep = p.repetition ? __ldg(p.repetition + b) : 1.0f;
  if (!(rep > 0.0f)) rep = 1.0f;
  const float freq = p.frequency ? __ldg(p.frequency + b) : 0.0f;
  const float pres = p.presence ? __ldg(p.presence + b) : 0.0f;
#pragma unroll 1
  for (int i = tid; i < found; i += kThreads) {
    const int at = list[i], v = v0 + at;
    if (!allowed(v)) continue;
    // (in place the slice holds it still: no mask met it)
    float y = as_float(z[v]);
    const unsigned w = met[at], times = w & ~(kMet | kBias);
    if (w & ~kBias) y = y > 0.0f ? y / rep : y * rep;
    if (times) y = y - freq * (float)times - pres;
    if (BIAS && (w & kBias)) y += __ldg(p.bias_values + biases.x + bias[at] - 1);
    out[v] = y;
  }
}

template <typename T, int E, bool BIAS>
cudaError_t launch(const kvq_adjust_params& p, cudaStream_t stream) {
  constexpr int kSlice = E * kThreads;
  constexpr int kBytes = kSlice * ((int)sizeof(unsigned) * (BIAS ? 2 : 1) + (int)sizeof(uint16_t));
  static std::atomic<unsigned long long> done{0};
  const cudaError_t e = once_per_device(done, [] {
    return cudaFuncSetAttribute(adjust_kernel<T, E, BIAS>,
                                cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes);
  });
  if (e != cudaSuccess) return e;
  const dim3 grid((p.vocab + 3 + kSlice - 1) / kSlice, p.rows);
  adjust_kernel<T, E, BIAS><<<grid, kThreads, kBytes, stream>>>(p);
  return cudaGetLastError();
}

// Slices of 4096 logits; 2048 while they leave SMs without two CTAs.
template <typename T, bool BIAS>
cudaError_t launch_slices(const kvq_adjust_params& p, cudaStream_t stream) {
  const long long logits = (long long)p.rows * p.vocab;
  if (logits > 300LL * 4096) return launch<T, 8, BIAS>(p, stream);
  return launch<T, 4, BIAS>(p, stream);
}

template <typename T>
cudaError_t launch_type(const kvq_adjust_params& p, cudaStream_t stream) {
  return p.bias_starts ? launch_slices<T, true>(p, stream) : launch_slices<T, false>(p, stream);
}

}  // namespace

cudaError_t launch_adjust(const kvq_adjust_params& p, cudaStream_t stream) {
  switch (p.dtype) {
    case KVQ_F16: return launch_type<__half>(p, stream);
    case KVQ_BF16: return launch_type<__nv_bfloat16>(p, stream);
    default: return launch_type<float>(p, stream);
  }
}

}  // namespace kvq
