// kvq_adjust_logits: penalties for repeated tokens, biases and a grammar's mask.
//
// A CTA owns a slice of one row's vocabulary, E neighbours' strides of 512 logits: its
// logits and mask words are on their way while it counts the history's tokens that lie in
// the slice in shared memory (a word a token: the top bit for a prompt's, the others for the
// times it was answered) and finds the last bias of each token there (the largest place in
// the list, so equal ids need no order).
#include "block8.cuh"

#include <cuda_bf16.h>

namespace kvq {

namespace {

constexpr int kThreads = 512;
constexpr unsigned kMet = 0x80000000u;

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

template <typename T, int E, bool BIAS>
__global__ void __launch_bounds__(kThreads)
adjust_kernel(const __grid_constant__ kvq_adjust_params p) {
  constexpr int kSlice = E * kThreads;
  extern __shared__ unsigned sm[];
  unsigned* met = sm;
  unsigned* bias = sm + kSlice;
  const int tid = threadIdx.x, lane = tid & 31, b = blockIdx.y, v0 = blockIdx.x * kSlice;
  const int n = min(kSlice, p.vocab - v0);
  const T* z = static_cast<const T*>(p.logits) + b * p.logits_stride + v0;
  float* out = p.out + b * p.out_stride + v0;
  // (in place: no read-only path)
  T x[E];
#pragma unroll
  for (int i = 0; i < E; ++i)
    if (i * kThreads + tid < n) x[i] = z[i * kThreads + tid];
  const int2 h = p.history_starts ? part_of(p.history_starts, b, p.n_history) : make_int2(0, 0);
  const int2 list = BIAS ? part_of(p.bias_starts, b, p.n_bias) : make_int2(0, 0);
  const int prompt = p.prompt_lengths ? __ldg(p.prompt_lengths + b) : 0;
  // lane i holds the mask's word of the warp's 32 tokens of stride i
  unsigned words = 0xffffffffu;
  if (p.mask) {
    const int m = p.mask_rows ? __ldg(p.mask_rows + b) : b;
    const int at = (lane & (E - 1)) * kThreads + (tid & ~31);
    if (m >= 0 && m < p.n_masks && at < n)
      words = (unsigned)__ldg(p.mask + m * p.mask_stride + ((v0 + at) >> 5));
  }
#pragma unroll
  for (int i = 0; i < E; ++i) {
    met[i * kThreads + tid] = 0u;
    if (BIAS) bias[i * kThreads + tid] = 0u;
  }
  __syncthreads();
  each_in(p.history, h, v0, n, [&](unsigned v, int place) {
    if (place >= prompt) atomicAdd(&met[v], 1u);
    else atomicOr(&met[v], kMet);
  });
  if (BIAS)
    each_in(p.bias_ids, list, v0, n,
            [&](unsigned v, int place) { atomicMax(&bias[v], (unsigned)place + 1u); });
  float rep = p.repetition ? __ldg(p.repetition + b) : 1.0f;
  if (!(rep > 0.0f)) rep = 1.0f;
  const float freq = p.frequency ? __ldg(p.frequency + b) : 0.0f;
  const float pres = p.presence ? __ldg(p.presence + b) : 0.0f;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const int at = i * kThreads + tid;
    float y = as_float(x[i]);
    const unsigned w = met[at];
    if (w) {
      y = y > 0.0f ? y / rep : y * rep;
      const unsigned times = w & ~kMet;
      if (times) y = y - freq * (float)times - pres;
    }
    if (BIAS) {
      const unsigned place = bias[at];
      if (place) y += __ldg(p.bias_values + list.x + place - 1);
    }
    if (!(__shfl_sync(0xffffffffu, words, i) >> lane & 1u)) y = -INFINITY;
    if (at < n) out[at] = y;
  }
}

template <typename T, int E, bool BIAS>
cudaError_t launch(const kvq_adjust_params& p, cudaStream_t stream) {
  constexpr int kSlice = E * kThreads;
  constexpr int kBytes = kSlice * (int)sizeof(unsigned) * (BIAS ? 2 : 1);
  static std::atomic<unsigned long long> done{0};
  const cudaError_t e = once_per_device(done, [] {
    return cudaFuncSetAttribute(adjust_kernel<T, E, BIAS>,
                                cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes);
  });
  if (e != cudaSuccess) return e;
  const dim3 grid((p.vocab + kSlice - 1) / kSlice, p.rows);
  adjust_kernel<T, E, BIAS><<<grid, kThreads, kBytes, stream>>>(p);
  return cudaGetLastError();
}

// Slices of 8192 logits; smaller ones while they leave SMs without two CTAs.
template <typename T, bool BIAS>
cudaError_t launch_slices(const kvq_adjust_params& p, cudaStream_t stream) {
  const long long logits = (long long)p.rows * p.vocab;
  if (logits > 300LL * 8192) return launch<T, 16, BIAS>(p, stream);
  if (logits > 300LL * 2048) return launch<T, 4, BIAS>(p, stream);
  return launch<T, 2, BIAS>(p, stream);
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
