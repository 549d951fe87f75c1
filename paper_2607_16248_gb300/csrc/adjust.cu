// kvq_adjust_logits: penalties for repeated tokens, biases and a grammar's mask.
//
// A CTA owns a slice of one row's vocabulary.  It counts the history's tokens that lie
// in the slice in shared memory (a word a token: the top bit for "met at all", the
// others for the times it was answered), finds the last bias of each token there (the
// largest place in the list, so equal ids need no order), then streams the slice once.
#include "block8.cuh"

#include <cuda_bf16.h>

namespace kvq {

namespace {

constexpr int kThreads = 512;
constexpr int kSlice = 8192;
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

template <typename T, bool BIAS>
__global__ void __launch_bounds__(kThreads)
adjust_kernel(const __grid_constant__ kvq_adjust_params p) {
  extern __shared__ unsigned sm[];
  unsigned* met = sm;
  unsigned* bias = sm + kSlice;
  const int tid = threadIdx.x, b = blockIdx.y, v0 = blockIdx.x * kSlice;
  const int n = min(kSlice, p.vocab - v0);
  for (int i = tid; i < kSlice; i += kThreads) {
    met[i] = 0u;
    if (BIAS) bias[i] = 0u;
  }
  __syncthreads();
  if (p.history_starts) {
    const int2 h = part_of(p.history_starts, b, p.n_history);
    const int prompt = p.prompt_lengths ? __ldg(p.prompt_lengths + b) : 0;
    for (int i = h.x + tid; i < h.y; i += kThreads) {
      const unsigned v = (unsigned)__ldg(p.history + i) - (unsigned)v0;
      if (v < (unsigned)n) {
        atomicOr(&met[v], kMet);
        if (i - h.x >= prompt) atomicAdd(&met[v], 1u);
      }
    }
  }
  int2 list = make_int2(0, 0);
  if (BIAS) {
    list = part_of(p.bias_starts, b, p.n_bias);
    for (int i = list.x + tid; i < list.y; i += kThreads) {
      const unsigned v = (unsigned)__ldg(p.bias_ids + i) - (unsigned)v0;
      if (v < (unsigned)n) atomicMax(&bias[v], (unsigned)(i - list.x) + 1u);
    }
  }
  __syncthreads();
  float rep = p.repetition ? __ldg(p.repetition + b) : 1.0f;
  if (!(rep > 0.0f)) rep = 1.0f;
  const float freq = p.frequency ? __ldg(p.frequency + b) : 0.0f;
  const float pres = p.presence ? __ldg(p.presence + b) : 0.0f;
  const int32_t* mask = nullptr;
  if (p.mask) {
    const int m = p.mask_rows ? __ldg(p.mask_rows + b) : b;
    if (m >= 0 && m < p.n_masks) mask = p.mask + m * p.mask_stride;
  }
  const T* z = static_cast<const T*>(p.logits) + b * p.logits_stride + v0;
  float* out = p.out + b * p.out_stride + v0;
  for (int i = tid; i < n; i += kThreads) {
    float x = as_float(z[i]);
    const unsigned w = met[i];
    if (w) {
      x = x > 0.0f ? x / rep : x * rep;
      const unsigned times = w & ~kMet;
      if (times) x = x - freq * (float)times - pres;
    }
    if (BIAS) {
      const unsigned at = bias[i];
      if (at) x += __ldg(p.bias_values + list.x + at - 1);
    }
    if (mask && !((unsigned)__ldg(mask + ((v0 + i) >> 5)) >> ((v0 + i) & 31) & 1u)) x = -INFINITY;
    out[i] = x;
  }
}

template <typename T, bool BIAS>
cudaError_t launch(const kvq_adjust_params& p, cudaStream_t stream) {
  const size_t bytes = kSlice * sizeof(unsigned) * (BIAS ? 2 : 1);
  static std::atomic<unsigned long long> done{0};
  const cudaError_t e = once_per_device(done, [&] {
    return cudaFuncSetAttribute(adjust_kernel<T, BIAS>,
                                cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  });
  if (e != cudaSuccess) return e;
  const dim3 grid((p.vocab + kSlice - 1) / kSlice, p.rows);
  adjust_kernel<T, BIAS><<<grid, kThreads, bytes, stream>>>(p);
  return cudaGetLastError();
}

template <typename T>
cudaError_t launch_type(const kvq_adjust_params& p, cudaStream_t stream) {
  return p.bias_starts ? launch<T, true>(p, stream) : launch<T, false>(p, stream);
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
