// kvq_adjust_logits: penalties for repeated tokens, biases and a grammar's mask, in one
// kernel or two.
//
// stream_kernel converts and masks every logit, four neighbours a thread and step: pure
// bandwidth (128 rows of 152063 bf16 logits: 25 us, 4.7 TB/s; 22 where the rows' ends are
// aligned).  Where logits stay in their place and no mask is given there is nothing to do.
// patch_kernel then gives the tokens that a list names, a few in a hundred, their values.  A
// CTA owns a slice of one row's vocabulary: a bit a token says which ones the lists name, the
// bits' running count numbers them, and the second pass over the lists counts by these
// numbers: the times a token was answered (a bit for a prompt's), and its last bias (the
// largest place in the list, so equal ids need no order).  All that runs while the first
// kernel still does; its tokens are then spread evenly over the threads.
//
// In one kernel, a counter for every token beside the slice's logits in registers
// (slice_kernel), each CTA spends most of its time on the chain of starts, list, counters and
// barriers, 47 us, but small calls are nothing but such a chain.
#include "block8.cuh"

#include <cuda_bf16.h>

#include <algorithm>

namespace kvq {

namespace {

constexpr int kThreads = 1024;         // of a patching CTA
constexpr int kSliceThreads = 512;     // of a CTA of the one kernel for small calls
constexpr int kStreamThreads = 256, kSteps = 2;  // 2048 logits a streaming CTA
constexpr int kMostSlice = 163840, kLeastSlice = 4096;  // tokens of a patching CTA
// One kernel takes calls of up to 2^23 logits (16 rows of 152063: 10.4 us where two kernels
// take 15; 128 rows: 53 where two take 39) and those of long lists (128 rows of 32768 with
// 8000 to 32768 tokens: 34 us, two kernels 62).  Slices of 4096, or of 1024 where they
// would not give every SM one (one row of 128256: 5.7 us, 6.4 in slices of 4096).
constexpr long long kOneKernel = 1LL << 23, kShortSlices = 300LL * 1024;
constexpr int kNumbers = 4096;         // tokens that it counts at a time
constexpr unsigned kMet = 0x80000000u;  // a counter's bit for a prompt's token

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
template <int THREADS, typename F>
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
  for (int i = a0 + 4 * tid; i < a1; i += 4 * THREADS) {
    const int4 x = __ldg(reinterpret_cast<const int4*>(ids + i));
    one(x.x, i);
    one(x.y, i + 1);
    one(x.z, i + 2);
    one(x.w, i + 3);
  }
}

// Four neighbouring logits on their way.  16-bit ones need not stand on an eight-byte
// boundary: the two eight-byte words that hold the first and the last of them (so that no
// word without a logit is touched).
template <typename T>
struct Four {
  uint2 a, c;
  __device__ __forceinline__ void load(const T* z) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(z);
    a = *reinterpret_cast<const uint2*>(at & ~(uintptr_t)7);
    c = *reinterpret_cast<const uint2*>((at + 7) & ~(uintptr_t)7);
  }
  __device__ __forceinline__ void values(const T* z, float (&x)[4]) const {
    const unsigned skew = (unsigned)reinterpret_cast<uintptr_t>(z) & 7u, bits = 8u * (skew & 3u);
    const bool odd = skew & 4u, two = skew != 0u;
    const unsigned w0 = odd ? a.y : a.x, w1 = odd ? c.x : a.y, w2 = odd ? c.y : c.x;
    const uint2 v = two ? make_uint2(__funnelshift_r(w0, w1, bits), __funnelshift_r(w1, w2, bits))
                        : a;
    const T* h = reinterpret_cast<const T*>(&v);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = as_float(h[i]);
  }
};
template <>
struct Four<float> {
  float4 v;
  __device__ __forceinline__ void load(const float* z) {
    if (reinterpret_cast<uintptr_t>(z) & 15u) v = make_float4(z[0], z[1], z[2], z[3]);
    else v = *reinterpret_cast<const float4*>(z);
  }
  __device__ __forceinline__ void values(const float*, float (&x)[4]) const {
    x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
  }
};

__device__ __forceinline__ const int32_t* mask_of(const kvq_adjust_params& p, int b) {
  if (!p.mask) return nullptr;
  const int m = p.mask_rows ? __ldg(p.mask_rows + b) : b;
  return m >= 0 && m < p.n_masks ? p.mask + m * p.mask_stride : nullptr;
}
__device__ __forceinline__ bool allowed(const int32_t* mask, int v) {
  return !mask || (unsigned)__ldg(mask + (v >> 5)) >> (v & 31) & 1u;
}

// Small calls: everything in one kernel.  A CTA owns a slice of one row, E strides of 512
// logits: they and their mask words are on their way while it counts the lists' tokens that
// lie there, a word a token.
template <typename T, int E, bool BIAS>
__global__ void __launch_bounds__(kSliceThreads)
slice_kernel(const __grid_constant__ kvq_adjust_params p) {
  constexpr int kSlice = E * kSliceThreads;
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
    if (i * kSliceThreads + tid < n) x[i] = z[i * kSliceThreads + tid];
  const int32_t* row_mask = mask_of(p, b);
  const int2 h = p.history_starts ? part_of(p.history_starts, b, p.n_history) : make_int2(0, 0);
  const int2 list = BIAS ? part_of(p.bias_starts, b, p.n_bias) : make_int2(0, 0);
  const int prompt = p.prompt_lengths ? __ldg(p.prompt_lengths + b) : 0;
  // lane i holds the mask's word of the warp's 32 tokens of stride i
  unsigned words = 0xffffffffu;
  if (row_mask) {
    const int at = (lane & (E - 1)) * kSliceThreads + (tid & ~31);
    if (at < n) words = (unsigned)__ldg(row_mask + ((v0 + at) >> 5));
  }
#pragma unroll
  for (int i = 0; i < E; ++i) {
    met[i * kSliceThreads + tid] = 0u;
    if (BIAS) bias[i * kSliceThreads + tid] = 0u;
  }
  __syncthreads();
  each_in<kSliceThreads>(p.history, h, v0, n, [&](unsigned v, int place) {
    if (place >= prompt) atomicAdd(&met[v], 1u);
    else atomicOr(&met[v], kMet);
  });
  if (BIAS)
    each_in<kSliceThreads>(p.bias_ids, list, v0, n,
            [&](unsigned v, int place) { atomicMax(&bias[v], (unsigned)place + 1u); });
  float rep = p.repetition ? __ldg(p.repetition + b) : 1.0f;
  if (!(rep > 0.0f)) rep = 1.0f;
  const float freq = p.frequency ? __ldg(p.frequency + b) : 0.0f;
  const float pres = p.presence ? __ldg(p.presence + b) : 0.0f;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const int at = i * kSliceThreads + tid;
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

template <typename T>
__global__ void __launch_bounds__(kStreamThreads)
stream_kernel(const __grid_constant__ kvq_adjust_params p) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  constexpr int kSlice = 4 * kSteps * kStreamThreads;
  const int tid = threadIdx.x, b = blockIdx.y;
  const T* z = static_cast<const T*>(p.logits) + b * p.logits_stride;
  float* out = p.out + b * p.out_stride;
  // slices begin at the row's results' 16-byte boundaries: the first ahead of the row
  const int first = (int)blockIdx.x * kSlice -
                    (int)((reinterpret_cast<uintptr_t>(out) >> 2) & 3u);
  const int end = min(first + kSlice, p.vocab);
  const int32_t* mask = mask_of(p, b);
  if (first >= 0 && first + kSlice <= p.vocab) {
    Four<T> raw[kSteps];
    unsigned lo[kSteps], hi[kSteps];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) raw[i].load(z + first + 4 * (i * kStreamThreads + tid));
    if (mask) {
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        const int v = first + 4 * (i * kStreamThreads + tid);
        lo[i] = (unsigned)__ldg(mask + (v >> 5));
        hi[i] = (unsigned)__ldg(mask + ((v + 3) >> 5));
      }
    }
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const int v = first + 4 * (i * kStreamThreads + tid);
      float x[4];
      raw[i].values(z + v, x);
      if (mask) {
        const unsigned bits = __funnelshift_r(lo[i], hi[i], v & 31);
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (!(bits >> k & 1u)) x[k] = -INFINITY;
      }
      *reinterpret_cast<float4*>(out + v) = make_float4(x[0], x[1], x[2], x[3]);
    }
  } else {
    for (int v = max(first, 0) + tid; v < end; v += kStreamThreads)
      out[v] = allowed(mask, v) ? as_float(z[v]) : -INFINITY;
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
patch_kernel(const __grid_constant__ kvq_adjust_params p, int slice) {
  extern __shared__ __align__(16) unsigned sm[];
  __shared__ int sums[kThreads / 32];
  const int tid = threadIdx.x, lane = tid & 31, b = blockIdx.y, v0 = blockIdx.x * slice;
  const int n = min(slice, p.vocab - v0), words = slice / 32;
  unsigned* bits = sm;             // [words]: the named tokens
  unsigned* rank = bits + words;   // [words]: how many there are before the word's
  unsigned* count = rank + words;  // [kNumbers]
  unsigned* place = count + kNumbers;
  const int2 h = p.history_starts ? part_of(p.history_starts, b, p.n_history) : make_int2(0, 0);
  const int2 biases = p.bias_starts ? part_of(p.bias_starts, b, p.n_bias) : make_int2(0, 0);
  const int prompt = p.prompt_lengths ? __ldg(p.prompt_lengths + b) : 0;
  const int32_t* mask = mask_of(p, b);
  float rep = p.repetition ? __ldg(p.repetition + b) : 1.0f;
  if (!(rep > 0.0f)) rep = 1.0f;
  const float freq = p.frequency ? __ldg(p.frequency + b) : 0.0f;
  const float pres = p.presence ? __ldg(p.presence + b) : 0.0f;
  for (int i = tid; i < words / 4; i += kThreads)
    reinterpret_cast<uint4*>(bits)[i] = make_uint4(0u, 0u, 0u, 0u);
  __syncthreads();
  const auto name = [&](unsigned v, int) {
    const unsigned bit = 1u << (v & 31);
    if (!(bits[v >> 5] & bit)) atomicOr(&bits[v >> 5], bit);
  };
  each_in<kThreads>(p.history, h, v0, n, name);
  each_in<kThreads>(p.bias_ids, biases, v0, n, name);
  __syncthreads();
  // the running count over the words, a run of them a thread
  const int run = (words + kThreads - 1) / kThreads;
  const int w0 = min(words, tid * run), w1 = min(words, w0 + run);
  int mine = 0;
  for (int w = w0; w < w1; ++w) mine += __popc(bits[w]);
  int inc = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += y;
  }
  if (lane == 31) sums[tid >> 5] = inc;
  __syncthreads();
  int at = inc - mine, total = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) {
    if (w < (tid >> 5)) at += sums[w];
    total += sums[w];
  }
  for (int w = w0; w < w1; ++w) {
    rank[w] = (unsigned)at;
    at += __popc(bits[w]);
  }
  const T* z = static_cast<const T*>(p.logits) + b * p.logits_stride;
  float* out = p.out + b * p.out_stride;
  for (int base = 0; base < total; base += kNumbers) {
    const int here = min(kNumbers, total - base);
    for (int i = tid; i < here; i += kThreads) count[i] = place[i] = 0u;
    __syncthreads();
    const auto number = [&](unsigned v) {
      return rank[v >> 5] + __popc(bits[v >> 5] & ((1u << (v & 31)) - 1u)) - (unsigned)base;
    };
    each_in<kThreads>(p.history, h, v0, n, [&](unsigned v, int i) {
      const unsigned k = number(v);
      if (k >= (unsigned)kNumbers) return;
      if (i >= prompt) atomicAdd(&count[k], 1u);
      else atomicOr(&count[k], kMet);
    });
    each_in<kThreads>(p.bias_ids, biases, v0, n, [&](unsigned v, int i) {
      const unsigned k = number(v);
      if (k < (unsigned)kNumbers) atomicMax(&place[k], (unsigned)i + 1u);
    });
    __syncthreads();
    if (base == 0) asm volatile("griddepcontrol.wait;" ::: "memory");  // all logits are there
    for (int i = tid; i < here; i += kThreads) {
      // token number base + i: the last word with no more before it, the bit by count
      int lo = 0, hi = words;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (rank[mid] <= (unsigned)(base + i)) lo = mid;
        else hi = mid;
      }
      unsigned word = bits[lo];
      for (int k = base + i - (int)rank[lo]; k > 0; --k) word &= word - 1u;
      const int v = v0 + 32 * lo + __ffs(word) - 1;
      // (in place a logit holds its value still unless a mask met it, and then it stays)
      if (!allowed(mask, v)) continue;
      float y = as_float(z[v]);
      const unsigned w = count[i], times = w & ~kMet, c = place[i];
      if (w) y = y > 0.0f ? y / rep : y * rep;
      if (times) y = y - freq * (float)times - pres;
      if (c) y += __ldg(p.bias_values + biases.x + c - 1);
      out[v] = y;
    }
    __syncthreads();
  }
  if (total == 0) asm volatile("griddepcontrol.wait;" ::: "memory");
}

// Tokens of a patching CTA's slice (a multiple of 128): a whole row while rows fill the GPU,
// else less, so that a long history's counting is spread.
int slice_of(const kvq_adjust_params& p) {
  int slice = std::min(kMostSlice, (p.vocab + 127) & ~127);
  while (slice > kLeastSlice && (long long)p.rows * ((p.vocab + slice - 1) / slice) < 128)
    slice = std::max(kLeastSlice, (slice / 2 + 127) & ~127);
  return slice;
}
int patch_bytes(int slice) { return (slice / 16 + 2 * kNumbers) * (int)sizeof(unsigned); }

template <typename T, int E, bool BIAS>
cudaError_t launch_slices(const kvq_adjust_params& p, cudaStream_t stream) {
  constexpr int kSlice = E * kSliceThreads;
  constexpr int kBytes = kSlice * (int)sizeof(unsigned) * (BIAS ? 2 : 1);
  const dim3 grid((p.vocab + kSlice - 1) / kSlice, p.rows);
  slice_kernel<T, E, BIAS><<<grid, kSliceThreads, kBytes, stream>>>(p);
  return cudaGetLastError();
}

template <typename T>
cudaError_t launch(const kvq_adjust_params& p, cudaStream_t stream) {
  const bool still = (const void*)p.out == p.logits && !p.mask;
  const long long logits = (long long)p.rows * p.vocab, named = (long long)p.n_history + p.n_bias;
  if (!still && (logits <= kOneKernel || named > (long long)kNumbers * p.rows)) {
    if (logits <= kShortSlices)
      return p.bias_starts ? launch_slices<T, 2, true>(p, stream)
                           : launch_slices<T, 2, false>(p, stream);
    return p.bias_starts ? launch_slices<T, 8, true>(p, stream)
                         : launch_slices<T, 8, false>(p, stream);
  }
  if (!still) {
    constexpr int kSlice = 4 * kSteps * kStreamThreads;
    const dim3 grid((p.vocab + 3 + kSlice - 1) / kSlice, p.rows);
    stream_kernel<T><<<grid, kStreamThreads, 0, stream>>>(p);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  if (!p.history_starts && !p.bias_starts) return cudaSuccess;
  static std::atomic<unsigned long long> done{0};
  const cudaError_t e = once_per_device(done, [] {
    return cudaFuncSetAttribute(patch_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                patch_bytes(kMostSlice));
  });
  if (e != cudaSuccess) return e;
  const int slice = slice_of(p);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((p.vocab + slice - 1) / slice, p.rows);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = patch_bytes(slice);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = still ? 0 : 1;  // only the first kernel lets it start early
  const cudaError_t l = cudaLaunchKernelEx(&cfg, patch_kernel<T>, p, slice);
  return l != cudaSuccess ? l : cudaGetLastError();
}

}  // namespace

cudaError_t launch_adjust(const kvq_adjust_params& p, cudaStream_t stream) {
  switch (p.dtype) {
    case KVQ_F16: return launch<__half>(p, stream);
    case KVQ_BF16: return launch<__nv_bfloat16>(p, stream);
    default: return launch<float>(p, stream);
  }
}

}  // namespace kvq
