// The next token of each row of logits (kvq_sample): one CTA per row.
//
// The order of the tokens (value descending, lowest index first) is the order
// of the 64-bit number (ordered bits of z) << 32 | ~index, descending.  A limit
// keeps the tokens at or above the largest threshold whose count (top-k) or
// mass (top-p) reaches its goal; the threshold is found bit by bit.

#include "common.cuh"

namespace kvq {

namespace {

using u64 = unsigned long long;
constexpr int kThreads = 1024, kMaxVocab = 262144;

// Bits of a float32 whose unsigned order is the numbers' (-0 as +0).
__device__ __forceinline__ uint32_t ordered(float z) {
  const uint32_t u = __float_as_uint(z == 0.0f ? 0.0f : z);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ u64 rank_key(float z, int i) {
  return ((u64)ordered(z) << 32) | (uint32_t)~i;
}

struct Sm {
  u64 part[32];
  u64 result;
};

template <typename F>
__device__ u64 reduce(Sm& s, u64 v, F f) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v = f(v, __shfl_xor_sync(0xffffffffu, v, o));
  __syncthreads();
  if ((threadIdx.x & 31) == 0) s.part[threadIdx.x >> 5] = v;
  __syncthreads();
  v = s.part[threadIdx.x & 31];
#pragma unroll
  for (int o = 16; o; o >>= 1) v = f(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
__device__ __forceinline__ u64 add(u64 a, u64 b) { return a + b; }
__device__ __forceinline__ u64 most(u64 a, u64 b) { return a > b ? a : b; }

// e in [0, 1] as a multiple of 2^-40.
__device__ __forceinline__ u64 mass_of(float e) { return (u64)__float2ull_rn(e * 0x1p40f); }

__global__ void __launch_bounds__(kThreads) sample_kernel(SampleCall p) {
  __shared__ Sm s;
  const int b = blockIdx.x, tid = threadIdx.x, V = p.vocab;
  const float* z = p.logits + b * p.logits_stride;
  const float* u = p.noise ? p.noise + b * p.noise_stride : nullptr;
  float T = p.temperature ? p.temperature[b] : 1.0f;
  const bool greedy = !(T > 0.0f) || !u;
  if (!(T > 0.0f)) T = 1.0f;
  u64 top = 0;
  for (int i = tid; i < V; i += kThreads) top = most(top, rank_key(z[i], i));
  top = reduce(s, top, most);
  const int best = (int)~(uint32_t)top;
  const float zmax = z[best];
  if (zmax == -INFINITY) {
    if (tid == 0) {
      p.token[b] = -1;
      if (p.logprob) p.logprob[b] = -INFINITY;
    }
    return;
  }
  const auto dist = [&](int i) { return __fdiv_rn(z[i] - zmax, T); };
  u64 total = 0;
  for (int i = tid; i < V; i += kThreads) total += mass_of(expf(dist(i)));
  total = reduce(s, total, add);
  int token = best;
  if (!greedy) {
    // the largest threshold at or above which there are `goal` tokens (or mass)
    const auto search = [&](u64 goal, bool mass) {
      u64 t = 0;
      for (int bit = 63; bit >= 0; --bit) {
        const u64 c = t | (1ull << bit);
        u64 n = 0;
        for (int i = tid; i < V; i += kThreads)
          if (rank_key(z[i], i) >= c) n += mass ? mass_of(expf(dist(i))) : 1ull;
        if (reduce(s, n, add) >= goal) t = c;
      }
      return t;
    };
    const int k = p.top_k ? p.top_k[b] : 0;
    const float tp = p.top_p ? p.top_p[b] : 1.0f, mp = p.min_p ? p.min_p[b] : 0.0f;
    u64 cut = k > 0 && k < V ? search((u64)k, false) : 0ull;
    if (tp < 1.0f) {
      u64 n = 0;
      for (int i = tid; i < V; i += kThreads)
        if (rank_key(z[i], i) >= cut) n += mass_of(expf(dist(i)));
      n = reduce(s, n, add);
      const u64 goal = tp > 0.0f ? (u64)ceil((double)tp * (double)n) : 0ull;
      cut = goal ? search(goal, true) : top;
    }
    u64 win = 0;
    for (int i = tid; i < V; i += kThreads) {
      const u64 r = rank_key(z[i], i);
      const float d = dist(i);
      if (r < cut || (expf(d) < mp && r != top) || z[i] == -INFINITY) continue;
      const float key = d - logf(-logf(u[i]));
      win = most(win, rank_key(key, i));
    }
    win = reduce(s, win, most);
    token = (int)~(uint32_t)win;
  }
  if (tid == 0) {
    p.token[b] = token;
    if (p.logprob) p.logprob[b] = dist(token) - logf((float)((double)total * 0x1p-40));
  }
}

}  // namespace

int sample_max_vocab() { return kMaxVocab; }

cudaError_t launch_sample(const SampleCall& call, cudaStream_t stream) {
  sample_kernel<<<call.batch, kThreads, 0, stream>>>(call);
  return cudaGetLastError();
}

}  // namespace kvq
