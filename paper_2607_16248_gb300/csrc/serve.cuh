// Launchers of the chunk attention and of sampling (what a serving loop adds to
// the decode step), called by api.cu.
#pragma once

#include "common.cuh"

#include <atomic>

namespace kvq {

// Runs `prepare` (function attributes) at a kernel's first launch on each device;
// `done` is the kernel's own.
template <typename F>
cudaError_t once_per_device(std::atomic<unsigned long long>& done, F prepare) {
  int dev = 0;
  const cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const unsigned long long bit = dev < 64 ? 1ull << dev : 0ull;
  if (done.load(std::memory_order_acquire) & bit) return cudaSuccess;
  const cudaError_t p = prepare();
  if (p == cudaSuccess) done.fetch_or(bit, std::memory_order_release);
  return p;
}

// Chunk attention (chunk.cu): kvq_chunk_params with the scale in the log2
// domain and the range of sequences.
struct ChunkCall {
  int n_q, window, sinks, batch_begin, batch_count;
  float scale_log2;
  long long q_stride[3], out_stride[3];
};
// The most units of work that the kernel can count for a call (full sequences).
long long chunk_most_units(const Dims& d, int n_q, int batch_count);
size_t chunk_workspace_bytes(const Dims& d, int n_q, int sm_count);
cudaError_t launch_chunk_attn(const Dims& d, const kvq_cache& cache, const __half* q, __half* out,
                              const ChunkCall& call, int sm_count, void* workspace,
                              cudaStream_t stream);
cudaError_t launch_chunk_wait_selftest(int role, int32_t* flag, uint32_t limit_cycles,
                                       cudaStream_t stream);

// Sampling (sample.cu).
struct SampleCall {
  const float *logits, *noise;
  long long logits_stride, noise_stride;
  int batch, vocab;
  const float* temperature;
  const int32_t* top_k;
  const float *top_p, *min_p;
  int32_t* token;
  float* logprob;
};
int sample_max_vocab();
cudaError_t launch_sample(const SampleCall& call, int sm_count, cudaStream_t stream);

}  // namespace kvq
