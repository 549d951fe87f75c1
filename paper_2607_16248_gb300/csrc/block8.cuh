// The block-8 cache's shared definitions: the call's sizes, a batch's sequences and
// the launchers that api.cu calls.
#pragma once

#include <cuda_bf16.h>

#include "serve.cuh"

namespace kvq {
namespace block8 {

constexpr int kRing = KVQ_BLOCK8_RING;
constexpr float kMaxCode = 448.0f;  // e4m3's largest

struct Dims8 {
  int batch, hq, hkv, gq, max_len, max_blocks, bf16;
};

struct AppendCall {
  Dims8 d;
  kvq_block8_cache cache;
  kvq_block8_batch batch;
  kvq_block8_append_params p;
};

struct AttnCall {
  Dims8 d;
  kvq_block8_cache cache;
  kvq_block8_batch batch;
  const uint16_t* q;
  uint16_t* out;
  int window, sinks;
  float scale_log2;
  long long q_stride[2], out_stride[2];
};

cudaError_t launch_append(const AppendCall& call, int sm_count, cudaStream_t stream);
size_t attn_workspace_bytes(const Dims8& d, int max_new, int sm_count);
// The most units of work that a call's kernels can count.
long long attn_most_units(const Dims8& d, int max_new);
// selftest: with a short limit and an arrival that never comes, so that a wait runs out.
cudaError_t launch_attn(const AttnCall& call, int sm_count, void* workspace, cudaStream_t stream,
                        bool selftest = false);

#ifdef __CUDACC__
// The rows [row, row + n) of sequence b, which has L tokens with them; n is 0 where it
// has none or what the batch says of it does not hold (`bad`: a KVQ_FLAG_*).
struct Seq {
  int row, n, L, bad;
};
__device__ __forceinline__ Seq seq_of(const Dims8& d, const kvq_block8_batch& batch, int b) {
  Seq s;
  s.bad = 0;
  s.L = __ldg(batch.lengths + b);
  if (batch.starts) {
    s.row = __ldg(batch.starts + b);
    const int end = __ldg(batch.starts + b + 1);
    s.n = end - s.row;
    if (s.row < 0 || end < s.row || end > batch.n_tokens || s.n > batch.max_new)
      s.bad = KVQ_FLAG_BAD_BATCH;
  } else {
    s.n = batch.max_new;
    s.row = b * s.n;
  }
  if (s.L > d.max_len) s.bad |= KVQ_FLAG_OVERFLOW;
  if (s.L < 0) s.bad |= KVQ_FLAG_BAD_BATCH;
  if (s.bad) s.n = 0;
  return s;
}
__device__ __forceinline__ void set_flag(const kvq_block8_cache& c, unsigned bit) {
  atomicOr(c.flags, bit);
}
#endif

}  // namespace block8

// Adjusted logits (adjust.cu).
cudaError_t launch_adjust(const kvq_adjust_params& p, cudaStream_t stream);

}  // namespace kvq
