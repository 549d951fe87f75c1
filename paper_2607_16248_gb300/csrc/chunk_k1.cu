// Chunk attention kernels for 1-bit keys (all value widths).

#include "chunk_core.cuh"

namespace kvq {
namespace chunk {

cudaError_t launch_k1(const Params& p, int ctas, cudaStream_t stream) {
  return launch_key_width<1>(p, ctas, stream);
}

}  // namespace chunk
}  // namespace kvq
