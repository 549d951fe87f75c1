// Chunk attention kernels for 4-bit keys (all value widths).

#include "chunk_core.cuh"

namespace kvq {
namespace chunk {

cudaError_t launch_k4(const Params& p, int ctas, cudaStream_t stream) {
  return launch_key_width<4>(p, ctas, stream);
}

}  // namespace chunk
}  // namespace kvq
