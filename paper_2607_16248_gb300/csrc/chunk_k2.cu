// Chunk attention kernels for 2-bit keys (all value widths).

#include "chunk_core.cuh"

namespace kvq {
namespace chunk {

cudaError_t launch_k2(const Params& p, int ctas, cudaStream_t stream) {
  return launch_key_width<2>(p, ctas, stream);
}

}  // namespace chunk
}  // namespace kvq
