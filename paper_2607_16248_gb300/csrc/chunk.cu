// Host side of the chunk attention: sizes of the work plan, workspace and the
// kernel of the cache's code widths.

#include "chunk_core.cuh"

namespace kvq {

namespace {

// Rows of a (sequence, kv-head) up to this many make one row tile of 128.
constexpr int kOneTileRows = chunk::kTile;

struct Plan {
  int tiles, streams_rows, rows;  // row tiles per pair, see Params; rows of an item
  size_t items, o_bytes, ml_bytes, total;
};

size_t up16(size_t x) { return (x + 15) / 16 * 16; }

Plan plan_of(const Dims& d, int n_q, int batch_count, int ctas) {
  Plan p;
  const long long rows = (long long)n_q * d.gq;
  p.streams_rows = rows > kOneTileRows ? 1 : 0;
  p.rows = chunk::kTile << p.streams_rows;
  p.tiles = (int)((rows + p.rows - 1) / p.rows);
  p.items = (size_t)p.tiles * d.hkv * batch_count;
  p.o_bytes = (size_t)2 * ctas * p.rows * kHeadDim * sizeof(float);
  p.ml_bytes = (size_t)2 * ctas * p.rows * sizeof(float2);
  p.total = p.o_bytes + p.ml_bytes + up16(p.items * sizeof(unsigned));
  return p;
}

}  // namespace

size_t chunk_workspace_bytes(const Dims& d, int n_q, int batch_count, int sm_count) {
  return plan_of(d, n_q, batch_count, sm_count).total;
}

cudaError_t launch_chunk_attn(const Dims& d, const kvq_cache& cache, const __half* q, __half* out,
                              const ChunkCall& call, int sm_count, void* workspace,
                              cudaStream_t stream) {
  const Plan plan = plan_of(d, call.n_q, call.batch_count, sm_count);
  chunk::Params p;
  p.d = d;
  p.cache = cache;
  p.q = q;
  p.out = out;
  p.c = call;
  p.tiles = plan.tiles;
  p.streams_rows = plan.streams_rows;
  p.gq_inverse = (uint32_t)((1ull << 32) / d.gq + 1);
  char* w = static_cast<char*>(workspace);
  p.part_o = reinterpret_cast<float*>(w);
  p.part_ml = reinterpret_cast<float2*>(w + plan.o_bytes);
  p.tickets = reinterpret_cast<unsigned*>(w + plan.o_bytes + plan.ml_bytes);
  switch (d.bits_k) {
    case 1: return chunk::launch_k1(p, sm_count, stream);
    case 2: return chunk::launch_k2(p, sm_count, stream);
    case 4: return chunk::launch_k4(p, sm_count, stream);
    default: return chunk::launch_k8(p, sm_count, stream);
  }
}

}  // namespace kvq
