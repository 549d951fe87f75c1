// Host side of kvq_block8_attn: which kernel takes which sequences, the workspace, and the
// kernel that joins the partials of shared items.
#include <algorithm>

#include "block8_plan.cuh"

namespace kvq {
namespace block8 {

namespace {

// The chunk kernel's partials to results: the CTAs (c, y) share the rows of the item that CTA c
// left.  (In that kernel itself it would fall to the CTA that comes last, whose roles have no
// registers for it.)  Up to four partials: eight rows a warp, four lanes a row, so that eight
// loads a lane are on their way (y = 0, 8, ...: 64 rows a CTA); more: a row a warp (join_row).
constexpr int kJoinWarps = 8, kFewParts = 4;

template <bool BF16>
__global__ void __launch_bounds__(32 * kJoinWarps)
join_kernel(const __grid_constant__ AttnParams p) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const Split sp = p.splits[blockIdx.x];
  const int n = sp.last - (int)blockIdx.x + 1;
  if (!sp.valid || (n <= kFewParts && (blockIdx.y & 7))) return;
  const Seq q = seq_of(p.c.d, p.c.batch, sp.b);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int n_rows = min(p.item_rows, q.n * p.c.d.gq - sp.row_tile * p.item_rows);
  const auto result = [&](int r) {
    return p.c.out + row_offset(p, p.c.out_stride, q.row, sp.head, sp.row_tile * p.item_rows + r);
  };
  if (n > kFewParts) {
    const int r = kJoinWarps * blockIdx.y + warp;
    if (r < n_rows) join_row<BF16>(p, blockIdx.x, sp.inside, n, r, result(r));
    return;
  }
  const int r = kJoinWarps * ((int)blockIdx.y + warp) + (lane >> 2);
  if (r >= n_rows) return;
  const auto slot = [&](int i) {
    return (long long)(2 * ((int)blockIdx.x + i) + (i == 0 ? sp.inside : 0)) * p.item_rows + r;
  };
  float2 ml[kFewParts];
  float m = -INFINITY, l = 0.0f;
#pragma unroll
  for (int i = 0; i < kFewParts; ++i) {
    ml[i] = i < n ? __ldcg(&p.part_ml[slot(i)]) : make_float2(0.0f, 0.0f);
    if (ml[i].y > 0.0f) m = fmaxf(m, ml[i].x);
  }
#pragma unroll
  for (int i = 0; i < kFewParts; ++i) {
    ml[i].x = ml[i].y > 0.0f ? exp2_fast(ml[i].x - m) : 0.0f;
    l += ml[i].y * ml[i].x;
  }
  const float f = l > 0.0f ? 1.0f / l : 0.0f;
  float4 out[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) out[j] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
  for (int i = 0; i < kFewParts; ++i) {
    const float x = ml[i].x * f;
    if (!(x > 0.0f)) continue;
    const float4* src =
        reinterpret_cast<const float4*>(p.part_o + slot(i) * kHeadDim) + (lane & 3);
    float4 v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = __ldcg(src + 4 * j);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      out[j].x = fmaf(v[j].x, x, out[j].x);
      out[j].y = fmaf(v[j].y, x, out[j].y);
      out[j].z = fmaf(v[j].z, x, out[j].z);
      out[j].w = fmaf(v[j].w, x, out[j].w);
    }
  }
  uint2* dst = reinterpret_cast<uint2*>(result(r)) + (lane & 3);
#pragma unroll
  for (int j = 0; j < 8; ++j)
    dst[4 * j] = make_uint2(pack16<BF16>(out[j].x, out[j].y), pack16<BF16>(out[j].z, out[j].w));
}

cudaError_t launch_join(const AttnParams& p, int ctas, int rows, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ctas, (rows + kJoinWarps - 1) / kJoinWarps);
  cfg.blockDim = dim3(32 * kJoinWarps);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const cudaError_t e = p.c.d.bf16 ? cudaLaunchKernelEx(&cfg, join_kernel<true>, p)
                                   : cudaLaunchKernelEx(&cfg, join_kernel<false>, p);
  return e != cudaSuccess ? e : cudaGetLastError();
}

// Rows of the items of both kernels; many: sequences of more than `few` rows may be there.
struct Plan {
  int few, chunk;
  bool many;
  size_t total;
};
// Rows up to which an item is one row tile of the chunk kernel, whose two streams then share
// the tokens.
constexpr int kOneTileRows = 128;
// Tickets (zero between calls) at the front, the same for every call that the workspace
// serves; then partials and splits.
size_t tickets_bytes(int ctas) { return ((size_t)ctas * sizeof(int) + 255) / 256 * 256; }
size_t parts_bytes(int ctas, int rows) {
  return tickets_bytes(ctas) +
         (size_t)2 * ctas * rows * (kHeadDim * sizeof(float) + sizeof(float2)) +
         (size_t)ctas * sizeof(Split);
}
Plan plan_of(const Dims8& d, int max_new, int ctas) {
  Plan p;
  const long long rows = (long long)max_new * d.gq;
  p.many = rows > kFewRows;
  // beside longer ones, single tokens alone: with more row groups the first kernel has fewer
  // registers to spare and its queries in shared memory (drafts beside a chunk are the second's)
  const int most = p.many ? d.gq : (int)rows;
  p.few = (most + 7) & ~7;
  p.chunk = rows > kOneTileRows ? 2 * kOneTileRows : kOneTileRows;
  // the kernels run one behind the other
  p.total = parts_bytes(ctas, p.many ? p.chunk : p.few);
  return p;
}

AttnParams params_of(const AttnCall& call, int ctas, int item_rows, void* workspace) {
  AttnParams p;
  p.c = call;
  p.gq_inverse = (uint32_t)((1ull << 32) / call.d.gq + 1);
  p.item_rows = item_rows;
  char* w = static_cast<char*>(workspace);
  p.tickets = reinterpret_cast<int*>(w);
  w += tickets_bytes(ctas);
  p.part_o = reinterpret_cast<float*>(w);
  w += (size_t)2 * ctas * item_rows * kHeadDim * sizeof(float);
  p.part_ml = reinterpret_cast<float2*>(w);
  w += (size_t)2 * ctas * item_rows * sizeof(float2);
  p.splits = reinterpret_cast<Split*>(w);
  return p;
}

}  // namespace

size_t attn_workspace_bytes(const Dims8& d, int max_new, int sm_count) {
  return plan_of(d, max_new, sm_count).total;
}
// Each kernel counts all of its items' units in 32 bits: the first a row tile a sequence, in
// blocks, the second row tiles of `chunk` rows in tiles of 128 tokens.
long long attn_most_units(const Dims8& d, int max_new) {
  const Plan plan = plan_of(d, max_new, 1);
  const long long pairs = (long long)d.batch * d.hkv, blocks = d.max_blocks;
  const long long few = pairs * (blocks * kMostWeight + kRowsItemCost);
  if (!plan.many) return few;
  const long long tiles = ((long long)max_new * d.gq + plan.chunk - 1) / plan.chunk;
  return std::max(few, pairs * tiles * ((blocks + 3) / 4 + kChunkItemCost));
}

cudaError_t launch_attn(const AttnCall& call, int sm_count, void* workspace, cudaStream_t stream,
                        bool selftest) {
  const Plan plan = plan_of(call.d, call.batch.max_new, sm_count);
  AttnParams p = params_of(call, sm_count, plan.few, workspace);
  p.min_rows = 1;
  p.max_rows = plan.few;
  cudaError_t e = cudaSuccess;
  if (call.batch.starts || !plan.many) {
    if ((e = launch_rows(p, sm_count, stream, selftest)) != cudaSuccess || !plan.many) return e;
  }
  p = params_of(call, sm_count, plan.chunk, workspace);
  p.min_rows = plan.few + 1;
  p.max_rows = 1 << 30;
  if ((e = launch_chunk(p, sm_count, stream, selftest)) != cudaSuccess) return e;
  const int rows = (int)std::min<long long>(plan.chunk, (long long)call.batch.max_new * call.d.gq);
  return launch_join(p, sm_count, rows, stream);
}

}  // namespace block8
}  // namespace kvq
