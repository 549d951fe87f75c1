// Host side of the chunk attention: sizes of the work plan, workspace and the
// kernel of the cache's code widths; the kernel that joins the partials of items
// that several CTAs shared.

#include <algorithm>

#include "chunk_core.cuh"

namespace kvq {

namespace {

constexpr int kJoinWarps = 8, kFewParts = 4;

// The partials of a split item to results: the CTAs (c, y) share the rows of the
// item that CTA c left.  (In the attention kernel itself it would fall to the CTA that
// comes last, behind all others, and take registers from the scores.)
//   up to four partials: eight rows a warp, four lanes a row, so that eight loads
//   a lane are on their way (y = 0, 8, ...: 64 rows a CTA);
//   more: a row a warp; each lane finds the weights of one of every 32 partials,
//   then the weighted rows are summed in the order of the tokens.
// A partial without a seen token weighs nothing, whatever it holds.
__global__ void __launch_bounds__(32 * kJoinWarps, 2)
join_kernel(const __grid_constant__ chunk::Params p) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const chunk::Split sp = p.splits[blockIdx.x];
  if (!sp.valid) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int tr = chunk::kTile << p.streams_rows, n = sp.last - (int)blockIdx.x + 1;
  const int n_rows = min(tr, p.c.n_q * p.d.gq - sp.row_tile * tr);
  const auto slot = [&](int i) {  // first row of the i-th partial
    return (long long)(2 * ((int)blockIdx.x + i) + (i == 0 ? sp.inside : 0)) * tr;
  };
  const auto result = [&](int r) {
    return p.out + chunk::row_offset(p, p.c.out_stride, sp.bl, sp.head, sp.row_tile * tr + r);
  };
  if (n <= kFewParts) {
    if (blockIdx.y & 7) return;
    const int r = kJoinWarps * ((int)blockIdx.y + warp) + (lane >> 2);
    if (r >= n_rows) return;
    float2 ml[kFewParts];
    float m = -INFINITY, l = 0.0f;
#pragma unroll
    for (int i = 0; i < kFewParts; ++i) {
      ml[i] = i < n ? __ldcg(&p.part_ml[slot(i) + r]) : make_float2(0.0f, 0.0f);
      if (ml[i].y > 0.0f) m = fmaxf(m, ml[i].x);
    }
#pragma unroll
    for (int i = 0; i < kFewParts; ++i) {
      ml[i].x = ml[i].y > 0.0f ? chunk::exp2_fast(ml[i].x - m) : 0.0f;
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
          reinterpret_cast<const float4*>(p.part_o + (slot(i) + r) * kHeadDim) + (lane & 3);
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
      dst[4 * j] = make_uint2(chunk::pack_half2(out[j].x, out[j].y),
                              chunk::pack_half2(out[j].z, out[j].w));
    return;
  }
  constexpr int kMost = (kMaxSplits + 31) / 32;  // partials a lane
  const int r = kJoinWarps * blockIdx.y + warp;
  if (r >= n_rows) return;
  float2 ml[kMost];
  float m = -INFINITY;
#pragma unroll
  for (int k = 0; k < kMost; ++k) {
    const int i = 32 * k + lane;
    ml[k] = i < n ? __ldcg(&p.part_ml[slot(i) + r]) : make_float2(0.0f, 0.0f);
    if (ml[k].y > 0.0f) m = fmaxf(m, ml[k].x);
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  float l = 0.0f;
#pragma unroll
  for (int k = 0; k < kMost; ++k) {
    ml[k].x = ml[k].y > 0.0f ? chunk::exp2_fast(ml[k].x - m) : 0.0f;
    l += ml[k].y * ml[k].x;
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
  const float f = l > 0.0f ? 1.0f / l : 0.0f;
  float4 out = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
  for (int k = 0; k < kMost; ++k) {
#pragma unroll 8
    for (int i = 32 * k; i < min(n, 32 * k + 32); ++i) {
      const float x = __shfl_sync(0xffffffffu, ml[k].x, i & 31) * f;
      const float4 v =
          __ldcg(reinterpret_cast<const float4*>(p.part_o + (slot(i) + r) * kHeadDim) + lane);
      if (x > 0.0f) {
        out.x = fmaf(v.x, x, out.x);
        out.y = fmaf(v.y, x, out.y);
        out.z = fmaf(v.z, x, out.z);
        out.w = fmaf(v.w, x, out.w);
      }
    }
  }
  reinterpret_cast<uint2*>(result(r))[lane] =
      make_uint2(chunk::pack_half2(out.x, out.y), chunk::pack_half2(out.z, out.w));
}

// The waits of the attention kernel's roles: the warps of `role` (0 softmax, 1
// loading, 2 issuing) wait with a short limit on a barrier at which nothing arrives,
// the softmax and loading warps otherwise with the usual one, the issuing warps have
// finished.  All leave when the first ones give up.
__global__ void __launch_bounds__(chunk::kThreads, 1)
wait_selftest_kernel(int role, int32_t* flag, uint32_t limit) {
  extern __shared__ __align__(1024) unsigned char raw[];
  chunk::Smem& s = *reinterpret_cast<chunk::Smem*>(raw);
  const int warp = threadIdx.x >> 5;
  const int mine = warp < chunk::kSoftmaxWarps ? 0 : warp < chunk::kIssueWarp ? 1 : 2;
  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      chunk::bar_init(&s.k_full[i], 1);
      chunk::bar_init(&s.drained[i], 1);
    }
    s.abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  if (mine == role) chunk::warp_wait(s, &s.k_full[0], 0, limit);
  else if (mine < 2) chunk::warp_wait(s, &s.k_full[1], 0);
  __syncwarp();
  chunk::leave(s, flag);
}

// Rows of a (sequence, kv-head) up to this many make one row tile of 128.
constexpr int kOneTileRows = chunk::kTile;

struct Plan {
  int tiles, streams_rows, rows;  // row tiles per pair, see Params; rows of an item
  size_t o_bytes, ml_bytes, total;
};

Plan plan_of(const Dims& d, int n_q, int ctas) {
  Plan p;
  const long long rows = (long long)n_q * d.gq;
  p.streams_rows = rows > kOneTileRows ? 1 : 0;
  p.rows = chunk::kTile << p.streams_rows;
  p.tiles = (int)((rows + p.rows - 1) / p.rows);
  p.o_bytes = (size_t)2 * ctas * p.rows * kHeadDim * sizeof(float);
  p.ml_bytes = (size_t)2 * ctas * p.rows * sizeof(float2);
  p.total = p.o_bytes + p.ml_bytes + (size_t)ctas * sizeof(chunk::Split);
  return p;
}

}  // namespace

long long chunk_most_units(const Dims& d, int n_q, int batch_count) {
  const long long items = (long long)plan_of(d, n_q, 1).tiles * d.hkv * batch_count;
  return items * ((d.max_len + chunk::kTile - 1LL) / chunk::kTile + chunk::kItemCost);
}

size_t chunk_workspace_bytes(const Dims& d, int n_q, int sm_count) {
  return plan_of(d, n_q, sm_count).total;
}

cudaError_t launch_chunk_wait_selftest(int role, int32_t* flag, uint32_t limit_cycles,
                                       cudaStream_t stream) {
  static std::atomic<unsigned long long> done{0};
  const cudaError_t e = once_per_device(done, [] {
    return cudaFuncSetAttribute(wait_selftest_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                (int)sizeof(chunk::Smem));
  });
  if (e != cudaSuccess) return e;
  wait_selftest_kernel<<<1, chunk::kThreads, sizeof(chunk::Smem), stream>>>(role, flag,
                                                                            limit_cycles);
  return cudaGetLastError();
}

cudaError_t launch_chunk_attn(const Dims& d, const kvq_cache& cache, const __half* q, __half* out,
                              const ChunkCall& call, int sm_count, void* workspace,
                              cudaStream_t stream) {
  const Plan plan = plan_of(d, call.n_q, sm_count);
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
  p.splits = reinterpret_cast<chunk::Split*>(w + plan.o_bytes + plan.ml_bytes);
  cudaError_t e;
  switch (d.bits_k) {
    case 1: e = chunk::launch_k1(p, sm_count, stream); break;
    case 2: e = chunk::launch_k2(p, sm_count, stream); break;
    case 4: e = chunk::launch_k4(p, sm_count, stream); break;
    default: e = chunk::launch_k8(p, sm_count, stream); break;
  }
  if (e != cudaSuccess) return e;
  const int rows = (int)std::min<long long>(plan.rows, (long long)call.n_q * d.gq);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(sm_count, (rows + kJoinWarps - 1) / kJoinWarps);
  cfg.blockDim = dim3(32 * kJoinWarps);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  e = cudaLaunchKernelEx(&cfg, join_kernel, p);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace kvq
