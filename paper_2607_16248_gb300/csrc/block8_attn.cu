// Host side of kvq_block8_attn: which kernel takes which sequences, the workspace, and the
// kernel that joins the partials of shared items.
#include <algorithm>

#include "block8_plan.cuh"

#include <cuda_fp8.h>

namespace kvq {
namespace block8 {

namespace {

__device__ __forceinline__ float4 half4(uint2 v, int bf16) {
  if (bf16)
    return make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u),
                       __uint_as_float(v.y << 16), __uint_as_float(v.y & 0xffff0000u));
  const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&v.x));
  const float2 b = __half22float2(*reinterpret_cast<const __half2*>(&v.y));
  return make_float4(a.x, a.y, b.x, b.y);
}
__device__ __forceinline__ float4 code4(uint32_t v) {
  const __half2_raw a = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(v & 0xffff), __NV_E4M3);
  const __half2_raw b = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(v >> 16), __NV_E4M3);
  const float2 x = __half22float2(__half2(a)), y = __half22float2(__half2(b));
  return make_float4(x.x, x.y, y.x, y.y);
}

__global__ void __launch_bounds__(256) simple_kernel(const __grid_constant__ AttnCall call,
                                                     int min_rows) {
  const int lane = threadIdx.x & 31;
  const long long task = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int row = (int)(task / call.d.hq), head = (int)(task - (long long)row * call.d.hq);
  if (row >= call.batch.n_tokens) return;
  int b = 0;
  Seq s{0, 0, 0, 0};
  for (; b < call.d.batch; ++b) {
    s = seq_of(call.d, call.batch, b);
    if (s.bad && lane == 0 && row == 0 && head == 0) set_flag(call.cache, s.bad);
    if (row >= s.row && row < s.row + s.n) break;
  }
  if (b == call.d.batch || s.n * call.d.gq < min_rows) return;
  const int h = head / call.d.gq, pos = s.L - s.n + row - s.row;
  const float4 q = half4(*reinterpret_cast<const uint2*>(
                             call.q + row * call.q_stride[0] + head * call.q_stride[1] + 4 * lane),
                         call.d.bf16);
  const long long ring = ((long long)b * call.d.hkv + h) * (kRing * kHeadDim);
  const int done = s.L / kGroup;
  float m = -INFINITY, l = 0.0f;
  float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  for (int j = 0; j <= pos; ++j) {
    if (call.window && j <= pos - call.window && j >= call.sinks) {
      j = pos - call.window;
      continue;
    }
    float4 k, v;
    if (j / kGroup < done) {
      const int page = call.cache.block_table[(long long)b * call.d.max_blocks + j / kGroup];
      if ((unsigned)page >= (unsigned)call.cache.n_pages) {
        if (lane == 0) set_flag(call.cache, KVQ_FLAG_BAD_PAGE);
        continue;
      }
      const long long at = (long long)page * call.d.hkv + h;
      const long long off = (at * kGroup + j % kGroup) * kHeadDim + 4 * lane;
      const float sk = call.cache.scales[2 * at], sv = call.cache.scales[2 * at + 1];
      k = code4(*reinterpret_cast<const uint32_t*>(call.cache.k_codes + off));
      v = code4(*reinterpret_cast<const uint32_t*>(call.cache.v_codes + off));
      k.x *= sk, k.y *= sk, k.z *= sk, k.w *= sk;
      v.x *= sv, v.y *= sv, v.z *= sv, v.w *= sv;
    } else {
      const long long off = ring + (j & (kRing - 1)) * kHeadDim + 4 * lane;
      k = half4(*reinterpret_cast<const uint2*>(call.cache.k_ring + off), call.d.bf16);
      v = half4(*reinterpret_cast<const uint2*>(call.cache.v_ring + off), call.d.bf16);
    }
    float x = q.x * k.x + q.y * k.y + q.z * k.z + q.w * k.w;
#pragma unroll
    for (int i = 16; i; i >>= 1) x += __shfl_xor_sync(0xffffffffu, x, i);
    x *= call.scale_log2;
    const float m1 = fmaxf(m, x), f = exp2f(m - m1), w = exp2f(x - m1);
    m = m1;
    l = l * f + w;
    o.x = o.x * f + w * v.x, o.y = o.y * f + w * v.y;
    o.z = o.z * f + w * v.z, o.w = o.w * f + w * v.w;
  }
  const float f = l > 0.0f ? 1.0f / l : 0.0f;
  uint2 r;
  if (call.d.bf16) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(o.x * f, o.y * f);
    const __nv_bfloat162 c = __floats2bfloat162_rn(o.z * f, o.w * f);
    r = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&c));
  } else {
    const __half2 a = __floats2half2_rn(o.x * f, o.y * f);
    const __half2 c = __floats2half2_rn(o.z * f, o.w * f);
    r = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&c));
  }
  *reinterpret_cast<uint2*>(call.out + row * call.out_stride[0] + head * call.out_stride[1] +
                            4 * lane) = r;
}

// The partials of a split item to results: the CTAs (c, y) share the rows of the item that
// CTA c left, a row a warp.  Each lane finds the weights of one of every 32 partials, then
// the weighted rows are summed in the order of the tokens.  A partial without a seen token
// weighs nothing, whatever it holds.
constexpr int kJoinWarps = 8;

template <bool BF16>
__global__ void __launch_bounds__(32 * kJoinWarps)
join_kernel(const __grid_constant__ AttnParams p) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const Split sp = p.splits[blockIdx.x];
  if (!sp.valid) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int n = sp.last - (int)blockIdx.x + 1;
  const Seq q = seq_of(p.c.d, p.c.batch, sp.b);
  const int r = kJoinWarps * blockIdx.y + warp;
  const int row = sp.row_tile * p.item_rows + r;
  if (r >= p.item_rows || row >= q.n * p.c.d.gq) return;
  const auto slot = [&](int i) {  // row r of the i-th partial
    return (long long)(2 * ((int)blockIdx.x + i) + (i == 0 ? sp.inside : 0)) * p.item_rows + r;
  };
  constexpr int kMost = (kMaxSplits + 31) / 32;  // partials a lane
  float2 ml[kMost];
  float m = -INFINITY;
#pragma unroll
  for (int k = 0; k < kMost; ++k) {
    const int i = 32 * k + lane;
    ml[k] = i < n ? __ldcg(&p.part_ml[slot(i)]) : make_float2(0.0f, 0.0f);
    if (ml[k].y > 0.0f) m = fmaxf(m, ml[k].x);
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  float l = 0.0f;
#pragma unroll
  for (int k = 0; k < kMost; ++k) {
    ml[k].x = ml[k].y > 0.0f ? exp2_fast(ml[k].x - m) : 0.0f;
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
          __ldcg(reinterpret_cast<const float4*>(p.part_o + slot(i) * kHeadDim) + lane);
      if (x > 0.0f) {
        out.x = fmaf(v.x, x, out.x);
        out.y = fmaf(v.y, x, out.y);
        out.z = fmaf(v.z, x, out.z);
        out.w = fmaf(v.w, x, out.w);
      }
    }
  }
  reinterpret_cast<uint2*>(p.c.out + row_offset(p, p.c.out_stride, q.row, sp.head, row))[lane] =
      make_uint2(pack16<BF16>(out.x, out.y), pack16<BF16>(out.z, out.w));
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

// Which kernels a call runs: `few`, rows of the items of the kernel for few rows.
struct Plan {
  int few;
  bool many;  // sequences of more rows may be there
  size_t total;
};
size_t parts_bytes(int ctas, int rows) {
  return (size_t)2 * ctas * rows * (kHeadDim * sizeof(float) + sizeof(float2)) +
         (size_t)ctas * sizeof(Split) + 256;
}
Plan plan_of(const Dims8& d, int max_new, int ctas) {
  Plan p;
  const long long rows = (long long)max_new * d.gq;
  p.many = rows > kFewRows;
  // beside longer ones, single tokens alone are short: more columns would cost them products
  const int most = p.many ? d.gq : (int)rows;
  p.few = most <= 8 ? 8 : most <= 16 ? 16 : 32;
  p.total = parts_bytes(ctas, p.few);
  return p;
}

AttnParams params_of(const AttnCall& call, int ctas, int item_rows, void* workspace) {
  AttnParams p;
  p.c = call;
  p.gq_inverse = (uint32_t)((1ull << 32) / call.d.gq + 1);
  p.item_rows = item_rows;
  char* w = static_cast<char*>(workspace);
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
long long attn_most_units(const Dims8& d, int max_new) {
  const Plan plan = plan_of(d, max_new, 1);
  const long long tiles = plan.many ? ((long long)max_new * d.gq + 255) / 256 : 1;
  return (long long)d.batch * d.hkv * (d.max_blocks + 8) * tiles;
}

cudaError_t launch_attn(const AttnCall& call, int sm_count, void* workspace, cudaStream_t stream) {
  const Plan plan = plan_of(call.d, call.batch.max_new, sm_count);
  AttnParams p = params_of(call, sm_count, plan.few, workspace);
  p.min_rows = 1;
  p.max_rows = plan.few;
  cudaError_t e = launch_rows(p, sm_count, stream);
  if (e != cudaSuccess) return e;
  if ((e = launch_join(p, sm_count, plan.few, stream)) != cudaSuccess || !plan.many) return e;
  const long long tasks = (long long)call.batch.n_tokens * call.d.hq;
  simple_kernel<<<(unsigned)((tasks + 7) / 8), 256, 0, stream>>>(call, plan.few + 1);
  return cudaGetLastError();
}

}  // namespace block8
}  // namespace kvq
