// kvq_block8_attn, the simple form: a warp per query row, a token at a time.
#include "block8.cuh"

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

__global__ void __launch_bounds__(256) rows_kernel(const __grid_constant__ AttnCall call) {
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
  if (b == call.d.batch) return;
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

}  // namespace

size_t attn_workspace_bytes(const Dims8&, int, int) { return 16; }
long long attn_most_units(const Dims8& d, int max_new) {
  return (long long)d.batch * d.hkv * (d.max_blocks + 8) * ((max_new * d.gq + 255) / 256);
}

cudaError_t launch_attn(const AttnCall& call, int, void*, cudaStream_t stream) {
  const long long tasks = (long long)call.batch.n_tokens * call.d.hq;
  rows_kernel<<<(unsigned)((tasks + 7) / 8), 256, 0, stream>>>(call);
  return cudaGetLastError();
}

}  // namespace block8
}  // namespace kvq
