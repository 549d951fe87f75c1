// Attention of a chunk of new tokens over the cache (kvq_chunk_attn): one CTA
// per 32 query rows of a (sequence, kv-head), in fp32 on the dequantized
// blocks, one 32-token block at a time with a running maximum and sum.

#include "common.cuh"

namespace kvq {

namespace {

constexpr int kRows = 32, kThreads = 256;

// Code of element (token t, channel c) of a page's key or value area.
__device__ __forceinline__ int code_at(const uint32_t* w, int bits, bool key, int t, int c) {
  if (bits == 1) {
    const int i = key ? key1_bit(t, c) : val1_bit(t, c);
    return (w[i >> 5] >> (i & 31)) & 1;
  }
  const int row = key ? c : (c >> 5) * 32 + t, i = (key ? t : c & 31) * bits;
  return (w[row * bits + (i >> 5)] >> (i & 31)) & ((1 << bits) - 1);
}

__global__ void __launch_bounds__(kThreads)
chunk_attn_kernel(Dims d, kvq_cache cache, const __half* __restrict__ q, __half* __restrict__ out,
                  ChunkCall p) {
  __shared__ float qs[kRows][kHeadDim], ks[kGroup][kHeadDim + 1], vs[kGroup][kHeadDim];
  __shared__ float ps[kRows][kGroup + 1], row_m[kRows], row_l[kRows], row_f[kRows];
  const int tid = threadIdx.x, h = blockIdx.y, bl = blockIdx.z, b = p.batch_begin + bl;
  const int L = cache.seq_len[b], lq = packed_len(L, d.residual);
  const int rows = p.n_q * d.gq, row0 = blockIdx.x * kRows;
  const auto pos_of = [&](int r) { return L - p.n_q + (row0 + r) / d.gq; };
  const auto row_ptr = [&](const long long* st, int r) {
    const int t = (row0 + r) / d.gq, i = h * d.gq + (row0 + r) % d.gq;
    return bl * st[0] + t * st[1] + i * st[2];
  };
  for (int i = tid; i < kRows * kHeadDim; i += kThreads) {
    const int r = i / kHeadDim, c = i % kHeadDim;
    qs[r][c] = row0 + r < rows ? __half2float(q[row_ptr(p.q_stride, r) + c]) : 0.0f;
  }
  if (tid < kRows) {
    row_m[tid] = -INFINITY;
    row_l[tid] = 0.0f;
  }
  float acc[16];
#pragma unroll
  for (int k = 0; k < 16; ++k) acc[k] = 0.0f;
  const int last = min(kRows, rows - row0) - 1;
  const int hi = pos_of(last), lo = p.window ? max(0, pos_of(0) - p.window + 1) : 0;
  const PageMap pm = page_map(d, cache, b, h);
  const long long ring = ((long long)b * d.hkv + h) * d.ring * kHeadDim;
  const __half* kr = reinterpret_cast<const __half*>(cache.k_resid) + ring;
  const __half* vr = reinterpret_cast<const __half*>(cache.v_resid) + ring;
  for (int t0 = 0; t0 <= hi; t0 += kGroup) {
    if (t0 >= p.sinks && t0 < lo / kGroup * kGroup) t0 = lo / kGroup * kGroup;
    __syncthreads();
    if (t0 < lq) {
      const char* page = pm.at(t0 / kGroup);
      if (!page && tid == 0)
        atomicOr(reinterpret_cast<unsigned*>(cache.seq_len + d.batch), KVQ_FLAG_BAD_PAGE);
      for (int i = tid; i < kGroup * kHeadDim; i += kThreads) {
        const int t = i / kHeadDim, c = i % kHeadDim;
        float kx = 0.0f, vx = 0.0f;
        if (page) {
          const __half* km = reinterpret_cast<const __half*>(page + page_off_kmeta(d.bits_k));
          const __half* vm =
              reinterpret_cast<const __half*>(page + page_off_vmeta(d.bits_k, d.bits_v));
          const int kc = code_at(reinterpret_cast<const uint32_t*>(page), d.bits_k, true, t, c);
          const int vc = code_at(reinterpret_cast<const uint32_t*>(page + page_off_vcodes(d.bits_k)),
                                 d.bits_v, false, t, c);
          const int vi = vmeta_index(c >> 5, t);
          kx = fmaf(__half2float(km[c]), (float)kc, __half2float(km[kHeadDim + c]));
          vx = fmaf(__half2float(vm[vi]), (float)vc, __half2float(vm[kHeadDim + vi]));
        }
        ks[t][c] = kx;
        vs[t][c] = vx;
      }
    } else {
      for (int i = tid; i < kGroup * kHeadDim; i += kThreads) {
        const int t = i / kHeadDim, c = i % kHeadDim, slot = (t0 + t) % d.ring;
        ks[t][c] = t0 + t < L ? __half2float(kr[slot * kHeadDim + c]) : 0.0f;
        vs[t][c] = t0 + t < L ? __half2float(vr[slot * kHeadDim + c]) : 0.0f;
      }
    }
    __syncthreads();
    {
      const int t = tid & 31, r0 = tid >> 5, j = t0 + t;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int r = r0 + 8 * k, pr = pos_of(r);
        float s = 0.0f;
        for (int c = 0; c < kHeadDim; ++c) s = fmaf(qs[r][c], ks[t][c], s);
        const bool seen = j <= pr && (!p.window || j > pr - p.window || j < p.sinks);
        s = seen ? s * p.scale_log2 : -INFINITY;
        float m = s;
#pragma unroll
        for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        const float old = row_m[r], now = fmaxf(old, m);
        const float e = seen ? exp2f(s - now) : 0.0f;
        ps[r][t] = e;
        float sum = e;
#pragma unroll
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        __syncwarp();
        if (t == 0) {
          const float f = old == -INFINITY ? 0.0f : exp2f(old - now);
          row_f[r] = f;
          row_l[r] = row_l[r] * f + sum;
          row_m[r] = now;
        }
      }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      const int r = (tid >> 7) + 2 * k, c = tid & 127;
      float o = acc[k] * row_f[r];
      for (int t = 0; t < kGroup; ++t) o = fmaf(ps[r][t], vs[t][c], o);
      acc[k] = o;
    }
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    const int r = (tid >> 7) + 2 * k, c = tid & 127;
    if (row0 + r >= rows) continue;
    const float l = row_l[r];
    out[row_ptr(p.out_stride, r) + c] = __float2half_rn(l > 0.0f ? acc[k] / l : 0.0f);
  }
}

}  // namespace

size_t chunk_workspace_bytes(const Dims&, int, int, int) { return 256; }

cudaError_t launch_chunk_attn(const Dims& d, const kvq_cache& cache, const __half* q, __half* out,
                              const ChunkCall& call, int, void*, cudaStream_t stream) {
  const dim3 grid((call.n_q * d.gq + kRows - 1) / kRows, d.hkv, call.batch_count);
  chunk_attn_kernel<<<grid, kThreads, 0, stream>>>(d, cache, q, out, call);
  return cudaGetLastError();
}

}  // namespace kvq
