// kvq_block8_append: rotation of queries and keys, the rings, and the codes of the
// blocks that the new tokens complete, in one launch.
//
// A warp's task is either one block's keys or values of one kv-head (32 x 128 elements,
// two rows at a time, all in its registers: the block's largest magnitude is known before
// the first code) or one token's queries of eight heads.  In both, 16 lanes share a row
// of 128 channels; a lane holds two groups of four channels such that it has both
// channels of its four rotated pairs (`Lane`), so a rotation needs no exchange and each
// cosine is read once.
//
// The codes need the keys' exact roundings: a key next to a border of its type changes
// its block's scale, and a quotient next to a border its code.  Products and sums
// therefore keep their low parts (two fp32 numbers), and the first rounding goes to odd,
// so that the second, to 16 bits, is the only one.
//
// A block that was begun by an earlier call has its first rows in the ring, in slots that
// this call's newest tokens may take.  Of the two blocks whose tokens go to the ring, the
// one with the same slots (an even number of blocks behind) is done by the same warp,
// after the begun block's rows are in its registers.
#include "block8.cuh"

#include <cuda_fp8.h>

namespace kvq {
namespace block8 {

namespace {

constexpr int kWarps = 8;
constexpr int kQueryHeads = 8;  // heads of a query task

__device__ __forceinline__ uint2 ld8(const uint16_t* p) {
  return __ldg(reinterpret_cast<const uint2*>(p));
}
// The ring is written by the same launch: no read-only path.
__device__ __forceinline__ uint2 ld8_ring(const uint16_t* p) {
  return __ldcg(reinterpret_cast<const uint2*>(p));
}
__device__ __forceinline__ void st8(uint16_t* p, uint2 v) { *reinterpret_cast<uint2*>(p) = v; }

template <bool BF16>
__device__ __forceinline__ float2 widen(uint32_t u) {
  if constexpr (BF16)
    return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
  else
    return __half22float2(*reinterpret_cast<const __half2*>(&u));
}
template <bool BF16>
__device__ __forceinline__ uint32_t narrow(float a, float b) {
  if constexpr (BF16) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  } else {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
}

// The two groups of four channels of lane c of 16, and its first pair (r = rot_dim / 2).
struct Lane {
  int g0, g1, pair;
  bool rotate, paired;
};
__device__ __forceinline__ Lane lane_of(int c, int r, bool paired) {
  Lane l;
  l.pair = 4 * c;
  l.rotate = 4 * c < r;
  l.paired = paired;
  if (paired || !l.rotate) {
    // pairs side by side; and the channels behind the rotated ones, 8 a lane
    l.g0 = 8 * c;
    l.g1 = 8 * c + 4;
  } else {
    l.g0 = 4 * c;
    l.g1 = r + 4 * c;
  }
  return l;
}

// x1 c - x2 s (or x1 c + x2 s with s negated) rounded to odd: exact products as two fp32
// numbers each, their sum as one and what it leaves.  Correct unless the low parts'
// own sum, 2^-48 of the products, decides.
__device__ __forceinline__ float rotate_odd(float x1, float c, float x2, float s) {
  const float p = __fmul_rn(x1, c), q = __fmul_rn(x2, s);
  const float ep = __fmaf_rn(x1, c, -p), eq = __fmaf_rn(x2, s, -q);
  const float d = __fsub_rn(p, q);
  const float t = __fsub_rn(d, p);
  const float ed = __fsub_rn(__fsub_rn(p, __fsub_rn(d, t)), __fadd_rn(q, t));
  const float low = __fadd_rn(ed, __fsub_rn(ep, eq));
  const float y = __fadd_rn(d, low);
  const float rest = __fadd_rn(__fsub_rn(d, y), low);  // exact: |low| <= |d| or both small
  // towards zero, then odd where anything is left
  uint32_t u = __float_as_uint(y);
  if (rest != 0.0f) {
    if ((rest < 0.0f) != (y < 0.0f)) --u;
    u |= 1u;
  }
  return __uint_as_float(u);
}

struct Angles {
  float4 c, s;
};
__device__ __forceinline__ Angles angles_of(const kvq_block8_append_params& p, const Lane& l,
                                            int pos) {
  Angles a;
  const long long at = (long long)pos * (p.rot_dim >> 1) + l.pair;
  a.c = __ldg(reinterpret_cast<const float4*>(p.cos + at));
  a.s = __ldg(reinterpret_cast<const float4*>(p.sin + at));
  return a;
}

// The table row of a token: its position, or its entry of `positions`.
__device__ __forceinline__ int table_row(const AppendCall& call, int row, int pos) {
  int at = call.p.positions ? __ldg(call.p.positions + row) : pos;
  if (at < 0 || at >= call.p.n_positions) {
    set_flag(call.cache, KVQ_FLAG_BAD_BATCH);
    at = at < 0 ? 0 : call.p.n_positions - 1;
  }
  return at;
}

template <bool BF16, bool KEY>
__device__ __forceinline__ void rotate(uint2& a, uint2& b, const Lane& l, const Angles& t) {
  const float2 a0 = widen<BF16>(a.x), a1 = widen<BF16>(a.y);
  const float2 b0 = widen<BF16>(b.x), b1 = widen<BF16>(b.y);
  float x1[4], x2[4];
  if (l.paired) {
    x1[0] = a0.x, x2[0] = a0.y, x1[1] = a1.x, x2[1] = a1.y;
    x1[2] = b0.x, x2[2] = b0.y, x1[3] = b1.x, x2[3] = b1.y;
  } else {
    x1[0] = a0.x, x1[1] = a0.y, x1[2] = a1.x, x1[3] = a1.y;
    x2[0] = b0.x, x2[1] = b0.y, x2[2] = b1.x, x2[3] = b1.y;
  }
  const float c[4] = {t.c.x, t.c.y, t.c.z, t.c.w}, s[4] = {t.s.x, t.s.y, t.s.z, t.s.w};
  float y1[4], y2[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (KEY) {
      y1[i] = rotate_odd(x1[i], c[i], x2[i], s[i]);
      y2[i] = rotate_odd(x2[i], c[i], x1[i], -s[i]);
    } else {
      y1[i] = x1[i] * c[i] - x2[i] * s[i];
      y2[i] = x2[i] * c[i] + x1[i] * s[i];
    }
  }
  if (l.paired) {
    a = make_uint2(narrow<BF16>(y1[0], y2[0]), narrow<BF16>(y1[1], y2[1]));
    b = make_uint2(narrow<BF16>(y1[2], y2[2]), narrow<BF16>(y1[3], y2[3]));
  } else {
    a = make_uint2(narrow<BF16>(y1[0], y1[1]), narrow<BF16>(y1[2], y1[3]));
    b = make_uint2(narrow<BF16>(y2[0], y2[1]), narrow<BF16>(y2[2], y2[3]));
  }
}

// Magnitudes of 16-bit floats compare as integers; a NaN stands above infinity.
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
  return __vmaxu2(a, b & 0x7fff7fffu);
}

template <bool BF16>
__device__ __forceinline__ uint32_t codes_of(uint2 v, float scale) {
  const float2 x = widen<BF16>(v.x), y = widen<BF16>(v.y);
  const __nv_fp8x2_storage_t a = __nv_cvt_float2_to_fp8x2(
      make_float2(__fdiv_rn(x.x, scale), __fdiv_rn(x.y, scale)), __NV_SATFINITE, __NV_E4M3);
  const __nv_fp8x2_storage_t b = __nv_cvt_float2_to_fp8x2(
      make_float2(__fdiv_rn(y.x, scale), __fdiv_rn(y.y, scale)), __NV_SATFINITE, __NV_E4M3);
  return (uint32_t)a | ((uint32_t)b << 16);
}

// Block `blk` of a sequence: keys (KEY) or values of kv-head h.
template <bool BF16, bool KEY>
__device__ __forceinline__ void block_task(const AppendCall& call, const Seq& s, int b, int blk,
                                           int h) {
  const int lane = threadIdx.x & 31, c = lane & 15, half = lane >> 4;
  const Lane l = lane_of(c, KEY ? call.p.rot_dim >> 1 : 0, KEY && call.p.paired);
  const int before = s.L - s.n, t0 = blk * kGroup;
  const bool whole = t0 + kGroup <= s.L;
  const uint16_t* src = KEY ? call.p.k : call.p.v;
  const int64_t* stride = KEY ? call.p.k_stride : call.p.v_stride;
  uint16_t* ring = (KEY ? call.cache.k_ring : call.cache.v_ring) +
                   ((long long)b * call.d.hkv + h) * (kRing * kHeadDim);
  const bool keep = blk >= s.L / kGroup - 1;  // the block's new tokens go to the ring
  src += h * stride[1];
  uint2 x[16][2];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int pos = t0 + 2 * i + half;
    x[i][0] = x[i][1] = make_uint2(0u, 0u);
    if (pos < before) {
      if (whole) {
        const uint16_t* r = ring + (pos & (kRing - 1)) * kHeadDim;
        x[i][0] = ld8_ring(r + l.g0);
        x[i][1] = ld8_ring(r + l.g1);
      }
    } else if (pos < s.L) {
      const uint16_t* r = src + (long long)(s.row + pos - before) * stride[0];
      x[i][0] = ld8(r + l.g0);
      x[i][1] = ld8(r + l.g1);
    }
  }
  if constexpr (KEY) {
    if (l.rotate) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int pos = t0 + 2 * i + half;
        if (pos >= before && pos < s.L)
          rotate<BF16, true>(x[i][0], x[i][1], l,
                             angles_of(call.p, l, table_row(call, s.row + pos - before, pos)));
      }
    }
  }
  if (keep) {
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int pos = t0 + 2 * i + half;
      if (pos >= before && pos < s.L) {
        uint16_t* r = ring + (pos & (kRing - 1)) * kHeadDim;
        st8(r + l.g0, x[i][0]);
        st8(r + l.g1, x[i][1]);
      }
    }
  }
  if (!whole) return;
  const int page = __ldg(call.cache.block_table + (long long)b * call.d.max_blocks + blk);
  if ((unsigned)page >= (unsigned)call.cache.n_pages) {
    if (lane == 0) set_flag(call.cache, KVQ_FLAG_BAD_PAGE);
    return;
  }
  uint32_t m = 0u;
#pragma unroll
  for (int i = 0; i < 16; ++i)
    m = larger(larger(m, x[i][0].x), larger(larger(x[i][0].y & 0x7fff7fffu, x[i][1].x), x[i][1].y));
  m = max(m & 0xffffu, m >> 16);
#pragma unroll
  for (int o = 16; o; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
  const float amax = widen<BF16>(m).x;
  const float scale =
      m ? fminf(fmaxf(__fdiv_rn(amax, kMaxCode), 0x1p-60f), 0x1p60f) : 1.0f;
  const long long at = (long long)page * call.d.hkv + h;
  if (lane == 0) call.cache.scales[2 * at + (KEY ? 0 : 1)] = scale;
  uint8_t* codes = (KEY ? call.cache.k_codes : call.cache.v_codes) + at * (kGroup * kHeadDim);
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    uint8_t* r = codes + (2 * i + half) * kHeadDim;
    *reinterpret_cast<uint32_t*>(r + l.g0) = codes_of<BF16>(x[i][0], scale);
    *reinterpret_cast<uint32_t*>(r + l.g1) = codes_of<BF16>(x[i][1], scale);
  }
}

// Blocks that hold new tokens of a sequence.
__device__ __forceinline__ int blocks_of(const Seq& s) {
  return s.n > 0 ? (s.L - 1) / kGroup - (s.L - s.n) / kGroup + 1 : 0;
}
// A sequence as appending takes it: the new tokens are among its tokens.
__device__ __forceinline__ Seq append_seq(const AppendCall& call, int b) {
  Seq s{0, 0, 0, 0};
  if (b < call.d.batch) s = seq_of(call.d, call.batch, b);
  if (s.n > s.L) s.n = 0, s.bad |= KVQ_FLAG_BAD_BATCH;
  return s;
}

// A warp looks through the batch 128 sequences at a time, four neighbours a lane: the
// loads of a step are on their way together.
constexpr int kPerLane = 4;

template <bool BF16>
__device__ __forceinline__ void kv_task(const AppendCall& call, int unit, int part) {
  const int lane = threadIdx.x & 31;
#pragma unroll 1
  for (int b0 = 0; b0 < call.d.batch; b0 += 32 * kPerLane) {
    Seq s[kPerLane];
    int mine = 0;
#pragma unroll
    for (int k = 0; k < kPerLane; ++k) {
      s[k] = append_seq(call, b0 + kPerLane * lane + k);
      mine += blocks_of(s[k]);
    }
    int inc = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += y;
    }
    const int all = __shfl_sync(0xffffffffu, inc, 31);
    if (unit >= all) {
      unit -= all;
      continue;
    }
    const int at = __ffs(__ballot_sync(0xffffffffu, inc > unit)) - 1;
    // the lane that has the unit picks its sequence
    int left = unit - (inc - mine), k = 0;
    Seq q = s[0];
#pragma unroll
    for (int i = 0; i < kPerLane - 1; ++i)
      if (k == i && left >= blocks_of(s[i])) {
        left -= blocks_of(s[i]);
        q = s[i + 1];
        k = i + 1;
      }
    q.row = __shfl_sync(0xffffffffu, q.row, at);
    q.n = __shfl_sync(0xffffffffu, q.n, at);
    q.L = __shfl_sync(0xffffffffu, q.L, at);
    const int b = b0 + kPerLane * at + __shfl_sync(0xffffffffu, k, at);
    const int before = q.L - q.n, first = before / kGroup, done = q.L / kGroup;
    int blk = first + __shfl_sync(0xffffffffu, left, at);
    // the block whose ring slots hold the first rows of a begun block that is completed
    int heir = done - ((done - first) & 1);
    if (before % kGroup == 0 || heir <= first || heir * kGroup >= q.L) heir = -1;
    if (blk == heir) return;
    for (;;) {
      if (part & 1) block_task<BF16, false>(call, q, b, blk, part >> 1);
      else block_task<BF16, true>(call, q, b, blk, part >> 1);
      if (blk != first || heir < 0) return;
      __syncwarp();
      blk = heir;
      heir = -1;
    }
  }
}

// Queries of token `row`, heads h0 .. h0 + 7.
template <bool BF16>
__device__ __forceinline__ void query_task(const AppendCall& call, int row, int h0) {
  const int lane = threadIdx.x & 31, half = lane >> 4;
  int pos = -1;
#pragma unroll 1
  for (int b0 = 0; b0 < call.d.batch; b0 += 32 * kPerLane) {
    int mine = -1;
#pragma unroll
    for (int k = 0; k < kPerLane; ++k) {
      const Seq s = append_seq(call, b0 + kPerLane * lane + k);
      if (mine < 0 && row >= s.row && row < s.row + s.n) mine = s.L - s.n + row - s.row;
    }
    const unsigned who = __ballot_sync(0xffffffffu, mine >= 0);
    if (who) {
      pos = __shfl_sync(0xffffffffu, mine, __ffs(who) - 1);
      break;
    }
  }
  if (pos < 0) return;
  const Lane l = lane_of(lane & 15, call.p.rot_dim >> 1, call.p.paired);
  const uint16_t* src = call.p.q + row * call.p.q_stride[0];
  uint16_t* dst = call.p.q_out + row * call.p.q_out_stride[0];
  uint2 x[kQueryHeads / 2][2];
#pragma unroll
  for (int i = 0; i < kQueryHeads / 2; ++i) {
    const int h = h0 + 2 * i + half;
    if (h < call.d.hq) {
      // (in place: no read-only path)
      const uint16_t* r = src + h * call.p.q_stride[1];
      x[i][0] = *reinterpret_cast<const uint2*>(r + l.g0);
      x[i][1] = *reinterpret_cast<const uint2*>(r + l.g1);
    }
  }
  if (l.rotate) {
    const Angles t = angles_of(call.p, l, table_row(call, row, pos));
#pragma unroll
    for (int i = 0; i < kQueryHeads / 2; ++i) rotate<BF16, false>(x[i][0], x[i][1], l, t);
  }
#pragma unroll
  for (int i = 0; i < kQueryHeads / 2; ++i) {
    const int h = h0 + 2 * i + half;
    if (h < call.d.hq) {
      uint16_t* r = dst + h * call.p.q_out_stride[1];
      st8(r + l.g0, x[i][0]);
      st8(r + l.g1, x[i][1]);
    }
  }
}

// Tasks of blocks, then of queries, a warp each; the last CTA looks over the batch's
// sizes for the flag word.
template <bool BF16>
__global__ void __launch_bounds__(32 * kWarps)
append_kernel(const __grid_constant__ AppendCall call, int kv_ctas, int groups) {
  const int warp = threadIdx.x >> 5;
  if (blockIdx.x == gridDim.x - 1) {
    for (int b = threadIdx.x; b < call.d.batch; b += 32 * kWarps) {
      const Seq s = append_seq(call, b);
      if (s.bad) set_flag(call.cache, s.bad);
    }
  } else if ((int)blockIdx.x < kv_ctas) {
    const int task = blockIdx.x * kWarps + warp, parts = 2 * call.d.hkv;
    kv_task<BF16>(call, task / parts, task % parts);
  } else {
    const int task = ((int)blockIdx.x - kv_ctas) * kWarps + warp;
    const int row = task / groups;
    if (row < call.batch.n_tokens) query_task<BF16>(call, row, (task - row * groups) * kQueryHeads);
  }
}

}  // namespace

cudaError_t launch_append(const AppendCall& call, cudaStream_t stream) {
  // A sequence of n new tokens touches at most (n - 1) / 32 + 2 blocks.
  const long long tokens = call.batch.n_tokens;
  const long long seqs = tokens < call.d.batch ? tokens : call.d.batch;
  const long long units = tokens / kGroup + 2 * seqs;
  const int kv_ctas = (int)((units * 2 * call.d.hkv + kWarps - 1) / kWarps);
  const int groups = (call.d.hq + kQueryHeads - 1) / kQueryHeads;
  const int q_ctas = call.p.q ? (int)((tokens * groups + kWarps - 1) / kWarps) : 0;
  const int grid = kv_ctas + q_ctas + 1;
  if (call.d.bf16) append_kernel<true><<<grid, 32 * kWarps, 0, stream>>>(call, kv_ctas, groups);
  else append_kernel<false><<<grid, 32 * kWarps, 0, stream>>>(call, kv_ctas, groups);
  return cudaGetLastError();
}

}  // namespace block8
}  // namespace kvq
