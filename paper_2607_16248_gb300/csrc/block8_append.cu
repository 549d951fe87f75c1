// kvq_block8_append: rotation of queries and keys, the rings, and the codes of the
// blocks that the new tokens complete, in one launch.
//
// A CTA of four warps takes one block's keys or values of one kv-head (32 x 128 elements in
// its registers: the block's largest magnitude is known before the first code), or a warp
// each takes one token's queries of eight heads.  16 lanes share a row of 128 channels; a
// lane holds two groups of four channels such that it has both channels of its four rotated
// pairs (`Lane`), so a rotation needs no exchange and each cosine is read once.
//
// The codes need the keys' exact roundings: a key next to a border of its type changes
// its block's scale, and a quotient next to a border its code.  Products and sums
// therefore keep their low parts (two fp32 numbers), and the first rounding goes to odd,
// so that the second, to 16 bits, is the only one.
//
// What bounds it.  32 tokens and a prompt of 8191 (32 heads over 8, fp16): 49 us, 3.9 TB/s;
// the queries alone take 17, the blocks alone 33: 1000 instructions a warp for a quarter of
// a block's keys (rotation with its two roundings, quotients with their borders), 58% of the
// issue slots.  With the seldom ways in their places the code passed the instruction
// cache: 62 us.  Keys and values of a head by one CTA, or five or ten CTAs an SM instead of
// eight: the same time.  One token: 5.6 us, launch and three dependent loads.
//
// A block that was begun by an earlier call has its first rows in the ring, in slots that
// this call's newest tokens may take.  Of the two blocks whose tokens go to the ring, the
// one with the same slots (an even number of blocks behind) is done by the same CTA,
// after the begun block's rows are in its registers.
#include "block8.cuh"

#include <cuda_fp8.h>

#include <algorithm>

namespace kvq {
namespace block8 {

namespace {

constexpr int kWarps = 4;
constexpr int kPlaces = 8;      // CTAs an SM
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
  bool rotate;
};
__device__ __forceinline__ Lane lane_of(int c, int r, bool paired) {
  Lane l;
  l.pair = 4 * c;
  l.rotate = 4 * c < r;
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
__device__ __noinline__ float rotate_odd(float x1, float c, float x2, float s) {
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

// Two neighbouring results of a type's word, y = x1 c - x2 s each.  Keys: rounded as if
// nothing had been rounded before.  The quick sum is within 2^-23 (|x1 c| + |x2 s|) of the
// exact one, so where both ends of that range round alike, so does the exact sum; the
// others (one fp16 number in 20) take the long way.
template <bool BF16, bool KEY>
__device__ __forceinline__ uint32_t rotate2(float x1, float c1, float x2, float s1, float w1,
                                            float c2, float w2, float s2) {
  const float p = x1 * c1, q = x2 * s1, u = w1 * c2, v = w2 * s2;
  const float y = p - q, z = u - v;
  if constexpr (!KEY) return narrow<BF16>(y, z);
  constexpr float kRange = 1.25f * 0x1p-23f;
  const float dy = (fabsf(p) + fabsf(q)) * kRange, dz = (fabsf(u) + fabsf(v)) * kRange;
  const uint32_t lo = narrow<BF16>(y - dy, z - dz), hi = narrow<BF16>(y + dy, z + dz);
  if (lo == hi) return lo;
  return narrow<BF16>(rotate_odd(x1, c1, x2, s1), rotate_odd(w1, c2, w2, s2));
}

template <bool BF16, bool KEY, bool PAIRED>
__device__ __forceinline__ void rotate(uint2& a, uint2& b, const Lane& l, const Angles& t) {
  const float2 a0 = widen<BF16>(a.x), a1 = widen<BF16>(a.y);
  const float2 b0 = widen<BF16>(b.x), b1 = widen<BF16>(b.y);
  if constexpr (PAIRED) {
    a.x = rotate2<BF16, KEY>(a0.x, t.c.x, a0.y, t.s.x, a0.y, t.c.x, a0.x, -t.s.x);
    a.y = rotate2<BF16, KEY>(a1.x, t.c.y, a1.y, t.s.y, a1.y, t.c.y, a1.x, -t.s.y);
    b.x = rotate2<BF16, KEY>(b0.x, t.c.z, b0.y, t.s.z, b0.y, t.c.z, b0.x, -t.s.z);
    b.y = rotate2<BF16, KEY>(b1.x, t.c.w, b1.y, t.s.w, b1.y, t.c.w, b1.x, -t.s.w);
  } else {
    a.x = rotate2<BF16, KEY>(a0.x, t.c.x, b0.x, t.s.x, a0.y, t.c.y, b0.y, t.s.y);
    a.y = rotate2<BF16, KEY>(a1.x, t.c.z, b1.x, t.s.z, a1.y, t.c.w, b1.y, t.s.w);
    b.x = rotate2<BF16, KEY>(b0.x, t.c.x, a0.x, -t.s.x, b0.y, t.c.y, a0.y, -t.s.y);
    b.y = rotate2<BF16, KEY>(b1.x, t.c.z, a1.x, -t.s.z, b1.y, t.c.w, a1.y, -t.s.w);
  }
}

// Magnitudes of 16-bit floats compare as integers; a NaN stands above infinity.
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
  return __vmaxu2(a, b & 0x7fff7fffu);
}

// Four codes.  A product with 1 / scale is within 2^-22 of the quotient; where it is not
// that near to a border of the codes (bits 0 .. 19 of the fp32 number at their middle, as
// long as the code is a normal number), it rounds as the quotient does.
__device__ __forceinline__ bool in_doubt(float q) {
  return ((__float_as_uint(q) & 0xfffffu) - 0x7fff8u) <= 16u || fabsf(q) < 0x1p-6f;
}
// Below 2^-6 codes are the multiples of 2^-9.
__device__ __forceinline__ bool near_border(float q) {
  const float t = fabsf(q) * 512.0f;
  if (t >= 8.0f) return ((__float_as_uint(q) & 0xfffffu) - 0x7fff8u) <= 16u;
  return fabsf(t - rintf(t)) > 0.5f - 0x1p-17f;
}
__device__ __forceinline__ uint32_t to_codes(float x, float y, float z, float w) {
  const __nv_fp8x2_storage_t a =
      __nv_cvt_float2_to_fp8x2(make_float2(x, y), __NV_SATFINITE, __NV_E4M3);
  const __nv_fp8x2_storage_t b =
      __nv_cvt_float2_to_fp8x2(make_float2(z, w), __NV_SATFINITE, __NV_E4M3);
  return (uint32_t)a | ((uint32_t)b << 16);
}
__device__ __noinline__ uint32_t careful_codes(float x, float y, float z, float w, float scale,
                                               float inv) {
  const float a = x * inv, b = y * inv, c = z * inv, d = w * inv;
  if (near_border(a) || near_border(b) || near_border(c) || near_border(d))
    return to_codes(__fdiv_rn(x, scale), __fdiv_rn(y, scale), __fdiv_rn(z, scale),
                    __fdiv_rn(w, scale));
  return to_codes(a, b, c, d);
}
template <bool BF16>
__device__ __forceinline__ uint32_t codes_of(uint2 v, float scale, float inv) {
  const float2 x = widen<BF16>(v.x), y = widen<BF16>(v.y);
  const float a = x.x * inv, b = x.y * inv, c = y.x * inv, d = y.y * inv;
  if (in_doubt(a) || in_doubt(b) || in_doubt(c) || in_doubt(d))
    return careful_codes(x.x, x.y, y.x, y.y, scale, inv);
  return to_codes(a, b, c, d);
}

// Keys (KEY) or values of kv-head h of a sequence.
template <bool BF16, bool KEY, bool PAIRED>
struct Task {
  const AppendCall& call;
  const Seq& s;
  int b, h, before;
  Lane l;
  const uint16_t* src;
  uint16_t* ring;
  __device__ __forceinline__ Task(const AppendCall& call, const Seq& s, int b, int h)
      : call(call), s(s), b(b), h(h), before(s.L - s.n) {
    l = lane_of(threadIdx.x & 15, KEY ? call.p.rot_dim >> 1 : 0, KEY && call.p.paired);
    src = (KEY ? call.p.k : call.p.v) + h * (KEY ? call.p.k_stride : call.p.v_stride)[1];
    ring = (KEY ? call.cache.k_ring : call.cache.v_ring) +
           ((long long)b * call.d.hkv + h) * (kRing * kHeadDim);
  }
  __device__ __forceinline__ const uint16_t* new_row(int pos) const {
    return src + (long long)(s.row + pos - before) * (KEY ? call.p.k_stride : call.p.v_stride)[0];
  }
  __device__ __forceinline__ uint16_t* ring_row(int pos) const {
    return ring + (pos & (kRing - 1)) * kHeadDim;
  }
  // N rows from pos on, every second one: rotated if they are new.
  template <int N>
  __device__ __forceinline__ void turn(uint2 (&x)[N][2], int pos) const {
    if constexpr (KEY) {
      if (!l.rotate) return;
      Angles t[N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int at = pos + 2 * i;
        const bool fresh = at >= before && at < s.L;
        t[i] = angles_of(call.p, l, fresh ? table_row(call, s.row + at - before, at) : 0);
      }
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int at = pos + 2 * i;
        if (at >= before && at < s.L) rotate<BF16, true, PAIRED>(x[i][0], x[i][1], l, t[i]);
      }
    }
  }

  // New tokens of a block that stays open: to the ring.
  __device__ __forceinline__ void open_block(int blk) const {
#pragma unroll 1
    for (int pos = max(blk * kGroup, before) + (threadIdx.x >> 4); pos < s.L;
         pos += 2 * kWarps) {
      uint2 x[1][2];
      x[0][0] = ld8(new_row(pos) + l.g0);
      x[0][1] = ld8(new_row(pos) + l.g1);
      turn<1>(x, pos);
      st8(ring_row(pos) + l.g0, x[0][0]);
      st8(ring_row(pos) + l.g1, x[0][1]);
    }
  }

  // A block that is whole now: codes, and the ring if it is among the last two.
  __device__ __forceinline__ void whole_block(int blk, uint32_t* share) const {
    constexpr int N = kGroup / (2 * kWarps);  // rows of a lane
    const int warp = threadIdx.x >> 5, r0 = 2 * N * warp + ((threadIdx.x >> 4) & 1);
    const int t0 = blk * kGroup + r0;
    const int page = __ldg(call.cache.block_table + (long long)b * call.d.max_blocks + blk);
    uint2 x[N][2];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int pos = t0 + 2 * i;
      const uint16_t* r = pos < before ? ring_row(pos) : new_row(pos);
      x[i][0] = ld8_ring(r + l.g0);
      x[i][1] = ld8_ring(r + l.g1);
    }
    turn<N>(x, t0);
    uint32_t m = 0u;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int k = 0; k < 2; ++k) m = larger(larger(m, x[i][k].x), x[i][k].y);
    m = __reduce_max_sync(0xffffffffu, max(m & 0xffffu, m >> 16));
    if ((threadIdx.x & 31) == 0) share[warp] = m;
    __syncthreads();  // and every row of the ring has been read
#pragma unroll
    for (int w = 0; w < kWarps; ++w) m = max(m, share[w]);
    if (blk >= s.L / kGroup - 1) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int pos = t0 + 2 * i;
        if (pos >= before) {
          st8(ring_row(pos) + l.g0, x[i][0]);
          st8(ring_row(pos) + l.g1, x[i][1]);
        }
      }
    }
    if ((unsigned)page >= (unsigned)call.cache.n_pages) {
      if (threadIdx.x == 0) set_flag(call.cache, KVQ_FLAG_BAD_PAGE);
      return;
    }
    const float amax = widen<BF16>(m).x;
    const float scale = m ? fminf(fmaxf(__fdiv_rn(amax, kMaxCode), 0x1p-60f), 0x1p60f) : 1.0f;
    const float inv = __frcp_rn(scale);
    const long long at = (long long)page * call.d.hkv + h;
    if (threadIdx.x == 0) call.cache.scales[2 * at + (KEY ? 0 : 1)] = scale;
    uint8_t* codes = (KEY ? call.cache.k_codes : call.cache.v_codes) + at * (kGroup * kHeadDim);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      uint8_t* r = codes + (r0 + 2 * i) * kHeadDim;
      *reinterpret_cast<uint32_t*>(r + l.g0) = codes_of<BF16>(x[i][0], scale, inv);
      *reinterpret_cast<uint32_t*>(r + l.g1) = codes_of<BF16>(x[i][1], scale, inv);
    }
  }

  __device__ __forceinline__ void block(int blk, uint32_t* share) const {
    if (blk * kGroup + kGroup <= s.L) whole_block(blk, share);
    else open_block(blk);
  }
};

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

// What a CTA's warps tell one another.
struct Share {
  uint32_t m[kWarps];
  int sum[kWarps];
  Seq s;
  int b, left;
};

// Parts `part` .. end - 1 (2 h: keys of kv-head h, 2 h + 1: its values) of unit `unit` of
// `units` (the batch's blocks with new tokens, in order).  The warps look through 32 sequences
// each.  Where ranges overlap there may be more blocks than units: a sequence that does not
// fit is left alone whole.
template <bool BF16, bool PAIRED>
__device__ __forceinline__ void kv_task(const AppendCall& call, int unit, int units, int part,
                                        int end, Share& sh) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, place = unit;
#pragma unroll 1
  for (int b0 = 0; b0 < call.d.batch; b0 += 32 * kWarps) {
    const int b = b0 + 32 * warp + lane;
    const Seq s = append_seq(call, b);
    const int mine = blocks_of(s);
    int inc = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += y;
    }
    if (lane == 31) sh.sum[warp] = inc;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      if (w == warp) before = all;
      all += sh.sum[w];
    }
    if (unit >= all) {
      unit -= all;
      __syncthreads();
      continue;
    }
    const int left = unit - before - (inc - mine);
    if (left >= 0 && left < mine) {
      sh.s = s;
      sh.b = b;
      sh.left = left;
    }
    __syncthreads();
    const Seq q = sh.s;
    const int old = q.L - q.n, first = old / kGroup, done = q.L / kGroup;
    if (place - sh.left + blocks_of(q) > units) return;
    int blk = first + sh.left;
    // the block whose ring slots hold the first rows of a begun block that is completed
    int heir = done - ((done - first) & 1);
    if (old % kGroup == 0 || heir <= first || heir * kGroup >= q.L) heir = -1;
    if (blk == heir) return;
    const int seq = sh.b;
#pragma unroll 1
    for (; part < end; ++part) {
#pragma unroll 1
      for (int at = blk;;) {
        if (part & 1) Task<BF16, false, PAIRED>(call, q, seq, part >> 1).block(at, sh.m);
        else Task<BF16, true, PAIRED>(call, q, seq, part >> 1).block(at, sh.m);
        if (at != first || heir < 0) break;
        __syncthreads();  // sh.m is written again
        at = heir;
      }
      if (part + 1 < end) __syncthreads();
    }
    return;
  }
}

// The first sequence that takes token `row`, for a warp: one whose range holds it, that is
// appended and whose blocks fit (kv_task).  Where a start is out of order; n is 0 for none.
__device__ __forceinline__ Seq taker_of(const AppendCall& call, int units, int row) {
  const int lane = threadIdx.x & 31;
  long long blocks = 0;
#pragma unroll 1
  for (int b0 = 0; b0 < call.d.batch; b0 += 32) {
    const Seq s = append_seq(call, b0 + lane);
    long long until = blocks_of(s);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, until, o);
      if (lane >= o) until += y;
    }
    until += blocks;
    const unsigned who = __ballot_sync(
        0xffffffffu, s.n > 0 && row >= s.row && row < s.row + s.n && until <= units);
    if (who) return append_seq(call, b0 + __ffs(who) - 1);
    blocks = __shfl_sync(0xffffffffu, until, 31);
  }
  return Seq{0, 0, 0, 0};
}

// Queries of token `row`, heads h0 .. h0 + 7.
template <bool BF16, bool PAIRED>
__device__ __forceinline__ void query_task(const AppendCall& call, int units, int row, int h0) {
  const int lane = threadIdx.x & 31, half = lane >> 4;
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
  int b = -1;
  bool down = false;  // a start is out of order
  if (!call.batch.starts) {
    b = row / call.batch.max_new;
  } else {
#pragma unroll 1
    for (int b0 = 0; b0 < call.d.batch; b0 += 32) {
      const int i = b0 + lane;
      bool mine = false;
      if (i < call.d.batch) {
        const int begin = __ldg(call.batch.starts + i), end = __ldg(call.batch.starts + i + 1);
        mine = row >= begin && row < end;
        down |= end < begin;
      }
      const unsigned who = __ballot_sync(0xffffffffu, mine);
      if (who) {
        b = b0 + __ffs(who) - 1;
        break;
      }
    }
    if (b < 0) return;
  }
  Seq s = append_seq(call, b);
  if (call.batch.starts && (s.n == 0 || __any_sync(0xffffffffu, down)))
    s = taker_of(call, units, row);
  if (s.n == 0) return;
  const int pos = s.L - s.n + row - s.row;
  if (l.rotate) {
    const Angles t = angles_of(call.p, l, table_row(call, row, pos));
#pragma unroll
    for (int i = 0; i < kQueryHeads / 2; ++i) rotate<BF16, false, PAIRED>(x[i][0], x[i][1], l, t);
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

// CTAs of blocks, then of queries; the last CTA looks over the batch's sizes for the flag
// word.
template <bool BF16, bool PAIRED>
__global__ void __launch_bounds__(32 * kWarps, kPlaces)
append_kernel(const __grid_constant__ AppendCall call, int units, int kv_ctas, int parts,
              int groups) {
  __shared__ Share share;
  if (blockIdx.x == gridDim.x - 1) {
    for (int b = threadIdx.x; b < call.d.batch; b += 32 * kWarps) {
      const Seq s = append_seq(call, b);
      if (s.bad) set_flag(call.cache, s.bad);
    }
  } else if ((int)blockIdx.x < kv_ctas) {
    const int all = 2 * call.d.hkv, shares = (all + parts - 1) / parts;
    const int unit = (int)blockIdx.x / shares, part = ((int)blockIdx.x - unit * shares) * parts;
    kv_task<BF16, PAIRED>(call, unit, units, part, min(part + parts, all), share);
  } else {
    const int task = ((int)blockIdx.x - kv_ctas) * kWarps + ((int)threadIdx.x >> 5);
    const int row = task / groups;
    if (row < call.batch.n_tokens)
      query_task<BF16, PAIRED>(call, units, row, (task - row * groups) * kQueryHeads);
  }
}

}  // namespace

cudaError_t launch_append(const AppendCall& call, int sm_count, cudaStream_t stream) {
  // A sequence of n new tokens touches at most (n + 30) / 32 + 1 blocks (no two the same rows,
  // unless a start is out of order).
  const long long tokens = call.batch.n_tokens;
  const long long seqs = tokens < call.d.batch ? tokens : call.d.batch;
  const long long units = std::min(tokens / kGroup + 2 * seqs,
                                   seqs * ((call.batch.max_new + 30LL) / kGroup + 1));
  // One part a CTA, or as many as leave four CTAs for each place on the GPU: a large batch's
  // CTAs look for their sequences longer than they take for a part (8192 single tokens of 8
  // kv-heads: 0.51 ms, 4.8 with a part each; 1024: 37 us and 103).
  const int all = 2 * call.d.hkv;
  const int parts =
      (int)std::max(1LL, std::min<long long>(all, units * all / (4LL * kPlaces * sm_count)));
  const int kv_ctas = (int)(units * ((all + parts - 1) / parts));
  const int groups = (call.d.hq + kQueryHeads - 1) / kQueryHeads;
  const int q_ctas = call.p.q ? (int)((tokens * groups + kWarps - 1) / kWarps) : 0;
  const int grid = kv_ctas + q_ctas + 1;
  const auto kernel = call.d.bf16
                          ? (call.p.paired ? append_kernel<true, true> : append_kernel<true, false>)
                          : (call.p.paired ? append_kernel<false, true>
                                           : append_kernel<false, false>);
  kernel<<<grid, 32 * kWarps, 0, stream>>>(call, (int)units, kv_ctas, parts, groups);
  return cudaGetLastError();
}

}  // namespace block8
}  // namespace kvq
