// kvq_block8_attn for many rows a kv-head (prompt chunks) on the 5th-generation tensor cores.
//
// A CTA and its roles, the two alternating streams and the order of products are those of
// chunk_core.cuh: per step (128 query rows, half a tile of 128 tokens) S = Q K^T with fp16
// operands in shared memory and fp32 in tensor memory, softmax by the four warps that own the
// rows of S, weights as fp16 over the same columns, O += W V with W from tensor memory.
//   warps 0-3, 4-7  softmax of streams 0 and 1, queries in, results out
//   warps 8-11      keys: a block of 32 tokens each, codes -> fp16 tile
//   warps 12-15     values, the same
//   warps 16, 17    issue the products of streams 0 and 1 (18, 19 idle)
// What differs: codes are exact in fp16, and both tiles take them in the order in which the
// pages hold them (tokens as rows, channels contiguous: the contraction of the scores, the
// columns of the results), so a lane's 16 codes become 32 neighbouring bytes.  A block's
// scales reach the softmax instead: scores times s_k in the exponent's factor, weights times
// s_v as 2^(x + log2 s_v) with the running maximum taken of that, and the sum of the
// softmax as that of w / s_v (block8_rows.cu has the same).  bf16 queries go to fp16 times a
// power of two, and so do the rows of the open block, keys and values of both types, each
// times its own: what one row holds, seen or not, does not touch the others.
//
// What bounds it.  Two prompts of 8191 tokens (32 heads over 8): 1.08 ms, 1.02 PFLOP/s of a
// cuBLAS product's 1.92 (bf16: 1.24).  When it took 1.04, it was 0.96 without the exponentials
// and 0.93 without the conversion of codes: softmax and loading warps share the issue slots,
// and the chain of a step (scores, softmax, weights, product) is not hidden whole by the other
// stream's.  The ordinary step's code has to stay in one piece: with the open block's in its
// midst 1.17 ms, with that of large scores too 1.27.
#include "block8_plan.cuh"
#include "chunk_core.cuh"

#include <type_traits>

namespace kvq {
namespace block8 {

namespace {

using chunk::add2;
using chunk::bar_arrive;
using chunk::bar_init;
using chunk::bar_try;
using chunk::elect_lane;
using chunk::fence_async;
using chunk::fma2;
using chunk::instr_desc;
using chunk::kColO;
using chunk::kColS;
using chunk::kHalfBytes;
using chunk::kIssueWarp;
using chunk::kLiftLog2;
using chunk::kLoadWarps;
using chunk::kRegsIssue;
using chunk::kRegsLaunch;
using chunk::kRescaleLog2;
using chunk::kSoftmaxWarps;
using chunk::kStep;
using chunk::kThreads;
using chunk::kTile;
using chunk::kTileBytes;
using chunk::kWaitLimit;
using chunk::mma_ss;
using chunk::mma_ts;
using chunk::pair;
using chunk::put_rows;
using chunk::rescale_row;
using chunk::sptr;
using chunk::st16;
using chunk::stage_row;
using chunk::step_major_k;
using chunk::step_major_mn;
using chunk::tc_after;
using chunk::tc_before;
using chunk::tc_commit;
using chunk::tile_at;
using chunk::tile_desc;
using chunk::tm_load32;
using chunk::tm_load8;
using chunk::tm_load_wait;
using chunk::tm_store16;
using chunk::tm_store32;
using chunk::tm_store8;
using chunk::tm_store_wait;
using chunk::unpair;
using chunk::warp_arrive;

constexpr int kTok = 7;       // tiles of 128 tokens
constexpr int kItemCost = kChunkItemCost;
constexpr int kScaleTiles = 8;  // tiles whose scales are kept: loading is at most five ahead
constexpr int kRegsLoad = 104, kRegsSoftmax = 112;
static_assert(32 * (kSoftmaxWarps * kRegsSoftmax + kLoadWarps * kRegsLoad + 4 * kRegsIssue) <=
                  kThreads * kRegsLaunch,
              "register shares exceed the launch's");
using ItemWalk = Walk<kTok, kItemCost>;

struct Smem {
  unsigned char q[2][kTileBytes];
  unsigned char k[2][kTileBytes];
  unsigned char v[2][kTileBytes];
  unsigned char stage[kSoftmaxWarps][32 * 64];  // results on their way out
  uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2];
  uint64_t s_full[2][2], p_ready[2][2], o_last[2], o_full[2];  // [stream][buffer], [stream]
  uint64_t q_full, meet, drained[2];
  int scan[32];
  ItemWalk walk[kSoftmaxWarps][2];     // a softmax warp's item and the next one
  Start start;
  uint32_t tmem, limit;                // cycles of a bounded wait
  int abort;
  float4 scale[kScaleTiles][4];        // a block's s_k, log2 s_v, 1 / s_v; 1 for the open one
  float2 open[kScaleTiles][kGroup];    // its tokens' s_k (from the keys' warp), log2 s_v
  float qf[2][2][kTile];               // [item][stream]: 1 / the factor of a row's queries
  float m[kTile], l[kTile], unit[kTile];  // stream 1's statistics of a shared row tile
};

// Waits are bounded: after the limit, or once another role has given up, they return
// false, and every role leaves its loop.
__device__ __forceinline__ bool warp_wait(Smem& s, uint64_t* b, uint32_t parity) {
  bool ok = bar_try(b, parity);
  if (!ok) {
    const uint32_t t0 = (uint32_t)clock();
#pragma unroll 1
    while (!(ok = bar_try(b, parity))) {
      if (*reinterpret_cast<volatile int*>(&s.abort) || (uint32_t)clock() - t0 > s.limit) {
        *reinterpret_cast<volatile int*>(&s.abort) = 1;
        break;
      }
    }
  }
  return __all_sync(0xffffffffu, ok);
}
__device__ __forceinline__ bool meet_softmax(Smem& s, uint32_t& n) {
  warp_arrive(&s.meet);
  return warp_wait(s, &s.meet, n++ & 1);
}
// All threads, once every role has left its loop.  If one gave up, the products in flight
// end (bounded) before tensor and shared memory are given back, and the flag word says so.
__device__ __forceinline__ void leave(Smem& s, const AttnParams& p) {
  tc_before();
  __syncthreads();
  tc_after();
  if (!*reinterpret_cast<volatile int*>(&s.abort)) return;
  const int x = (int)(threadIdx.x >> 5) - kIssueWarp;
  if (x == 0 || x == 1) {
    tc_commit(elect_lane(), &s.drained[x]);
    const uint32_t t0 = (uint32_t)clock();
    while (!bar_try(&s.drained[x], 0) && (uint32_t)clock() - t0 < kWaitLimit) {
    }
  }
  if (threadIdx.x == 0) set_flag(p.c.cache, KVQ_FLAG_WAIT_TIMEOUT);
  __syncthreads();
}

// ---------------------------------------------------------------------------
// Loading
// ---------------------------------------------------------------------------

__device__ __forceinline__ uint32_t wide_lo(uint32_t v) {
  uint32_t r;
  asm("{\n .reg .b16 a, b;\n mov.b32 {a, b}, %1;\n cvt.rn.f16x2.e4m3x2 %0, a;\n}"
      : "=r"(r)
      : "r"(v));
  return r;
}
__device__ __forceinline__ uint32_t wide_hi(uint32_t v) {
  uint32_t r;
  asm("{\n .reg .b16 a, b;\n mov.b32 {a, b}, %1;\n cvt.rn.f16x2.e4m3x2 %0, b;\n}"
      : "=r"(r)
      : "r"(v));
  return r;
}
template <bool BF16>
__device__ __forceinline__ uint32_t to_half2(uint32_t u, float f) {
  if constexpr (!BF16) return u;
  return pack16<false>(__uint_as_float(u << 16) * f, __uint_as_float(u & 0xffff0000u) * f);
}
template <bool BF16>
__device__ __forceinline__ uint4 to_half8(uint4 v, float f) {
  return make_uint4(to_half2<BF16>(v.x, f), to_half2<BF16>(v.y, f), to_half2<BF16>(v.z, f),
                    to_half2<BF16>(v.w, f));
}
// The power of two that takes a magnitude (bf16 bits) to [2^14, 2^15); at least 2^-100 counts.
__device__ __forceinline__ float lift_of(uint32_t bits) {
  const int e = max((int)(bits >> 7), 27) - 127;
  return bits ? __uint_as_float((uint32_t)(14 - e + 127) << 23) : 1.0f;
}
__device__ __forceinline__ uint32_t largest(const uint4& v) {
  uint32_t m = __vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu);
  m = __vmaxu2(m, __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu));
  return max(m & 0xffffu, m >> 16);
}

// A block's codes in a warp's registers: rows 4 k + lane / 8, 16 channels each, and their way
// into a tile: the second half's lanes write their upper eight channels first, so that the
// eight lanes of a store phase meet different banks.
struct Codes {
  uint4 w[8];
};
__device__ __forceinline__ void load_codes(Codes& c, int k, const uint8_t* at) {
  c.w[k] = __ldg(reinterpret_cast<const uint4*>(at + 512 * k) + (threadIdx.x & 31));
}
__device__ __forceinline__ void restore_codes(const Codes& c, int k, unsigned char* tile, int j) {
  const int lane = threadIdx.x & 31, col = lane & 7, half = col >> 2;
  const int row = 32 * j + 4 * k + (lane >> 3), chunk = 2 * (col & 3);
  const uint4 lo = make_uint4(wide_lo(c.w[k].x), wide_hi(c.w[k].x), wide_lo(c.w[k].y),
                              wide_hi(c.w[k].y));
  const uint4 hi = make_uint4(wide_lo(c.w[k].z), wide_hi(c.w[k].z), wide_lo(c.w[k].w),
                              wide_hi(c.w[k].w));
  st16(tile, tile_at(half, row, chunk + half), half ? hi : lo);
  st16(tile, tile_at(half, row, chunk + 1 - half), half ? lo : hi);
}

// The open block's rows (`valid` of them, the others zero) by a warp, 16 lanes a row, as many at
// a time as fit registers, since each time waits for memory; what becomes of their factors in
// `open`: a key's in x, log2 of a value's in y.
template <bool BF16, bool KEY>
__device__ __forceinline__ void open_block(const uint16_t* rows, int valid, unsigned char* tile,
                                           int j, float2* open) {
  const int lane = threadIdx.x & 31, m = lane & 15;
  constexpr int N = KEY ? 8 : 4;  // (values' least magnitudes take some too)
#pragma unroll 1
  for (int h = 0; h < 32; h += 2 * N) {
    uint4 v[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = h + 2 * i + (lane >> 4);
      v[i] = make_uint4(0u, 0u, 0u, 0u);
      if (r < valid) v[i] = *(reinterpret_cast<const uint4*>(rows + r * kHeadDim) + m);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = h + 2 * i + (lane >> 4);
      // the row's largest magnitude, and (values) above it what its least (least2) lacks to 0xffff
      uint32_t x = largest(v[i]);
      if (!KEY) {
        uint32_t y = least2(least2(least2(least2(~0u, v[i].x), v[i].y), v[i].z), v[i].w);
        x |= ~min(y & 0xffffu, y >> 16) << 16;
      }
#pragma unroll
      for (int o = 8; o; o >>= 1) x = __vmaxu2(x, __shfl_xor_sync(0xffffffffu, x, o));
      const int e = KEY ? key_lift<BF16>(x) : value_lift<BF16>(x & 0xffffu, ~x >> 16);
      st16(tile, tile_at(m >> 3, 32 * j + r, m & 7), lifted8<BF16>(v[i], pow2(e)));
      if (m == 0) {
        if (KEY) open[r].x = pow2(-e);
        else open[r].y = (float)-e;
      }
    }
  }
}
// Whether a block's values are all zero; for a warp of the keys (the values' loads it
// just before, so it is near).
__device__ __forceinline__ bool no_value(const uint8_t* codes) {
  uint32_t any = 0u;
#pragma unroll 2
  for (int k = 0; k < 8; ++k) {
    const uint4 x = __ldg(reinterpret_cast<const uint4*>(codes + 512 * k) + (threadIdx.x & 31));
    any |= x.x | x.y | x.z | x.w;
  }
  return !__any_sync(0xffffffffu, (any & 0x7f7f7f7fu) != 0u);
}
__device__ __forceinline__ void zero_block(unsigned char* tile, int j) {
  const int lane = threadIdx.x & 31, m = lane & 15;
#pragma unroll 1
  for (int i = 0; i < 32; i += 2)
    st16(tile, tile_at(m >> 3, 32 * j + i + (lane >> 4), m & 7), make_uint4(0u, 0u, 0u, 0u));
}

// A loading warp: block j of every key (or value) tile of the CTA's share.  As soon as a
// part of a block is in its tile, the same part of the next block is loaded into its
// registers; the block after that comes to L2, and the table's entry of the one after that
// is on its way.  The keys' warps leave the block's scales beside the tile.
constexpr int kAhead = 2;

template <bool BF16, bool TEST>
__device__ __forceinline__ void load_role(const AttnParams& p, Smem& s, int u0, int u1, int j,
                                          bool key) {
  const int lane = threadIdx.x & 31;
  unsigned char(*tiles)[kTileBytes] = key ? s.k : s.v;
  uint64_t* full = key ? s.k_full : s.v_full;
  uint64_t* empty = key ? s.k_empty : s.v_empty;
  const uint8_t* pool = key ? p.c.cache.k_codes : p.c.cache.v_codes;
  uint32_t n = 0;
  ItemWalk w;
  w.begin(p, s.start, u0, u1);
  for (; w.next(p); w.advance(p)) {
    const int32_t* table = p.c.cache.block_table + (long long)w.b * p.c.d.max_blocks;
    const int whole = w.q.L & ~(kGroup - 1);
    const auto seen = [&](int t0) {
      return t0 <= w.s.p1 && (t0 + kGroup > w.s.lo || t0 < p.c.sinks);
    };
    const auto token = [&](int i) { return w.s.tile(i) * kTile + j * kGroup; };
    // whether unit i's block is read as codes, its page (looked at no sooner than needed),
    // and its place in the pools, -1 for none
    const auto reads = [&](int i) {
      const int t0 = token(i);
      return i < w.i1 && t0 < whole && seen(t0);
    };
    const auto entry = [&](int i) { return reads(i) ? __ldg(table + (token(i) >> 5)) : -1; };
    const auto place = [&](int i, int e) -> int {
      if (!reads(i)) return -1;
      if ((unsigned)e < (unsigned)p.c.cache.n_pages) return e * p.c.d.hkv + w.head;
      if (lane == 0) set_flag(p.c.cache, KVQ_FLAG_BAD_PAGE);
      return -1;
    };
    const auto prefetch = [&](int e) {
      if ((unsigned)e < (unsigned)p.c.cache.n_pages)
        asm volatile("prefetch.global.L2 [%0];" ::"l"(
            pool + ((long long)e * p.c.d.hkv + w.head) * (kGroup * kHeadDim) + 128 * lane));
    };
    Codes c;
    float2 scale = make_float2(1.0f, 1.0f);
    int at0 = -1, at1 = place(w.i0, entry(w.i0));
    int e[kAhead];  // entries behind at1's
#pragma unroll
    for (int k = 0; k < kAhead; ++k) e[k] = entry(w.i0 + 1 + k);
#pragma unroll
    for (int k = 0; k < kAhead - 1; ++k) prefetch(e[k]);
    // i = i0 - 1 only loads the first block
#pragma unroll 1
    for (int i = w.i0 - 1; i < w.i1; ++i) {
      const int buf = n & 1, far = entry(i + 2 + kAhead);
      unsigned char* tile = tiles[buf];
      if (i >= w.i0) {
        if (!warp_wait(s, &empty[buf], ((n >> 1) & 1) ^ 1)) return;
        bool none = false, open = false;  // the block counts for nothing; is the open one
        if (at0 < 0) {
          const int ta = token(i);
          none = !(ta >= whole && ta < w.q.L && seen(ta));
          if (none) {
            zero_block(tile, j);
          } else {
            const long long at =
                (((long long)w.b * p.c.d.hkv + w.head) * kRing + (ta & (kRing - 1))) * kHeadDim;
            const int valid = w.q.L - ta;
            float2* factors = s.open[n & (kScaleTiles - 1)];
            if (key) open_block<BF16, true>(p.c.cache.k_ring + at, valid, tile, j, factors);
            else open_block<BF16, false>(p.c.cache.v_ring + at, valid, tile, j, factors);
            open = true;
          }
          c = Codes{};  // (nothing is in it: so it takes no registers from the lines above)
        }
        // (the scores' product waits for the keys' warps alone: they write all of it; the values'
        // factors of the open block are waited for)
        if (key && at0 >= 0 && scale.y == 1.0f &&
            no_value(p.c.cache.v_codes + (long long)at0 * (kGroup * kHeadDim)))
          scale.y = kNoValue;
        if (key && lane == 0)
          s.scale[n & (kScaleTiles - 1)][j] =
              none   ? make_float4(1.0f, -INFINITY, 1.0f, 0.0f)
              : open ? make_float4(1.0f, 0.0f, 0.0f, 1.0f)
                     : make_float4(scale.x, log2_fast(scale.y), 1.0f / scale.y, 0.0f);
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        if (at0 >= 0) restore_codes(c, k, tile, j);
        if (at1 >= 0) load_codes(c, k, pool + (long long)at1 * (kGroup * kHeadDim));
      }
      if (key && at1 >= 0) scale = __ldg(reinterpret_cast<const float2*>(p.c.cache.scales) + at1);
      if (i >= w.i0) {
        fence_async();
        if (!TEST || !key || j != 1 || n != 1) warp_arrive(&full[buf]);
        ++n;
      }
      at0 = at1;
      at1 = place(i + 2, e[0]);
      prefetch(e[kAhead - 1]);
#pragma unroll
      for (int k = 0; k < kAhead - 1; ++k) e[k] = e[k + 1];
      e[kAhead - 1] = far;
    }
  }
}

// ---------------------------------------------------------------------------
// Products
// ---------------------------------------------------------------------------

// The products of stream x, by one warp.  two: items of 256 rows (a row tile and both halves
// of every token tile per stream), else of 128 (a half of the token tiles per stream).
__device__ __forceinline__ void issue_role(const AttnParams& p, Smem& s, int u0, int u1, int x,
                                           int two) {
  constexpr uint32_t kIdS = instr_desc(false, kStep), kIdO = instr_desc(true, kHeadDim);
  constexpr int kHalf = kStep * 128;  // where the second half of a tile's tokens begins
  const uint32_t tm = __shfl_sync(0xffffffffu, s.tmem, 0) + 128 * x, leader = elect_lane();
  const uint64_t q = tile_desc(sptr(s.q[two ? x : 0]), false);
  uint32_t nt = 0, ns = 0, items = 0;  // tiles, steps and items done
  ItemWalk w;
  w.begin(p, s.start, u0, u1);
#pragma unroll 1
  for (; w.next(p); w.advance(p), ++items) {
    const int steps = (w.i1 - w.i0) << two;
    if (!warp_wait(s, &s.q_full, items & 1)) return;
    tc_after();
    // scores run two steps ahead
#pragma unroll 1
    for (int st = -2; st < steps; ++st) {
      const uint32_t k = ns + st, b = k & 1;  // the step counted over all items, its buffer
      const uint32_t ts = tm + kColS + kStep * b;
      if (st >= 0) {
        const uint32_t t = nt + (st >> two), buf = t & 1;
        const int half = two ? st & 1 : x;
        if (!warp_wait(s, &s.p_ready[x][b], (k >> 1) & 1)) return;
        if ((!two || half == 0) && !warp_wait(s, &s.v_full[buf], (t >> 1) & 1)) return;
        tc_after();
        const uint64_t v = tile_desc(sptr(s.v[buf]) + half * kHalf, true);
#pragma unroll
        for (int ks = 0; ks < kStep / 16; ++ks)
          mma_ts(leader, tm + kColO, ts + 8 * ks, v + step_major_mn(ks), kIdO, st > 0 || ks > 0);
        if (!two || half == 1) tc_commit(leader, &s.v_empty[buf]);
        // the last two products of an item tell that they are in; the others are when the
        // scores issued behind them are
        if (st + 2 >= steps) tc_commit(leader, st + 1 == steps ? &s.o_full[x] : &s.o_last[x]);
      }
      if (st + 2 < steps) {
        const uint32_t t = nt + ((st + 2) >> two), buf = t & 1;
        const int half = two ? st & 1 : x;
        if (!two || half == 0) {
          if (!warp_wait(s, &s.k_full[buf], (t >> 1) & 1)) return;
          tc_after();
        }
        const uint64_t kd = tile_desc(sptr(s.k[buf]) + half * kHalf, false);
#pragma unroll
        for (int ks = 0; ks < kHeadDim / 16; ++ks)
          mma_ss(leader, ts, q + step_major_k(ks), kd + step_major_k(ks), kIdS, ks > 0);
        tc_commit(leader, &s.s_full[x][b]);
        if (!two || half == 1) tc_commit(leader, &s.k_empty[buf]);
      }
    }
    nt += w.i1 - w.i0;
    ns += steps;
  }
}

// ---------------------------------------------------------------------------
// Softmax, results
// ---------------------------------------------------------------------------

// The running maximum of x + log2 s_v is m + e: e is 0 until it passes kFar (from then on
// log2 s_v alone, and every step goes by differences of scores, which are exact where it counts).
// l: lifted sum of w / s_v.
struct Row {
  float m, e, l;
};
constexpr float kFar = 32768.0f;  // rounded to fp32, a sum with m is good to 2^-9

// A warp's 32 rows, from row r0 of the sequence and row `row` of the tile on: 16 lanes a row.
template <bool BF16>
__device__ __forceinline__ void load_queries(const AttnParams& p, const ItemWalk& w, int r0,
                                             unsigned char* tile, int row, float* qf) {
  const int lane = threadIdx.x & 31, m = lane & 15, rows = w.q.n * p.c.d.gq;
#pragma unroll 1
  for (int h = 0; h < 32; h += 16) {
    uint4 v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = h + 2 * i + (lane >> 4);
      v[i] = make_uint4(0u, 0u, 0u, 0u);
      if (r0 + r < rows)
        v[i] = __ldg(reinterpret_cast<const uint4*>(
                         p.c.q + row_offset(p, p.c.q_stride, w.q.row, w.head, r0 + r)) + m);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = row + h + 2 * i + (lane >> 4);
      float f = 1.0f;
      if constexpr (BF16) {
        uint32_t x = largest(v[i]);
#pragma unroll
        for (int o = 8; o; o >>= 1) x = max(x, __shfl_xor_sync(0xffffffffu, x, o));
        f = lift_of(x);
        if (m == 0) qf[r] = 1.0f / f;
      }
      st16(tile, tile_at(m >> 3, r, m & 7), to_half8<BF16>(v[i], f));
    }
  }
}

// The thread's row of scores with -inf where a column is not seen: column n is seen when n is
// at most hi and above lo, or below sink (all less the step's first token).  Only steps at
// an edge come here; the scores are rewritten in tensor memory by a short loop.
__device__ __forceinline__ void mask_row(uint32_t ts, int hi, int lo, int sink) {
#pragma unroll 1
  for (int c = 0; c < kStep; c += 32) {
    uint32_t r[32];
    tm_load32(ts + c, r);
    tm_load_wait();
#pragma unroll
    for (int n = 0; n < 32; ++n) {
      const int t = c + n;
      if (t > hi || (t <= lo && t >= sink)) r[n] = 0xff800000u;
    }
    tm_store32(ts + c, r);
  }
  tm_store_wait();
}

// A step in which tokens have factors of their own (the open block's: w of its scale is 1), or
// in which scores are so large that only their differences are fit for fp32 (`far`): the best of a
// thread's row by x + log2 s_v first, then all weights against it.  Returns the row and what the
// results so far have to be multiplied with.  Few steps come here, so the numbers stay in tensor
// memory, 16 at a time, and the code out of the others' way.
__device__ __noinline__ float4 apart_step(uint32_t sb, const float4* sc, const float2* open,
                                          float sl, bool first, bool far, float row_m,
                                          float row_e, float l) {
  // s_k, log2 s_v of columns c .. c + 15, one or each: the first's place and its distance to the next
  const auto factors = [&](int c, int& stride) {
    stride = sc[c >> 5].w != 0.0f ? 1 : 0;
    return stride ? open + (c & 31) : reinterpret_cast<const float2*>(sc + (c >> 5));
  };
  float best = -INFINITY, best_lv = 0.0f;
#pragma unroll 1
  for (int c = 0; c < kStep; c += 8) {
    uint32_t r[8];
    int stride;
    const float2* f = factors(c, stride);
    tm_load8(sb + c, r);
    tm_load_wait();
#pragma unroll
    for (int n = 0; n < 8; ++n) {
      const float2 s = f[n * stride];
      const float x = __fmul_rn(__uint_as_float(r[n]), fmaxf(s.x * sl, kLeastFactor));
      if ((x - best) + (s.y - best_lv) > 0.0f) best = x, best_lv = s.y;
      r[n] = __float_as_uint(x);
    }
    tm_store8(sb + c, r);
  }
  tm_store_wait();
  // (-inf - -inf is NaN, and no reason for a new maximum)
  const float d = (best - row_m) + (best_lv - row_e);
  float z = 1.0f;
  if (first || d > kRescaleLog2) {
    const float sum = best + best_lv;
    const bool split = far || fabsf(sum) > kFar;
    z = exp2_fast(-d);
    l = first ? 0.0f : l * z;
    row_m = split ? best : sum;
    row_e = split ? best_lv : 0.0f;
  }
  const float m = row_m == -INFINITY ? 0.0f : row_m, e = row_e - kLiftLog2;
#pragma unroll 1
  for (int c = 0; c < kStep; c += 16) {
    uint32_t r[2][8], h[8];
    int stride;
    const float2* f = factors(c, stride);
    tm_load8(sb + c, r[0]);
    tm_load8(sb + c + 8, r[1]);
    tm_load_wait();
#pragma unroll
    for (int n = 0; n < 16; n += 2) {
      const float lv0 = f[n * stride].y, lv1 = f[(n + 1) * stride].y;
      const float y0 = (__uint_as_float(r[n >> 3][n & 7]) - m) + (lv0 - e);
      const float y1 = (__uint_as_float(r[n >> 3][(n & 7) + 1]) - m) + (lv1 - e);
      const float w0 = exp2_fast(y0), w1 = exp2_fast(y1);
      if (w0 > 0.0f) l = fmaf(w0, exp2_fast(-lv0), l);
      if (w1 > 0.0f) l = fmaf(w1, exp2_fast(-lv1), l);
      h[n >> 1] = pack16<false>(w0, w1);
    }
    // (words 8 c / 16 ..: what stood there has been read)
    tm_store8(sb + (c >> 1), h);
  }
  tm_store_wait();
  return make_float4(row_m, row_e, l, z);
}

template <bool BF16>
__device__ __forceinline__ void softmax_role(const AttnParams& p, Smem& s, int u0, int u1,
                                             const Shares& shares, int two) {
  const int warp = threadIdx.x >> 5, x = warp >> 2, lane_row = threadIdx.x & 127;
  const uint32_t lanes = (uint32_t)(warp & 3) << 21;  // 32 lanes a warp, in bits 16 up
  const uint32_t tm = __shfl_sync(0xffffffffu, s.tmem, 0) + 128 * x;
  const uint32_t ts = tm + lanes + kColS, to = tm + lanes + kColO;
  const int tr = kTile << two;
  // steps and tiles of the stream, meetings, items and phases of o_last so far
  uint32_t ns = 0, nt = 0, met = 0, items = 0, lasts = 0;
  const auto queries = [&](const ItemWalk& w, uint32_t item) {
    const int r0 = w.row_tile * tr + (two ? kTile * x : 0) + (lane_row & ~31);
    load_queries<BF16>(p, w, r0, s.q[x], lane_row & ~31, s.qf[item & 1][x]);
    fence_async();
    warp_arrive(&s.q_full);
  };
  // The item and the next one are kept in shared memory: their fields would take
  // registers from the scores.
  bool more;
  {
    ItemWalk first;
    first.begin(p, s.start, u0, u1);
    more = first.next(p);
    s.walk[warp][0] = first;
    __syncwarp();
    if (more && (two || x == 0)) queries(first, 0);
  }
#pragma unroll 1
  while (more) {
    const ItemWalk& w = s.walk[warp][items & 1];
    const int rows = w.q.n * p.c.d.gq;
    const int tr_row = (two ? kTile * x : 0) + lane_row;  // row in the item
    const int g = w.row_tile * tr + tr_row, g_warp = g - (threadIdx.x & 31);
    const bool valid = g < rows;
    const bool live = g_warp < rows;  // the warp has a row
    const int pos = w.q.L - w.q.n + token_of_row(p, g);
    Row row{-INFINITY, 0.0f, 0.0f};
    bool far = false;  // a row of the warp has its maximum beyond kFar
    float sl = p.c.scale_log2;
    const int steps = (w.i1 - w.i0) << two;
#pragma unroll 1
    for (int st = 0; st < steps; ++st, ++ns) {
      const int b = ns & 1;
      const uint32_t sb = ts + kStep * b;
      if (!warp_wait(s, &s.s_full[x][b], (ns >> 1) & 1)) return;
      tc_after();
      if (live) {
        if (BF16 && st == 0) sl *= s.qf[items & 1][two ? x : 0][lane_row];
        const int half = two ? st & 1 : x;
        const int t0 = w.s.tile(w.i0 + (st >> two)) * kTile + kStep * half;
        // every token of the step is seen by every row of the item, and nothing is special
        const bool whole = !far && w.s.p0 >= t0 + kStep - 1 &&
                           (!p.c.window || t0 > w.s.p1 - p.c.window || t0 <= p.c.sinks - kStep);
        const int slot = (nt + (st >> two)) & (kScaleTiles - 1);
        const float4* sc = &s.scale[slot][2 * half];
        // The product before this step's has to be in: the next scores are issued behind it;
        // an item's last step has none behind.
        const auto rescale = [&](float z) {
          if (st + 1 < steps ? !warp_wait(s, &s.s_full[x][b ^ 1], ((ns + 1) >> 1) & 1)
                             : !warp_wait(s, &s.o_last[x], lasts & 1))
            return false;
          tc_after();
          rescale_row(to, z);
          return true;
        };
        if (!whole) {
          // the last token behind the window, -1 if there is none (positions and windows
          // each reach 2^31)
          const int behind = p.c.window ? max(max(pos, 0) - p.c.window, -1) : -1;
          mask_row(sb, (valid ? pos : -1) - t0, behind - t0, p.c.sinks - t0);
          // (the open block ends behind every row's position: no step with it is whole)
          if (far || sc[0].w != 0.0f || sc[1].w != 0.0f) goto apart;
        }
        {
          uint32_t r[2][32];
          tm_load32(sb, r[0]);
          tm_load32(sb + 32, r[1]);
          const float2 f =
              make_float2(fmaxf(sc[0].x * sl, kLeastFactor), fmaxf(sc[1].x * sl, kLeastFactor));
          const float2 lv = make_float2(sc[0].y, sc[1].y);
          tm_load_wait();
          float mc[2];
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const uint32_t* y = r[c];
            float a = fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
            float d = fmaxf(__uint_as_float(y[2]), __uint_as_float(y[3]));
#pragma unroll
            for (int n = 4; n < 32; n += 4) {
              a = fmaxf(fmaxf(a, __uint_as_float(y[n])), __uint_as_float(y[n + 1]));
              d = fmaxf(fmaxf(d, __uint_as_float(y[n + 2])), __uint_as_float(y[n + 3]));
            }
            mc[c] = fmaxf(a, d);
          }
          const float mx = fmaxf(fmaf(mc[0], f.x, lv.x), fmaf(mc[1], f.y, lv.y));
          if (st == 0) {
            far = __any_sync(0xffffffffu, mx > -INFINITY && fabsf(mx) > kFar);
            if (far) goto apart;
            row.m = mx;
          } else {
            const bool up = mx > row.m + kRescaleLog2;
            if (__any_sync(0xffffffffu, up)) {
              far = __any_sync(0xffffffffu, up && fabsf(mx) > kFar);
              if (far) goto apart;
              const float z = up ? exp2_fast(row.m - mx) : 1.0f;
              if (up) row.m = mx;
              row.l *= z;
              if (!rescale(z)) return;
            }
          }
          const float base = row.m == -INFINITY ? 0.0f : kLiftLog2 - row.m;
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const float fc = c ? f.y : f.x, oc = base + (c ? lv.y : lv.x);
            const uint64_t sl2 = pair(fc, fc), of = pair(oc, oc);
            uint64_t acc[2] = {0ull, 0ull};
            uint32_t h[16];
#pragma unroll
            for (int n = 0; n < 16; ++n) {
              float y0, y1;
              unpair(fma2(pair(__uint_as_float(r[c][2 * n]), __uint_as_float(r[c][2 * n + 1])),
                          sl2, of),
                     y0, y1);
              y0 = exp2_fast(y0);
              y1 = exp2_fast(y1);
              acc[n & 1] = add2(acc[n & 1], pair(y0, y1));
              h[n] = pack16<false>(y0, y1);
            }
            tm_store16(sb + 16 * c, h);
            float y0, y1;
            unpair(add2(acc[0], acc[1]), y0, y1);
            row.l = fmaf(y0 + y1, sc[c].z, row.l);
          }
          tm_store_wait();
        }
        if (false) {  // (behind the others' code, so that theirs stays in one piece)
        apart:
          const uint32_t t = nt + (st >> two);
          if (!warp_wait(s, &s.v_full[t & 1], (t >> 1) & 1)) return;
          const float4 next =
              apart_step(sb, sc, s.open[slot], sl, st == 0, far, row.m, row.e, row.l);
          row = Row{next.x, next.y, next.z};
          far |= __any_sync(0xffffffffu, row.e != 0.0f ||
                                             (row.m > -INFINITY && fabsf(row.m) > kFar)) != 0;
          if (st > 0 && __any_sync(0xffffffffu, next.w != 1.0f) && !rescale(next.w)) return;
        }
      }
      tc_before();
      warp_arrive(&s.p_ready[x][b]);
    }
    lasts += steps > 1;
    nt += w.i1 - w.i0;
    // The next item's queries: all scores of this one are done (an item of one row tile
    // has the other stream's too).
    {
      ItemWalk next = w;
      next.advance(p);
      more = next.next(p);
      s.walk[warp][(items + 1) & 1] = next;
      __syncwarp();
      if (more && (two || x == 0)) {
        if (!two && !warp_wait(s, &s.s_full[1][(ns - 1) & 1], ((ns - 1) >> 1) & 1)) return;
        queries(next, items + 1);
      }
    }
    // the accumulator is complete; items of one row tile need both streams'
    if (!warp_wait(s, &s.o_full[x], items & 1)) return;
    if (!two && x == 0 && !warp_wait(s, &s.o_full[1], items & 1)) return;
    tc_after();
    // one number again for the maximum; what it leaves of the two goes to the results
    float unit = 1.0f;
    if (far && row.m > -INFINITY) {
      const float m = row.m + row.e;
      unit = exp2_fast((row.m - m) + row.e);
      row.l *= unit;
      row.m = m;
    }
    if (!two && x == 1) {
      s.m[lane_row] = row.m;
      s.l[lane_row] = row.l;
      s.unit[lane_row] = unit;
    }
    if (!two && !meet_softmax(s, met)) return;
    const bool direct = w.whole();
    if ((two || x == 0) && live) {
      float f0 = unit, f1 = 0.0f, m = row.m, l = row.l;
      if (!two) {
        const float m1 = s.m[lane_row], l1 = s.l[lane_row];
        m = fmaxf(row.m, m1);
        if (m > -INFINITY) {
          f0 = exp2_fast(row.m - m);
          f1 = exp2_fast(m1 - m);
        }
        l = row.l * f0 + l1 * f1;
        f0 *= unit;
        f1 *= s.unit[lane_row];
      }
      const float scale = direct ? (l > 0.0f ? 1.0f / l : 0.0f) : 1.0f;
      f0 *= scale;
      f1 *= scale;
      const int pr = w.slot(u0) * tr + tr_row;
      const int lane = threadIdx.x & 31;
      chunk::Rows at;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int r = (lane >> 2) + 8 * k;
        char* row_at =
            direct ? reinterpret_cast<char*>(
                         p.c.out + row_offset(p, p.c.out_stride, w.q.row, w.head, g_warp + r))
                   : reinterpret_cast<char*>(p.part_o + (long long)(pr - lane + r) * kHeadDim);
        at.at[k] = g_warp + r < rows ? row_at + 16 * (lane & 3) : nullptr;
      }
#pragma unroll 1
      for (int c = 0; c < kHeadDim; c += 32) {
        uint32_t r[32];
        float o[32];
        tm_load32(to + c, r);
        if (two) {
          tm_load_wait();
#pragma unroll
          for (int k = 0; k < 32; ++k) o[k] = __uint_as_float(r[k]) * f0;
        } else {
          uint32_t r1[32];
          tm_load32(to + 128 + c, r1);
          tm_load_wait();
#pragma unroll
          for (int k = 0; k < 32; ++k)
            o[k] = fmaf(__uint_as_float(r1[k]), f1, __uint_as_float(r[k]) * f0);
        }
        uint4 v[4];
        if (direct) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float* y = o + 8 * k;
            v[k] = make_uint4(pack16<BF16>(y[0], y[1]), pack16<BF16>(y[2], y[3]),
                              pack16<BF16>(y[4], y[5]), pack16<BF16>(y[6], y[7]));
          }
          stage_row(s.stage[warp], v);
          put_rows(s.stage[warp], at, 2 * c);
        } else {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const float* y = o + 16 * h + 4 * k;
              v[k] = make_uint4(__float_as_uint(y[0]), __float_as_uint(y[1]),
                                __float_as_uint(y[2]), __float_as_uint(y[3]));
            }
            stage_row(s.stage[warp], v);
            put_rows(s.stage[warp], at, 4 * (c + 16 * h));
          }
        }
      }
      if (valid && !direct) p.part_ml[pr] = make_float2(m, l);
      tc_before();
    }
    if (!direct && w.i0 == 0 && threadIdx.x == 0)
      p.splits[blockIdx.x] =
          Split{1, u0 < w.base ? 1 : 0, shares.owner(w.last_unit()), w.b,
                w.row_tile, w.head};
    if (!meet_softmax(s, met)) return;  // s.m, s.l and both accumulators may be written again
    ++items;
  }
}

// ---------------------------------------------------------------------------
// Kernel
// ---------------------------------------------------------------------------

// TEST: a short bound of the waits, and an arrival for the second tile of keys is left out.
template <bool BF16, bool TEST>
__global__ void __launch_bounds__(kThreads, 1)
chunk_kernel(const __grid_constant__ AttnParams p) {
  extern __shared__ __align__(1024) unsigned char raw[];
  Smem& s = *reinterpret_cast<Smem*>(raw);
  const int tid = threadIdx.x, warp = tid >> 5;
  const int two = p.item_rows > kTile ? 1 : 0;
  if (tid == 0) {
    p.splits[blockIdx.x].valid = 0;
    for (int i = 0; i < 2; ++i) {
      bar_init(&s.k_full[i], 4);
      bar_init(&s.v_full[i], 4);
      bar_init(&s.k_empty[i], 2);  // a commit of either stream
      bar_init(&s.v_empty[i], 2);
      bar_init(&s.o_full[i], 1);
      bar_init(&s.o_last[i], 1);
      bar_init(&s.drained[i], 1);
      for (int b = 0; b < 2; ++b) {
        bar_init(&s.s_full[i][b], 1);
        bar_init(&s.p_ready[i][b], 4);
      }
    }
    bar_init(&s.q_full, 4 << two);
    bar_init(&s.meet, kSoftmaxWarps);
    s.abort = 0;
    s.limit = TEST ? kWaitLimit / 100 : kWaitLimit;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  Shares shares;
  int u0, u1;
  if (!plan_share<kTok, kItemCost>(p, s.scan, &s.start, 1, shares, u0, u1)) return;
  if (warp == kIssueWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(
                     sptr(&s.tmem))
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    tc_before();
  }
  __syncthreads();
  tc_after();
  const uint32_t tm = *reinterpret_cast<volatile uint32_t*>(&s.tmem);

  if (warp < kSoftmaxWarps) {
    chunk::regs_up<kRegsSoftmax>();
    softmax_role<BF16>(p, s, u0, u1, shares, two);
    __syncwarp();
  } else if (warp < kIssueWarp) {
    chunk::regs_up<kRegsLoad>();
    load_role<BF16, TEST>(p, s, u0, u1, warp & 3, warp < kSoftmaxWarps + 4);
    __syncwarp();
  } else {
    chunk::regs_down<kRegsIssue>();
    if (warp < kIssueWarp + 2) issue_role(p, s, u0, u1, warp - kIssueWarp, two);
    __syncwarp();
  }
  leave(s, p);
  if (warp == kIssueWarp)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tm));
}

template <bool BF16, bool TEST>
cudaError_t launch(const AttnParams& p, int ctas, cudaStream_t stream) {
  static std::atomic<unsigned long long> done{0};
  const cudaError_t e = once_per_device(done, [] {
    const cudaError_t e = cudaFuncSetAttribute(
        chunk_kernel<BF16, TEST>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Smem));
    if (e != cudaSuccess) return e;
    // the register shares wait for registers that a smaller launch would lack
    cudaFuncAttributes attr;
    const cudaError_t ea = cudaFuncGetAttributes(&attr, chunk_kernel<BF16, TEST>);
    if (ea != cudaSuccess) return ea;
    return attr.numRegs < kRegsLaunch ? cudaErrorInvalidConfiguration : cudaSuccess;
  });
  if (e != cudaSuccess) return e;
  chunk_kernel<BF16, TEST><<<ctas, kThreads, sizeof(Smem), stream>>>(p);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_chunk(const AttnParams& p, int ctas, cudaStream_t stream, bool selftest) {
  if (selftest)
    return p.c.d.bf16 ? cudaErrorNotSupported : launch<false, true>(p, ctas, stream);
  return p.c.d.bf16 ? launch<true, false>(p, ctas, stream)
                    : launch<false, false>(p, ctas, stream);
}

}  // namespace block8
}  // namespace kvq
