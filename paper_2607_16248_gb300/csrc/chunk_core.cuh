// Device code of the chunk attention kernel (kvq_chunk_attn): an attention
// over the packed cache on the 5th-generation tensor cores.  Included by one
// translation unit per key width (chunk_k*.cu).
//
// Work.  The query rows of a (sequence, kv-head) are its n_q tokens times the
// gq heads that share the kv-head, row = t * gq + head, so one dequantized
// tile of keys and values serves every head of the group.  An item is one row
// tile (128 or 256 rows) of one (sequence, kv-head); its units are the
// 128-token tiles that any of its rows can see.  All items' units lie end to
// end and every CTA (one per SM) takes an equal contiguous share: a long cache
// with few rows is split over many CTAs and a whole prompt leaves no tail of
// half-empty waves.  An item that is shared leaves partials (unnormalised
// row, maximum, sum) in the workspace; the CTA that finishes last merges them
// in the order of the tokens, so results repeat bit for bit.
//
// A CTA.  Per step: S = Q K^T (M 128 rows x N 128 tokens, fp16 operands in
// shared memory, fp32 in tensor memory), softmax by the four warps that own
// the 128 lanes of S (a thread per row), P as fp16 over the same tensor memory
// columns, O += P V with P read from tensor memory.  Two such streams
// alternate, so that one's softmax runs under the other's products: two row
// tiles on the same key tiles, or (items of at most 128 rows) the same row
// tile on alternate key tiles, joined at the end.
//   warps 0-3, 4-7  softmax of streams 0 and 1 (and queries in, results out)
//   warps 8-11      keys: one 32-token block each, codes -> fp16 tile
//   warps 12-15     values, the same
//   warp 16         issues the products
// The running maximum of a row moves only when a score is more than 8 (in log2)
// above it, so the accumulator is rescaled rarely; weights stay below 2^8.
//
// Tile layouts (128-byte swizzle, [half][row][128 bytes]).  Tokens of an
// 8-token run stand in the order 0 4 1 5 2 6 3 7 and so do the channels of the
// accumulator: two elements four apart come out of a code word in one
// extraction.  Codes of 2, 4, 8 bits leave a lane with 32 tokens of one
// channel (keys) or 32 channels of one token (values), which is what tiles
// with the token (the channel) contiguous take; 1-bit codes come in pairs
// along the other axis (the order the decode kernel reads them in) and fill
// tiles with the contraction contiguous, keys with the channels permuted
// (q1_offset; the queries alike).
#pragma once

#include "common.cuh"

namespace kvq {
namespace chunk {

constexpr int kTile = 128;                  // tokens of a key / value tile, rows of a product
constexpr int kTileBytes = kTile * kHeadDim * 2;
constexpr int kHalfBytes = kTileBytes / 2;  // 64 elements of the contiguous axis
constexpr int kSoftmaxWarps = 8, kLoadWarps = 8;
constexpr int kThreads = 32 * (kSoftmaxWarps + kLoadWarps + 1);
constexpr long long kWaitLimit = 4000000000LL;  // cycles of a bounded wait (~2 s)
constexpr float kRescaleLog2 = 8.0f;

struct Smem {
  unsigned char q[2][kTileBytes];
  unsigned char k[2][kTileBytes];
  unsigned char v[2][kTileBytes];
  uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2], s_full[2], p_ready[2], o_full[2], q_full;
  uint64_t meet, drained;
  long long scan[32];
  long long start_unit;
  int start_group, start_head, start_step;
  uint32_t tmem;
  int abort, last;
  float m[kTile], l[kTile];
};

struct Params {
  Dims d;
  kvq_cache cache;
  const __half* q;
  __half* out;
  ChunkCall c;
  int tiles;         // row tiles per (sequence, kv-head)
  int streams_rows;  // 1: items of 256 rows (a row tile per stream), 0: of 128
  float* part_o;     // [2 * CTAs][rows of an item][128]
  float2* part_ml;   // [2 * CTAs][rows of an item]
  unsigned* tickets; // [items]
};

// ---------------------------------------------------------------------------
// PTX
// ---------------------------------------------------------------------------

__device__ __forceinline__ uint32_t sptr(const void* p) {
  return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}
__device__ __forceinline__ void bar_init(uint64_t* b, uint32_t n) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(sptr(b)), "r"(n) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint64_t* b) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(sptr(b)) : "memory");
}
__device__ __forceinline__ bool bar_try(uint64_t* b, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n .reg .pred p;\n"
      " mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n"
      " selp.u32 %0, 1, 0, p;\n}"
      : "=r"(ok)
      : "r"(sptr(b)), "r"(parity)
      : "memory");
  return ok != 0;
}
// Bounded: after the limit, or once another role has given up, it returns
// false; every role then leaves its loop.
__device__ __forceinline__ bool bar_wait(Smem& s, uint64_t* b, uint32_t parity) {
  if (bar_try(b, parity)) return true;
  const long long t0 = clock64();
  while (!bar_try(b, parity)) {
    if (*reinterpret_cast<volatile int*>(&s.abort)) return false;
    if (clock64() - t0 > kWaitLimit) {
      *reinterpret_cast<volatile int*>(&s.abort) = 1;
      return false;
    }
  }
  return true;
}
// The same for a whole warp (all lanes leave together).
__device__ __forceinline__ bool warp_wait(Smem& s, uint64_t* b, uint32_t parity) {
  return __all_sync(0xffffffffu, bar_wait(s, b, parity));
}
// All softmax threads meet (bounded, unlike a hardware barrier).
__device__ __forceinline__ bool meet_softmax(Smem& s, uint32_t& n) {
  bar_arrive(&s.meet);
  return warp_wait(s, &s.meet, n++ & 1);
}
__device__ __forceinline__ void fence_async() {
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}
__device__ __forceinline__ void tc_before() {
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
}
__device__ __forceinline__ void tc_after() {
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
}
__device__ __forceinline__ void tc_commit(uint64_t* b) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(
                   sptr(b))
               : "memory");
}

// D[128 x 128] (+)= A B, fp16 in, fp32 out, K = 16.  A in shared memory.
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc,
                                       uint32_t acc) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(acc)
      : "memory");
}
// The same with A in tensor memory.
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc,
                                       uint32_t acc) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(acc)
      : "memory");
}
__device__ __forceinline__ void tm_load32(uint32_t addr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,"
      "%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
        "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
        "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
        "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
        "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(addr));
}
__device__ __forceinline__ void tm_load_wait() {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tm_store32(uint32_t addr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,"
      "%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};" ::"r"(r[0]),
      "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
      "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
      "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]),
      "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]),
      "r"(r[30]), "r"(r[31]), "r"(addr)
      : "memory");
}
__device__ __forceinline__ void tm_store16(uint32_t addr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,"
      "%13,%14,%15};" ::"r"(r[0]),
      "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
      "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
      "r"(addr)
      : "memory");
}
__device__ __forceinline__ void tm_store_wait() {
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ __half2 as_half2(uint32_t u) {
  return *reinterpret_cast<const __half2*>(&u);
}
__device__ __forceinline__ uint32_t as_u32(__half2 h) {
  return *reinterpret_cast<const uint32_t*>(&h);
}

// Shared-memory descriptor of a swizzled tile: 8-row groups 1024 bytes apart;
// where the contiguous axis is not the contraction, its 64-element halves are
// kHalfBytes apart.
__device__ __forceinline__ uint64_t tile_desc(uint32_t addr, bool mn) {
  return (uint64_t)((addr & 0x3ffffu) >> 4) | ((uint64_t)(mn ? kHalfBytes >> 4 : 1) << 16) |
         ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
// Descriptor advance (in 16-byte units) of contraction step ks (16 elements).
__device__ __forceinline__ uint32_t step_major_k(int ks) {
  return ((ks >> 2) * kHalfBytes + (ks & 3) * 32) >> 4;
}
__device__ __forceinline__ uint32_t step_major_mn(int ks) { return (ks * 2048) >> 4; }

// fp32 accumulator, fp16 operands, M = N = 128; b_mn: B's contiguous axis is N.
__host__ __device__ constexpr uint32_t instr_desc(bool b_mn) {
  return (1u << 4) | ((b_mn ? 1u : 0u) << 16) | ((128u >> 3) << 17) | ((128u >> 4) << 24);
}

// ---------------------------------------------------------------------------
// Items
// ---------------------------------------------------------------------------

// What one row tile of a sequence sees: key tiles 0 .. n_sink - 1, then from
// first on; n of them in all.
struct Span {
  int L, p0, p1;    // positions of the first and last valid row (p1 may be < 0)
  int lo;           // first token of the window of the first row
  int n_sink, first, n;
  __device__ __forceinline__ int tile(int i) const { return i < n_sink ? i : first + i - n_sink; }
};

__device__ __forceinline__ Span span_of(const Params& p, int bl, int tile) {
  Span s;
  const int gq = p.d.gq, tr = kTile << p.streams_rows;
  s.L = p.cache.seq_len[p.c.batch_begin + bl];
  const int r0 = tile * tr, r1 = min(r0 + tr, p.c.n_q * gq) - 1;
  s.p0 = s.L - p.c.n_q + r0 / gq;
  s.p1 = s.L - p.c.n_q + r1 / gq;
  s.lo = p.c.window ? max(0, max(s.p0, 0) - p.c.window + 1) : 0;
  s.first = s.lo / kTile;
  s.n_sink = p.c.window ? min((p.c.sinks + kTile - 1) / kTile, s.first) : 0;
  s.n = s.n_sink + max(s.p1, 0) / kTile - s.first + 1;
  return s;
}

// The items of this CTA's share of the units, in order; every role walks them.
struct Walk {
  long long u, end, base;  // next unit, end of the share, first unit of the item
  int group, head, step;   // group = sequence * tiles + row tile
  Span s;
  int i0, i1;              // the item's units in this share
  __device__ __forceinline__ void begin(const Smem& sm, long long u0, long long u1) {
    u = u0;
    end = u1;
    group = sm.start_group;
    head = sm.start_head;
    step = sm.start_step;
    base = u0 - step;
  }
  __device__ __forceinline__ bool next(const Params& p) {
    if (u >= end) return false;
    s = span_of(p, group / p.tiles, group % p.tiles);
    i0 = step;
    i1 = (int)min((long long)s.n, step + (end - u));
    return true;
  }
  __device__ __forceinline__ void advance(const Params& p) {
    u += i1 - i0;
    base += s.n;
    step = 0;
    if (++head == p.d.hkv) {
      head = 0;
      ++group;
    }
  }
};

// ---------------------------------------------------------------------------
// Codes to fp16 tiles
// ---------------------------------------------------------------------------

// Position of token (channel) t of an 8-run in the order 0 4 1 5 2 6 3 7.
__device__ __forceinline__ int run_pos(int t) { return t < 4 ? 2 * t : 2 * t - 7; }

// Byte address of 16-byte chunk `chunk` of row `row` in half `half`.
__device__ __forceinline__ uint32_t tile_at(int half, int row, int chunk) {
  return half * kHalfBytes + row * 128 + ((chunk ^ (row & 7)) << 4);
}
__device__ __forceinline__ void st16(unsigned char* tile, uint32_t off, uint4 v) {
  *reinterpret_cast<uint4*>(tile + off) = v;
}

// Elements 8k .. 8k + 7 of a group of B-bit codes (B >= 2) as zero + scale *
// code, one rounding, in the run order.  A code k bits up in the mantissa of
// 1024 reads 1024 + 2^k code; the next product with 2^-k is exact.
template <int B>
__device__ __forceinline__ uint4 restore8(const uint32_t (&w)[B], int k, __half2 s, __half2 z) {
  uint32_t r[4];
  if constexpr (B == 8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t x = __byte_perm(w[2 * k], w[2 * k + 1], 0x0400 + i * 0x0101);
      const __half2 c = __hsub2(as_half2(((x & 0x00ff00ffu)) | 0x64006400u), __float2half2_rn(1024.0f));
      r[i] = as_u32(__hfma2(c, s, z));
    }
  } else if constexpr (B == 4) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t x = i < 2 ? w[k] : w[k] >> 8;
      const uint32_t y = (x & (i & 1 ? 0x00f000f0u : 0x000f000fu)) | 0x64006400u;
      const __half2 c = __hfma2(as_half2(y), __float2half2_rn(i & 1 ? 0.0625f : 1.0f),
                                __float2half2_rn(i & 1 ? -64.0f : -1024.0f));
      r[i] = as_u32(__hfma2(c, s, z));
    }
  } else {
    const uint32_t x = __byte_perm(w[k >> 1], 0u, (k & 1) ? 0x4342 : 0x4140);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t y = (x & (0x00030003u << (2 * i))) | 0x64006400u;
      const float f = 1.0f / (1 << (2 * i));
      const __half2 c = __hfma2(as_half2(y), __float2half2_rn(f), __float2half2_rn(-1024.0f * f));
      r[i] = as_u32(__hfma2(c, s, z));
    }
  }
  return make_uint4(r[0], r[1], r[2], r[3]);
}

// Queries and 1-bit keys: byte offset of channels 4x .. 4x + 3 (x = 4 ks + tig
// of the page's channel split) of a row in the permuted contraction order.
// Channel c = 16 ks + 4 tig + i goes to half tig / 2, chunk (tig mod 2) * 4 +
// (ks / 2, its bit 1 flipped in the second half), 8-byte part ks mod 2: a
// lane's codes of one token fill 64 contiguous bytes, and the eight lanes of a
// store phase hit eight different banks.
__device__ __forceinline__ uint32_t q1_offset(int row, int x) {
  const int ks = x >> 2, tig = x & 3, half = tig >> 1;
  return tile_at(half, row, (tig & 1) * 4 + ((ks >> 1) ^ (half << 1))) + (ks & 1) * 8;
}
// A row's 16-byte chunk m (channels 8m .. 8m + 7).
template <int BK>
__device__ __forceinline__ void put_key_row(unsigned char* tile, int row, int m, uint4 v) {
  if constexpr (BK == 1) {
    *reinterpret_cast<uint2*>(tile + q1_offset(row, 2 * m)) = make_uint2(v.x, v.y);
    *reinterpret_cast<uint2*>(tile + q1_offset(row, 2 * m + 1)) = make_uint2(v.z, v.w);
  } else {
    st16(tile, tile_at(m >> 3, row, m & 7), v);
  }
}
// 8 fp16 numbers in the run order.
__device__ __forceinline__ uint4 run_order(uint4 v) {
  return make_uint4(__byte_perm(v.x, v.z, 0x5410), __byte_perm(v.x, v.z, 0x7632),
                    __byte_perm(v.y, v.w, 0x5410), __byte_perm(v.y, v.w, 0x7632));
}
// Row of the value tile (channel-major, 1-bit) that holds channel c.
__device__ __forceinline__ int value_row(int c) { return (c & ~7) + run_pos(c & 7); }

// A packed block's codes and scales on their way to a tile (registers).
// 1-bit: 16 bytes of codes and the pairs of scales and zeros they meet;
// others: four groups of B words with a scale and a zero each.
template <int B>
struct Codes {
  uint32_t w[4][B];
  uint32_t sz[4];
};
template <>
struct Codes<1> {
  uint32_t w[4];
  uint32_t s[16], z[16];
};

template <int B, bool kKey>
__device__ __forceinline__ void load_codes(Codes<B>& c, const char* codes, const __half* meta) {
  const int lane = threadIdx.x & 31;
  if constexpr (B == 1) {
    const uint4 w = __ldg(reinterpret_cast<const uint4*>(codes) + lane);
    c.w[0] = w.x, c.w[1] = w.y, c.w[2] = w.z, c.w[3] = w.w;
    if constexpr (kKey) {
      const int tig = lane & 3;
#pragma unroll
      for (int ks = 0; ks < 8; ++ks) {
        const uint2 a = __ldg(reinterpret_cast<const uint2*>(meta + 16 * ks + 4 * tig));
        const uint2 b = __ldg(reinterpret_cast<const uint2*>(meta + kHeadDim + 16 * ks + 4 * tig));
        c.s[2 * ks] = a.x, c.s[2 * ks + 1] = a.y;
        c.z[2 * ks] = b.x, c.z[2 * ks + 1] = b.y;
      }
    } else {
      const int tig = lane & 3;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const uint4 a = __ldg(reinterpret_cast<const uint4*>(meta + 32 * g + 8 * tig));
        const uint4 b = __ldg(reinterpret_cast<const uint4*>(meta + kHeadDim + 32 * g + 8 * tig));
        c.s[4 * g] = a.x, c.s[4 * g + 1] = a.y, c.s[4 * g + 2] = a.z, c.s[4 * g + 3] = a.w;
        c.z[4 * g] = b.x, c.z[4 * g + 1] = b.y, c.z[4 * g + 2] = b.z, c.z[4 * g + 3] = b.w;
      }
    }
  } else {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const char* src = codes + (32 * g + lane) * (4 * B);
      if constexpr (B == 2) {
        const uint2 a = __ldg(reinterpret_cast<const uint2*>(src));
        c.w[g][0] = a.x, c.w[g][1] = a.y;
      } else {
#pragma unroll
        for (int i = 0; i < B / 4; ++i) {
          const uint4 a = __ldg(reinterpret_cast<const uint4*>(src) + i);
          c.w[g][4 * i] = a.x, c.w[g][4 * i + 1] = a.y;
          c.w[g][4 * i + 2] = a.z, c.w[g][4 * i + 3] = a.w;
        }
      }
      const int mi = kKey ? 32 * g + lane : vmeta_index(g, lane);
      const __half2 sz = __halves2half2(meta[mi], meta[kHeadDim + mi]);
      c.sz[g] = as_u32(sz);
    }
  }
}

// The block's part of a tile: tokens 32 j .. 32 j + 31 of its 128.
template <int B, bool kKey>
__device__ __forceinline__ void restore_block(const Codes<B>& c, unsigned char* tile, int j) {
  const int lane = threadIdx.x & 31;
  if constexpr (B == 1) {
    const int gid = lane >> 2, tig = lane & 3;
    if constexpr (kKey) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        __half2 s[4];
#pragma unroll
        for (int r = 0; r < 4; ++r)
          s[r] = __hmul2(as_half2(c.s[4 * k + r]), __float2half2_rn(0.5f));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t o[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            // the token's two codes at bits 14 and 30: 0 or 2.0
            const uint32_t x = __funnelshift_l(c.w[k], c.w[k], 4 * r + 4 - i) & 0x40004000u;
            o[r] = as_u32(__hfma2(as_half2(x), s[r], as_half2(c.z[4 * k + r])));
          }
          const int t = 4 * gid + i, row = 32 * j + (t & 24) + run_pos(t & 7), half = tig >> 1;
          st16(tile, tile_at(half, row, (tig & 1) * 4 + (k ^ (half << 1))),
               make_uint4(o[0], o[1], o[2], o[3]));
        }
      }
    } else {
      const int flip = (gid & 1) << 1;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        __half2 s[4];
#pragma unroll
        for (int r = 0; r < 4; ++r)
          s[r] = __hmul2(as_half2(c.s[4 * g + r]), __float2half2_rn(0.5f));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int ch = i ^ flip;  // so that a store phase meets eight banks
          const uint32_t w = __funnelshift_l(c.w[g], c.w[g], 4 - ch);
          uint32_t o[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const uint32_t x = __funnelshift_l(w, w, 4 * r) & 0x40004000u;
            o[r] = as_u32(__hfma2(as_half2(x), s[r], as_half2(c.z[4 * g + r])));
          }
          st16(tile, tile_at(j >> 1, 32 * g + 8 * (gid >> 1) + 2 * ch + (gid & 1), (j & 1) * 4 + tig),
               make_uint4(o[0], o[1], o[2], o[3]));
        }
      }
    }
  } else {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const __half2 s = __low2half2(as_half2(c.sz[g])), z = __high2half2(as_half2(c.sz[g]));
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint4 v = restore8<B>(c.w[g], k, s, z);
        if constexpr (kKey) {
          st16(tile, tile_at(j >> 1, 32 * g + lane, (j & 1) * 4 + k), v);
        } else {
          const int row = 32 * j + (lane & 24) + run_pos(lane & 7);
          st16(tile, tile_at(g >> 1, row, (g & 1) * 4 + k), v);
        }
      }
    }
  }
}

// The same for a block of the fp16 window, whose token t is at rows + slot *
// 128, slot = (t0 + t) mod ring; tokens from `valid` on are zero.
template <int B, bool kKey>
__device__ __noinline__ void window_block(const __half* rows, int t0, int ring, int valid,
                                          unsigned char* tile, int j) {
  const int lane = threadIdx.x & 31;
  if constexpr ((B == 1) == kKey) {  // rows of the tile are tokens
    const int row = 32 * j + (lane & 24) + run_pos(lane & 7);
    const uint4* src =
        reinterpret_cast<const uint4*>(rows + (long long)((t0 + lane) % ring) * kHeadDim);
#pragma unroll 4
    for (int m = 0; m < 16; ++m) {
      const uint4 v = lane < valid ? src[m] : make_uint4(0u, 0u, 0u, 0u);
      if constexpr (kKey) put_key_row<1>(tile, row, m, v);
      else st16(tile, tile_at(m >> 3, row, m & 7), run_order(v));
    }
  } else {  // rows are channels
    const unsigned short* src = reinterpret_cast<const unsigned short*>(rows);
    for (int g = 0; g < 4; ++g) {
      const int c = 32 * g + lane, row = kKey ? c : value_row(c);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        uint32_t x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int t = 8 * k + i;
          x[i] = t < valid ? src[(long long)((t0 + t) % ring) * kHeadDim + c] : 0u;
        }
        st16(tile, tile_at(j >> 1, row, (j & 1) * 4 + k),
             make_uint4(x[0] | x[4] << 16, x[1] | x[5] << 16, x[2] | x[6] << 16, x[3] | x[7] << 16));
      }
    }
  }
}
template <int B, bool kKey>
__device__ __noinline__ void zero_block(unsigned char* tile, int j) {
  const int lane = threadIdx.x & 31;
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
  if constexpr ((B == 1) == kKey) {
    for (int m = 0; m < 16; ++m) st16(tile, tile_at(m >> 3, 32 * j + lane, m & 7), zero);
  } else {
    for (int i = 0; i < 16; ++i)
      st16(tile, tile_at(j >> 1, 32 * (i >> 2) + lane, (j & 1) * 4 + (i & 3)), zero);
  }
}

// A loading warp: block j of every key (or value) tile of the CTA's share.
template <int B, bool kKey>
__device__ __forceinline__ void load_role(const Params& p, Smem& s, long long u0, long long u1,
                                          int j) {
  const int lane = threadIdx.x & 31;
  unsigned char(*tiles)[kTileBytes] = kKey ? s.k : s.v;
  uint64_t* full = kKey ? s.k_full : s.v_full;
  uint64_t* empty = kKey ? s.k_empty : s.v_empty;
  uint32_t n = 0;
  Walk w;
  w.begin(s, u0, u1);
  for (; w.next(p); w.advance(p)) {
    const int b = p.c.batch_begin + w.group / p.tiles;
    const PageMap pm = page_map(p.d, p.cache, b, w.head);
    const __half* rows =
        reinterpret_cast<const __half*>(kKey ? p.cache.k_resid : p.cache.v_resid) +
        ((long long)b * p.d.hkv + w.head) * p.d.ring * kHeadDim;
    const int lq = packed_len(w.s.L, p.d.residual);
    const int codes = kKey ? 0 : page_off_vcodes(p.d.bits_k);
    const int meta = kKey ? page_off_kmeta(p.d.bits_k) : page_off_vmeta(p.d.bits_k, p.d.bits_v);
    // the block of unit i, by kind: 0 nothing to see, 1 packed, 2 window
    const auto kind_of = [&](int t0) {
      const bool seen = t0 <= w.s.p1 && (t0 + kGroup > w.s.lo || t0 < p.c.sinks);
      return !seen ? 0 : t0 < lq ? 1 : 2;
    };
    Codes<B> c;
    const auto fetch = [&](int i) {
      const int t0 = w.s.tile(i) * kTile + j * kGroup;
      int kind = kind_of(t0);
      if (kind == 1) {
        const char* page = pm.at(t0 / kGroup);
        if (page) {
          load_codes<B, kKey>(c, page + codes, reinterpret_cast<const __half*>(page + meta));
        } else {
          kind = 0;
          if (lane == 0)
            atomicOr(reinterpret_cast<unsigned*>(p.cache.seq_len + p.d.batch), KVQ_FLAG_BAD_PAGE);
        }
      }
      return kind;
    };
    int kind = fetch(w.i0);
    for (int i = w.i0; i < w.i1; ++i, ++n) {
      const int buf = n & 1;
      if (!warp_wait(s, &empty[buf], ((n >> 1) & 1) ^ 1)) return;
      const int t0 = w.s.tile(i) * kTile + j * kGroup;
      if (kind == 1) restore_block<B, kKey>(c, tiles[buf], j);
      else if (kind == 2)
        window_block<B, kKey>(rows, t0, p.d.ring, w.s.L - t0, tiles[buf], j);
      else
        zero_block<B, kKey>(tiles[buf], j);
      fence_async();
      __syncwarp();
      if (lane == 0) bar_arrive(&full[buf]);
      if (i + 1 < w.i1) kind = fetch(i + 1);
    }
  }
}

// ---------------------------------------------------------------------------
// Products
// ---------------------------------------------------------------------------

constexpr uint32_t kColS = 0, kColO = 256;  // tensor memory columns: S0 S1 O0 O1, 128 each

template <int BK, int BV>
__device__ __forceinline__ void mma_role(const Params& p, Smem& s, long long u0, long long u1) {
  constexpr uint32_t kIdS = instr_desc(BK != 1), kIdO = instr_desc(BV != 1);
  const uint32_t tm = s.tmem;
  uint32_t nk = 0, nv = 0, ns[2] = {0, 0}, items = 0;
  const int two = p.streams_rows;  // a key tile serves two steps
  Walk w;
  w.begin(s, u0, u1);
  for (; w.next(p); w.advance(p), ++items) {
    const int steps = (w.i1 - w.i0) << two;
    if (!bar_wait(s, &s.q_full, items & 1)) return;
    tc_after();
    const auto scores = [&](int st) {
      const int x = st & 1, buf = nk & 1;
      if (!two || x == 0) {
        if (!bar_wait(s, &s.k_full[buf], (nk >> 1) & 1)) return false;
        tc_after();
      }
      const uint64_t a = tile_desc(sptr(s.q[two ? x : 0]), false),
                     b = tile_desc(sptr(s.k[buf]), BK != 1);
#pragma unroll
      for (int ks = 0; ks < 8; ++ks)
        mma_ss(tm + kColS + 128 * x, a + step_major_k(ks),
               b + (BK == 1 ? step_major_k(ks) : step_major_mn(ks)), kIdS, ks > 0);
      tc_commit(&s.s_full[x]);
      if (!two || x == 1) {
        tc_commit(&s.k_empty[buf]);
        ++nk;
      }
      return true;
    };
    if (!scores(0)) return;
    if (steps > 1 && !scores(1)) return;
    for (int st = 0; st < steps; ++st) {
      const int x = st & 1, buf = nv & 1;
      if (!bar_wait(s, &s.p_ready[x], ns[x] & 1)) return;
      ++ns[x];
      if ((!two || x == 0) && !bar_wait(s, &s.v_full[buf], (nv >> 1) & 1)) return;
      tc_after();
      const uint64_t b = tile_desc(sptr(s.v[buf]), BV != 1);
#pragma unroll
      for (int ks = 0; ks < 8; ++ks)
        mma_ts(tm + kColO + 128 * x, tm + kColS + 128 * x + 8 * ks,
               b + (BV == 1 ? step_major_k(ks) : step_major_mn(ks)), kIdO, st > 1 || ks > 0);
      if (!two || x == 1) {
        tc_commit(&s.v_empty[buf]);
        ++nv;
      }
      if (st + 2 >= steps) tc_commit(&s.o_full[x]);
      else if (!scores(st + 2)) return;
    }
  }
}

// ---------------------------------------------------------------------------
// Softmax, results
// ---------------------------------------------------------------------------

// Column n of a key tile holds token 8 (n / 8) + run_token(n mod 8).
__host__ __device__ constexpr int run_token(int n) { return (n & 1) * 4 + (n >> 1); }

struct Row {
  float m, l;    // running maximum (of scores times scale, log2 domain) and sum
};

template <int BK>
__device__ __forceinline__ void load_queries(const Params& p, const __half* src,
                                             unsigned char* tile, int row) {
  (void)p;
  const uint4* q = reinterpret_cast<const uint4*>(src);
#pragma unroll
  for (int m = 0; m < 16; ++m)
    put_key_row<BK>(tile, row, m, src ? q[m] : make_uint4(0u, 0u, 0u, 0u));
}

// Scores at columns [32 c, 32 c + 32) of the thread's row, masked: column n is
// seen when its token (less the tile's first) is at most hi and above lo, or
// below sink.
__device__ __forceinline__ void mask32(uint32_t (&r)[32], int c, int hi, int lo, int sink) {
#pragma unroll
  for (int n = 0; n < 32; ++n) {
    const int t = 32 * c + (n & ~7) + run_token(n & 7);
    if (t > hi || (t <= lo && t >= sink)) r[n] = 0xff800000u;
  }
}

// One step of a stream's softmax for a row (a thread); `first`: no accumulator
// yet.
__device__ __forceinline__ void softmax_step(uint32_t ts, uint32_t to, float sl2, bool first,
                                             bool masked, int hi, int lo, int sink, Row& row) {
  float mx = -INFINITY;
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    uint32_t r[32];
    tm_load32(ts + 32 * c, r);
    tm_load_wait();
    if (masked) mask32(r, c, hi, lo, sink);
#pragma unroll
    for (int n = 0; n < 32; ++n) mx = fmaxf(mx, __uint_as_float(r[n]));
  }
  mx *= sl2;
  if (first) {
    row.m = mx;
    row.l = 0.0f;
  } else {
    const bool up = mx > row.m + kRescaleLog2;
    if (__any_sync(0xffffffffu, up)) {
      const float f = up ? exp2_fast(row.m - mx) : 1.0f;
      if (up) row.m = mx;
      row.l *= f;
#pragma unroll 1
      for (int c = 0; c < 4; ++c) {
        uint32_t r[32];
        tm_load32(to + 32 * c, r);
        tm_load_wait();
#pragma unroll
        for (int n = 0; n < 32; ++n) r[n] = __float_as_uint(__uint_as_float(r[n]) * f);
        tm_store32(to + 32 * c, r);
      }
    }
  }
  const float off = row.m == -INFINITY ? 0.0f : -row.m;
  float l0 = 0.0f, l1 = 0.0f;
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    uint32_t r[32], h[16];
    tm_load32(ts + 32 * c, r);
    tm_load_wait();
    if (masked) mask32(r, c, hi, lo, sink);
#pragma unroll
    for (int n = 0; n < 16; ++n) {
      const float a = exp2_fast(fmaf(__uint_as_float(r[2 * n]), sl2, off));
      const float b = exp2_fast(fmaf(__uint_as_float(r[2 * n + 1]), sl2, off));
      l0 += a;
      l1 += b;
      h[n] = pack_half2(a, b);
    }
    tm_store16(ts + 16 * c, h);
  }
  row.l += l0 + l1;
  tm_store_wait();
}

// Write 32 accumulator columns times f: fp16 results or fp32 partials, in
// channel order.
__device__ __forceinline__ void put_half(__half* dst, int c, const float (&o)[32]) {
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      // channels 2i and 2i + 1 of the run
      const int a = 2 * i < 4 ? 4 * i : 4 * i - 7;
      w[i] = pack_half2(o[8 * g + a], o[8 * g + a + 2]);
    }
    *reinterpret_cast<uint4*>(dst + 32 * c + 8 * g) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}
__device__ __forceinline__ void put_float(float* dst, int c, const float (&o)[32]) {
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const float* x = o + 8 * g;
    *reinterpret_cast<float4*>(dst + 32 * c + 8 * g) = make_float4(x[0], x[2], x[4], x[6]);
    *reinterpret_cast<float4*>(dst + 32 * c + 8 * g + 4) = make_float4(x[1], x[3], x[5], x[7]);
  }
}

template <int BK>
__device__ __forceinline__ void softmax_role(const Params& p, Smem& s, long long u0, long long u1,
                                             long long total, long long n_cta) {
  const int warp = threadIdx.x >> 5, x = warp >> 2, lane_row = threadIdx.x & 127;
  const uint32_t lanes = (uint32_t)(warp & 3) << 21;  // 32 lanes a warp, in bits 16 up
  const uint32_t ts = s.tmem + lanes + kColS + 128 * x, to = s.tmem + lanes + kColO + 128 * x;
  const int two = p.streams_rows, tr = kTile << two, rows = p.c.n_q * p.d.gq, gq = p.d.gq;
  uint32_t ns = 0, no[2] = {0, 0}, met = 0;
  Walk w;
  w.begin(s, u0, u1);
  for (; w.next(p); w.advance(p)) {
    const int bl = w.group / p.tiles, tile = w.group % p.tiles;
    const int tr_row = (two ? kTile * x : 0) + lane_row;  // row in the item
    const int g = tile * tr + tr_row;
    const bool valid = g < rows;
    const int t = g / gq, head = w.head * gq + g % gq;
    const int pos = w.s.L - p.c.n_q + t;
    if (two || x == 0) {
      const long long off = bl * p.c.q_stride[0] + t * p.c.q_stride[1] + head * p.c.q_stride[2];
      load_queries<BK>(p, valid ? p.q + off : nullptr, s.q[x], lane_row);
      fence_async();
      bar_arrive(&s.q_full);
    }
    const bool live = __any_sync(0xffffffffu, valid);
    Row row{-INFINITY, 0.0f};
    const int n = w.i1 - w.i0;
    bool first = true;
    for (int i = two ? 0 : x; i < n; i += two ? 1 : 2, ++ns, first = false) {
      if (!warp_wait(s, &s.s_full[x], ns & 1)) return;
      tc_after();
      if (live) {
        const int t0 = w.s.tile(w.i0 + i) * kTile;
        // every token of the tile is seen by every row of the item
        const bool whole = w.s.p0 >= t0 + kTile - 1 &&
                           (!p.c.window || t0 > w.s.p1 - p.c.window || t0 + kTile <= p.c.sinks);
        softmax_step(ts, to, p.c.scale_log2, first, !whole, (valid ? pos : -1) - t0,
                     p.c.window ? pos - p.c.window - t0 : -1 - t0, p.c.sinks - t0, row);
      }
      tc_before();
      bar_arrive(&s.p_ready[x]);
    }
    // both accumulators complete (a stream without a step has none)
    const bool has1 = two || n > 1;
    if (x == 0 || two) {
      if (!warp_wait(s, &s.o_full[x], no[x] & 1)) return;
    }
    if (!two && x == 0 && has1 && !warp_wait(s, &s.o_full[1], no[1] & 1)) return;
    if (two) ++no[x];
    else {
      ++no[0];
      if (has1) ++no[1];
    }
    tc_after();
    if (!two && x == 1) {
      s.m[lane_row] = row.m;
      s.l[lane_row] = row.l;
    }
    if (!two && !meet_softmax(s, met)) return;
    const bool direct = w.i0 == 0 && w.i1 == w.s.n;
    const int slot = 2 * blockIdx.x + (w.u == u0 ? 0 : 1);
    if ((two || x == 0) && live) {
      float f0 = 1.0f, f1 = 0.0f, m = row.m, l = row.l;
      if (!two && has1) {
        const float m1 = s.m[lane_row], l1 = s.l[lane_row];
        m = fmaxf(row.m, m1);
        if (m > -INFINITY) {
          f0 = exp2_fast(row.m - m);
          f1 = exp2_fast(m1 - m);
        }
        l = row.l * f0 + l1 * f1;
      }
      const float scale = direct ? (l > 0.0f ? 1.0f / l : 0.0f) : 1.0f;
      f0 *= scale;
      f1 *= scale;
      const long long off =
          bl * p.c.out_stride[0] + t * p.c.out_stride[1] + head * p.c.out_stride[2];
      const long long pr = (long long)slot * tr + tr_row;
#pragma unroll 1
      for (int c = 0; c < 4; ++c) {
        uint32_t r[32];
        float o[32];
        __syncwarp();
        tm_load32(to + 32 * c, r);
        tm_load_wait();
#pragma unroll
        for (int k = 0; k < 32; ++k) o[k] = __uint_as_float(r[k]) * f0;
        if (!two && has1) {
          tm_load32(to + 128 + 32 * c, r);
          tm_load_wait();
#pragma unroll
          for (int k = 0; k < 32; ++k) o[k] = fmaf(__uint_as_float(r[k]), f1, o[k]);
        }
        if (valid) {
          if (direct) put_half(p.out + off, c, o);
          else put_float(p.part_o + pr * kHeadDim, c, o);
        }
      }
      if (valid && !direct) p.part_ml[pr] = make_float2(m, l);
      tc_before();
    }
    if (!direct) {
      // the last of the item's CTAs merges its partials, in the order of the
      // tokens
      const long long a = w.base, z = w.base + w.s.n - 1;
      const int c0 = (int)(((a + 1) * n_cta - 1) / total), c1 = (int)(((z + 1) * n_cta - 1) / total);
      const long long item = (long long)w.group * p.d.hkv + w.head;
      __threadfence();
      if (!meet_softmax(s, met)) return;
      if (threadIdx.x == 0) {
        s.last = atomicAdd(&p.tickets[item], 1u) == (unsigned)(c1 - c0);
        __threadfence();
      }
      if (!meet_softmax(s, met)) return;
      if (s.last) {
        if (threadIdx.x == 0) p.tickets[item] = 0u;
        const int n_rows = min(tr, rows - tile * tr);
        // a CTA's slot 0 holds the item its share begins in
        const auto slot_of = [&](int c) { return 2 * c + (c * total / n_cta < a ? 1 : 0); };
        for (int r = threadIdx.x >> 5; r < n_rows; r += kSoftmaxWarps) {
          const int ch = 4 * (threadIdx.x & 31);
          float m = -INFINITY, l = 0.0f;
          float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
          for (int c = c0; c <= c1; ++c) {
            const long long pr = (long long)slot_of(c) * tr + r;
            const float2 ml = __ldcg(&p.part_ml[pr]);
            if (!(ml.y > 0.0f)) continue;
            const float4 v = __ldcg(reinterpret_cast<const float4*>(p.part_o + pr * kHeadDim + ch));
            const float mm = fmaxf(m, ml.x), fa = exp2_fast(m - mm), fb = exp2_fast(ml.x - mm);
            m = mm;
            l = l * fa + ml.y * fb;
            o.x = o.x * fa + v.x * fb;
            o.y = o.y * fa + v.y * fb;
            o.z = o.z * fa + v.z * fb;
            o.w = o.w * fa + v.w * fb;
          }
          const float f = l > 0.0f ? 1.0f / l : 0.0f;
          const int gr = tile * tr + r, tt = gr / gq, hh = w.head * gq + gr % gq;
          __half* dst = p.out + bl * p.c.out_stride[0] + tt * p.c.out_stride[1] +
                        hh * p.c.out_stride[2] + ch;
          *reinterpret_cast<uint2*>(dst) =
              make_uint2(pack_half2(o.x * f, o.y * f), pack_half2(o.z * f, o.w * f));
        }
      }
    }
    if (!meet_softmax(s, met)) return;  // s.m, s.last and both accumulators may be written again
  }
}

// ---------------------------------------------------------------------------
// Kernel
// ---------------------------------------------------------------------------

template <int BK, int BV>
__global__ void __launch_bounds__(kThreads, 1) chunk_attn_kernel(const __grid_constant__ Params p) {
  extern __shared__ __align__(1024) unsigned char raw[];
  Smem& s = *reinterpret_cast<Smem*>(raw);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  // Units of every (sequence, row tile), summed over the threads in order.
  const int groups = p.c.batch_count * p.tiles;
  const int per = (groups + kThreads - 1) / kThreads;
  const int g0 = min(groups, tid * per), g1 = min(groups, g0 + per);
  long long mine = 0;
  for (int g = g0; g < g1; ++g) mine += (long long)span_of(p, g / p.tiles, g % p.tiles).n * p.d.hkv;
  long long inc = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += y;
  }
  if (lane == 31) s.scan[warp] = inc;
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      bar_init(&s.k_full[i], 4);
      bar_init(&s.v_full[i], 4);
      bar_init(&s.k_empty[i], 1);
      bar_init(&s.v_empty[i], 1);
      bar_init(&s.s_full[i], 1);
      bar_init(&s.p_ready[i], kTile);
      bar_init(&s.o_full[i], 1);
    }
    bar_init(&s.q_full, kTile << p.streams_rows);
    bar_init(&s.meet, 32 * kSoftmaxWarps);
    bar_init(&s.drained, 1);
    s.abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  long long before = 0, total = 0;
  for (int i = 0; i < kThreads / 32; ++i) {
    if (i < warp) before += s.scan[i];
    total += s.scan[i];
  }
  before += inc - mine;
  const long long n_cta = min((long long)gridDim.x, total);
  if (blockIdx.x >= n_cta) return;  // fewer units than CTAs
  const long long u0 = blockIdx.x * total / n_cta, u1 = (blockIdx.x + 1) * total / n_cta;
  if (before <= u0 && u0 < before + mine) {
    long long at = before;
    for (int g = g0; g < g1; ++g) {
      const int n = span_of(p, g / p.tiles, g % p.tiles).n;
      if (u0 < at + (long long)n * p.d.hkv) {
        s.start_group = g;
        s.start_head = (int)((u0 - at) / n);
        s.start_step = (int)((u0 - at) % n);
        break;
      }
      at += (long long)n * p.d.hkv;
    }
  }
  if (warp == kSoftmaxWarps + kLoadWarps) {
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
    softmax_role<BK>(p, s, u0, u1, total, n_cta);
  } else if (warp < kSoftmaxWarps + 4) {
    load_role<BK, true>(p, s, u0, u1, warp - kSoftmaxWarps);
  } else if (warp < kSoftmaxWarps + 8) {
    load_role<BV, false>(p, s, u0, u1, warp - kSoftmaxWarps - 4);
  } else {
    if (lane == 0) {
      mma_role<BK, BV>(p, s, u0, u1);
      if (*reinterpret_cast<volatile int*>(&s.abort)) {
        // products in flight end before the tile memory is given back
        tc_commit(&s.drained);
        const long long t0 = clock64();
        while (!bar_try(&s.drained, 0) && clock64() - t0 < kWaitLimit) {
        }
        atomicOr(reinterpret_cast<unsigned*>(p.cache.seq_len + p.d.batch), KVQ_FLAG_WAIT_TIMEOUT);
      }
    }
    __syncwarp();
  }
  tc_before();
  __syncthreads();
  tc_after();
  if (warp == kSoftmaxWarps + kLoadWarps)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tm));
}

template <int BK, int BV>
cudaError_t launch_widths(const Params& p, int ctas, cudaStream_t stream) {
  const cudaError_t e =
      cudaFuncSetAttribute(chunk_attn_kernel<BK, BV>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                           (int)sizeof(Smem));
  if (e != cudaSuccess) return e;
  chunk_attn_kernel<BK, BV><<<ctas, kThreads, sizeof(Smem), stream>>>(p);
  return cudaGetLastError();
}

template <int BK>
cudaError_t launch_key_width(const Params& p, int ctas, cudaStream_t stream) {
  switch (p.d.bits_v) {
    case 1: return launch_widths<BK, 1>(p, ctas, stream);
    case 2: return launch_widths<BK, 2>(p, ctas, stream);
    case 4: return launch_widths<BK, 4>(p, ctas, stream);
    default: return launch_widths<BK, 8>(p, ctas, stream);
  }
}

// chunk_k*.cu
cudaError_t launch_k1(const Params& p, int ctas, cudaStream_t stream);
cudaError_t launch_k2(const Params& p, int ctas, cudaStream_t stream);
cudaError_t launch_k4(const Params& p, int ctas, cudaStream_t stream);
cudaError_t launch_k8(const Params& p, int ctas, cudaStream_t stream);

}  // namespace chunk
}  // namespace kvq
