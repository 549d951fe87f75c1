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
// row, maximum, sum) in the workspace; a second, small kernel (chunk.cu) joins
// them in the order of the tokens, so results repeat bit for bit.
//
// A CTA.  Per step (128 rows, half a key tile of 64 tokens): S = Q K^T (fp16
// operands in shared memory, fp32 in tensor memory), softmax by the four warps
// that own the 128 lanes of S (a thread per row), P as fp16 over the same
// tensor memory columns, O += P V with P read from tensor memory.  Two such
// streams of steps alternate: two row tiles on the same key tiles, or (items of
// at most 128 rows) the two halves of the key tiles, joined at the end.  Each
// stream has two buffers of scores, so a softmax does not wait for the products
// around it: with steps of 128 tokens and one buffer, a step's chain of score
// product, softmax and value product set the pace.
//   warps 0-3, 4-7  softmax of streams 0 and 1, queries in, results out
//   warps 8-11      keys: one 32-token block each, codes -> fp16 tile
//   warps 12-15     values, the same
//   warps 16, 17    issue the products of streams 0 and 1 (18, 19 idle)
// The running maximum of a row moves only when a score is more than 8 (in log2)
// above it, so the accumulator is rescaled rarely; weights are written with a factor
// of 2^7 and stay at or below 2^15.
//
// What bounds it.  A prompt chunk: the tensor cores by count (4 * 128 flops a
// query, visible key and head), measured the chain around them: 1.23 PFLOP/s of a
// cuBLAS product's 1.92 for a chunk of 2048 tokens over 64k (K1V1, groups of 5,
// 2.2 ms).  Counters of chunks over 4k at 1, 2 and 4 bits: the tensor pipe 34 to 41%
// of the active cycles, issue slots 52 to 60, no unit full; warps wait for loads and
// for one another.  Few rows over a long cache: the restoring of every code into a
// whole tile, whatever the rows that use it (four drafts in 16 sequences of 8k to 32k,
// K2V2: 212 us, 1.6 us a tile and SM), where the bytes take 39.  The smallest calls:
// the chain of launch, lengths, first tile, partials and their join, 18 to 22 us.
// Tried and dropped: products issued by a lane of a diverged warp, one warp for both
// streams' products, steps of 128 tokens with one score buffer a stream, all 128
// scores of a row in registers, a block's loads held in a second set of registers,
// the weights' sum in place of the row maximum as the sign for a new maximum.
//
// Roundings.  Operands are fp16: keys, values and weights are rounded once each, which
// leaves 3e-4 to 9e-4 of the results' rms where the rounding of exact results leaves
// 2e-4; most of it comes from keys with channels far above the others.  The scales
// cannot move to the queries, as the decode kernel has it: every 32-token block has its
// own, and one tile of queries meets them all.  The keys' low parts in a second product
// would add half to the products and 64 KB of tiles to the 215 KB in use.  Sums, maxima
// and accumulators are fp32.
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

#include "serve.cuh"

namespace kvq {
namespace chunk {

constexpr int kTile = 128;                  // tokens of a key / value tile, rows of a product
constexpr int kStep = 64;                   // tokens of a step
constexpr int kTileBytes = kTile * kHeadDim * 2;
constexpr int kHalfBytes = kTileBytes / 2;  // 64 elements of the contiguous axis
constexpr int kSoftmaxWarps = 8, kLoadWarps = 8;
constexpr int kThreads = 32 * (kSoftmaxWarps + kLoadWarps + 4);
// Registers a thread: at launch, then by role.  The loading warps' parts of 1 and
// 8 bits are the largest.  The shares must not exceed what the launch got.
constexpr int kRegsLaunch = 96, kRegsIssue = 48;
template <int BK, int BV>
struct Regs {
  static constexpr int kLoad = BK == 1 || BV == 1 || BK == 8 || BV == 8 ? 112 : 96;
  static constexpr int kSoftmax = 216 - kLoad;
  static_assert(32 * (kSoftmaxWarps * kSoftmax + kLoadWarps * kLoad + 4 * kRegsIssue) <=
                    kThreads * kRegsLaunch,
                "register shares exceed the launch's");
};
// Fixed cost of an item in units (a unit is a 128-token tile): queries in, results
// out, the first tile's way through the pipeline.
constexpr int kItemCost = 3;
constexpr uint32_t kWaitLimit = 2000000000u;  // cycles of a bounded wait (~1 s)
constexpr int kAhead = 2;  // blocks behind the next whose table entry (and L2 copy) is on its way
constexpr float kRescaleLog2 = 8.0f;
// Weights are written as 2^(score - maximum + kLiftLog2): with the maximum up to
// kRescaleLog2 behind they stay at or below 2^15, inside fp16, and keep all 11 bits
// down to 2^-21 of the maximum's, some down to 2^-32.  Without the lift a first token
// with 0.999 of the weight and no value left 4% of error in the tail of 4096 tokens.
// The sums carry the factor too, so quotients and joins need not know it.
constexpr float kLiftLog2 = 7.0f;

struct Smem {
  unsigned char q[2][kTileBytes];
  unsigned char k[2][kTileBytes];
  unsigned char v[2][kTileBytes];
  unsigned char stage[kSoftmaxWarps][32 * 64];  // results on their way out
  uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2];
  uint64_t s_full[2][2], p_ready[2][2], o_last[2], o_full[2];  // [stream][buffer], [stream]
  uint64_t q_full, meet, drained[2];
  int scan[32];
  int walk[kSoftmaxWarps][2][16];      // a softmax warp's item and the next one (Walk)
  int start_seq, start_tile, start_head, start_step;
  uint32_t tmem;
  int abort;
  float m[kTile], l[kTile];            // stream 1's statistics of a shared row tile
};

// An item that the shares of CTAs c .. last divide, left by CTA c for the kernel
// that joins the partials.
struct Split {
  int valid, inside, last, bl, row_tile, head;
};

struct Params {
  Dims d;
  kvq_cache cache;
  const __half* q;
  __half* out;
  ChunkCall c;
  int tiles;         // row tiles per (sequence, kv-head)
  uint32_t gq_inverse;  // floor(2^32 / gq) + 1
  int streams_rows;  // 1: items of 256 rows (a row tile per stream), 0: of 128
  float* part_o;     // [2 * CTAs][rows of an item][128]
  float2* part_ml;   // [2 * CTAs][rows of an item]
  Split* splits;     // [CTAs]
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
// One try, suspended for up to ~10 us in hardware: a warp that polls takes
// issue slots from the others on its scheduler.
__device__ __forceinline__ bool bar_try(uint64_t* b, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n .reg .pred p;\n"
      " mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, 10000;\n"
      " selp.u32 %0, 1, 0, p;\n}"
      : "=r"(ok)
      : "r"(sptr(b)), "r"(parity)
      : "memory");
  return ok != 0;
}
// Bounded: after the limit, or once another role has given up, it returns
// false; every role then leaves its loop.
__device__ __forceinline__ bool bar_wait(Smem& s, uint64_t* b, uint32_t parity,
                                         uint32_t limit = kWaitLimit) {
  if (bar_try(b, parity)) return true;
  const uint32_t t0 = (uint32_t)clock();
#pragma unroll 1
  while (!bar_try(b, parity)) {
    if (*reinterpret_cast<volatile int*>(&s.abort) || (uint32_t)clock() - t0 > limit) {
      *reinterpret_cast<volatile int*>(&s.abort) = 1;
      return false;
    }
  }
  return true;
}
// The same for a whole warp (all lanes leave together).
__device__ __forceinline__ bool warp_wait(Smem& s, uint64_t* b, uint32_t parity,
                                          uint32_t limit = kWaitLimit) {
  return __all_sync(0xffffffffu, bar_wait(s, b, parity, limit));
}
// One arrival for a warp, behind what all its lanes did (32 arrivals on one
// barrier are served one by one).
__device__ __forceinline__ void warp_arrive(uint64_t* b) {
  __syncwarp();
  if ((threadIdx.x & 31) == 0) bar_arrive(b);
}
// All softmax threads meet (bounded, unlike a hardware barrier).
__device__ __forceinline__ bool meet_softmax(Smem& s, uint32_t& n) {
  warp_arrive(&s.meet);
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
__device__ __forceinline__ void tc_commit(uint32_t leader, uint64_t* b) {
  asm volatile(
      "{\n .reg .pred e;\n setp.ne.b32 e, %1, 0;\n"
      " @e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}" ::"r"(
          sptr(b)),
      "r"(leader)
      : "memory");
}

// One of the warp's lanes, the same each time.
__device__ __forceinline__ uint32_t elect_lane() {
  uint32_t e;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}"
               : "=r"(e));
  return e;
}
constexpr int kIssueWarp = kSoftmaxWarps + kLoadWarps;
// All threads, once every role has left its loop.  If one gave up, whichever it was,
// the products in flight end (bounded) before tensor and shared memory are given back,
// and the flag word says so.
__device__ __forceinline__ void leave(Smem& s, int32_t* flag) {
  tc_before();
  __syncthreads();
  tc_after();
  if (!*reinterpret_cast<volatile int*>(&s.abort)) return;  // nobody writes it any more
  const int x = (int)(threadIdx.x >> 5) - kIssueWarp;
  if (x == 0 || x == 1) {
    tc_commit(elect_lane(), &s.drained[x]);
    const uint32_t t0 = (uint32_t)clock();
    while (!bar_try(&s.drained[x], 0) && (uint32_t)clock() - t0 < kWaitLimit) {
    }
  }
  if (threadIdx.x == 0) atomicOr(reinterpret_cast<unsigned*>(flag), KVQ_FLAG_WAIT_TIMEOUT);
  __syncthreads();
}

// D[128 x N] (+)= A B, fp16 in, fp32 out, K = 16, by the warp's elected lane
// (`leader`); all lanes run it, so that the descriptors stay uniform.
// A in shared memory.
__device__ __forceinline__ void mma_ss(uint32_t leader, uint32_t d, uint64_t a, uint64_t b,
                                       uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n .reg .pred p, e;\n setp.ne.b32 p, %4, 0;\n setp.ne.b32 e, %5, 0;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(acc), "r"(leader)
      : "memory");
}
// The same with A in tensor memory.
__device__ __forceinline__ void mma_ts(uint32_t leader, uint32_t d, uint32_t a, uint64_t b,
                                       uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n .reg .pred p, e;\n setp.ne.b32 p, %4, 0;\n setp.ne.b32 e, %5, 0;\n"
      " @e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(acc), "r"(leader)
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
__device__ __forceinline__ void tm_load8(uint32_t addr, uint32_t (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]),
                 "=r"(r[6]), "=r"(r[7])
               : "r"(addr));
}
__device__ __forceinline__ void tm_store8(uint32_t addr, const uint32_t (&r)[8]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};" ::"r"(r[0]),
      "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(addr)
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
// Two fp32 numbers in one 64-bit register, for the packed instructions.
__device__ __forceinline__ uint64_t pair(float a, float b) {
  uint64_t v;
  asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b));
  return v;
}
__device__ __forceinline__ void unpair(uint64_t v, float& a, float& b) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v));
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t v;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(v) : "l"(a), "l"(b), "l"(c));
  return v;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t v;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(a), "l"(b));
  return v;
}
template <int N>
__device__ __forceinline__ void regs_up() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
}
template <int N>
__device__ __forceinline__ void regs_down() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
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

// fp32 accumulator, fp16 operands, M = 128; b_mn: B's contiguous axis is N.
__host__ __device__ constexpr uint32_t instr_desc(bool b_mn, int n) {
  return (1u << 4) | ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | ((128u >> 4) << 24);
}

// ---------------------------------------------------------------------------
// Items
// ---------------------------------------------------------------------------

// Row r of an item's sequence: its token.  Rows stay below 2^28 (checked on the
// host), where the product with gq_inverse gives the exact quotient.
__device__ __forceinline__ int token_of_row(const Params& p, int r) {
  return p.d.gq == 1 ? r : (int)__umulhi((uint32_t)r, p.gq_inverse);
}

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
  s.L = p.cache.seq_len[p.c.batch_begin + bl];
  const int shift = 7 + p.streams_rows;
  const int r1 = min((tile + 1) << shift, p.c.n_q * p.d.gq) - 1;
  s.p0 = s.L - p.c.n_q + token_of_row(p, tile << shift);
  s.p1 = s.L - p.c.n_q + token_of_row(p, r1);
  s.lo = p.c.window ? max(0, max(s.p0, 0) - p.c.window + 1) : 0;
  s.first = s.lo >> 7;
  // sinks is 0 without a window; the sum passes 2^31 in the largest caches
  s.n_sink = min((int)(((uint32_t)p.c.sinks + (kTile - 1)) >> 7), s.first);
  s.n = s.n_sink + (max(s.p1, 0) >> 7) - s.first + 1;
  return s;
}

// CTA c's share of the units: [begin(c), begin(c + 1)), equal to within one.
struct Shares {
  int q, r, n;  // units = n q + r over n CTAs
  __device__ __forceinline__ int begin(int c) const { return c * q + min(c, r); }
  __device__ __forceinline__ int owner(int u) const {
    const int wide = (q + 1) * r;  // units of the CTAs that have q + 1
    return u < wide ? (int)((uint32_t)u / (uint32_t)(q + 1))
                    : r + (int)((uint32_t)(u - wide) / (uint32_t)q);
  }
};

// The items of this CTA's share of the units, in order (sequence, row tile,
// kv-head); every role walks them.
struct Walk {
  int u, end, base;        // next unit, end of the share, first unit of the item
  int bl, row_tile, head;
  Span s;
  int i0, i1;              // the item's tiles in this share
  __device__ __forceinline__ void begin(const Smem& sm, int u0, int u1) {
    u = u0;
    end = u1;
    bl = sm.start_seq;
    row_tile = sm.start_tile;
    head = sm.start_head;
    base = u0 - sm.start_step;
  }
  __device__ __forceinline__ bool next(const Params& p) {
    while (u < end) {
      s = span_of(p, bl, row_tile);
      const int local = u - base, stop = min(s.n + kItemCost, local + end - u);
      i0 = max(local - kItemCost, 0);
      i1 = stop - kItemCost;
      if (i1 > i0) return true;
      advance(p);  // nothing but a piece of the item's fixed cost
    }
    return false;
  }
  __device__ __forceinline__ void advance(const Params& p) {
    base += s.n + kItemCost;
    u = min(base, end);
    if (++head == p.d.hkv) {
      head = 0;
      if (++row_tile == p.tiles) {
        row_tile = 0;
        ++bl;
      }
    }
  }
};

static_assert(sizeof(Walk) <= sizeof(Smem::walk[0][0]), "an item's walk fits its place");

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

// Keys and values share one body of code per width (`key` is a runtime flag):
// the hot loops of all roles have to stay in the instruction cache together.

// A part (a quarter) of a packed block on its way to a tile, in registers.
// B >= 2: part k is group k, B words with a scale and a zero a lane.  1 bit:
// word k of the lane's 16 bytes and the pairs of scales and zeros it meets.
template <int B>
struct Part {
  uint32_t w[B];
  __half s, z;  // kept apart: packing them would wait for the loads
};
template <>
struct Part<1> {
  uint32_t w[1], s[4], z[4];
};

template <int B>
__device__ __forceinline__ void load_part(Part<B>& c, int k, const char* codes, bool key) {
  const int lane = threadIdx.x & 31, tig = lane & 3;
  const __half* meta = reinterpret_cast<const __half*>(codes + 512 * B) + 32 * k;
  if constexpr (B == 1) {
    c.w[0] = __ldg(reinterpret_cast<const uint32_t*>(codes) + 4 * lane + k);
    meta += key ? 4 * tig : 8 * tig;
    const __half* second = meta + (key ? 16 : 4);
    const uint2 a = __ldg(reinterpret_cast<const uint2*>(meta));
    const uint2 b = __ldg(reinterpret_cast<const uint2*>(second));
    const uint2 d = __ldg(reinterpret_cast<const uint2*>(meta + kHeadDim));
    const uint2 e = __ldg(reinterpret_cast<const uint2*>(second + kHeadDim));
    c.s[0] = a.x, c.s[1] = a.y, c.s[2] = b.x, c.s[3] = b.y;
    c.z[0] = d.x, c.z[1] = d.y, c.z[2] = e.x, c.z[3] = e.y;
  } else {
    const char* src = codes + (32 * k + lane) * (4 * B);
    if constexpr (B == 2) {
      const uint2 a = __ldg(reinterpret_cast<const uint2*>(src));
      c.w[0] = a.x, c.w[1] = a.y;
    } else {
#pragma unroll
      for (int i = 0; i < B / 4; ++i) {
        const uint4 a = __ldg(reinterpret_cast<const uint4*>(src) + i);
        c.w[4 * i] = a.x, c.w[4 * i + 1] = a.y, c.w[4 * i + 2] = a.z, c.w[4 * i + 3] = a.w;
      }
    }
    const __half* m = meta + (key ? lane : vmeta_index(0, lane));
    c.s = m[0];
    c.z = m[kHeadDim];
  }
}

template <int B>
__device__ __forceinline__ void restore_part(const Part<B>& c, int k, unsigned char* tile, int j,
                                             bool key) {
  const int lane = threadIdx.x & 31;
  if constexpr (B == 1) {
    const int gid = lane >> 2, tig = lane & 3;
    // keys: token 4 gid + n; values: channel 4 gid + n of the group, the odd
    // gids in another order so that a store phase meets eight banks
    const int flip = key ? 0 : (gid & 1) << 1;
    const int half = key ? tig >> 1 : j >> 1;
    const int chunk = key ? (tig & 1) * 4 + (k ^ (tig & 2)) : (j & 1) * 4 + tig;
    const int row = 32 * (key ? j : k) + 8 * (gid >> 1) + (gid & 1);
    unsigned char* base = tile + half * kHalfBytes + row * 128;
    const uint32_t x0 = (uint32_t)(chunk ^ (gid & 1)) << 4;
    // Halves of the scales, to meet codes that read 2.0: exact down to 2^-13; below, the
    // last bit of a scale (the spacing of the inputs there, 2^-24) may be lost.
    __half2 s[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) s[r] = __hmul2(as_half2(c.s[r]), __float2half2_rn(0.5f));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int n = i ^ flip;
      const uint32_t w = __funnelshift_l(c.w[0], c.w[0], 4 - n);
      uint32_t o[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        // two codes at bits 14 and 30: 0 or 2.0
        const uint32_t x = __funnelshift_l(w, w, 4 * r) & 0x40004000u;
        o[r] = as_u32(__hfma2(as_half2(x), s[r], as_half2(c.z[r])));
      }
      st16(base, n * 256 + (x0 ^ (n << 5)), make_uint4(o[0], o[1], o[2], o[3]));
    }
  } else {
    const __half2 s = __half2half2(c.s), z = __half2half2(c.z);
    const int row = key ? 32 * k + lane : 32 * j + (lane & 24) + run_pos(lane & 7);
    const uint32_t at = key ? tile_at(j >> 1, row, (j & 1) * 4) : tile_at(k >> 1, row, (k & 1) * 4);
#pragma unroll
    for (int q = 0; q < 4; ++q) st16(tile, at ^ (q << 4), restore8<B>(c.w, q, s, z));
  }
}

// The same for a block of the fp16 window: `rows` is its first token's row (the
// ring holds a whole number of blocks, so a block does not wrap); tokens from
// `valid` on are zero.
template <int B>
__device__ __forceinline__ void window_block(const __half* rows, int valid, unsigned char* tile,
                                             int j, bool key) {
  const int lane = threadIdx.x & 31;
  if ((B == 1) == key) {  // rows of the tile are tokens
    const int row = 32 * j + (lane & 24) + run_pos(lane & 7);
    const uint4* src = reinterpret_cast<const uint4*>(rows + lane * kHeadDim);
#pragma unroll 1
    for (int h = 0; h < 2; ++h) {
      uint4 v[8];
#pragma unroll
      for (int m = 0; m < 8; ++m) v[m] = lane < valid ? src[8 * h + m] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
      for (int m = 0; m < 8; ++m) {
        if constexpr (B == 1) put_key_row<1>(tile, row, 8 * h + m, v[m]);
        else st16(tile, tile_at(h, row, m), run_order(v[m]));
      }
    }
  } else {  // rows are channels, two a lane
    const uint32_t* src = reinterpret_cast<const uint32_t*>(rows) + lane;
#pragma unroll 1
    for (int g = 0; g < 2; ++g) {  // 64 channels at a time
      const int c = 64 * g + 2 * lane;
      uint32_t x[32];
#pragma unroll
      for (int t = 0; t < 32; ++t) x[t] = t < valid ? src[t * (kHeadDim / 2) + 32 * g] : 0u;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int row = key ? c + e : value_row(c + e);
        const uint32_t sel = e ? 0x7632 : 0x5410;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t* y = x + 8 * k;
          st16(tile, tile_at(j >> 1, row, (j & 1) * 4 + k),
               make_uint4(__byte_perm(y[0], y[4], sel), __byte_perm(y[1], y[5], sel),
                          __byte_perm(y[2], y[6], sel), __byte_perm(y[3], y[7], sel)));
        }
      }
    }
  }
}
template <int B>
__device__ __forceinline__ void zero_block(unsigned char* tile, int j, bool key) {
  const int lane = threadIdx.x & 31;
  const bool tokens = (B == 1) == key;
#pragma unroll 1
  for (int i = 0; i < 16; ++i)
    st16(tile, tokens ? tile_at(i >> 3, 32 * j + lane, i & 7)
                      : tile_at(j >> 1, 32 * (i >> 2) + lane, (j & 1) * 4 + (i & 3)),
         make_uint4(0u, 0u, 0u, 0u));
}

// A loading warp: block j of every key (or value) tile of the CTA's share.  As
// soon as a part of a block is restored, the same part of the next block is
// loaded into its registers; the block after that is brought into L2, and the
// table entry of the one after that is on its way.
template <int B>
__device__ __forceinline__ void load_role(const Params& p, Smem& s, int u0, int u1, int j,
                                          bool key) {
  const int lane = threadIdx.x & 31;
  unsigned char(*tiles)[kTileBytes] = key ? s.k : s.v;
  uint64_t* full = key ? s.k_full : s.v_full;
  uint64_t* empty = key ? s.k_empty : s.v_empty;
  const int codes = key ? 0 : page_off_vcodes(p.d.bits_k);
  uint32_t n = 0;
  Walk w;
  w.begin(s, u0, u1);
  for (; w.next(p); w.advance(p)) {
    const int b = p.c.batch_begin + w.bl;
    // block n at base + index * stride: its number, or its entry of the table
    const int32_t* table =
        p.cache.block_table ? p.cache.block_table + (long long)b * p.d.max_blocks : nullptr;
    const int page = (int)p.d.page_bytes, stride = table ? page * p.d.hkv : page;
    const int limit = table ? p.cache.n_pages : p.d.max_blocks;
    const char* base = static_cast<const char*>(p.cache.pages) + codes +
                       (table ? (long long)w.head * page
                              : ((long long)b * p.d.hkv + w.head) * p.d.max_blocks * page);
    const int lq = packed_len(w.s.L, p.d.residual);
    const auto seen = [&](int t0) {
      return t0 <= w.s.p1 && (t0 + kGroup > w.s.lo || t0 < p.c.sinks);
    };
    const auto token = [&](int i) { return w.s.tile(i) * kTile + j * kGroup; };
    // index of unit i's block; kNone where there is nothing to restore
    constexpr int kNone = -0x7fffffff - 1;
    const auto index = [&](int i) {
      if (i >= w.i1) return kNone;
      const int t0 = token(i);
      if (t0 >= lq || !seen(t0)) return kNone;
      return table ? max(__ldg(table + (t0 >> 5)), kNone + 1) : t0 >> 5;  // (as much outside)
    };
    const auto address = [&](int e) -> const char* {
      if (e >= 0 && e < limit) return base + (long long)e * stride;
      if (e != kNone && lane == 0)
        atomicOr(reinterpret_cast<unsigned*>(p.cache.seq_len + p.d.batch), KVQ_FLAG_BAD_PAGE);
      return nullptr;
    };
    const auto prefetch = [&](int e) {
      if (e >= 0 && e < limit && lane < 4 * B + 4)
        asm volatile("prefetch.global.L2 [%0];" ::"l"(base + (long long)e * stride + 128 * lane));
    };
    Part<B> c[4];
    const char* at0 = nullptr;
    const char* at1 = address(index(w.i0));
    int e[kAhead];  // indexes of the blocks behind at1's
#pragma unroll
    for (int k = 0; k < kAhead; ++k) e[k] = index(w.i0 + 1 + k);
#pragma unroll
    for (int k = 0; k < kAhead - 1; ++k) prefetch(e[k]);
    // i = i0 - 1 only loads the first block
#pragma unroll 1
    for (int i = w.i0 - 1; i < w.i1; ++i) {
      const int buf = n & 1, far = index(i + 2 + kAhead);
      unsigned char* tile = tiles[buf];
      if (i >= w.i0) {
        if (!warp_wait(s, &empty[buf], ((n >> 1) & 1) ^ 1)) return;
        if (!at0) {
          const int ta = token(i);
          if (ta >= lq && seen(ta)) {
            const __half* rows =
                reinterpret_cast<const __half*>(key ? p.cache.k_resid : p.cache.v_resid) +
                (((long long)b * p.d.hkv + w.head) * p.d.ring + ta % p.d.ring) * kHeadDim;
            window_block<B>(rows, w.s.L - ta, tile, j, key);
          } else {
            zero_block<B>(tile, j, key);
          }
        }
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (at0) restore_part<B>(c[k], k, tile, j, key);
        if (at1) load_part<B>(c[k], k, at1, key);
      }
      if (i >= w.i0) {
        fence_async();
        warp_arrive(&full[buf]);
        ++n;
      }
      at0 = at1;
      at1 = address(e[0]);
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

constexpr uint32_t kColS = 0, kColO = 256;  // tensor memory columns: S0 S1 O0 O1, 128 each

// The products of stream x, by one warp.
template <int BK, int BV>
__device__ __forceinline__ void issue_role(const Params& p, Smem& s, int u0, int u1, int x) {
  constexpr uint32_t kIdS = instr_desc(BK != 1, kStep), kIdO = instr_desc(BV != 1, kHeadDim);
  // where the second half of a tile's tokens begins
  constexpr int kHalfK = BK == 1 ? kStep * 128 : kHalfBytes;
  constexpr int kHalfV = BV == 1 ? kHalfBytes : kStep * 128;
  const int two = p.streams_rows;  // two steps a tile (the stream takes both halves)
  const uint32_t tm = __shfl_sync(0xffffffffu, s.tmem, 0) + 128 * x, leader = elect_lane();
  const uint64_t q = tile_desc(sptr(s.q[two ? x : 0]), false);
  uint32_t nt = 0, ns = 0, items = 0;  // tiles, steps and items done
  Walk w;
  w.begin(s, u0, u1);
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
        const uint64_t v = tile_desc(sptr(s.v[buf]) + half * kHalfV, BV != 1);
#pragma unroll
        for (int ks = 0; ks < kStep / 16; ++ks)
          mma_ts(leader, tm + kColO, ts + 8 * ks,
                 v + (BV == 1 ? step_major_k(ks) : step_major_mn(ks)), kIdO, st > 0 || ks > 0);
        if (!two || half == 1) tc_commit(leader, &s.v_empty[buf]);
        // the last two products of an item tell that they are in; the others
        // are when the scores issued behind them are
        if (st + 2 >= steps) tc_commit(leader, st + 1 == steps ? &s.o_full[x] : &s.o_last[x]);
      }
      if (st + 2 < steps) {
        const uint32_t t = nt + ((st + 2) >> two), buf = t & 1;
        const int half = two ? st & 1 : x;
        if (!two || half == 0) {
          if (!warp_wait(s, &s.k_full[buf], (t >> 1) & 1)) return;
          tc_after();
        }
        const uint64_t kd = tile_desc(sptr(s.k[buf]) + half * kHalfK, BK != 1);
#pragma unroll
        for (int ks = 0; ks < kHeadDim / 16; ++ks)
          mma_ss(leader, ts, q + step_major_k(ks),
                 kd + (BK == 1 ? step_major_k(ks) : step_major_mn(ks)), kIdS, ks > 0);
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

// Column n of a key tile holds token 8 (n / 8) + run_token(n mod 8).
__host__ __device__ constexpr int run_token(int n) { return (n & 1) * 4 + (n >> 1); }

struct Row {
  float m, l;    // running maximum (of scores times scale, log2 domain), lifted sum
};

// Row r (of the sequence's n_q * gq) of a [sequence][token][head] array.
__device__ __forceinline__ long long row_offset(const Params& p, const long long (&stride)[3],
                                                int bl, int kv_head, int r) {
  const int t = token_of_row(p, r);
  return bl * stride[0] + t * stride[1] + (kv_head * p.d.gq + r - t * p.d.gq) * stride[2];
}

// A warp's 32 rows, from row r0 of the sequence and row `row` of the tile on:
// 16 lanes a row.
template <int BK>
__device__ __forceinline__ void load_queries(const Params& p, const Walk& w, int r0,
                                             unsigned char* tile, int row) {
  const int lane = threadIdx.x & 31, m = lane & 15, rows = p.c.n_q * p.d.gq;
#pragma unroll 1
  for (int h = 0; h < 32; h += 16) {
    uint4 v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = h + 2 * i + (lane >> 4);
      v[i] = make_uint4(0u, 0u, 0u, 0u);
      if (r0 + r < rows)
        v[i] = __ldg(reinterpret_cast<const uint4*>(
                         p.q + row_offset(p, p.c.q_stride, w.bl, w.head, r0 + r)) + m);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) put_key_row<BK>(tile, row + h + 2 * i + (lane >> 4), m, v[i]);
  }
}

// The thread's row of scores with -inf where a column is not seen: column n is
// seen when its token (less the tile's first) is at most hi and above lo, or
// below sink.  Only tiles at an edge come here; the scores are rewritten in
// tensor memory by a short loop to keep the code of the others small.
__device__ __forceinline__ void mask_row(uint32_t ts, int hi, int lo, int sink) {
#pragma unroll 1
  for (int c = 0; c < kStep; c += 32) {
    uint32_t r[32];
    tm_load32(ts + c, r);
    tm_load_wait();
#pragma unroll
    for (int n = 0; n < 32; ++n) {
      const int t = c + (n & ~7) + run_token(n & 7);
      if (t > hi || (t <= lo && t >= sink)) r[n] = 0xff800000u;
    }
    tm_store32(ts + c, r);
  }
  tm_store_wait();
}

// Multiply the thread's row of the accumulator by f.
__device__ __forceinline__ void rescale_row(uint32_t to, float f) {
#pragma unroll 1
  for (int c = 0; c < kHeadDim; c += 8) {
    uint32_t o[8];
    tm_load8(to + c, o);
    tm_load_wait();
#pragma unroll
    for (int n = 0; n < 8; ++n) o[n] = __float_as_uint(__uint_as_float(o[n]) * f);
    tm_store8(to + c, o);
  }
}

// Results leave through shared memory, 64 bytes a row at a time: each lane
// writes its own row, then four lanes copy a row to memory.  Chunk m of row r is
// at m ^ (r / 2 mod 4), so neither side meets a bank twice.
struct Rows {
  char* at[4];  // rows lane / 4 + 8 k, this lane's 16 bytes; nullptr past the end
};
__device__ __forceinline__ void stage_row(unsigned char* stage, const uint4 (&v)[4]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int m = 0; m < 4; ++m) st16(stage, lane * 64 + ((m ^ ((lane >> 1) & 3)) << 4), v[m]);
}
__device__ __forceinline__ void put_rows(const unsigned char* stage, const Rows& rows,
                                         int offset) {
  const int lane = threadIdx.x & 31;
  __syncwarp();
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int r = (lane >> 2) + 8 * k;
    const uint4 x = *reinterpret_cast<const uint4*>(
        stage + r * 64 + (((lane & 3) ^ ((r >> 1) & 3)) << 4));
    if (rows.at[k]) *reinterpret_cast<uint4*>(rows.at[k] + offset) = x;
  }
  __syncwarp();
}

template <int BK>
__device__ __forceinline__ void softmax_role(const Params& p, Smem& s, int u0, int u1,
                                             const Shares& shares) {
  const int warp = threadIdx.x >> 5, x = warp >> 2, lane_row = threadIdx.x & 127;
  const uint32_t lanes = (uint32_t)(warp & 3) << 21;  // 32 lanes a warp, in bits 16 up
  const uint32_t tm = __shfl_sync(0xffffffffu, s.tmem, 0) + 128 * x;
  const uint32_t ts = tm + lanes + kColS, to = tm + lanes + kColO;
  const int two = p.streams_rows, tr = kTile << two, rows = p.c.n_q * p.d.gq;
  // steps of the stream, meetings, items and phases of o_last so far
  uint32_t ns = 0, met = 0, items = 0, lasts = 0;
  const float sl2 = p.c.scale_log2;
  const auto queries = [&](const Walk& w) {
    const int r0 = w.row_tile * tr + (two ? kTile * x : 0) + (lane_row & ~31);
    load_queries<BK>(p, w, r0, s.q[x], lane_row & ~31);
    fence_async();
    warp_arrive(&s.q_full);
  };
  // The item and the next one are kept in shared memory: their fields would take
  // registers from the scores.
  const auto walk = [&](uint32_t i) -> Walk& {
    return *reinterpret_cast<Walk*>(s.walk[warp][i & 1]);
  };
  bool more;
  {
    Walk first;
    first.begin(s, u0, u1);
    more = first.next(p);
    walk(0) = first;
    __syncwarp();
    if (more && (two || x == 0)) queries(first);
  }
#pragma unroll 1
  while (more) {
    const Walk& w = walk(items);
    const int tr_row = (two ? kTile * x : 0) + lane_row;  // row in the item
    const int g = w.row_tile * tr + tr_row, g_warp = g - (threadIdx.x & 31);
    const bool valid = g < rows;
    const bool live = g_warp < rows;  // the warp has a row
    const int pos = w.s.L - p.c.n_q + token_of_row(p, g);
    Row row{-INFINITY, 0.0f};
    const int steps = (w.i1 - w.i0) << two;
#pragma unroll 1
    for (int st = 0; st < steps; ++st, ++ns) {
      const int b = ns & 1;
      const uint32_t sb = ts + kStep * b;
      if (!warp_wait(s, &s.s_full[x][b], (ns >> 1) & 1)) return;
      tc_after();
      if (live) {
        const int t0 = w.s.tile(w.i0 + (st >> two)) * kTile + kStep * (two ? st & 1 : x);
        // every token of the step is seen by every row of the item
        const bool whole = w.s.p0 >= t0 + kStep - 1 &&
                           (!p.c.window || t0 > w.s.p1 - p.c.window || t0 <= p.c.sinks - kStep);
        // the last token behind the window, -1 if there is none (positions and
        // windows each reach 2^31)
        const int behind = p.c.window ? max(max(pos, 0) - p.c.window, -1) : -1;
        if (!whole) mask_row(sb, (valid ? pos : -1) - t0, behind - t0, p.c.sinks - t0);
        uint32_t r[2][32];
        tm_load32(sb, r[0]);
        tm_load32(sb + 32, r[1]);
        tm_load_wait();
        float mc[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const uint32_t* y = &r[c >> 1][16 * (c & 1)];
          mc[c] = fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
#pragma unroll
          for (int n = 2; n < 16; n += 2)
            mc[c] = fmaxf(fmaxf(mc[c], __uint_as_float(y[n])), __uint_as_float(y[n + 1]));
        }
        const float mx = fmaxf(fmaxf(mc[0], mc[1]), fmaxf(mc[2], mc[3])) * sl2;
        if (st == 0) {
          row.m = mx;
        } else {
          const bool up = mx > row.m + kRescaleLog2;
          if (__any_sync(0xffffffffu, up)) {
            const float f = up ? exp2_fast(row.m - mx) : 1.0f;
            if (up) row.m = mx;
            row.l *= f;
            // The product before this step's has to be in: the next scores are
            // issued behind it; an item's last step has none behind.
            if (st + 1 < steps ? !warp_wait(s, &s.s_full[x][b ^ 1], ((ns + 1) >> 1) & 1)
                               : !warp_wait(s, &s.o_last[x], lasts & 1))
              return;
            tc_after();
            rescale_row(to, f);
          }
        }
        const float off = row.m == -INFINITY ? 0.0f : kLiftLog2 - row.m;
        const uint64_t sl = pair(sl2, sl2), of = pair(off, off);
        uint64_t acc[2] = {0ull, 0ull};
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          uint32_t h[16];
#pragma unroll
          for (int n = 0; n < 16; ++n) {
            float y0, y1;
            unpair(fma2(pair(__uint_as_float(r[c][2 * n]), __uint_as_float(r[c][2 * n + 1])), sl,
                        of),
                   y0, y1);
            y0 = exp2_fast(y0);
            y1 = exp2_fast(y1);
            acc[n & 1] = add2(acc[n & 1], pair(y0, y1));
            h[n] = pack_half2(y0, y1);
          }
          tm_store16(sb + 16 * c, h);
        }
        float y0, y1;
        unpair(add2(acc[0], acc[1]), y0, y1);
        row.l += y0 + y1;
        tm_store_wait();
      }
      tc_before();
      warp_arrive(&s.p_ready[x][b]);
    }
    lasts += steps > 1;
    // The next item's queries: all scores of this one are done (an item of one
    // row tile has the other stream's too).
    {
      Walk next = w;
      next.advance(p);
      more = next.next(p);
      walk(items + 1) = next;
      __syncwarp();
      if (more && (two || x == 0)) {
        if (!two && !warp_wait(s, &s.s_full[1][(ns - 1) & 1], ((ns - 1) >> 1) & 1)) return;
        queries(next);
      }
    }
    // the accumulator is complete; items of one row tile need both streams'
    if (!warp_wait(s, &s.o_full[x], items & 1)) return;
    if (!two && x == 0 && !warp_wait(s, &s.o_full[1], items & 1)) return;
    tc_after();
    if (!two && x == 1) {
      s.m[lane_row] = row.m;
      s.l[lane_row] = row.l;
    }
    if (!two && !meet_softmax(s, met)) return;
    const bool direct = w.i0 == 0 && w.i1 == w.s.n;
    if ((two || x == 0) && live) {
      float f0 = 1.0f, f1 = 0.0f, m = row.m, l = row.l;
      if (!two) {
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
      // slot 0 of a CTA: the item its share begins in
      const int pr = (2 * blockIdx.x + (u0 < w.base ? 1 : 0)) * tr + tr_row;
      const int lane = threadIdx.x & 31;
      Rows at;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int r = (lane >> 2) + 8 * k;
        char* row_at =
            direct ? reinterpret_cast<char*>(
                         p.out + row_offset(p, p.c.out_stride, w.bl, w.head, g_warp + r))
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
        // accumulator columns stand in the run order
        uint4 v[4];
        if (direct) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float* y = o + 8 * k;
            v[k] = make_uint4(pack_half2(y[0], y[2]), pack_half2(y[4], y[6]),
                              pack_half2(y[1], y[3]), pack_half2(y[5], y[7]));
          }
          stage_row(s.stage[warp], v);
          put_rows(s.stage[warp], at, 2 * c);
        } else {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const float* y = o + 16 * h + 8 * (k >> 1) + (k & 1);
              v[k] = make_uint4(__float_as_uint(y[0]), __float_as_uint(y[2]),
                                __float_as_uint(y[4]), __float_as_uint(y[6]));
            }
            stage_row(s.stage[warp], v);
            put_rows(s.stage[warp], at, 4 * (c + 16 * h));
          }
        }
      }
      if (valid && !direct) p.part_ml[pr] = make_float2(m, l);
      tc_before();
    }
    if (!direct && w.i0 == 0 && threadIdx.x == 0) {
      const int first = w.base + kItemCost;
      p.splits[blockIdx.x] = Split{1, u0 < w.base ? 1 : 0, shares.owner(first + w.s.n - 1), w.bl,
                                   w.row_tile, w.head};
    }
    if (!meet_softmax(s, met)) return;  // s.m, s.l and both accumulators may be written again
    ++items;
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

  if (tid == 0) p.splits[blockIdx.x].valid = 0;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  // Units of every (sequence, row tile), summed over the threads in order.
  const int groups = p.c.batch_count * p.tiles;
  const int per = (int)((uint32_t)(groups + kThreads - 1) / kThreads);
  const int g0 = min(groups, tid * per), g1 = min(groups, g0 + per);
  const int seq0 = (int)((uint32_t)g0 / (uint32_t)p.tiles), tile0 = g0 - seq0 * p.tiles;
  int mine = 0;
#pragma unroll 1
  for (int g = g0, sq = seq0, tl = tile0; g < g1; ++g) {
    mine += (span_of(p, sq, tl).n + kItemCost) * p.d.hkv;
    if (++tl == p.tiles) tl = 0, ++sq;
  }
  int inc = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += y;
  }
  if (lane == 31) s.scan[warp] = inc;
  if (tid == 0) {
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
    bar_init(&s.q_full, 4 << p.streams_rows);
    bar_init(&s.meet, kSoftmaxWarps);
    s.abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  int warps = lane < kThreads / 32 ? s.scan[lane] : 0;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, warps, o);
    if (lane >= o) warps += y;
  }
  const int total = __shfl_sync(0xffffffffu, warps, 31);
  int before = __shfl_sync(0xffffffffu, warps, warp > 0 ? warp - 1 : 0);
  if (warp == 0) before = 0;
  before += inc - mine;
  Shares shares;
  shares.n = min((int)gridDim.x, total);
  if ((int)blockIdx.x >= shares.n) return;  // fewer units than CTAs
  shares.q = (int)((uint32_t)total / (uint32_t)shares.n);
  shares.r = total - shares.q * shares.n;
  const int u0 = shares.begin(blockIdx.x), u1 = shares.begin(blockIdx.x + 1);
  if (before <= u0 && u0 < before + mine) {
#pragma unroll 1
    for (int at = before, sq = seq0, tl = tile0;;) {
      const int n = span_of(p, sq, tl).n + kItemCost;
      if (u0 < at + n * p.d.hkv) {
        s.start_seq = sq;
        s.start_tile = tl;
        s.start_head = (int)((uint32_t)(u0 - at) / (uint32_t)n);
        s.start_step = u0 - at - s.start_head * n;
        break;
      }
      at += n * p.d.hkv;
      if (++tl == p.tiles) tl = 0, ++sq;
    }
  }
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
    regs_up<Regs<BK, BV>::kSoftmax>();
    softmax_role<BK>(p, s, u0, u1, shares);
    __syncwarp();
  } else if (warp < kIssueWarp) {
    regs_up<Regs<BK, BV>::kLoad>();
    const bool key = warp < kSoftmaxWarps + 4;
    if constexpr (BK == BV) load_role<BK>(p, s, u0, u1, warp & 3, key);
    else if (key) load_role<BK>(p, s, u0, u1, warp & 3, true);
    else load_role<BV>(p, s, u0, u1, warp & 3, false);
    __syncwarp();
  } else {
    regs_down<kRegsIssue>();
    if (warp < kIssueWarp + 2) issue_role<BK, BV>(p, s, u0, u1, warp - kIssueWarp);
    __syncwarp();
  }
  leave(s, p.cache.seq_len + p.d.batch);
  if (warp == kIssueWarp)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tm));
}

template <int BK, int BV>
cudaError_t launch_widths(const Params& p, int ctas, cudaStream_t stream) {
  static std::atomic<unsigned long long> done{0};
  const cudaError_t e = once_per_device(done, [] {
    const cudaError_t e = cudaFuncSetAttribute(chunk_attn_kernel<BK, BV>,
                                               cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               (int)sizeof(Smem));
    if (e != cudaSuccess) return e;
    // the register shares wait for registers that a smaller launch would lack
    cudaFuncAttributes attr;
    const cudaError_t ea = cudaFuncGetAttributes(&attr, chunk_attn_kernel<BK, BV>);
    if (ea != cudaSuccess) return ea;
    return attr.numRegs < kRegsLaunch ? cudaErrorInvalidConfiguration : cudaSuccess;
  });
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
