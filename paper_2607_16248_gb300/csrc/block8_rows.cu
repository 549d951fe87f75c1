// kvq_block8_attn for few rows a kv-head (single tokens, drafts): the cache is read once
// at memory speed, the arithmetic stays out of its way.
//
// A warp takes whole blocks of 32 tokens.  TMA brings a block's keys and values (2 x 4 KB,
// 128-byte swizzle) into the warp's own ring of slots; the block's scales follow by a small
// asynchronous copy on the same barrier.  Scores S^T = K Q^T by m16n8k16 products with the
// codes as A (tokens x channels) and eight query rows as B; O^T += V^T W^T with the codes
// as A again (channels x tokens).  Codes become fp16 exactly, two at a time.  The sum over
// a product's index may run in any order, so a lane takes 32 neighbouring channels of a
// key (and of its query row), and 16 neighbouring channels of eight values; with the
// swizzle no load of 16 bytes meets a bank twice.  Tokens of a value pair come together by
// a byte permutation, weights get from the scores' layout to B's by an 8 x 8 transposition
// in registers.
//
// Scales.  A score is (codes . q) * s_k: s_k joins the factor of the exponent.  A weight
// times s_v is 2^(x + log2 s_v): the running maximum is taken of x + log2 s_v, fp16 weights
// are w = 2^(x + log2 s_v - m + kLift), and the sum of the softmax is that of w / s_v, in
// fp32.  So neither scale rounds a code, and weights stay within fp16 whatever the scales.
// The maximum is kept in its two parts, m = x_max and e = log2 s_v there, and a weight's
// exponent is (x - m) + (log2 s_v + kLift - e) with x rounded: the difference of two scores
// is exact where it counts, however large they are.  In one sum with x, a product's rounding
// and that of kLift - m passed fp16's range from scores of 2^28 on.
//
// The tokens behind the last whole block are a block of 16-bit elements that two warps take
// from the ring, 16 tokens each, by asynchronous copies ahead of the item: behind full rings each
// load waits for microseconds, and their largest magnitudes make two passes.  Values, and bf16 keys, go to fp16 times a power of two, each token's its own:
// what one token holds, seen or not, does not touch the others.
//
// What bounds it.  HBM where there is enough to read: 32 ragged chats of 2k to 32k tokens,
// query groups of eight, bf16: 183 us, 6.1 TB/s; without the arithmetic 171.  Drafts of one
// to five tokens in 16 chats of 8k to 32k (one to three row groups): 124 us, 5.5 TB/s, two
// of them the open tokens' own factors.  One chat of 32k: 24.6 us, of which the cache's bytes
// take 9 at 7.4 TB/s; the others are the chain of launch, plan (2.6), table (1.3), first block
// (1.4), merge (1.1), partial and ticket (1.7), and the join (4).
#include <cuda.h>

#include <cfloat>
#include <type_traits>

#include "block8_plan.cuh"

namespace kvq {
namespace block8 {

namespace {

constexpr int kTok = 5;            // 32 tokens a unit
constexpr int kItemCost = kRowsItemCost;
constexpr int kHalfPage = kGroup * kHeadDim;  // bytes of a block's keys (or values)
constexpr float kLift = 7.0f;      // weights stay below 2^(kLift + kLag)
constexpr float kLag = 8.0f;       // how far a score may pass the running maximum
constexpr float kNone = -FLT_MAX;  // the maximum before any token
constexpr long long kWaitCycles = 4000000000LL;  // bound of a wait (~2 s)
constexpr long long kTestCycles = 20000000LL;    // in the self-test (~10 ms)

// Eight warps with two slots each: 128 KB of copies on their way in an SM.  More only make
// everything else wait behind them (ragged batch of 32 single tokens: 198 us; three slots
// 214, twelve warps 209).
template <int NT>
struct Smem {
  static constexpr int kWarps = 8, kSlots = 2;
  static constexpr int kMergers = 4;  // warps whose results change hands at a time
  unsigned char page[kWarps][kSlots][2 * kHalfPage];
  float4 merge[kMergers][NT * 8][32];
  float m[kWarps][8 * NT], l[kWarps][8 * NT];
  uint2 q[NT <= 2 ? 1 : NT][8][32];  // queries of more row groups than fit registers
  uint4 tail[2][2][16][16];  // 16 open tokens' keys and values each: chunk c of row r at c ^ r mod 8
  float qf[8 * NT];
  float2 scale[kWarps][kSlots];
  uint64_t full[kWarps][kSlots];
  int scan[32];
  Start start;
  int join;  // this CTA's partial is the item's last
  Walk<kTok, kItemCost> ahead[kWarps];  // the item whose blocks are being fetched
};

__device__ __forceinline__ uint32_t sptr(const void* p) {
  return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                    uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
      "{%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// Two fp32 operations at once.
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 v;
  asm("{\n .reg .b64 x, y;\n mov.b64 x, {%2, %3};\n mov.b64 y, {%4, %5};\n"
      " mul.rn.f32x2 x, x, y;\n mov.b64 {%0, %1}, x;\n}"
      : "=f"(v.x), "=f"(v.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return v;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 v;
  asm("{\n .reg .b64 x, y;\n mov.b64 x, {%2, %3};\n mov.b64 y, {%4, %5};\n"
      " add.rn.f32x2 x, x, y;\n mov.b64 {%0, %1}, x;\n}"
      : "=f"(v.x), "=f"(v.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return v;
}
// Codes 2 i, 2 i + 1 of a word as fp16.
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

template <int NT>
struct State {
  // queries in registers while there is room for them beside the results
  static constexpr bool kOwnQueries = NT <= 2;
  float m[NT][2], e[NT][2];  // of rows 8 nt + 2 tig, + 1
  float l[NT][2];            // of this lane's tokens alone
  float o[NT][8][4];         // channels 16 gid + 2 i (0, 1) and + 1 (2, 3), the same rows
  uint2 q[kOwnQueries ? NT : 1][8];  // of row 8 nt + gid, channels 32 tig ..
  const uint2* shared_q;             // [NT][8][32] of the CTA
  float f[NT][2];            // factor of a score in the exponent
  __device__ __forceinline__ uint2 query(int n, int step) const {
    if constexpr (kOwnQueries) return q[n][step];
    else return shared_q[(8 * n + step) * 32 + (threadIdx.x & 31)];
  }
};

// What masks a block's tokens: the rows' positions.
struct Rows {
  int first;  // of row 0
  __device__ __forceinline__ int pos(const AttnParams& p, int n, int j) const {
    return first + token_of_row(p, 8 * n + 2 * (threadIdx.x & 3) + j);
  }
};

// The softmax of a block's scores s[half of 16 tokens][nt][4], and its weights as B.
// t0: the block's first token; edge: some row may not see some token.
template <int N, int NT>
__device__ __forceinline__ void weights(const AttnParams& p, State<NT>& st, const Rows& rows,
                                        float (&s)[2][N][4], int t0, bool edge, float sk,
                                        float sv, uint32_t (&w)[2][N][2]) {
  const int gid = (threadIdx.x & 31) >> 2;
  if (edge) {
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int pos = rows.pos(p, n, j);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int t = t0 + 16 * h + 8 * i + gid;
            if (t > pos || (p.c.window && t <= pos - p.c.window && t >= p.c.sinks))
              s[h][n][j + 2 * i] = -INFINITY;
          }
      }
  }
  const float lsv = log2_fast(sv), inv = 1.0f / sv;
  const auto factor = [&](int n, int j) { return fmaxf(sk * st.f[n][j], kLeastFactor); };
  // how far a score of row j of group n is above the reference
  const auto above = [&](int n, int j, float s) {
    return __fsub_rn(__fmul_rn(s, factor(n, j)), st.m[n][j]) + (lsv - st.e[n][j]);
  };
  bool up = false;
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const float mx = fmaxf(fmaxf(s[0][n][j], s[0][n][j + 2]), fmaxf(s[1][n][j], s[1][n][j + 2]));
      up |= above(n, j, mx) > kLag;
    }
  if (__any_sync(0xffffffffu, up)) {
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float mx = fmaxf(fmaxf(s[0][n][j], s[0][n][j + 2]), fmaxf(s[1][n][j], s[1][n][j + 2]));
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
        const float d = above(n, j, mx);
        float f = 1.0f;
        if (d > 0.0f) {
          f = exp2_fast(-d);
          st.m[n][j] = __fmul_rn(mx, factor(n, j));
          st.e[n][j] = lsv;
        }
        st.l[n][j] *= f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          st.o[n][i][j] *= f;
          st.o[n][i][j + 2] *= f;
        }
      }
  }
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const float2 f = make_float2(factor(n, 0), factor(n, 1));
    const float2 c = make_float2(lsv + kLift - st.e[n][0], lsv + kLift - st.e[n][1]);
    float2 sum = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        // (m by single subtractions: a packed one would be fused with the product)
        const float2 x = mul2(make_float2(s[h][n][2 * i], s[h][n][2 * i + 1]), f);
        float2 y = add2(make_float2(__fsub_rn(x.x, st.m[n][0]), __fsub_rn(x.y, st.m[n][1])), c);
        y.x = exp2_fast(y.x);
        y.y = exp2_fast(y.y);
        sum = add2(sum, y);
        w[h][n][i] = transpose(pack16<false>(y.x, y.y));
      }
    st.l[n][0] = fmaf(sum.x, inv, st.l[n][0]);
    st.l[n][1] = fmaf(sum.y, inv, st.l[n][1]);
  }
}

// Whether a block's values are all zero; for a warp.
__device__ __forceinline__ bool no_value(const unsigned char* codes) {
  uint32_t any = 0u;
#pragma unroll
  for (int k = 0; k < kHalfPage / 512; ++k) {
    const uint4 x = reinterpret_cast<const uint4*>(codes + 512 * k)[threadIdx.x & 31];
    any |= x.x | x.y | x.z | x.w;
  }
  return !__any_sync(0xffffffffu, (any & 0x7f7f7f7fu) != 0u);
}

// One block of codes in shared memory; the first N of the item's row groups are in use.
template <int N, int NT>
__device__ __forceinline__ void block(const AttnParams& p, State<NT>& st, const Rows& rows,
                                      const unsigned char* page, float2 scale, int t0, bool edge) {
  const int lane = threadIdx.x & 31, gid = lane >> 2, tig = lane & 3;
  float s[2][N][4];
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[h][n][i] = 0.0f;
  const unsigned char* kr = page + gid * kHeadDim;
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const unsigned char* at = kr + (((2 * tig + c) ^ gid) << 4);
    uint4 x[2], y[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      x[h] = *reinterpret_cast<const uint4*>(at + h * 16 * kHeadDim);
      y[h] = *reinterpret_cast<const uint4*>(at + (h * 16 + 8) * kHeadDim);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      uint2 q[N];
#pragma unroll
      for (int n = 0; n < N; ++n) q[n] = st.query(n, 4 * c + k);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t xw = k == 0 ? x[h].x : k == 1 ? x[h].y : k == 2 ? x[h].z : x[h].w;
        const uint32_t yw = k == 0 ? y[h].x : k == 1 ? y[h].y : k == 2 ? y[h].z : y[h].w;
        const uint32_t a0 = wide_lo(xw), a1 = wide_lo(yw), a2 = wide_hi(xw), a3 = wide_hi(yw);
#pragma unroll
        for (int n = 0; n < N; ++n) mma(s[h][n], a0, a1, a2, a3, q[n].x, q[n].y);
      }
    }
  }
  uint32_t w[2][N][2];
  weights<N, NT>(p, st, rows, s, t0, edge, scale.x, scale.y, w);
  const unsigned char* vb = page + kHalfPage;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint4 x[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = 16 * h + 8 * i + 2 * tig + e;
        x[i][e] = *reinterpret_cast<const uint4*>(vb + r * kHeadDim + ((gid ^ (r & 7)) << 4));
      }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const auto word = [&](int i, int e) {
        return k == 0 ? x[i][e].x : k == 1 ? x[i][e].y : k == 2 ? x[i][e].z : x[i][e].w;
      };
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        const uint32_t u = __byte_perm(word(0, 0), word(0, 1), z ? 0x7362 : 0x5140);
        const uint32_t v = __byte_perm(word(1, 0), word(1, 1), z ? 0x7362 : 0x5140);
        const uint32_t a0 = wide_lo(u), a1 = wide_hi(u), a2 = wide_lo(v), a3 = wide_hi(v);
#pragma unroll
        for (int n = 0; n < N; ++n)
          mma(st.o[n][2 * k + z], a0, a1, a2, a3, w[h][n][0], w[h][n][1]);
      }
    }
  }
}

// 16-bit elements of a word as fp16, times f.
template <bool BF16>
__device__ __forceinline__ uint32_t to_half2(uint32_t u, float f) {
  if constexpr (!BF16) return u;
  return pack16<false>(__uint_as_float(u << 16) * f, __uint_as_float(u & 0xffff0000u) * f);
}
// The power of two that takes a magnitude (bf16 bits) to [2^14, 2^15).
__device__ __forceinline__ float lift_of(uint32_t bits) {
  const int e = max((int)(bits >> 7), 27) - 127;  // at least 2^-100
  return bits ? __uint_as_float((uint32_t)(14 - e + 127) << 23) : 1.0f;
}
__device__ __forceinline__ uint32_t largest(uint32_t m, const uint4& v) {
  m = __vmaxu2(m, v.x & 0x7fff7fffu);
  m = __vmaxu2(m, v.y & 0x7fff7fffu);
  m = __vmaxu2(m, v.z & 0x7fff7fffu);
  return __vmaxu2(m, v.w & 0x7fff7fffu);
}

// The softmax of the scores of 16 open tokens from t0 on, each of which has factors of its own: ks
// and 2^lift, of tokens 8 i + gid.  The reference is the row's best token by x + log2 of its
// value's factor.
template <int NT>
__device__ __forceinline__ void tail_weights(const AttnParams& p, State<NT>& st,
                                             const Rows& rows, float (&s)[NT][4], int t0,
                                             const float (&ks)[2], const int (&lift)[2],
                                             uint32_t (&w)[NT][2]) {
  const int gid = (threadIdx.x & 31) >> 2;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    float y[4];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int pos = rows.pos(p, n, j);
      float best = -INFINITY, best_lv = 0.0f;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int t = t0 + 8 * i + gid;
        float x = __fmul_rn(s[n][j + 2 * i], fmaxf(ks[i] * st.f[n][j], kLeastFactor));
        if (t > pos || (p.c.window && t <= pos - p.c.window && t >= p.c.sinks)) x = -INFINITY;
        const float lv = (float)-lift[i];
        if ((x - best) + (lv - best_lv) > 0.0f) best = x, best_lv = lv;
        y[j + 2 * i] = x;
      }
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) {
        const float x = __shfl_xor_sync(0xffffffffu, best, o);
        const float lv = __shfl_xor_sync(0xffffffffu, best_lv, o);
        const float d = (x - best) + (lv - best_lv);
        if (d > 0.0f || (d == 0.0f && x > best)) best = x, best_lv = lv;
      }
      if (best > -INFINITY) {  // a token is seen
        st.m[n][j] = best;
        st.e[n][j] = best_lv;
      } else {
        best = 0.0f;
      }
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float lv = (float)-lift[i];
        const float x = exp2_fast((y[j + 2 * i] - best) + (lv - best_lv) + kLift);
        sum = fmaf(x, pow2(lift[i]), sum);
        y[j + 2 * i] = x;
      }
      st.l[n][j] = sum;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) w[n][i] = transpose(pack16<false>(y[2 * i], y[2 * i + 1]));
  }
}

// An item's open tokens: the first one's position, and how many.
__device__ __forceinline__ int2 open_tokens(const Walk<kTok, kItemCost>& w) {
  const int t0 = w.s.tile(w.s.n - 1) * kGroup;
  return make_int2(t0, w.q.L - t0);
}
// The ring's rows of 16 of an item's open tokens (from the t-th on) on their way to shared
// memory, by a warp; rows behind the last are zero.
__device__ __forceinline__ void fetch_tail(const AttnParams& p, const Walk<kTok, kItemCost>& w,
                                           int t, uint4 (&tail)[2][16][16]) {
  const int lane = threadIdx.x & 31, c = lane & 15;
  const int2 open = open_tokens(w);
  const long long at =
      (((long long)w.b * p.c.d.hkv + w.head) * kRing + ((open.x + t) & (kRing - 1))) * kHeadDim;
#pragma unroll 1
  for (int r = lane >> 4; r < 16; r += 2) {
    const bool valid = t + r < open.y;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint16_t* src = (i ? p.c.cache.v_ring : p.c.cache.k_ring) + at + 8 * c +
                            (valid ? r * kHeadDim : 0);
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(
                       sptr(&tail[i][r][c ^ (r & 7)])),
                   "l"(src), "r"(valid ? 16 : 0)
                   : "memory");
    }
  }
}

// 16 open tokens from t0 on, from shared memory; the warp's first of the item, so its results are
// its own.
template <int NT, bool BF16>
__device__ __forceinline__ void tail_block(const AttnParams& p, State<NT>& st, const Rows& rows,
                                           const uint4 (&tail)[2][16][16], int t0) {
  const int lane = threadIdx.x & 31, gid = lane >> 2, tig = lane & 3;
  const auto load = [&](int i, int r, int chunk) { return tail[i][r][chunk ^ (r & 7)]; };
  // the largest magnitude of a row of which four lanes hold a quarter each, and the least (least2)
  const auto row_most = [&](const uint4 (&x)[4]) {
    uint32_t m = 0u;
#pragma unroll
    for (int c = 0; c < 4; ++c) m = largest(m, x[c]);
    m = max(m & 0xffffu, m >> 16);
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
    return max(m, __shfl_xor_sync(0xffffffffu, m, 2));
  };
  const auto row_least = [&](const uint4 (&x)[4]) {
    uint32_t m = ~0u;
#pragma unroll
    for (int c = 0; c < 4; ++c)
      m = least2(least2(least2(least2(m, x[c].x), x[c].y), x[c].z), x[c].w);
    m = min(m & 0xffffu, m >> 16);
    m = min(m, __shfl_xor_sync(0xffffffffu, m, 1));
    return min(m, __shfl_xor_sync(0xffffffffu, m, 2));
  };
  float s[NT][4], ks[2] = {1.0f, 1.0f}, f[2] = {1.0f, 1.0f};
  int lift[2];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) s[n][i] = 0.0f;
  uint4 x[2][4];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
#pragma unroll
    for (int c = 0; c < 4; ++c) x[e][c] = load(1, 8 * e + gid, 4 * tig + c);
    lift[e] = value_lift<BF16>(row_most(x[e]), row_least(x[e]));
  }
#pragma unroll
  for (int e = 0; e < 2; ++e) {
#pragma unroll
    for (int c = 0; c < 4; ++c) x[e][c] = load(0, 8 * e + gid, 4 * tig + c);
    if constexpr (BF16) {
      const int z = key_lift<BF16>(row_most(x[e]));
      f[e] = pow2(z);
      ks[e] = pow2(-z);
    }
  }
#pragma unroll
  for (int c = 0; c < 4; ++c) {  // 8 channels: two steps of the product
    const uint32_t xw[4] = {x[0][c].x, x[0][c].y, x[0][c].z, x[0][c].w};
    const uint32_t yw[4] = {x[1][c].x, x[1][c].y, x[1][c].z, x[1][c].w};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t a0 = to_half2<BF16>(xw[2 * i], f[0]), a1 = to_half2<BF16>(yw[2 * i], f[1]);
      const uint32_t a2 = to_half2<BF16>(xw[2 * i + 1], f[0]),
                     a3 = to_half2<BF16>(yw[2 * i + 1], f[1]);
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const uint2 q = st.query(n, 2 * c + i);
        mma(s[n], a0, a1, a2, a3, q.x, q.y);
      }
    }
  }
  uint32_t w[NT][2];
  tail_weights<NT>(p, st, rows, s, t0, ks, lift, w);
  uint4 v[2][2][2];
  float g[2][2];  // of rows 8 i + 2 tig + e: lanes 4 (2 tig + e) know them
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
#pragma unroll
      for (int c = 0; c < 2; ++c) v[i][e][c] = load(1, 8 * i + 2 * tig + e, 2 * gid + c);
      g[i][e] = pow2(__shfl_sync(0xffffffffu, lift[i], 8 * tig + 4 * e));
    }
#pragma unroll
  for (int c = 0; c < 2; ++c) {  // 8 channels each
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const auto word = [&](int i, int e) {
        const uint4& y = v[i][e][c];
        return lifted2<BF16>(k == 0 ? y.x : k == 1 ? y.y : k == 2 ? y.z : y.w, g[i][e]);
      };
      const uint32_t w00 = word(0, 0), w01 = word(0, 1), w10 = word(1, 0), w11 = word(1, 1);
      const uint32_t a0 = __byte_perm(w00, w01, 0x5410), a1 = __byte_perm(w00, w01, 0x7632);
      const uint32_t a2 = __byte_perm(w10, w11, 0x5410), a3 = __byte_perm(w10, w11, 0x7632);
#pragma unroll
      for (int n = 0; n < NT; ++n) mma(st.o[n][4 * c + k], a0, a1, a2, a3, w[n][0], w[n][1]);
    }
  }
}

// Queries of an item's row group n: row 8 n + gid's channels 32 tig .. 32 tig + 31, bf16 ones
// times a power of two, which is returned.
template <bool BF16>
__device__ __forceinline__ float load_group(const AttnParams& p, const Seq& q, int head, int n,
                                            uint2 (&out)[8]) {
  const int lane = threadIdx.x & 31, r = 8 * n + (lane >> 2);
  uint4 x[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = make_uint4(0u, 0u, 0u, 0u);
  if (r < q.n * p.c.d.gq) {
    const uint4* src = reinterpret_cast<const uint4*>(
        p.c.q + row_offset(p, p.c.q_stride, q.row, head, r) + 32 * (lane & 3));
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __ldg(src + i);
  }
  float f = 1.0f;
  if constexpr (BF16) {
    uint32_t m = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) m = largest(m, x[i]);
    m = max(m & 0xffffu, m >> 16);
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
    f = lift_of(m);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    out[2 * i] = make_uint2(to_half2<BF16>(x[i].x, f), to_half2<BF16>(x[i].y, f));
    out[2 * i + 1] = make_uint2(to_half2<BF16>(x[i].z, f), to_half2<BF16>(x[i].w, f));
  }
  return f;
}

// An item's queries, its rows' factors and positions, and empty results.  By all threads.
template <int NT, bool BF16>
__device__ __forceinline__ void begin_item(const AttnParams& p, const Seq& q, int head,
                                           Smem<NT>& sm, State<NT>& st, Rows& rows) {
  const int lane = threadIdx.x & 31, tig = lane & 3;
  if constexpr (!State<NT>::kOwnQueries) {
    const int warp = threadIdx.x >> 5;
    if (warp < NT) {  // (nobody reads the last item's any more: its parts have met)
      uint2 x[8];
      const float f = load_group<BF16>(p, q, head, warp, x);
#pragma unroll
      for (int i = 0; i < 8; ++i) sm.q[warp][i][lane] = x[i];
      if (tig == 0) sm.qf[8 * warp + (lane >> 2)] = f;
    }
    __syncthreads();
    st.shared_q = &sm.q[0][0][0];
  }
  rows.first = q.L - q.n;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    float f = 1.0f;
    if constexpr (State<NT>::kOwnQueries) f = load_group<BF16>(p, q, head, n, st.q[n]);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      float g = 1.0f;
      if constexpr (BF16) {
        if constexpr (State<NT>::kOwnQueries) g = __shfl_sync(0xffffffffu, f, 8 * tig + 4 * j);
        else g = sm.qf[8 * n + 2 * tig + j];
      }
      st.f[n][j] = p.c.scale_log2 / g;
      st.m[n][j] = kNone;
      st.e[n][j] = 0.0f;
      st.l[n][j] = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) st.o[n][i][j] = 0.0f;
  }
}

// TEST: a short bound, and no copies of the third warp's second block.
template <int NT, bool BF16, bool TEST>
__global__ void __launch_bounds__(32 * Smem<NT>::kWarps, 1)
rows_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ CUtensorMap k_map,
            const __grid_constant__ CUtensorMap v_map) {
  extern __shared__ __align__(1024) unsigned char raw[];
  Smem<NT>& sm = *reinterpret_cast<Smem<NT>*>(raw);
  constexpr int kSlots = Smem<NT>::kSlots, kWarps = Smem<NT>::kWarps;
  constexpr int kMergers = Smem<NT>::kMergers;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, gid = lane >> 2, tig = lane & 3;
  if (lane == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(warp & 1 ? &k_map : &v_map) : "memory");
    for (int i = 0; i < kSlots; ++i)
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 2;" ::"r"(sptr(&sm.full[warp][i]))
                   : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  Shares shares;
  int u0, u1;
  if (!plan_share<kTok, kItemCost>(p, sm.scan, &sm.start, 4 * kWarps, shares, u0, u1)) return;

  // Units of an item before the 16-bit ones are whole blocks; warp w takes every eighth.
  const auto whole_units = [](const Walk<kTok, kItemCost>& w) {
    return w.s.tile(w.s.n - 1) * kGroup + kGroup > w.q.L ? min(w.i1, w.s.n - 1) : w.i1;
  };
  // This warp's next block, over all items of the share: its item is in shared memory (its
  // fields would take registers from the results), `next` its unit, `limit` the item's last,
  // `entry` this lane's table entry of the 32 units from `entries` on.
  Walk<kTok, kItemCost>& ahead = sm.ahead[warp];
  int next = 0, limit = 0, entry = 0, entries = -1;
  bool some;  // the share has a tile
  {
    Walk<kTok, kItemCost> first;
    first.begin(p, sm.start, u0, u1);
    some = first.next(p);
    if (some) {
      next = first.i0 + warp;
      limit = whole_units(first);
    }
    ahead = first;
    __syncwarp();
  }
  // An item's queries come to L2 ahead of its blocks, its open tokens to shared memory if that
  // is free (`held`: the first unit of the item whose tokens it has): behind full rings a load
  // waits its turn of several microseconds.  The last two warps, which never have more blocks
  // than the others, take 16 open tokens each.
  const int half = warp - (kWarps - 2);
  const auto has_tail = [&](const Walk<kTok, kItemCost>& f) {
    const int open = open_tokens(f).y;
    return half >= 0 && f.i1 == f.s.n && open < kGroup && open > 16 * half;
  };
  int held = -1;
  const auto fetch_small = [&](const Walk<kTok, kItemCost>& f) {
    if (half < 0) return;
    const auto line = [](const void* at) {
      asm volatile("prefetch.global.L2 [%0];" ::"l"(at));
    };
    if (half && lane < f.q.n * p.c.d.gq) {
      const uint16_t* at = p.c.q + row_offset(p, p.c.q_stride, f.q.row, f.head, lane);
      line(at);
      line(at + 64);
    }
    if (held < 0 && has_tail(f)) {
      fetch_tail(p, f, 16 * half, sm.tail[half]);
      held = f.base;
    }
  };
  if (some) fetch_small(ahead);
  int fed = 0;  // TEST: this warp's blocks
  // The next block goes to slot `slot`.
  const auto feed = [&](int slot) {
    if (next >= limit) {
      Walk<kTok, kItemCost> f = ahead;
      while (next >= limit) {
        if (f.u >= f.end) break;
        f.advance(p);
        if (f.next(p)) {
          next = f.i0 + warp;
          limit = whole_units(f);
          fetch_small(f);
        }
      }
      entries = -1;
      __syncwarp();
      ahead = f;
      __syncwarp();
      if (next >= limit) return;  // the end of the share
    }
    if (entries < 0 || next >= entries + 32 * kWarps) {
      entries = next;
      const int i = next + kWarps * lane;
      entry = i < limit ? __ldg(p.c.cache.block_table + (long long)ahead.b * p.c.d.max_blocks +
                                ahead.s.tile(i))
                        : 0;
    }
    const int page = __shfl_sync(0xffffffffu, entry, (next - entries) / kWarps);
    next += kWarps;
    if (lane == 0) {
      const uint32_t bar = sptr(&sm.full[warp][slot]);
      if ((unsigned)page < (unsigned)p.c.cache.n_pages) {
        const int at = page * p.c.d.hkv + ahead.head;
        const uint32_t dst = sptr(sm.page[warp][slot]);
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar),
                     "r"(2 * kHalfPage)
                     : "memory");
        if (TEST && warp == 2 && fed++ == 1) return;
        asm volatile(
            "cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], "
            "[%1, {%2, %3}], [%4];" ::"r"(dst),
            "l"(&k_map), "r"(0), "r"(at * kGroup), "r"(bar)
            : "memory");
        asm volatile(
            "cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], "
            "[%1, {%2, %3}], [%4];" ::"r"(dst + kHalfPage),
            "l"(&v_map), "r"(0), "r"(at * kGroup), "r"(bar)
            : "memory");
        asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(
                         sptr(&sm.scale[warp][slot])),
                     "l"(p.c.cache.scales + 2ll * at)
                     : "memory");
        asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
      } else {
        set_flag(p.c.cache, KVQ_FLAG_BAD_PAGE);
        sm.scale[warp][slot] = make_float2(-1.0f, -1.0f);
        asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], 2;" ::"r"(bar) : "memory");
      }
    }
  };
#pragma unroll
  for (int i = 0; i < kSlots; ++i) feed(i);

  int slot = 0;
  uint32_t phase = 0;
  const auto arrived = [&](int i, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, 10000;\n"
        " selp.u32 %0, 1, 0, p;\n}"
        : "=r"(ok)
        : "r"(sptr(&sm.full[warp][i])), "r"(parity)
        : "memory");
    return ok != 0;
  };
  // Bounded; for a whole warp.
  const auto wait = [&](int i, uint32_t parity) {
    bool ok = arrived(i, parity);
    if (!ok) {
      const long long begun = clock64();
      while (!(ok = arrived(i, parity)) && clock64() - begun < (TEST ? kTestCycles : kWaitCycles)) {
      }
    }
    return __all_sync(0xffffffffu, ok) != 0;
  };
  bool lost = false;  // a wait ran out: the warp only keeps the others company
  Walk<kTok, kItemCost> w;
  w.begin(p, sm.start, u0, u1);
#pragma unroll 1
  for (; w.next(p); w.advance(p)) {
    State<NT> st;
    Rows rows;
    begin_item<NT, BF16>(p, w.q, w.head, sm, st, rows);
    const int whole = whole_units(w);
    if (has_tail(w)) {
      const auto copied = [] {
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncwarp();
      };
      copied();
      if (held != w.base) {  // (another item's, or none)
        fetch_tail(p, w, 16 * half, sm.tail[half]);
        copied();
      }
      tail_block<NT, BF16>(p, st, rows, sm.tail[half], open_tokens(w).x + 16 * half);
      held = -1;
      __syncwarp();
    }
    const auto blocks = [&](auto used) {
      constexpr int N = decltype(used)::value;
#pragma unroll 1
      for (int i = w.i0 + warp; i < whole; i += kWarps) {
        const int t0 = w.s.tile(i) * kGroup;
        if (lost || !wait(slot, phase)) {
          if (!lost && lane == 0) set_flag(p.c.cache, KVQ_FLAG_WAIT_TIMEOUT);
          lost = true;
          break;
        }
        float2 scale = sm.scale[warp][slot];
        if (scale.x > 0.0f) {
          if (scale.y == 1.0f && no_value(sm.page[warp][slot] + kHalfPage)) scale.y = kNoValue;
          const bool edge = t0 + kGroup - 1 > w.s.p0 ||
                            (p.c.window && t0 <= w.s.p1 - p.c.window && t0 + kGroup > p.c.sinks);
          block<N, NT>(p, st, rows, sm.page[warp][slot], scale, t0, edge);
        }
        __syncwarp();
        feed(slot);
        if (++slot == kSlots) slot = 0, phase ^= 1;
      }
    };
    const int used = (w.q.n * p.c.d.gq + 7) >> 3;
    if (NT == 1 || used <= 1) blocks(std::integral_constant<int, 1>{});
    else if (NT == 2 || used == 2) blocks(std::integral_constant<int, NT < 2 ? NT : 2>{});
    else if (NT == 3 || used == 3) blocks(std::integral_constant<int, NT < 3 ? NT : 3>{});
    else blocks(std::integral_constant<int, NT>{});
    // The warps' parts of the item meet in shared memory, always in the same order.
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float l = st.l[n][j];
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
        // one number for the maximum from here on; what it leaves of the two goes to sum and
        // results
        const float m = st.m[n][j] + st.e[n][j];
        st.e[n][j] += st.m[n][j] - m;
        st.m[n][j] = m;
        if (gid == 0) {
          sm.m[warp][8 * n + 2 * tig + j] = m;
          sm.l[warp][8 * n + 2 * tig + j] = l * exp2_fast(st.e[n][j]);
        }
      }
    __syncthreads();
    float mm[NT][2], ll[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int r = 8 * n + 2 * tig + j;
        float m = kNone, l = 0.0f;
#pragma unroll
        for (int k = 0; k < kWarps; ++k) m = fmaxf(m, sm.m[k][r]);
#pragma unroll
        for (int k = 0; k < kWarps; ++k) l = fmaf(sm.l[k][r], exp2_fast(sm.m[k][r] - m), l);
        mm[n][j] = m;
        ll[n][j] = l;
        const float g = exp2_fast((st.m[n][j] - m) + st.e[n][j]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          st.o[n][i][j] *= g;
          st.o[n][i][j + 2] *= g;
        }
      }
    // Four parts at a time go to slots 0 .. 3; two and one to slots that their own warps
    // were the last to read.
#pragma unroll
    for (int alive = kWarps; alive > 1;) {
      const int keep = alive > 2 * kMergers ? alive - kMergers : alive / 2;
      const bool four = alive - keep == kMergers;
      if (warp >= keep && warp < alive) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 8; ++i)
            sm.merge[four ? warp - keep : warp][8 * n + i][lane] =
                make_float4(st.o[n][i][0], st.o[n][i][1], st.o[n][i][2], st.o[n][i][3]);
      }
      __syncthreads();
      if (warp < alive - keep) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float4 x = sm.merge[four ? warp : warp + keep][8 * n + i][lane];
            st.o[n][i][0] += x.x, st.o[n][i][1] += x.y;
            st.o[n][i][2] += x.z, st.o[n][i][3] += x.w;
          }
      }
      alive = keep;
      if (alive >= 2 * kMergers) __syncthreads();
    }
    const int n_rows = w.q.n * p.c.d.gq;
    const bool direct = w.whole();
    if (warp == 0) {
      const int slot_row = w.slot(u0) * p.item_rows;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int r = 8 * n + 2 * tig + j;
          if (r >= n_rows) continue;
          if (direct) {
            const float f = ll[n][j] > 0.0f ? 1.0f / ll[n][j] : 0.0f;
            uint32_t x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
              x[i] = pack16<BF16>(st.o[n][i][j] * f, st.o[n][i][j + 2] * f);
            uint4* dst = reinterpret_cast<uint4*>(
                p.c.out + row_offset(p, p.c.out_stride, w.q.row, w.head, r) + 16 * gid);
            dst[0] = make_uint4(x[0], x[1], x[2], x[3]);
            dst[1] = make_uint4(x[4], x[5], x[6], x[7]);
          } else {
            float4* dst = reinterpret_cast<float4*>(
                p.part_o + (long long)(slot_row + r) * kHeadDim + 16 * gid);
#pragma unroll
            for (int i = 0; i < 4; ++i)
              dst[i] = make_float4(st.o[n][2 * i][j], st.o[n][2 * i][j + 2],
                                   st.o[n][2 * i + 1][j], st.o[n][2 * i + 1][j + 2]);
            if (gid == 0) p.part_ml[slot_row + r] = make_float2(mm[n][j], ll[n][j]);
          }
        }
    }
    if (direct) continue;
    // Whoever brings an item's last partial joins them, in the order of the tokens.  The
    // tickets are zero between calls.
    const int c0 = shares.owner(w.first_unit()), parts = shares.owner(w.last_unit()) - c0 + 1;
    if (warp == 0) {
      __threadfence();
      __syncwarp();
      if (lane == 0) {
        const bool last = atomicAdd(p.tickets + c0, 1) == parts - 1;
        if (last) p.tickets[c0] = 0;
        __threadfence();
        sm.join = last;
      }
    }
    __syncthreads();
    if (sm.join) {
      const int inside = shares.begin(c0) < w.base ? 1 : 0;
      for (int r = warp; r < n_rows; r += kWarps)
        join_row<BF16>(p, c0, inside, parts, r,
                       p.c.out + row_offset(p, p.c.out_stride, w.q.row, w.head, r));
    }
  }
  // copies that are still on their way get their time before the memory goes
  if (lost)
    for (int i = 0; i < kSlots; ++i)
      wait((slot + i) % kSlots, slot + i < kSlots ? phase : phase ^ 1);
}

// The tensor map of codes [rows][128], 32 rows a copy.
cudaError_t make_map(CUtensorMap* map, const void* base, long long rows) {
  using Encode = decltype(&cuTensorMapEncodeTiled);
  static std::atomic<Encode> found{nullptr};
  Encode encode = found.load(std::memory_order_acquire);
  if (!encode) {
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult r;
    const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000,
                                                           cudaEnableDefault, &r);
    if (e != cudaSuccess) return e;
    if (r != cudaDriverEntryPointSuccess || !fn) return cudaErrorNotSupported;
    encode = reinterpret_cast<Encode>(fn);
    found.store(encode, std::memory_order_release);
  }
  const cuuint64_t dims[2] = {(cuuint64_t)kHeadDim, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)kHeadDim};
  const cuuint32_t box[2] = {(cuuint32_t)kHeadDim, (cuuint32_t)kGroup}, one[2] = {1, 1};
  const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims,
                            strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

template <int NT, bool BF16, bool TEST = false>
cudaError_t launch(const AttnParams& p, int ctas, cudaStream_t stream) {
  static std::atomic<unsigned long long> done{0};
  cudaError_t e = once_per_device(done, [] {
    return cudaFuncSetAttribute(rows_kernel<NT, BF16, TEST>,
                                cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Smem<NT>));
  });
  if (e != cudaSuccess) return e;
  CUtensorMap k, v;
  const long long rows = (long long)p.c.cache.n_pages * p.c.d.hkv * kGroup;
  if ((e = make_map(&k, p.c.cache.k_codes, rows)) != cudaSuccess) return e;
  if ((e = make_map(&v, p.c.cache.v_codes, rows)) != cudaSuccess) return e;
  rows_kernel<NT, BF16, TEST><<<ctas, 32 * Smem<NT>::kWarps, sizeof(Smem<NT>), stream>>>(p, k, v);
  return cudaGetLastError();
}

template <int NT>
cudaError_t launch_type(const AttnParams& p, int ctas, cudaStream_t stream) {
  return p.c.d.bf16 ? launch<NT, true>(p, ctas, stream) : launch<NT, false>(p, ctas, stream);
}

}  // namespace

cudaError_t launch_rows(const AttnParams& p, int ctas, cudaStream_t stream, bool selftest) {
  if (selftest)
    return p.item_rows == 8 && !p.c.d.bf16 ? launch<1, false, true>(p, ctas, stream)
                                           : cudaErrorNotSupported;
  switch (p.item_rows) {
    case 8: return launch_type<1>(p, ctas, stream);
    case 16: return launch_type<2>(p, ctas, stream);
    case 24: return launch_type<3>(p, ctas, stream);
    default: return launch_type<4>(p, ctas, stream);
  }
}

}  // namespace block8
}  // namespace kvq
