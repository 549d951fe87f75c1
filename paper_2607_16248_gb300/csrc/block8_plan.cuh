// Work of kvq_block8_attn's kernels: who does what, and how shared items meet again.
//
// An item is one row tile of one (sequence, kv-head): rows t * gq + head of the sequence's
// new tokens t and the gq heads that share the kv-head.  Its units are the tiles of
// 2^TOK tokens that any of its rows sees, after a fixed cost in units; a tile counts as many
// units as the kernel says it takes for the item's rows (`weight`).  All items' units
// lie end to end (sequence, row tile, kv-head) and every CTA takes an equal contiguous
// share.  An item that several CTAs share leaves partials (unnormalised rows, maximum,
// sum) that are joined in the order of the tokens: by the CTA that comes last, or by a second
// kernel.
#pragma once

#include <type_traits>

#include "block8.cuh"

namespace kvq {
namespace block8 {

// An item that the shares of CTAs c .. last divide, left by CTA c for the join.
struct Split {
  int valid, inside, last, b, row_tile, head;
};

constexpr int kMostWeight = 7;  // units of a block with four groups of eight rows
// Fixed cost of an item in units.  Few rows (a block's are 4 to 7): queries, merge.  Many
// (units are tiles of 128 tokens): queries in, results out, the pipeline's filling.
constexpr int kRowsItemCost = 16, kChunkItemCost = 3;

struct AttnParams {
  AttnCall c;
  uint32_t gq_inverse;      // floor(2^32 / gq) + 1
  int min_rows, max_rows;   // the sequences this kernel takes, by their rows n * gq
  int item_rows;            // rows of an item and of a partial
  float* part_o;            // [2 * CTAs][item_rows][128]
  float2* part_ml;          // [2 * CTAs][item_rows]
  Split* splits;            // [CTAs]: for the kernel that joins
  int* tickets;             // [CTAs]: for CTAs that join, by the item's first CTA
};

#ifdef __CUDACC__
// Row r of a sequence: its token.  Rows stay below 2^28 (checked on the host), where the
// product with gq_inverse gives the exact quotient.
__device__ __forceinline__ int token_of_row(const AttnParams& p, int r) {
  return p.c.d.gq == 1 ? r : (int)__umulhi((uint32_t)r, p.gq_inverse);
}
// Offset of row r of (sequence with first row `row`, kv-head) in an array of queries.
__device__ __forceinline__ long long row_offset(const AttnParams& p,
                                                const long long (&stride)[2], int row,
                                                int kv_head, int r) {
  const int t = token_of_row(p, r);
  return (row + t) * stride[0] + (kv_head * p.c.d.gq + r - t * p.c.d.gq) * stride[1];
}

// A sequence as this kernel takes it: n is 0 where it is another kernel's.
__device__ __forceinline__ Seq attn_seq(const AttnParams& p, int b) {
  Seq s = seq_of(p.c.d, p.c.batch, b);
  const long long rows = (long long)s.n * p.c.d.gq;
  if (rows < p.min_rows || rows > p.max_rows) s.n = 0;
  return s;
}

// What one row tile of a sequence sees: token tiles 0 .. n_sink - 1, then from first on;
// n of them in all.
struct Span {
  int p0, p1;  // positions of the first and last row (may be < 0)
  int lo;      // first token of the window of the first row
  int n_sink, first, n;
  __device__ __forceinline__ int tile(int i) const { return i < n_sink ? i : first + i - n_sink; }
};
template <int TOK>
__device__ __forceinline__ Span span_of(const AttnParams& p, const Seq& q, int row_tile) {
  Span s;
  const int r0 = row_tile * p.item_rows;
  const int r1 = min(r0 + p.item_rows, q.n * p.c.d.gq) - 1;
  s.p0 = q.L - q.n + token_of_row(p, r0);
  s.p1 = q.L - q.n + token_of_row(p, r1);
  s.lo = p.c.window ? max(0, max(s.p0, 0) - p.c.window + 1) : 0;
  s.first = s.lo >> TOK;
  // sinks is 0 without a window; the sum passes 2^31 in the largest caches
  s.n_sink = min((int)(((uint32_t)p.c.sinks + ((1u << TOK) - 1)) >> TOK), s.first);
  s.n = s.n_sink + (max(s.p1, 0) >> TOK) - s.first + 1;
  return s;
}
__device__ __forceinline__ int row_tiles(const AttnParams& p, const Seq& q) {
  return q.n > 0 ? (int)((uint32_t)(q.n * p.c.d.gq + p.item_rows - 1) / (uint32_t)p.item_rows)
                 : 0;
}

// CTA c's share of the units: [begin(c), begin(c + 1)).
// Over all items: equal to within one unit.  Over items of one size (`even`), each divided
// among as many CTAs (`parts`): a share that crosses from an item to the next costs its CTA
// the next one's queries, merge and partial, 4 us of one chat's 27.
struct Shares {
  int q, r, n;      // units = n q + r over n CTAs
  int even, parts;  // an item's units, 0: shares over all items
  __device__ __forceinline__ int begin(int c) const {
    if (even) {
      const int i = (int)((uint32_t)c / (uint32_t)parts);
      return i * even + (int)((uint32_t)((c - i * parts) * even) / (uint32_t)parts);
    }
    return c * q + min(c, r);
  }
  __device__ __forceinline__ int owner(int u) const {
    if (even) {
      const int i = (int)((uint32_t)u / (uint32_t)even);
      return i * parts + (int)(((uint32_t)(u - i * even + 1) * (uint32_t)parts - 1u) /
                               (uint32_t)even);
    }
    const int wide = (q + 1) * r;  // units of the CTAs that have q + 1
    return u < wide ? (int)((uint32_t)u / (uint32_t)(q + 1))
                    : r + (int)((uint32_t)(u - wide) / (uint32_t)q);
  }
};

// Where a CTA's share begins.
struct Start {
  int b, row_tile, head, step;
};

// Units of a token tile for a sequence's rows.  Few rows: each row group more is more
// products, and what a block takes beside its bytes shows while bytes and products share
// the time (16 chats with one to five drafts: 148 us by blocks alone, CTAs between 92 and
// 145 us busy).
template <int TOK>
__device__ __forceinline__ int weight(const AttnParams& p, const Seq& q) {
  if constexpr (TOK == 7) return 1;
  else return kMostWeight - 4 + min((q.n * p.c.d.gq + 7) >> 3, 4);
}
// Units of all sequences, this CTA's share and where it begins, by all threads of the CTA
// (at most 32 warps).  At least `least` units a CTA.  Ends behind a barrier; false where
// the CTA has no share.
template <int TOK, int COST>
__device__ __forceinline__ bool plan_share(const AttnParams& p, int* scan, Start* start,
                                           int least, Shares& shares, int& u0, int& u1) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, threads = blockDim.x;
  const int per = (p.c.d.batch + threads - 1) / threads;
  const int b0 = min(p.c.d.batch, tid * per), b1 = min(p.c.d.batch, b0 + per);
  const auto units = [&](const Seq& q) {
    int n = 0;
    const int tiles = row_tiles(p, q), wt = weight<TOK>(p, q);
#pragma unroll 1
    for (int t = 0; t < tiles; ++t) n += (span_of<TOK>(p, q, t).n * wt + COST) * p.c.d.hkv;
    return n;
  };
  int mine = 0;
#pragma unroll 1
  for (int b = b0; b < b1; ++b) {
    const Seq q = attn_seq(p, b);
    if (q.bad && blockIdx.x == 0) set_flag(p.c.cache, q.bad);
    mine += units(q);
  }
  int inc = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += y;
  }
  if (lane == 31) scan[warp] = inc;
  // few sequences' items of one size: that size (in a place that no warp's sum has)
  if (TOK != 7 && warp == 0) {
    const int size = mine / p.c.d.hkv, most = __reduce_max_sync(0xffffffffu, size);
    const bool one = __all_sync(0xffffffffu, size == 0 || size == most);
    if (lane == 0) scan[31] = one && p.c.d.batch <= 32 && most < 1 << 20 ? most : 0;
  }
  __syncthreads();
  int warps = lane < threads / 32 ? scan[lane] : 0;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, warps, o);
    if (lane >= o) warps += y;
  }
  const int total = __shfl_sync(0xffffffffu, warps, 31);
  int before = __shfl_sync(0xffffffffu, warps, warp > 0 ? warp - 1 : 0);
  if (warp == 0) before = 0;
  before += inc - mine;
  shares.n = min((int)gridDim.x, (int)(((uint32_t)total + least - 1) / (uint32_t)least));
  shares.even = 0;
  if (TOK != 7 && scan[31]) {
    // as many CTAs an item as there are, or as have `least` units; unless a tenth of the GPU
    // would be left
    const int size = scan[31], items = (int)((uint32_t)total / (uint32_t)size);
    const int fill = (int)gridDim.x / items, need = max(size / least, 1);
    if (fill >= 1 && (need <= fill || fill * items * 10 >= (int)gridDim.x * 9)) {
      shares.even = size;
      shares.parts = min(fill, need);
      shares.n = shares.parts * items;
    }
  }
  if ((int)blockIdx.x >= shares.n) return false;
  shares.q = (int)((uint32_t)total / (uint32_t)shares.n);
  shares.r = total - shares.q * shares.n;
  u0 = shares.begin(blockIdx.x);
  u1 = shares.begin(blockIdx.x + 1);
  if (before <= u0 && u0 < before + mine) {
    int at = before;
#pragma unroll 1
    for (int b = b0; b < b1; ++b) {
      const Seq q = attn_seq(p, b);
      const int tiles = row_tiles(p, q);
#pragma unroll 1
      for (int t = 0; t < tiles; ++t) {
        const int n = span_of<TOK>(p, q, t).n * weight<TOK>(p, q) + COST;
        if (u0 >= at && u0 < at + n * p.c.d.hkv) {
          start->b = b;
          start->row_tile = t;
          start->head = (int)((uint32_t)(u0 - at) / (uint32_t)n);
          start->step = u0 - at - start->head * n;
        }
        at += n * p.c.d.hkv;
      }
    }
  }
  __syncthreads();
  return true;
}

// The items of a share, in order; every role walks them.
template <int TOK, int COST>
struct Walk {
  int u, end, base;       // next unit, end of the share, first unit of the item
  int b, row_tile, head;
  Seq q;                  // the item's sequence
  Span s;
  std::conditional_t<TOK == 7, std::integral_constant<int, 1>, int> wt;  // units of a tile
  int i0, i1;             // the item's tiles in this share: those whose first unit lies there
  __device__ __forceinline__ void begin(const AttnParams& p, const Start& st, int u0, int u1) {
    u = u0;
    end = u1;
    b = st.b;
    row_tile = st.row_tile;
    head = st.head;
    base = u0 - st.step;
    if (u < end) {
      q = attn_seq(p, b);
      s = span_of<TOK>(p, q, row_tile);
      if constexpr (TOK != 7) wt = weight<TOK>(p, q);
    }
  }
  // The first tile that begins at unit x of the item or behind it.
  __device__ __forceinline__ int tile_from(int x) const {
    return TOK == 7 ? x : (int)((uint32_t)(x + wt - 1) / (uint32_t)wt);
  }
  // The item's first unit, and the last tile's.
  __device__ __forceinline__ int first_unit() const { return base + COST; }
  __device__ __forceinline__ int last_unit() const { return base + COST + (s.n - 1) * wt; }
  // The current item's part of the share; false at the end.
  __device__ __forceinline__ bool next(const AttnParams& p) {
    while (u < end) {
      const int local = u - base, stop = min(s.n * wt + COST, local + end - u);
      i0 = tile_from(max(local - COST, 0));
      i1 = tile_from(max(stop - COST, 0));
      if (i1 > i0) return true;
      advance(p);  // nothing but a piece of the item's fixed cost or of a tile
    }
    return false;
  }
  __device__ __forceinline__ void advance(const AttnParams& p) {
    base += s.n * wt + COST;
    u = min(base, end);
    if (++head < p.c.d.hkv || u >= end) return;
    head = 0;
    if (++row_tile == row_tiles(p, q)) {
      row_tile = 0;
      do {
        q = attn_seq(p, ++b);
      } while (q.n == 0);  // the share ends behind another item
    }
    s = span_of<TOK>(p, q, row_tile);
    if constexpr (TOK != 7) wt = weight<TOK>(p, q);
  }
  __device__ __forceinline__ bool whole() const { return i0 == 0 && i1 == s.n; }
  // Slot of the CTA's partial: 0 for the item that its share begins in.
  __device__ __forceinline__ int slot(int u0) const { return 2 * blockIdx.x + (u0 < base ? 1 : 0); }
};

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float log2_fast(float x) {
  float y;
  asm("lg2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
template <bool BF16>
__device__ __forceinline__ uint32_t pack16(float a, float b) {
  if constexpr (BF16) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  } else {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
}

// Elements of the open block go to fp16 times 2^lift, and two rows share nothing.  Keys: their
// row's largest magnitude to 2^14, bits from 2^-100 on; elements are exact down to 2^-24 of
// the largest.  Values, bits from 2^-80 on (sums of 2^lift stay within fp32): to 2^8, where the
// codes are, because an element shares fp16's range with its weight, which has 2^-lift in it
// (with 2^14 a first token without a value cost the newest ones theirs); higher, up to 2^14,
// where the row's smallest element would lose bits.  Rows of nothing as if they were the
// smallest, so that their weights count beside any others'.
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
template <bool BF16>
__device__ __forceinline__ int exponent_of(uint32_t bits) {
  const float m = BF16 ? __uint_as_float(bits << 16) : __half2float(__ushort_as_half(bits));
  return (int)(__float_as_uint(m) >> 23) - 127;
}
template <bool BF16>
__device__ __forceinline__ int key_lift(uint32_t bits) {
  const int lift = bits ? 14 - max(exponent_of<BF16>(bits), -100) : 0;
  return BF16 ? lift : max(lift, 0);  // (fp16's smallest would not stand 2^-1)
}
// (least: the smallest magnitude but 0, less 1; 0xffff for none)
__device__ __forceinline__ uint32_t least2(uint32_t m, uint32_t x) {
  return __vminu2(m, __vsub2(x & 0x7fff7fffu, 0x00010001u));
}
template <bool BF16>
__device__ __forceinline__ int value_lift(uint32_t most, uint32_t least) {
  if (!most) return 60;  // 2^-60: kNoValue
  const int e = max(exponent_of<BF16>(most), -80);
  return min(14 - e, max(8 - e, (BF16 ? -17 : -14) - exponent_of<BF16>(least + 1)));
}
template <bool BF16>
__device__ __forceinline__ uint32_t lifted2(uint32_t u, float f) {
  if constexpr (BF16)
    return pack16<false>(__uint_as_float(u << 16) * f, __uint_as_float(u & 0xffff0000u) * f);
  const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&u));
  return pack16<false>(x.x * f, x.y * f);
}
template <bool BF16>
__device__ __forceinline__ uint4 lifted8(const uint4& v, float f) {
  return make_uint4(lifted2<BF16>(v.x, f), lifted2<BF16>(v.y, f), lifted2<BF16>(v.z, f),
                    lifted2<BF16>(v.w, f));
}
// What stands for the scale of a block whose values are all zero.  By the format it is 1, but a
// weight is held with its value's scale in it, and beside small values those of a large
// scale would lose the others' bits.
constexpr float kNoValue = 0x1p-60f;
// A score's factor in the exponent is at least this: masked scores are -inf, and their product
// with 0 would be NaN; no score is large enough to show the difference.
constexpr float kLeastFactor = 0x1p-126f;

// Row r of an item's partials to its result, by a warp.  CTA c0 + i left the i-th, CTA c0 in
// its slot `inside`.  Each lane finds the weights of one of every 32, then the weighted rows
// are summed in order.  A partial without a seen token weighs nothing, whatever it holds.
template <bool BF16>
__device__ __forceinline__ void join_row(const AttnParams& p, int c0, int inside, int n, int r,
                                         uint16_t* out) {
  const int lane = threadIdx.x & 31;
  const auto slot = [&](int i) {
    return (long long)(2 * (c0 + i) + (i == 0 ? inside : 0)) * p.item_rows + r;
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
  float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
  for (int k = 0; k < kMost; ++k) {
#pragma unroll 8
    for (int i = 32 * k; i < min(n, 32 * k + 32); ++i) {
      const float x = __shfl_sync(0xffffffffu, ml[k].x, i & 31) * f;
      const float4 v =
          __ldcg(reinterpret_cast<const float4*>(p.part_o + slot(i) * kHeadDim) + lane);
      if (x > 0.0f) {
        sum.x = fmaf(v.x, x, sum.x);
        sum.y = fmaf(v.y, x, sum.y);
        sum.z = fmaf(v.z, x, sum.z);
        sum.w = fmaf(v.w, x, sum.w);
      }
    }
  }
  reinterpret_cast<uint2*>(out)[lane] =
      make_uint2(pack16<BF16>(sum.x, sum.y), pack16<BF16>(sum.z, sum.w));
}
#endif

// Launchers of the kernels: few rows (block8_rows.cu), many (block8_chunk.cu).
constexpr int kFewRows = 32;
cudaError_t launch_rows(const AttnParams& p, int ctas, cudaStream_t stream, bool selftest);
cudaError_t launch_chunk(const AttnParams& p, int ctas, cudaStream_t stream, bool selftest);

}  // namespace block8
}  // namespace kvq
