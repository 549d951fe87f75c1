// The next token of each row of logits (kvq_sample).
//
// The order of the tokens (value descending, lowest index first) is the order
// of the 64-bit number (ordered bits of z) << 32 | ~index, descending: a limit
// keeps the tokens at or above a threshold of that number.  What a row's limits
// keep is usually a small part of it, so a row is read once:
//   sample   8192 logits spread over the row give a bound tau below which the
//            limits will hardly reach (counts of a coarse histogram);
//   stream   tokens at or above tau go to a list in shared memory, the weights
//            of the others to a sum;
//   select   on the list: a histogram over 2048 value ranges finds the range in
//            which a limit falls, the few tokens of that range are ranked exactly;
//   draw     the kept token with the largest d - ln(-ln u).
// Up to eight CTAs (a cluster) stream a row when rows are few; their lists are
// joined in the first.  When the list does not hold what the limits need (a flat
// row, a limit near 1, ties beyond the list) the row itself takes its place in
// the last two steps: the result is the same, later.
//
// Bound: many rows, the stream, 4 bytes a logit, and what follows it on the lists
// (128 rows of 152063 by top-p 0.9, about 12000 tokens a list: 67 us, where the bytes
// take 11); one row, the chain of a dozen barriers and two cluster exchanges (128256:
// 13 us greedy, 22 with top-k and top-p).  The row in place of its list costs 60 us
// (128256, 20 free tokens, k 50) to 250 (128 rows of 152064 by top-p 0.99).
//
// Sums that decide what is kept are of integers (weights in units of 2^-40) or,
// for the weights left out of the list, of fp32 numbers in a fixed order.

#include "serve.cuh"

namespace kvq {

namespace {

using u64 = unsigned long long;
constexpr int kThreads = 1024, kWarps = kThreads / 32, kMaxVocab = 262144;
constexpr int kCap = 20480;      // list entries of a CTA
constexpr int kBins = 2048;      // value ranges of the selection
constexpr int kEdge = 1024;      // tokens of one range ranked directly
constexpr int kSample = 8 * kThreads, kCoarse = 512;  // sampled logits, ranges of 1/16 nat
constexpr float kPerNat = 16.0f;
// An unlimited draw is made in the stream with keys relative to the sampled maximum.
// They are taken when the row's maximum is at most this many units of T above it: the
// three roundings of a key that can win then add up to less than 1e-5.  Further up the
// noise would be lost in the rounding of (z - m0) / T.
constexpr float kDrawReach = 32.0f;

struct Entry {
  float z;
  int i;
};
struct Sm {
  Entry list[kCap];
  uint32_t count[kBins], mass[3][kBins];  // 14-bit pieces of the weights
  u64 edge_key[kEdge], edge_mass[kEdge];
  u64 part[kWarps], part2[kWarps];
  float fpart[kWarps];
  u64 before_c, before_m, cut_key, cut_mass;
  float tau, tail;
  int n, n_edge, range, peer_n[8];
  u64 best;
  float best_z;
};

// Bits of a float32 whose unsigned order is the numbers' (-0 as +0).
__device__ __forceinline__ uint32_t ordered(float z) {
  const uint32_t u = __float_as_uint(z == 0.0f ? 0.0f : z);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ u64 rank_key(float z, int i) {
  return ((u64)ordered(z) << 32) | (uint32_t)~i;
}
__device__ __forceinline__ float key_value(u64 k) {
  const uint32_t u = (uint32_t)(k >> 32);
  return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ int key_index(u64 k) { return (int)~(uint32_t)k; }

// A reduction over the CTA; every thread gets the result.
template <typename F>
__device__ __forceinline__ u64 reduce(Sm& s, u64 v, F f) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v = f(v, __shfl_xor_sync(0xffffffffu, v, o));
  __syncthreads();
  if ((threadIdx.x & 31) == 0) s.part[threadIdx.x >> 5] = v;
  __syncthreads();
  v = s.part[threadIdx.x & 31];
#pragma unroll
  for (int o = 16; o; o >>= 1) v = f(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
// The larger of a and of b over the CTA, in one go.
__device__ __forceinline__ void most2(Sm& s, u64& a, u64& b) {
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    const u64 x = __shfl_xor_sync(0xffffffffu, a, o), y = __shfl_xor_sync(0xffffffffu, b, o);
    a = a > x ? a : x;
    b = b > y ? b : y;
  }
  __syncthreads();
  if ((threadIdx.x & 31) == 0) s.part[threadIdx.x >> 5] = a, s.part2[threadIdx.x >> 5] = b;
  __syncthreads();
  a = s.part[threadIdx.x & 31];
  b = s.part2[threadIdx.x & 31];
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    const u64 x = __shfl_xor_sync(0xffffffffu, a, o), y = __shfl_xor_sync(0xffffffffu, b, o);
    a = a > x ? a : x;
    b = b > y ? b : y;
  }
}
__device__ __forceinline__ u64 add(u64 a, u64 b) { return a + b; }
__device__ __forceinline__ u64 most(u64 a, u64 b) { return a > b ? a : b; }

// e in [0, 1] as a multiple of 2^-40.
__device__ __forceinline__ u64 mass_of(float e) { return (u64)__float2ull_rn(e * 0x1p40f); }

struct Row {
  const float *z, *u;
  int V;
  float T;                 // > 0
  bool greedy;
  int k;                   // 0: no limit
  float p, m;              // >= 1, <= 0: no limit
};

// Where the tokens of a selection are: the list, or the whole row.
struct ListSource {
  static constexpr int kAtOnce = 1;
  const Entry* list;
  int n;
  __device__ __forceinline__ int size() const { return n; }
  __device__ __forceinline__ Entry at(int j) const { return list[j]; }
};
struct RowSource {
  static constexpr int kAtOnce = 8;
  const float* z;
  int V;
  __device__ __forceinline__ int size() const { return V; }
  __device__ __forceinline__ Entry at(int j) const { return Entry{z[j], j}; }
};

// f on every token of a source that is not -inf; eight loads at a time from memory
// (one by one, a row of 152064 by top-p 0.99 took 284 us and takes 221).
template <typename S, typename F>
__device__ __forceinline__ void for_each(const S& src, F f) {
  constexpr int kAtOnce = S::kAtOnce;
  const int n = src.size();
#pragma unroll 1
  for (int j0 = threadIdx.x; j0 < n; j0 += kAtOnce * kThreads) {
    Entry e[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int j = j0 + k * kThreads;
      e[k] = j < n ? src.at(j) : Entry{-INFINITY, 0};
    }
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k)
      if (e[k].z > -INFINITY) f(e[k]);
  }
}

// Prefix of the ranges: the first range at which `goal` tokens (or weights) are
// reached, and the count and weight before it; -1 if it is not reached.  By warp
// 0: 64 ranges a lane, then the 64 of the lane where it happens, two a lane.
// Results in s.range, s.before_c, s.before_m.
__device__ __forceinline__ u64 range_mass(const Sm& s, int b) {
  return s.mass[0][b] + ((u64)s.mass[1][b] << 14) + ((u64)s.mass[2][b] << 28);
}
__device__ void find_range(Sm& s, u64 goal, bool by_mass) {
  constexpr int kPer = kBins / 32;
  const int lane = threadIdx.x;
  if (threadIdx.x < 32) {
    u64 c = 0, m = 0;
#pragma unroll 4
    for (int j = 0; j < kPer; ++j) {
      const int b = lane * kPer + ((j + lane) & (kPer - 1));
      c += s.count[b];
      m += range_mass(s, b);
    }
    u64 ci = c, mi = m;
    for (int o = 1; o < 32; o <<= 1) {
      const u64 x = __shfl_up_sync(0xffffffffu, ci, o), y = __shfl_up_sync(0xffffffffu, mi, o);
      if (lane >= o) ci += x, mi += y;
    }
    const unsigned hit = __ballot_sync(0xffffffffu, (by_mass ? mi : ci) >= goal);
    if (!hit) {
      if (lane == 0) s.range = -1;
    } else {
      const int at = __ffs(hit) - 1, b = at * kPer + 2 * lane;
      const u64 c0 = __shfl_sync(0xffffffffu, ci - c, at);
      const u64 m0 = __shfl_sync(0xffffffffu, mi - m, at);
      const u64 ca = s.count[b], cb = s.count[b + 1], ma = range_mass(s, b),
                mb = range_mass(s, b + 1);
      u64 cs = ca + cb, ms = ma + mb;
      for (int o = 1; o < 32; o <<= 1) {
        const u64 x = __shfl_up_sync(0xffffffffu, cs, o), y = __shfl_up_sync(0xffffffffu, ms, o);
        if (lane >= o) cs += x, ms += y;
      }
      const unsigned inner = __ballot_sync(0xffffffffu, (by_mass ? m0 + ms : c0 + cs) >= goal);
      if (lane == __ffs(inner) - 1) {
        const u64 before_c = c0 + cs - ca - cb, before_m = m0 + ms - ma - mb;
        const bool second = (by_mass ? before_m + ma : before_c + ca) < goal;
        s.range = b + (second ? 1 : 0);
        s.before_c = before_c + (second ? ca : 0ull);
        s.before_m = before_m + (second ? ma : 0ull);
      }
    }
  }
  __syncthreads();
}

// The threshold of a limit: the largest rank key at or above which there are
// `goal` tokens (or weights), 0 if the source has fewer.  *weight: the weights
// at or above it.
template <typename S, typename BinOf, typename MassOf>
__device__ u64 threshold(Sm& s, const S& src, BinOf bin_of, MassOf weight_of, u64 goal,
                         bool by_mass, u64* weight) {
  const int tid = threadIdx.x;
  find_range(s, goal, by_mass);
  const int range = s.range;
  const u64 before_c = s.before_c, before_m = s.before_m;
  if (tid == 0) s.n_edge = 0, s.cut_key = 0, s.cut_mass = 0;
  __syncthreads();  // ahead of any return: the next limit's find_range writes s.range again
  if (range < 0) return 0;
  for_each(src, [&](const Entry& e) {
    if (bin_of(e.z) == range) {
      const int at = atomicAdd(&s.n_edge, 1);
      if (at < kEdge) {
        s.edge_key[at] = rank_key(e.z, e.i);
        s.edge_mass[at] = weight_of(e.z);
      }
    }
  });
  __syncthreads();
  const int n = s.n_edge;
  if (n <= kEdge) {
    if (tid < n) {
      const u64 mine = s.edge_key[tid];
      u64 c = before_c, m = before_m;
      for (int j = 0; j < n; ++j)
        if (s.edge_key[j] > mine) {
          ++c;
          m += s.edge_mass[j];
        }
      // the token with which the goal is reached
      if ((by_mass ? m : c) < goal && (by_mass ? m + s.edge_mass[tid] : c + 1) >= goal) {
        s.cut_key = mine;
        s.cut_mass = m + s.edge_mass[tid];
      }
    }
    __syncthreads();
    *weight = s.cut_mass;
    return s.cut_key;
  }
  // more tokens than can be ranked at once (ties): bit by bit
  u64 t = 0;
  for (int bit = 63; bit >= 0; --bit) {
    const u64 c = t | (1ull << bit);
    u64 sum = 0;
    for_each(src, [&](const Entry& e) {
      if (rank_key(e.z, e.i) >= c) sum += by_mass ? weight_of(e.z) : 1ull;
    });
    if (reduce(s, sum, add) >= goal) t = c;
  }
  u64 sum = 0;
  for_each(src, [&](const Entry& e) {
    if (rank_key(e.z, e.i) >= t) sum += weight_of(e.z);
  });
  *weight = reduce(s, sum, add);
  return t;
}

// Selection and draw on a source.  tau: the source holds every token at or above
// it; tail: the weights of the others, relative to a logit of m0.  *weight: all
// tokens' weights.  given: the winner of an unlimited draw made relative to m0, or 0.
// False: the source does not hold what the limits need, or m0 was too low for the draw.
template <typename S>
__device__ bool choose(Sm& s, const Row& r, const S& src, float tau, float m0, float tail,
                       u64 given, int* token, u64* weight) {
  const int tid = threadIdx.x;
  const bool limits = !r.greedy && !given && (r.k > 0 || r.p < 1.0f);
  u64 top = 0, low = 0;  // largest key, complement of the least
  for_each(src, [&](const Entry& e) {
    const u64 key = rank_key(e.z, e.i);
    top = most(top, key);
    low = most(low, ~key);
  });
  if (limits) {
    for (int j = tid; j < kBins; j += kThreads) {
      s.count[j] = 0;
      s.mass[0][j] = s.mass[1][j] = s.mass[2][j] = 0;
    }
  }
  most2(s, top, low);
  if (top == 0) return false;
  const float zmax = key_value(top);
  const auto dist = [&](float z) { return __fdiv_rn(z - zmax, r.T); };
  if (given && !(dist(m0) >= -kDrawReach)) return false;
  const auto weight_of = [&](float z) { return mass_of(expf(dist(z))); };
  // ranges of equal width from the largest value to the least of the source
  const float width = zmax - key_value(~low);
  const float scale = width > 0.0f && width < INFINITY ? (kBins - 1) / width : 0.0f;
  const auto bin_of = [&](float z) {
    return min((int)__fmul_rn(__fsub_rn(zmax, z), scale), kBins - 1);
  };
  u64 sum = 0;
  for_each(src, [&](const Entry& e) {
    const u64 q = weight_of(e.z);
    sum += q;
    if (limits) {
      const int b = bin_of(e.z);
      if (r.k > 0) atomicAdd(&s.count[b], 1u);
      if (q && r.p < 1.0f) {
        atomicAdd(&s.mass[0][b], (uint32_t)(q & 0x3fffu));
        if (q >> 14) atomicAdd(&s.mass[1][b], (uint32_t)(q >> 14) & 0x3fffu);
        if (q >> 28) atomicAdd(&s.mass[2][b], (uint32_t)(q >> 28));
      }
    }
  });
  sum = reduce(s, sum, add);
  const u64 total = sum + (tail > 0.0f ? mass_of(tail * expf(dist(m0))) : 0ull);
  u64 win = top;
  if (given) {
    win = given;
  } else if (!r.greedy) {
    // a limit that the source ends before is as good as none where min-p ends
    // earlier still
    const bool enough = r.m > 0.0f && expf(dist(tau)) < r.m;
    u64 cut = 0, kept = total;
    if (r.k > 0) {
      u64 w = 0;
      cut = threshold(s, src, bin_of, weight_of, (u64)r.k, false, &w);
      if (cut) kept = w;
      else if (tau > -INFINITY && (!enough || r.p < 1.0f)) return false;
    }
    if (r.p < 1.0f) {
      // the least whole number >= p * kept, p in units of 2^-32 (64-bit floating
      // point would take longer than the rest)
      const u64 p32 = (u64)__float2ull_rn(fmaxf(r.p, 0.0f) * 0x1p32f);
      const u64 frac = kept * p32, whole = __umul64hi(kept, p32);
      const u64 goal = (whole << 32 | frac >> 32) + ((uint32_t)frac ? 1 : 0);
      u64 w;
      const u64 c = goal ? threshold(s, src, bin_of, weight_of, goal, true, &w) : top;
      if (c) cut = most(cut, c);
      else if (tau > -INFINITY && !enough) return false;
    }
    if (r.k <= 0 && r.p >= 1.0f && tau > -INFINITY && !enough) return false;
    u64 best = 0;
    for_each(src, [&](const Entry& e) {
      const u64 key = rank_key(e.z, e.i);
      if (key < cut) return;
      const float d = dist(e.z);
      if (expf(d) < r.m && key != top) return;
      best = most(best, rank_key(d - logf(-logf(r.u[e.i])), e.i));
    });
    win = reduce(s, best, most);
  }
  *token = key_index(win);
  *weight = total;
  if (tid == 0) s.best_z = zmax;
  return true;
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile(
      "barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::
          : "memory");
}
__device__ __forceinline__ uint32_t peer(const void* p, uint32_t rank) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;"
               : "=r"(a)
               : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
  return a;
}
__device__ __forceinline__ uint32_t peer_u32(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ u64 peer_u64(uint32_t a) {
  u64 v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(a) : "memory");
  return v;
}

// kCl CTAs a row.
template <int kCl>
__global__ void __launch_bounds__(kThreads, 1) sample_kernel(SampleCall p) {
  extern __shared__ __align__(16) unsigned char raw[];
  Sm& s = *reinterpret_cast<Sm*>(raw);
  const int tid = threadIdx.x, lane = tid & 31, b = blockIdx.x / kCl;
  const int rank = kCl > 1 ? (int)cluster_rank() : 0;
  Row r;
  r.z = p.logits + b * p.logits_stride;
  r.u = p.noise ? p.noise + b * p.noise_stride : nullptr;
  r.V = p.vocab;
  r.T = p.temperature ? p.temperature[b] : 1.0f;
  r.greedy = !(r.T > 0.0f) || !r.u;
  r.T = r.T > 0.0f ? fminf(fmaxf(r.T, 1e-30f), 1e30f) : 1.0f;  // 1 / T stays finite
  r.k = p.top_k ? p.top_k[b] : 0;
  if (r.k < 0 || r.k >= r.V) r.k = 0;
  r.p = p.top_p ? p.top_p[b] : 1.0f;
  r.m = p.min_p ? p.min_p[b] : 0.0f;
  const bool all = !r.greedy && r.k <= 0 && !(r.p < 1.0f) && !(r.m > 0.0f);
  const float per_t = 1.0f / r.T;

  // Sample: every CTA of the row takes the same logits and finds the same tau.
  float x[8];
  float m0 = -INFINITY;
  const int taken = min(r.V, kSample);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int at = r.V <= kSample ? j * kThreads + tid
                                  : (int)((long long)j * (r.V - kThreads) / 7) + tid;
    x[j] = at < r.V ? r.z[at] : -INFINITY;
    m0 = fmaxf(m0, x[j]);
  }
  for (int j = tid; j < kCoarse; j += kThreads) s.count[j] = 0;
  if (tid == 0) s.n = 0;
  m0 = key_value(reduce(s, rank_key(m0, 0), most));
  const bool seen = m0 > -INFINITY;  // else the sample says nothing: the row itself
  if (seen && (r.greedy || all)) {
    if (tid == 0) s.tau = m0;
  } else if (seen) {
    const float scale = kPerNat * per_t;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (x[j] > -INFINITY) atomicAdd(&s.count[min((int)((m0 - x[j]) * scale), kCoarse - 1)], 1u);
    __syncthreads();
    if (tid < 32) {
      // counts and weights up to each range, 16 ranges a lane
      constexpr int kPer = kCoarse / 32;
      float c[kPer], w[kPer], cs = 0.0f, ws = 0.0f;
      for (int j = 0; j < kPer; ++j) {
        c[j] = (float)s.count[lane * kPer + j];
        w[j] = c[j] * __expf(-(lane * kPer + j + 0.5f) / kPerNat);
        cs += c[j];
        ws += w[j];
      }
      float ci = cs, wi = ws;
      for (int o = 1; o < 32; o <<= 1) {
        const float a = __shfl_up_sync(0xffffffffu, ci, o), d = __shfl_up_sync(0xffffffffu, wi, o);
        if (lane >= o) ci += a, wi += d;
      }
      const float all_w = __shfl_sync(0xffffffffu, wi, 31);
      // The weights of the first tokens of the sample say little about the row (one
      // far above the rest stands for V / 8192 others): those up to the range that
      // reaches eight tokens do not count.
      float head = 0.0f;
      {
        float cc = ci - cs, ww = wi - ws;
        bool there = false;
        for (int j = 0; j < kPer; ++j) {
          cc += c[j];
          ww += w[j];
          if (!there && cc >= 8.0f) there = true, head = ww;
        }
        const unsigned reached = __ballot_sync(0xffffffffu, there);
        head = __shfl_sync(0xffffffffu, head, reached ? __ffs(reached) - 1 : 31);
      }
      const float rate = (float)taken / (float)r.V;
      // how many sampled tokens and which weight the list should reach down to
      const float most_c = 0.6f * kCap * rate;
      float want_c = 0.0f, want_w = 0.0f;
      if (r.k > 0) {
        // the first k hold about k * rate sampled tokens, six deviations more at most
        want_c = 1.5f * r.k * rate + 6.0f * sqrtf(r.k * rate) + 8.0f;
      } else if (r.p < 1.0f) {
        want_c = 2048.0f * rate;
        want_w = all_w - 0.125f * (1.0f - r.p) * (all_w - head);
      }
      int mine = kCoarse;  // first range that reaches both
      int last = -1;       // last range within the list's room
      float cc = ci - cs, ww = wi - ws;
      for (int j = 0; j < kPer; ++j) {
        cc += c[j];
        ww += w[j];
        if (mine == kCoarse && cc >= want_c && ww >= want_w) mine = lane * kPer + j;
        if (cc <= most_c) last = lane * kPer + j;
      }
      for (int o = 16; o; o >>= 1) {
        mine = min(mine, __shfl_xor_sync(0xffffffffu, mine, o));
        last = max(last, __shfl_xor_sync(0xffffffffu, last, o));
      }
      int range = min(mine, max(last, 0));
      if (r.m > 0.0f) {
        // nothing is kept below min-p of the sample's maximum, nor of the row's
        const int floor_range = max(0, (int)fminf(-logf(r.m) * kPerNat + 1.0f, (float)kCoarse));
        if (r.k <= 0 && !(r.p < 1.0f)) range = floor_range;
        else if (r.k <= 0 || !(r.p < 1.0f)) range = min(range, floor_range);  // p needs all of k
      }
      if (lane == 0)
        s.tau = range >= kCoarse - 1 && mine < kCoarse ? -INFINITY
                                                       : m0 - (range + 1) / kPerNat * r.T;
    }
  }
  __syncthreads();
  const float tau = seen ? s.tau : 0.0f;

  // Stream: this CTA's part of the row.
  if (seen) {
    const int per = (r.V + kCl - 1) / kCl, lo = min(r.V, rank * per), hi = min(r.V, lo + per);
    const float c2 = per_t * 1.4426950408889634f;
    float tail[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    float best_key = -INFINITY;
    int best_i = -1;  // of an unlimited draw
    // places in the list for the warp's `mine` tokens a lane
    const auto reserve = [&](int mine) {
      int sum = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += y;
      }
      int at = 0;
      if (lane == 31 && sum) at = atomicAdd(&s.n, sum);
      return __shfl_sync(0xffffffffu, at, 31) + sum - mine;
    };
    const auto wanted = [&](float z) { return z >= tau && z > -INFINITY; };
    const auto one = [&](float z, int i, float& sum) {
      float e;
      asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"((z - m0) * c2));
      sum += z < tau ? e : 0.0f;
      if (all && z > -INFINITY) {
        const float key = __fdiv_rn(z - m0, r.T) - logf(-logf(r.u[i]));
        if (best_i < 0 || key > best_key || (key == best_key && i < best_i))
          best_key = key, best_i = i;
      }
    };
    // up to three logits before the first 16-byte boundary, then four at a time
    const int head = min(hi - lo, (int)((4 - ((reinterpret_cast<uintptr_t>(r.z + lo) >> 2) & 3)) & 3));
    const int quads = (hi - lo - head) / 4, body = lo + head, end = body + 4 * quads;
    const float4* z4 = reinterpret_cast<const float4*>(r.z + body);
    constexpr int kUnroll = 4;
#pragma unroll 1
    for (int q0 = 0; q0 < quads; q0 += kUnroll * kThreads) {
      float4 v[kUnroll];
      int mine = 0;
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) {
        const int q = q0 + k * kThreads + tid;
        v[k] = q < quads ? __ldg(z4 + q)
                         : make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
      }
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) {
        const int i = body + 4 * (q0 + k * kThreads + tid);
        const float y[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          one(y[c], i + c, tail[c]);
          mine += wanted(y[c]);
        }
      }
      if (__any_sync(0xffffffffu, mine)) {
        int at = reserve(mine);
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) {
          const int i = body + 4 * (q0 + k * kThreads + tid);
          const float y[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
#pragma unroll
          for (int c = 0; c < 4; ++c)
            if (wanted(y[c])) {
              if (at < kCap) s.list[at] = Entry{y[c], i + c};
              ++at;
            }
        }
      }
    }
    if (tid < 32) {  // the ragged ends
      const int i = lane < head ? lo + lane : end + lane - head;
      const float z = i < hi && (lane < head || i >= end) ? r.z[i] : -INFINITY;
      one(z, i, tail[0]);
      const int at = reserve(wanted(z));
      if (wanted(z) && at < kCap) s.list[at] = Entry{z, i};
    }
    float t = (tail[0] + tail[1]) + (tail[2] + tail[3]);
#pragma unroll
    for (int o = 16; o; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
    if (lane == 0) s.fpart[tid >> 5] = t;
    const u64 best = all ? reduce(s, best_i < 0 ? 0ull : rank_key(best_key, best_i), most) : 0ull;
    __syncthreads();
    if (tid == 0) {
      float sum = 0.0f;
      for (int w = 0; w < kWarps; ++w) sum += s.fpart[w];
      s.tail = sum;
      s.best = best;
    }
  }
  __syncthreads();

  // The first CTA joins the lists.
  bool fits = seen && s.n <= kCap;
  u64 given = 0;
  float tail = 0.0f;
  int n = 0;
  if (kCl > 1) {
    cluster_sync();
    if (rank == 0 && seen) {
      if (tid < kCl) {  // all peers at once: a remote read takes about a microsecond
        s.peer_n[tid] = (int)peer_u32(peer(&s.n, tid));
        s.fpart[tid] = __uint_as_float(peer_u32(peer(&s.tail, tid)));
        s.part[tid] = peer_u64(peer(&s.best, tid));
      }
      __syncthreads();
      int first[kCl];
#pragma unroll
      for (int c = 0; c < kCl; ++c) {
        first[c] = n;
        n += min(s.peer_n[c], kCap);
        fits = fits && s.peer_n[c] <= kCap;
        tail += s.fpart[c];
        given = most(given, s.part[c]);
      }
      fits = fits && n <= kCap;
      if (fits) {
#pragma unroll
        for (int c = 1; c < kCl; ++c) {
          const uint32_t src = peer(s.list, c);
          const int m = s.peer_n[c];
          for (int j = tid; j < m; j += kThreads) {
            const u64 v = peer_u64(src + 8 * j);
            s.list[first[c] + j] = Entry{__uint_as_float((uint32_t)v), (int)(v >> 32)};
          }
        }
      }
    }
    cluster_sync();
    if (rank) return;
  } else if (seen) {
    n = s.n;
    tail = s.tail;
    given = s.best;
  }
  __syncthreads();

  int token = -1;
  u64 weight = 0;
  bool done = false;
  if (fits) {
    done = choose(s, r, ListSource{s.list, n}, tau, m0, tail, given, &token, &weight);
    __syncthreads();
  }
  if (!done) choose(s, r, RowSource{r.z, r.V}, -INFINITY, 0.0f, 0.0f, 0ull, &token, &weight);
  if (tid == 0) {
    p.token[b] = token;
    if (p.logprob)
      p.logprob[b] =
          token < 0 ? -INFINITY : __fdiv_rn(r.z[token] - s.best_z, r.T) -
                                          logf(__ull2float_rn(weight) * 0x1p-40f);
  }
}

template <int kCl>
cudaError_t launch_cluster(const SampleCall& call, cudaStream_t stream) {
  static std::atomic<unsigned long long> done{0};
  cudaError_t e = once_per_device(done, [] {
    return cudaFuncSetAttribute(sample_kernel<kCl>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                (int)sizeof(Sm));
  });
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(call.batch * kCl);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = sizeof(Sm);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = kCl;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = kCl > 1 ? 1 : 0;
  e = cudaLaunchKernelEx(&cfg, sample_kernel<kCl>, call);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

int sample_max_vocab() { return kMaxVocab; }

// CTAs per row: as many as run in one wave.  The CTAs of a cluster share a
// neighbourhood of the GPU, so larger ones do not fill it, and those left over wait for
// a second wave.  Rows of 152064 by top-p 0.9, one, two, four and eight CTAs a row:
// 12 rows 63, 51, 46 and 43 us; 16 rows 63, 51, 47 and 57; 32 rows 64, 52, 47 and 73;
// 64 rows 64, 52, 87 and 113; 80 rows 64, 98, 97 and 138.  (From 31 rows on four CTAs
// would need more clusters than 152 SMs are sure to hold, so two are taken there.)
cudaError_t launch_sample(const SampleCall& call, int sm_count, cudaStream_t stream) {
  if (call.batch * 12 <= sm_count) return launch_cluster<8>(call, stream);
  if (call.batch * 5 <= sm_count) return launch_cluster<4>(call, stream);
  if (call.batch * 2 <= sm_count) return launch_cluster<2>(call, stream);
  return launch_cluster<1>(call, stream);
}

}  // namespace kvq
