// Log probabilities of given tokens from stored logits, with the entropy of their
// distribution, its log-sum-exp and the best alternatives, and the gradient of the
// logits.  With l = logit_scale * z over a row's vocabulary:
//   lse = log sum exp l,  logprob = l_y - lse,  q = exp(l - lse)
//   H   = lse - sum q l = log S - E / S,  S = sum exp(l - m),  E = sum (l - m) exp(l - m)
//   dz  = logit_scale ( r (1[j = y] - q_j) - h q_j (log q_j + H) )
// for upstream gradients r of logprob and h of H.
//
// Forward: one pass over the logits.  A block takes a row, or, where there are few rows,
// the blocks of a cluster take a run of its columns each and join over distributed shared
// memory.  A thread keeps the maximum, S and E of its elements in registers and rescales
// once a tile.  The alternatives come out of the same pass: the numbers of 16-byte vectors
// whose largest element reaches a threshold go into a list of the warp's, and when the row
// has ended those vectors, a few times `top`, are read again (out of L2) and the best of
// their elements kept.  (Elements or vectors put aside as they come cost as much as the
// sums.)  The threshold comes from the threads' running maxima: of a warp's 32 the want-th
// largest, and of those values the m-th largest over the warps, want * m >= top, is reached by
// at least `top` different elements.  It is formed again with each of the first tiles and then
// with every fourth (64 and 128 alternatives of 4096 x 163840, us: 307 and 367; with tiles 1, 2,
// 4, 8, ... 325 and 517, with every tile 350 and 406).  After
// the first tile the warps run without a barrier until the row ends; nothing is called within
// the loop, because what lives across a call is stored with every tile.  A warp whose list
// does not hold all (a row that ascends) reads its part again.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstddef>
#include <cstdio>
#include <type_traits>

#include "../../include/muon.h"
#include "ptx.cuh"

namespace muon {
void set_last_error(const char* msg);
}

namespace {

namespace ptx = muon::ptx;

constexpr int kThreads = 256;  // forward: or kShortThreads
constexpr int kVectors = 4;    // gradient: 16-byte loads a thread
constexpr int kTileVectors = kThreads * kVectors;
// Blocks on an SM: five leave a thread 48 registers, four 64, three 80.  (us, with 64
// alternatives: 4096 x 163840 bf16 380 with 3, 337 with 4, 325 with 5, 2048 x 163840 fp32 263,
// 279 and 329, whose registers spill; without: bf16 220 with 4, 213 with 5, 229 with 6, fp32
// 211 with 4, 214 with 5.)
constexpr int blocks_per_sm(bool fp32, bool top, int threads) { return (top ? (fp32 ? 3 : 5) : fp32 ? 4 : 5) * kThreads / threads; }
// Short rows that a block takes alone: blocks of half the threads, twice as many, whose starts
// and ends overlap.  (us, 4000 tokens, bf16, blocks of 256 and of 128 threads: 2000 columns 22.1
// and 15.7, 16384 34.0 and 31.1, 50021 73.0 and 72.1; with 20 alternatives 2000 92.7 and 39.1,
// 16384 75.3 and 62.4; with 64 50021 176 and 160, 100000 229 and 235; fp32 8192 32.0 and 25.9,
// 32000 79.3 and 80.3, with 64 155 and 135.)  Twice the vectors where there are alternatives.
constexpr int kShortThreads = 128;
constexpr int kShortVectors = 4096;
// Candidates up to which a thread each finds its place; of more, the best are found first.
// (4096 x 163840 bf16 with 64: 357 us, with 256 in its place 363.)
constexpr int kOrdered = 128;
constexpr int kVectorList = 256;  // of a warp
constexpr int kMaxTop = 128;
static_assert(kMaxTop <= kOrdered && kOrdered <= kShortThreads, "what is left is put in order");
constexpr int kKeys = kMaxTop + 32 * 8;  // candidates of a warp: the best, and a vector a lane
constexpr int kMaxCluster = 8;
constexpr int kSorted = 2048;  // where a block of a cluster leaves its best in the list of candidates
static_assert(kMaxCluster == kThreads / 32, "a warp reads a block's list");
static_assert(kMaxCluster * kMaxTop <= kSorted && kSorted + kMaxTop <= kThreads / 32 * kKeys, "a cluster's best fit before a block's");
constexpr float kLn2 = 0.693147180559945309f;
constexpr float kLog2e = 1.44269504088896341f;
constexpr float kFloor = -200.0f;  // exponents of 2 from here down give 0, and stay finite in products
// A logit whose exponent of 2 is this far from 0 is a mask, or no logit at all, and counts as the
// infinity of its sign: the differences below are exact but for the rounding of the reference, at
// most 64 up to here, of which 2^64 times 2^24 columns is a number.
constexpr float kFar = 2147483648.0f;
// The gradient's q = exp(l - lse) needs an lse whose last place is below 1.
constexpr float kFarLse = 16777216.0f;

struct LogitsParams {
  const void* z;
  long long ld;
  int tokens, vocab, top;
  float scale2;  // logit_scale * log2(e)
  const int64_t* targets;
  float* logprob;
  float* entropy;
  float* lse;
  int64_t* top_ids;
  float* top_logits;
  float* top_logprob;
  int index_bits;  // of a column number
};

struct GradParams {
  const void* z;
  void* dz;
  long long ld, ld_dz;
  int tokens, vocab;
  float scale;
  const int64_t* targets;
  const float* entropy;
  const float* lse;
  const float* r;
  const float* h;
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Larger of two; a NaN shows.
__device__ __forceinline__ float max_nan(float a, float b) {
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}

// Larger of three; a NaN does not show.
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// Pairs of floats in one instruction each.
__device__ __forceinline__ uint64_t pair(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}

__device__ __forceinline__ void unpair(uint64_t v, float& lo, float& hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}

__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}

__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

// Elements of a 16-byte vector.
template <bool kFp32>
struct Cells {
  using T = std::conditional_t<kFp32, float, __nv_bfloat16>;
  static constexpr int kEach = kFp32 ? 4 : 8;
  // Of one tile a thread: 32 elements, whose arithmetic covers the next tile's loads.  (2048 x
  // 163840 fp32 without and with 64 alternatives, us: 223 and 391 with 4, 212 and 282 with 8.)
  static constexpr int kVectors = kFp32 ? 8 : 4;
  static constexpr uint32_t kLowest = kFp32 ? 0xFF800000u : 0xFF80FF80u;  // -inf throughout
  static __device__ __forceinline__ float value(const uint4& v, int e) {
    if constexpr (kFp32) {
      return __uint_as_float(e == 0 ? v.x : e == 1 ? v.y : e == 2 ? v.z : v.w);
    } else {
      const uint32_t w = e < 2 ? v.x : e < 4 ? v.y : e < 6 ? v.z : v.w;
      return __uint_as_float(e & 1 ? w & 0xFFFF0000u : w << 16);
    }
  }
};

// A vector's largest element (a NaN does not show): of bf16 as the larger of its even and of
// its odd elements, without taking them apart.
template <bool kFp32>
struct Largest {
  std::conditional_t<kFp32, float, __nv_bfloat162> x;
  static __device__ __forceinline__ __nv_bfloat162 two(uint32_t w) { return *reinterpret_cast<const __nv_bfloat162*>(&w); }
  static __device__ __forceinline__ Largest of(const uint4& v) {
    Largest l;
    if constexpr (kFp32) l.x = fmaxf(max3(__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z)), __uint_as_float(v.w));
    else l.x = __hmax2(__hmax2(two(v.x), two(v.y)), __hmax2(two(v.z), two(v.w)));
    return l;
  }
  __device__ __forceinline__ void join(const Largest& o) {
    if constexpr (kFp32) x = fmaxf(x, o.x);
    else x = __hmax2(x, o.x);
  }
  __device__ __forceinline__ float value() const {
    if constexpr (kFp32) return x;
    else return fmaxf(__low2float(x), __high2float(x));
  }
};

// Vector `index` of a row from the 16-byte boundary at or below its start, `shift`
// elements before it; -inf outside the row.
template <bool kFp32>
__device__ __forceinline__ uint4 load_vector(const typename Cells<kFp32>::T* row, int vocab, int shift, int index, int end) {
  constexpr int kEach = Cells<kFp32>::kEach;
  constexpr uint32_t kLow = Cells<kFp32>::kLowest;
  uint4 v = make_uint4(kLow, kLow, kLow, kLow);
  if (index < end) {
    const int at = index * kEach - shift;
    if (at >= 0 && at + kEach <= vocab) {
      v = __ldcs(reinterpret_cast<const uint4*>(row + at));
    } else {
      uint32_t w[4] = {kLow, kLow, kLow, kLow};
#pragma unroll
      for (int e = 0; e < kEach; ++e)
        if (at + e >= 0 && at + e < vocab) {
          if constexpr (kFp32) {
            w[e] = __float_as_uint(row[at + e]);
          } else {
            const uint32_t b = __bfloat16_as_ushort(row[at + e]);
            w[e >> 1] = e & 1 ? (w[e >> 1] & 0xFFFFu) | (b << 16) : (w[e >> 1] & 0xFFFF0000u) | b;
          }
        }
      v = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
  return v;
}

// Ascending whole numbers for ascending floats; both zeros are one value and a NaN is -inf.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t b = __float_as_uint(x != x ? -INFINITY : x + 0.0f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o); }

constexpr uint32_t kLowestOrdered = 0x007FFFFFu;  // of minus infinity

// Value above, column counted down below: larger keys come first, equal logits by column.
// The lower half of a bf16 logit's 32 bits says nothing and is left out.
typedef unsigned long long Key;
template <bool kFp32>
__device__ __forceinline__ Key make_key(const LogitsParams& P, float x, int column) {
  return (static_cast<Key>(ordered(x) >> (kFp32 ? 0 : 16)) << P.index_bits) | static_cast<unsigned>(P.vocab - 1 - column);
}
template <bool kFp32>
__device__ __forceinline__ float value_of(const LogitsParams& P, Key k) {
  const uint32_t o = static_cast<uint32_t>(k >> P.index_bits);
  return unordered(kFp32 ? o : (o << 16) | (o & 0x8000u ? 0u : 0xFFFFu));
}

// Running statistics in powers of 2: y = z scale2, reference m = the largest y, rounded,
// S and E against it, E in units of log2.  All of a row's differences are formed as one
// fused z scale2 - m, so that the rounding of m cancels.
struct Sums {
  float m, s, e;
};

// The reference that a largest logit of exponent y asks for.
__device__ __forceinline__ float reference_of(float y) { return y >= kFar ? INFINITY : y > -kFar ? y : -INFINITY; }

// (s, e) against a larger reference.
__device__ __forceinline__ void rescale(Sums& a, float m) {
  const float d = a.m == m ? 0.f : max_nan(a.m - m, kFloor);
  const float f = ex2(d);
  a.e = f * fmaf(d, a.s, a.e);
  a.s *= f;
  a.m = m;
}

__device__ __forceinline__ Sums join(Sums a, Sums b) {
  const float m = fmaxf(a.m, b.m);
  rescale(a, m);
  rescale(b, m);
  return Sums{m, a.s + b.s, a.e + b.e};
}

// The sum of d 2^d over a thread's elements, read again, with exponents from kFloor on: where a
// thread has met minus infinity.  (us, 4096 x 163840 bf16, 64 alternatives: 219 and 317 without,
// 432 and 512 with one such column at the row's end, 490 and 844 with nine of ten so.)
template <bool kFp32, int kThreads>
__device__ __noinline__ float weighted_again(const uint4* cells, int begin, int end, float scale2, float base) {
  float sum = 0.f;
#pragma unroll 1
  for (int i = begin + static_cast<int>(threadIdx.x); i < end; i += kThreads) {
    const uint4 v = cells[i];
    float part = 0.f;
#pragma unroll
    for (int e = 0; e < Cells<kFp32>::kEach; ++e) {
      const float d = max_nan(fmaf(Cells<kFp32>::value(v, e), scale2, base), kFloor);
      part = fmaf(ex2(d), d, part);
    }
    sum += part;
  }
  return sum;
}

__device__ __forceinline__ Sums from_lane(const Sums& a, int lane) {
  return Sums{__shfl_sync(0xFFFFFFFFu, a.m, lane), __shfl_sync(0xFFFFFFFFu, a.s, lane), __shfl_sync(0xFFFFFFFFu, a.e, lane)};
}

template <int kThreads>
struct Shared {
  static constexpr int kWarps = kThreads / 32;
  Key list[kWarps * kKeys];  // candidates: kKeys a warp, at the end the block's first `count`
  int vectors[kWarps][kVectorList];
  int listed[kWarps];  // more than kVectorList where some found no room
  int count, counts[kWarps];
  uint32_t reached[2][kWarps];  // ordered; of the first tile, and of all so far
  Sums sums[kWarps];
  Sums all;
};

// How many of the first n keys are larger.
__device__ __forceinline__ int place_of(const Key* list, int n, Key mine) {
  int place = 0;
#pragma unroll 8
  for (int i = 0; i < n; ++i) place += list[i] > mine;
  return place;
}

// The `top` largest of the n > top candidates, to the front in their order, by one warp.
// Two bisections, of 32-bit numbers: for the top-th largest logit, and, where others equal
// it, for the column up to which they stay.
struct Cut {
  uint32_t value;   // candidates above it stay,
  uint32_t behind;  // and those of this value from here on (columns are counted down)
};

// The largest x that at least `top` of the lanes' numbers reach; fewer reach hi.
template <typename Count>
__device__ __forceinline__ uint32_t bisect(int top, uint32_t lo, uint32_t hi, int* reach, Count count_from) {
  while (hi - lo > 1) {
    const uint32_t mid = lo + (hi - lo) / 2;
    const int c = __reduce_add_sync(0xFFFFFFFFu, count_from(mid));
    if (c >= top) {
      lo = mid;
      *reach = c;
      if (c == top) break;
    } else {
      hi = mid;
    }
  }
  return lo;
}

template <int kEach>  // candidates a lane
__device__ __forceinline__ Cut find_cut(const Key* list, int n, int top, int bits, int lane) {
  uint32_t value[kEach], column[kEach], low = 0xFFFFFFFFu, high = 0u;
  const uint32_t columns = (1u << bits) - 1u;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const bool there = i * 32 + lane < n;
    const Key k = there ? list[i * 32 + lane] : 0;
    value[i] = static_cast<uint32_t>(k >> bits);
    column[i] = static_cast<uint32_t>(k) & columns;
    low = min(low, there ? value[i] : 0xFFFFFFFFu);
    high = max(high, value[i]);
  }
  low = __reduce_min_sync(0xFFFFFFFFu, low);
  high = __reduce_max_sync(0xFFFFFFFFu, high);
  Cut cut = {low, 0u};
  int reach = n;
  cut.value = bisect(top, low, high + 1u, &reach, [&](uint32_t x) {
    int c = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) c += value[i] >= x;
    return c;
  });
  if (reach > top) {
    int above = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) above += value[i] > cut.value;
    above = __reduce_add_sync(0xFFFFFFFFu, above);
    cut.behind = bisect(top - above, 0u, columns + 1u, &reach, [&](uint32_t x) {
      int c = 0;
#pragma unroll
      for (int i = 0; i < kEach; ++i) c += value[i] == cut.value && column[i] >= x;
      return c;
    });
  }
  return cut;
}

__device__ __noinline__ void keep_best(Key* list, int n, int top, int bits, int lane) {
  static_assert(kThreads / 32 * kMaxTop <= 32 * 32 && kKeys <= 32 * 32, "all candidates in registers");
  __syncwarp();
  const Cut cut = n <= 64 ? find_cut<2>(list, n, top, bits, lane)
                  : n <= 192 ? find_cut<6>(list, n, top, bits, lane)
                  : n <= 384 ? find_cut<12>(list, n, top, bits, lane) : find_cut<32>(list, n, top, bits, lane);
  int kept = 0;
  for (int i = 0; i < n; i += 32) {
    const Key k = i + lane < n ? list[i + lane] : 0;
    const uint32_t value = static_cast<uint32_t>(k >> bits), column = static_cast<uint32_t>(k) & ((1u << bits) - 1u);
    const bool keep = i + lane < n && (value > cut.value || (value == cut.value && column >= cut.behind));
    const unsigned who = __ballot_sync(0xFFFFFFFFu, keep);
    if (keep) list[kept + __popc(who & ((1u << lane) - 1u))] = k;  // at or before its place: read already
    kept += __popc(who);
    __syncwarp();
  }
}

// A value that at least `want` of the warp's 32 maxima reach: the largest such, but for a
// 64th of their range.
__device__ __forceinline__ uint32_t reached_by(uint32_t mine, int want) {
  const uint32_t high = __reduce_max_sync(0xFFFFFFFFu, mine);
  if (want == 1) return high;
  uint32_t lo = __reduce_min_sync(0xFFFFFFFFu, mine), step = high - lo;
#pragma unroll
  for (int i = 0; i < 6; ++i) {
    step = (step + 1) >> 1;
    if (__popc(__ballot_sync(0xFFFFFFFFu, mine >= lo + step)) >= want) lo += step;
  }
  return lo;
}

// The m-th largest of the warps' values.
template <int kWarps>
__device__ __forceinline__ uint32_t mth_of(const volatile uint32_t* v, int m, int lane) {
  const uint32_t mine = v[lane & (kWarps - 1)];
  int not_less = 0;
#pragma unroll
  for (int i = 0; i < kWarps; ++i) not_less += v[i] >= mine;
  // of the values that at least m reach the largest
  return __reduce_max_sync(0xFFFFFFFFu, not_less >= m ? mine : 0u);
}

// The elements from `threshold` on of a warp's vectors as candidates; at most kMaxTop stay,
// the `top` largest where they are cut.
template <bool kFp32>
struct Collector {
  const LogitsParams& P;
  Key* keys;
  const uint4* cells;
  int shift, lane, count;
  float threshold;

  __device__ __forceinline__ uint4 read(int index) { return index >= 0 ? cells[index] : make_uint4(0u, 0u, 0u, 0u); }

  // a vector a lane, or none (negative)
  __device__ __forceinline__ void take(int index, const uint4& v) {
    using C = Cells<kFp32>;
    const bool all = !(threshold > -INFINITY);
    unsigned keep = 0;
    if (index >= 0) {
#pragma unroll
      for (int e = 0; e < C::kEach; ++e) keep |= static_cast<unsigned>(C::value(v, e) >= threshold || all) << e;
    }
    // places in the order of the lanes
    int at = __popc(keep);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int below = __shfl_up_sync(0xFFFFFFFFu, at, o);
      if (lane >= o) at += below;
    }
    const int added = __shfl_sync(0xFFFFFFFFu, at, 31);
    at += count - __popc(keep);
    for (; keep != 0; keep &= keep - 1) {
      const int e = __ffs(keep) - 1, word = kFp32 ? e : e >> 1;
      const uint32_t bits = word == 0 ? v.x : word == 1 ? v.y : word == 2 ? v.z : v.w;
      const float x = __uint_as_float(kFp32 ? bits : e & 1 ? bits & 0xFFFF0000u : bits << 16);
      keys[at++] = make_key<kFp32>(P, x, index * C::kEach - shift + e);
    }
    __syncwarp();
    count += added;
    if (count > kMaxTop) {
      keep_best(keys, count, P.top, P.index_bits, lane);
      count = P.top;
    }
  }
};

// Of the vectors that the warp put in its list, or, where it did not hold all, of every one of
// its part that qualifies.  `first_tile`: threshold of the first tile, later elements equal to
// which come after the top that there are.
template <bool kFp32, int kThreads>
__device__ __noinline__ int collect(const LogitsParams& P, Shared<kThreads>& sh, const uint4* cells, int shift, int begin, int end,
                                    float first_tile, float threshold) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  Collector<kFp32> c = {P, sh.list + warp * kKeys, cells, shift, lane, 0, threshold};
  __syncwarp();
  const int listed = sh.listed[warp];
  if (listed <= kVectorList) {
    constexpr int kAtOnce = 4;  // loads in flight
    for (int first = 0; first < listed; first += 32 * kAtOnce) {
      int index[kAtOnce];
      uint4 v[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const int at = first + i * 32 + lane;
        index[i] = at < listed ? sh.vectors[warp][at] : -1;
        v[i] = c.read(index[i]);
      }
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i)
        if (first + i * 32 < listed) c.take(index[i], v[i]);
    }
  } else {
    for (int v0 = begin + static_cast<int>(threadIdx.x) - lane; v0 < end; v0 += kThreads) {
      const int index = v0 + lane;
      const bool early = v0 < begin + kThreads * Cells<kFp32>::kVectors;
      bool mark = false;
      if (index < end) {
        const float x = Largest<kFp32>::of(cells[index]).value();
        mark = early ? x >= threshold || !(threshold > -INFINITY) : x >= threshold && x > first_tile;
      }
      if (__any_sync(0xFFFFFFFFu, mark)) c.take(mark ? index : -1, c.read(mark ? index : -1));
    }
  }
  return c.count;
}

template <bool kFp32, bool kTop, int kThreads>
__global__ void __launch_bounds__(kThreads, blocks_per_sm(kFp32, kTop, kThreads)) logprob_kernel(const __grid_constant__ LogitsParams P) {
  using C = Cells<kFp32>;
  constexpr int kEach = C::kEach, kVectors = C::kVectors, kTileVectors = kThreads * kVectors, kWarps = kThreads / 32;
  using Shared = Shared<kThreads>;
  extern __shared__ __align__(16) unsigned char raw[];
  Shared& sh = *reinterpret_cast<Shared*>(raw);
  __shared__ float s_target;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int parts = static_cast<int>(gridDim.x), part = static_cast<int>(blockIdx.x);
  const long long token = blockIdx.y;
  const typename C::T* row = static_cast<const typename C::T*>(P.z) + token * P.ld;
  if (P.targets != nullptr) {
    const int64_t y = P.targets[token];
    if (y < 0 || y >= P.vocab) {  // masked: nothing of it is read
      if (part == 0) {
        if (tid == 0) {
          if (P.logprob != nullptr) P.logprob[token] = 0.f;
          if (P.entropy != nullptr) P.entropy[token] = 0.f;
          if (P.lse != nullptr) P.lse[token] = 0.f;
        }
        if (kTop)
          for (int k = tid; k < P.top; k += kThreads) {
            const long long at = token * P.top + k;
            if (P.top_ids != nullptr) P.top_ids[at] = -1;
            if (P.top_logits != nullptr) P.top_logits[at] = 0.f;
            if (P.top_logprob != nullptr) P.top_logprob[at] = 0.f;
          }
      }
      return;  // every block of the cluster alike
    }
    if (part == 0 && tid == 0) {
      if constexpr (kFp32) s_target = row[y];
      else s_target = __bfloat162float(row[y]);
    }
  }
  // vectors from the 16-byte boundary at or below the row's start; the ones that lie in the row
  // as a whole are dealt out to the blocks, the elements before and behind them (at most two
  // vectors less two elements) go to one lane each at the end
  const int shift = static_cast<int>((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(typename C::T));
  const uint4* const cells = reinterpret_cast<const uint4*>(row - shift);
  const int whole0 = shift > 0 ? 1 : 0, whole1 = max(whole0, static_cast<int>((static_cast<long long>(shift) + P.vocab) / kEach));
  const int begin = whole0 + static_cast<int>(static_cast<long long>(whole1 - whole0) * part / parts);
  const int end = whole0 + static_cast<int>(static_cast<long long>(whole1 - whole0) * (part + 1) / parts);

  Sums a = {-INFINITY, 0.f, 0.f};
  float threshold = -INFINITY, most = -INFINITY;  // `most`: of the thread's elements so far
  // `active` warps whose threads all have elements: m of them, and want maxima of each, make
  // top; want > 32: everything is a candidate
  const int active = min(kWarps, (end - begin) / 32), want = active > 0 ? (P.top + active - 1) / active : 33;
  const int m = (P.top + want - 1) / want;
  auto note_reached = [&](int tile) {
    const uint32_t t = want <= 32 && warp < active ? reached_by(ordered(most), want) : kLowestOrdered;
    if (lane == 0) {
      volatile uint32_t* mine = &sh.reached[0][warp];
      if (tile == 0) mine[0] = t;
      mine[kWarps] = t;
    }
  };
  float bound = -INFINITY, first = -INFINITY;  // a vector is listed from `bound` on
  if (kTop && lane == 0) sh.listed[warp] = 0;
  __syncwarp();
  const uint64_t scale = pair(P.scale2, P.scale2);
  uint4 v[kVectors];
  auto load = [&](int v0, int i, bool whole) {
    const uint4* src = cells + v0 + i * kThreads + tid;
    if (whole) return __ldcs(src);
    return v0 + i * kThreads + tid < end ? __ldcs(src) : make_uint4(C::kLowest, C::kLowest, C::kLowest, C::kLowest);
  };
#pragma unroll
  for (int i = 0; i < kVectors; ++i) v[i] = load(begin, i, begin + kTileVectors <= end);
  int tile = 0, v0 = begin;
  // full: this tile and the next one lie in the part as a whole
  auto take_tile = [&](auto full) {
    constexpr bool kFull = decltype(full)::value;
    Largest<kFp32> largest[kVectors];
#pragma unroll
    for (int i = 0; i < kVectors; ++i) largest[i] = Largest<kFp32>::of(v[i]);
    Largest<kFp32> all_of = largest[0];
#pragma unroll
    for (int i = 1; i < kVectors; ++i) all_of.join(largest[i]);
    const float here = all_of.value();
    most = fmaxf(most, here);
    if (kTop && (tile < 4 || (tile & 3) == 3)) {
      note_reached(tile);
      if (tile == 0) __syncthreads();
      // Of the first tile only its own: `first` has to be reached by elements that come before
      // all later tiles'.  Afterwards others' may be of earlier tiles, and lower, or of later ones.
      threshold = fmaxf(threshold, unordered(mth_of<kWarps>(sh.reached[tile > 0], m, lane)));
      bound = fmaxf(bound, threshold);
    }
    const float reference = most * P.scale2;
    if (reference > fmaxf(a.m, -kFar)) rescale(a, reference_of(reference));
    const float base = a.m == -INFINITY ? 0.f : -a.m;
    const uint64_t from = pair(base, base);
    uint64_t s = 0, w = 0;  // pairs of zeros
    const int left = end - v0 - tid;
    const bool more = kFull || v0 + kTileVectors < end, whole = kFull || v0 + 2 * kTileVectors <= end;
#pragma unroll
    for (int i = 0; i < kVectors; ++i) {
      if (kFull || i * kThreads < left) {
#pragma unroll
        for (int e = 0; e < kEach; e += 2) {
          const uint64_t d = fma2(pair(C::value(v[i], e), C::value(v[i], e + 1)), scale, from);
          float d0, d1;
          unpair(d, d0, d1);
          const uint64_t p = pair(ex2(d0), ex2(d1));
          s = add2(s, p);
          w = fma2(p, d, w);
        }
      }
      // the next tile's vector takes the place
      if (more) v[i] = load(v0 + kTileVectors, i, whole);
    }
    float lo, hi;
    unpair(w, lo, hi);
    a.e += lo + hi;
    unpair(s, lo, hi);
    a.s += lo + hi;

    if constexpr (kTop) {
      const bool every = tile == 0 && !(bound > -INFINITY);  // NaNs, too
      if (here >= bound || every) {
#pragma unroll
        for (int i = 0; i < kVectors; ++i)
          if ((largest[i].value() >= bound || every) && (kFull || i * kThreads < left)) {
            const int at = atomicAdd(&sh.listed[warp], 1);
            if (at < kVectorList) sh.vectors[warp][at] = v0 + i * kThreads + tid;
          }
      }
      // later elements have larger columns: one that equals the first tile's threshold comes
      // after the top that there are
      if (tile == 0) {
        first = bound;
        bound = unordered(ordered(bound) + 1u);
      }
    }
    ++tile;
    v0 += kTileVectors;
  };
  while (v0 + 2 * kTileVectors <= end) take_tile(std::true_type{});
  while (v0 < end) take_tile(std::false_type{});
  // 0 times an exponent of minus infinity, or a NaN
  if (!(a.e == a.e)) a.e = weighted_again<kFp32, kThreads>(cells, begin, end, P.scale2, a.m == -INFINITY ? 0.f : -a.m);

  // elements outside whole vectors
  float extra = 0.f;
  int extra_at = -1;
  if (part == 0 && warp == 0) {
    const int head = whole0 * kEach - shift, behind = min(P.vocab, whole1 * kEach - shift);
    const int column = lane < min(head, P.vocab) ? lane : behind + lane - min(head, P.vocab);
    const bool mine = column < P.vocab;
    const float x = mine ? static_cast<float>(row[column]) : -INFINITY;
    const float m = fmaxf(a.m, reference_of(x * P.scale2));
    if (mine) {
      rescale(a, m);
      // as in the loop; a NaN, which m does not show, shows here
      const float d = max_nan(fmaf(x, P.scale2, m == -INFINITY ? 0.f : -m), kFloor), p = ex2(d);
      a.s += p;
      a.e = fmaf(p, d, a.e);
    }
    extra = x;
    extra_at = mine ? column : -1;
  }

  // statistics: warp, block, cluster
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    a = join(a, from_lane(a, lane ^ o));
  }
  if (lane == 0) sh.sums[warp] = a;
  if (kTop) {
    int count = collect<kFp32, kThreads>(P, sh, cells, shift, begin, end, first, threshold);
    if (warp == 0) {
      const unsigned who = __ballot_sync(0xFFFFFFFFu, extra_at >= 0);
      if (extra_at >= 0) sh.list[count + __popc(who & ((1u << lane) - 1u))] = make_key<kFp32>(P, extra, extra_at);
      count += __popc(who);
      __syncwarp();
      if (count > kMaxTop) {
        keep_best(sh.list, count, P.top, P.index_bits, lane);
        count = P.top;
      }
    }
    if (lane == 0) sh.counts[warp] = count;
    // all warps' candidates one behind the other; what goes down is read first
    __syncthreads();
    int before = 0, n = 0;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) {
      const int c = sh.counts[i];
      before += i < warp ? c : 0;
      n += c;
    }
    Key mine[kMaxTop / 32];
#pragma unroll
    for (int i = 0; i < kMaxTop / 32; ++i)
      if (i * 32 + lane < count) mine[i] = sh.list[warp * kKeys + i * 32 + lane];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kMaxTop / 32; ++i)
      if (i * 32 + lane < count) sh.list[before + i * 32 + lane] = mine[i];
    __syncthreads();
    const bool cut = n > kOrdered;
    if (cut) {
      if (warp == 0) keep_best(sh.list, n, P.top, P.index_bits, lane);
      n = P.top;
      if (parts > 1) __syncthreads();
    }
    // a block of a cluster leaves its best in order
    if (parts > 1 && tid < n) {
      const int place = place_of(sh.list, n, sh.list[tid]);
      if (place < P.top) sh.list[kSorted + place] = sh.list[tid];
    }
    if (tid == 0) sh.count = parts > 1 ? min(n, P.top) : n;
  }
  __syncthreads();
  if (warp == 0) {
    a = sh.sums[lane & (kWarps - 1)];
#pragma unroll
    for (int o = kWarps / 2; o > 0; o >>= 1) a = join(a, from_lane(a, lane ^ o));
    if (lane == 0) sh.all = a;
  }
  __syncthreads();
  int candidates = kTop ? sh.count : 0;
  if (parts > 1) {
    ptx::cluster_sync_all();
    if (part == 0) {
      // the other blocks' lists behind this one's, a warp for each block, and their sums into this one's
      auto word = [&](int block, size_t at) {
        uint32_t x;
        const uint32_t theirs = ptx::map_to_cta(ptx::smem_u32(raw), static_cast<uint32_t>(block)) + static_cast<uint32_t>(at);
        asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(x) : "r"(theirs));
        return x;
      };
      if (kTop) {
        const int theirs = lane < parts ? static_cast<int>(word(lane, offsetof(Shared, count))) : 0;
        int before = 0, n = 0;
#pragma unroll
        for (int r = 0; r < kMaxCluster; ++r) {
          const int c = __shfl_sync(0xFFFFFFFFu, theirs, r);
          if (r < warp) before += c;
          if (r == warp) n = c;
          candidates += r > 0 ? c : 0;
        }
        for (int i = lane; i < n; i += 32) {
          const size_t at = 8 * static_cast<size_t>(kSorted + i);
          const Key lo = word(warp, at), hi = word(warp, at + 4);
          sh.list[before + i] = lo | (hi << 32);
        }
      }
      if (warp == 0) {
        a = Sums{-INFINITY, 0.f, 0.f};
        if (lane < parts)
          a = Sums{__uint_as_float(word(lane, offsetof(Shared, all))), __uint_as_float(word(lane, offsetof(Shared, all) + 4)),
                   __uint_as_float(word(lane, offsetof(Shared, all) + 8))};
#pragma unroll
        for (int o = kMaxCluster / 2; o > 0; o >>= 1) a = join(a, from_lane(a, lane ^ o));
        if (lane == 0) sh.all = a;
      }
      __syncthreads();
      if (candidates > kOrdered) {
        if (kTop && warp == 0) keep_best(sh.list, candidates, P.top, P.index_bits, lane);
        candidates = P.top;
      }
    }
    ptx::cluster_sync_all();  // lists stay until they are read
    if (part != 0) return;
  }

  const Sums all = sh.all;
  const float log2_s = log2f(all.s);
  const bool nothing = all.m == -INFINITY && all.s == 0.f;  // no logit above -inf
  auto log_prob = [&](float z) { return nothing ? -INFINITY : (fmaf(z, P.scale2, -all.m) - log2_s) * kLn2; };
  if (tid == 0) {
    if (P.logprob != nullptr) P.logprob[token] = log_prob(s_target);
    if (P.entropy != nullptr) P.entropy[token] = nothing ? 0.f : (log2_s - all.e / all.s) * kLn2;
    if (P.lse != nullptr) P.lse[token] = nothing ? -INFINITY : fmaf(all.m, kLn2, log2_s * kLn2);
  }
  if (kTop && tid < candidates) {
    const Key mine = sh.list[tid];
    const int place = place_of(sh.list, candidates, mine);
    if (place >= P.top) return;
    const float z = value_of<kFp32>(P, mine);
    const long long at = token * P.top + place;
    if (P.top_ids != nullptr) P.top_ids[at] = P.vocab - 1 - static_cast<int>(mine & ((1ull << P.index_bits) - 1));
    if (P.top_logits != nullptr) P.top_logits[at] = z;
    if (P.top_logprob != nullptr) P.top_logprob[at] = log_prob(z);
  }
}

// Gradient of the logits, one tile of a row a block.
template <bool kFp32>
__global__ void __launch_bounds__(kThreads) grad_kernel(const __grid_constant__ GradParams P) {
  using C = Cells<kFp32>;
  using T = typename C::T;
  constexpr int kEach = C::kEach;
  const int tid = threadIdx.x;
  const long long token = blockIdx.y;
  const T* row = static_cast<const T*>(P.z) + token * P.ld;
  T* out = static_cast<T*>(P.dz) + token * P.ld_dz;
  const int shift = static_cast<int>((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
  const int vectors = static_cast<int>((static_cast<long long>(shift) + P.vocab + kEach - 1) / kEach);
  const int v0 = static_cast<int>(blockIdx.x) * kTileVectors;
  if (v0 >= vectors) return;
  int64_t y = -1;
  bool counts = true;
  if (P.targets != nullptr) {
    y = P.targets[token];
    counts = y >= 0 && y < P.vocab;
  }
  uint4 v[kVectors];
  if (counts) {
#pragma unroll
    for (int i = 0; i < kVectors; ++i) v[i] = load_vector<kFp32>(row, P.vocab, shift, v0 + i * kThreads + tid, vectors);
  }
  const float lse = P.lse[token], h = P.h != nullptr ? P.h[token] : 0.f, r = P.r != nullptr ? P.r[token] : 0.f;
  const float entropy = P.h != nullptr ? P.entropy[token] : 0.f;
  const bool nothing = !counts || fabsf(lse) >= kFarLse;  // not for a NaN
  const float c0 = -(r + h * entropy) * P.scale, c1 = -h * P.scale;
  const int target = static_cast<int>(y);
  const float at_target = r * P.scale;
  const uint64_t scale = pair(P.scale, P.scale), minus_lse = pair(-lse, -lse), log2e = pair(kLog2e, kLog2e);
  const uint64_t factor0 = pair(c0, c0), factor1 = pair(c1, c1);
  const bool vec = (reinterpret_cast<uintptr_t>(out - shift) & 15) == 0;
#pragma unroll
  for (int i = 0; i < kVectors; ++i) {
    const int index = v0 + i * kThreads + tid, at = index * kEach - shift;
    if (index >= vectors) continue;
    float g[kEach];
#pragma unroll
    for (int e = 0; e < kEach; e += 2) {
      g[e] = g[e + 1] = 0.f;
      if (!nothing) {
        float l0, l1, x0, x1;
        unpair(fma2(pair(C::value(v[i], e), C::value(v[i], e + 1)), scale, minus_lse), l0, l1);
        const uint64_t log_q = pair(max_nan(l0, kFloor), max_nan(l1, kFloor));
        unpair(mul2(log_q, log2e), x0, x1);
        unpair(mul2(pair(ex2(x0), ex2(x1)), fma2(log_q, factor1, factor0)), g[e], g[e + 1]);
      }
    }
    if (!nothing && target >= at && target < at + kEach) {
#pragma unroll
      for (int e = 0; e < kEach; ++e)
        if (at + e == target) g[e] += at_target;
    }
    if (vec && at >= 0 && at + kEach <= P.vocab) {
      uint32_t w[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if constexpr (kFp32) {
          w[k] = __float_as_uint(g[k]);
        } else {
          const __nv_bfloat162 two = __floats2bfloat162_rn(g[2 * k], g[2 * k + 1]);
          w[k] = *reinterpret_cast<const uint32_t*>(&two);
        }
      }
      __stcs(reinterpret_cast<uint4*>(out + at), make_uint4(w[0], w[1], w[2], w[3]));
    } else {
#pragma unroll
      for (int e = 0; e < kEach; ++e)
        if (at + e >= 0 && at + e < P.vocab) {
          if constexpr (kFp32) out[at + e] = g[e];
          else out[at + e] = __float2bfloat16_rn(g[e]);
        }
    }
  }
}

int fail(int code, const char* msg) {
  muon::set_last_error(msg);
  return code;
}

struct DeviceGuard {
  int before = -1;
  cudaError_t set(int device) {
    cudaError_t e = cudaGetDevice(&before);
    return e == cudaSuccess && before != device ? cudaSetDevice(device) : e;
  }
  ~DeviceGuard() {
    int now = -1;
    if (before >= 0 && cudaGetDevice(&now) == cudaSuccess && now != before) cudaSetDevice(before);
  }
};

#define LOGITS_CUDA(call)                                                      \
  do {                                                                         \
    cudaError_t e_ = (call);                                                   \
    if (e_ != cudaSuccess) return fail(MUON_ERR_CUDA, cudaGetErrorString(e_)); \
  } while (0)

bool misaligned(const void* p, unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }

int check(const muon_logits_args* a) {
  if (!a) return fail(MUON_ERR_INVALID_ARG, "args is null");
  if (a->tokens < 0 || a->vocab <= 0) return fail(MUON_ERR_INVALID_ARG, "tokens must not be negative, vocab must be positive");
  if (a->tokens > (1 << 24) || a->vocab > (1 << 24)) return fail(MUON_ERR_UNSUPPORTED, "more than 2^24 tokens or vocabulary entries");
  if (a->dtype != MUON_DTYPE_BF16 && a->dtype != MUON_DTYPE_FP32) return fail(MUON_ERR_UNSUPPORTED, "logits must be bf16 or fp32");
  if (a->top < 0 || a->top > kMaxTop) return fail(MUON_ERR_UNSUPPORTED, "0 to 128 alternatives per token");
  if (a->top > a->vocab) return fail(MUON_ERR_INVALID_ARG, "more alternatives than vocabulary entries");
  const float scale2 = a->logit_scale * kLog2e;
  if (!std::isfinite(scale2) || !(scale2 > 0.f)) return fail(MUON_ERR_INVALID_ARG, "logit_scale must be positive and finite in fp32");
  if (a->tokens == 0) return MUON_OK;
  if (!a->logits) return fail(MUON_ERR_INVALID_ARG, "logits is null");
  if (a->ld < a->vocab) return fail(MUON_ERR_INVALID_ARG, "row stride smaller than vocab");
  if (misaligned(a->logits, a->dtype == MUON_DTYPE_FP32 ? 4 : 2) || misaligned(a->targets, 8) || misaligned(a->logprob, 4) ||
      misaligned(a->entropy, 4) || misaligned(a->lse, 4) || misaligned(a->top_ids, 8) || misaligned(a->top_logits, 4) ||
      misaligned(a->top_logprob, 4))
    return fail(MUON_ERR_ALIGNMENT, "pointer not aligned to its element size");
  return MUON_OK;
}

// The grid's second dimension holds 65535 rows.
constexpr int kRowsAtOnce = 65535;

// Blocks that share a row: enough for a few on every SM, each with half a tile at least.
int parts_for(int tokens, long long vectors, int sms) {
  int parts = 1;
  while (parts < kMaxCluster && static_cast<long long>(tokens) * parts * 2 <= 4ll * sms && vectors >= 2ll * parts * kTileVectors / 2) parts *= 2;
  return parts;
}

template <bool kFp32, bool kTop, int kThreads>
cudaError_t launch_of(const LogitsParams& P, int rows, int parts, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(parts), static_cast<unsigned>(rows));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = sizeof(Shared<kThreads>);
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = static_cast<unsigned>(parts);
  attr.val.clusterDim.y = 1;
  attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, logprob_kernel<kFp32, kTop, kThreads>, P);
}

template <bool kFp32, bool kTop>
cudaError_t launch(const LogitsParams& P, int rows, int parts, cudaStream_t stream) {
  // (of its four warps each has 32 maxima for a fourth of `top`)
  const bool brief = parts == 1 && P.vocab / Cells<kFp32>::kEach <= (kTop ? 2 : 1) * kShortVectors && P.top <= kMaxTop / 2;
  return brief ? launch_of<kFp32, kTop, kShortThreads>(P, rows, parts, stream) : launch_of<kFp32, kTop, kThreads>(P, rows, parts, stream);
}

}  // namespace

extern "C" int muon_logits_logprob(const muon_logits_args* a, int device, void* stream_v) {
  const int rc = check(a);
  if (rc != MUON_OK) return rc;
  if (a->logprob && !a->targets && a->tokens > 0) return fail(MUON_ERR_INVALID_ARG, "logprob without targets");
  const bool top = a->top > 0 && (a->top_ids || a->top_logits || a->top_logprob);
  if (!top && !a->logprob && !a->entropy && !a->lse && a->tokens > 0) return fail(MUON_ERR_INVALID_ARG, "no output wanted");
  if (a->tokens == 0) return MUON_OK;
  DeviceGuard guard;
  LOGITS_CUDA(guard.set(device));
  int sms = 0;
  LOGITS_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device));
  const bool fp32 = a->dtype == MUON_DTYPE_FP32;
  const int parts = parts_for(a->tokens, a->vocab / (fp32 ? 4 : 8), sms);
  int bits = 1;
  while ((1 << bits) < a->vocab) ++bits;
  for (int first = 0; first < a->tokens; first += kRowsAtOnce) {
    const int rows = a->tokens - first < kRowsAtOnce ? a->tokens - first : kRowsAtOnce;
    const long long entries = static_cast<long long>(first) * a->top;
    LogitsParams P = {};
    P.z = static_cast<const char*>(a->logits) + first * a->ld * (fp32 ? 4 : 2);
    P.ld = a->ld;
    P.tokens = rows;
    P.vocab = a->vocab;
    P.top = top ? a->top : 0;
    P.scale2 = a->logit_scale * kLog2e;
    P.targets = a->targets ? a->targets + first : nullptr;
    P.logprob = a->logprob ? a->logprob + first : nullptr;
    P.entropy = a->entropy ? a->entropy + first : nullptr;
    P.lse = a->lse ? a->lse + first : nullptr;
    P.top_ids = a->top_ids ? a->top_ids + entries : nullptr;
    P.top_logits = a->top_logits ? a->top_logits + entries : nullptr;
    P.top_logprob = a->top_logprob ? a->top_logprob + entries : nullptr;
    P.index_bits = bits;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_v);
    if (fp32) LOGITS_CUDA(top ? (launch<true, true>(P, rows, parts, stream)) : (launch<true, false>(P, rows, parts, stream)));
    else LOGITS_CUDA(top ? (launch<false, true>(P, rows, parts, stream)) : (launch<false, false>(P, rows, parts, stream)));
  }
  return MUON_OK;
}

extern "C" int muon_logits_logprob_grad(const muon_logits_args* a, const float* g_logprob, const float* g_entropy, void* dlogits,
                                        int64_t ld_dlogits, int device, void* stream_v) {
  const int rc = check(a);
  if (rc != MUON_OK) return rc;
  if (a->tokens == 0) return MUON_OK;
  if (!dlogits || !a->lse) return fail(MUON_ERR_INVALID_ARG, "dlogits or lse is null");
  if (g_logprob && !a->targets) return fail(MUON_ERR_INVALID_ARG, "g_logprob without targets");
  if (g_entropy && !a->entropy) return fail(MUON_ERR_INVALID_ARG, "g_entropy without the entropy");
  if (ld_dlogits < a->vocab) return fail(MUON_ERR_INVALID_ARG, "row stride smaller than vocab");
  const bool fp32 = a->dtype == MUON_DTYPE_FP32;
  if (misaligned(dlogits, fp32 ? 4 : 2) || misaligned(g_logprob, 4) || misaligned(g_entropy, 4))
    return fail(MUON_ERR_ALIGNMENT, "pointer not aligned to its element size");
  if (dlogits == a->logits && ld_dlogits != a->ld) return fail(MUON_ERR_INVALID_ARG, "in place with another row stride");
  DeviceGuard guard;
  LOGITS_CUDA(guard.set(device));
  const int each = fp32 ? 4 : 8;
  const int tiles = static_cast<int>((static_cast<long long>(a->vocab) + each - 1 + each - 1 + static_cast<long long>(each) * kTileVectors - 1) /
                                     (static_cast<long long>(each) * kTileVectors));
  for (int first = 0; first < a->tokens; first += kRowsAtOnce) {
    const int rows = a->tokens - first < kRowsAtOnce ? a->tokens - first : kRowsAtOnce;
    GradParams P = {};
    P.z = static_cast<const char*>(a->logits) + first * a->ld * (fp32 ? 4 : 2);
    P.dz = static_cast<char*>(dlogits) + first * ld_dlogits * (fp32 ? 4 : 2);
    P.ld = a->ld;
    P.ld_dz = ld_dlogits;
    P.tokens = rows;
    P.vocab = a->vocab;
    P.scale = a->logit_scale;
    P.targets = a->targets ? a->targets + first : nullptr;
    P.entropy = a->entropy ? a->entropy + first : nullptr;
    P.lse = a->lse + first;
    P.r = g_logprob ? g_logprob + first : nullptr;
    P.h = g_entropy ? g_entropy + first : nullptr;
    const dim3 grid(static_cast<unsigned>(tiles), static_cast<unsigned>(rows));
    cudaStream_t stream = static_cast<cudaStream_t>(stream_v);
    if (fp32) grad_kernel<true><<<grid, kThreads, 0, stream>>>(P);
    else grad_kernel<false><<<grid, kThreads, 0, stream>>>(P);
    LOGITS_CUDA(cudaGetLastError());
  }
  return MUON_OK;
}
