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
// once a tile.  The alternatives come out of the same pass: elements above the running
// threshold go into a list in shared memory, and where the list is long its `top` best
// raise the threshold.  A first threshold comes from the threads' maxima over the first
// tile, of which the top-th largest is below top different elements.
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

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kVectors = 4;  // 16-byte loads of one tile a thread
constexpr int kTileVectors = kThreads * kVectors;
constexpr int kList = 2048;  // candidates in shared memory; a cluster's lists fit one
constexpr int kMaxTop = 128;
constexpr int kMaxCluster = 8;
static_assert(kMaxCluster * kMaxTop <= kList, "the joined lists");
constexpr float kLn2 = 0.693147180559945309f;
constexpr float kLog2e = 1.44269504088896341f;
constexpr float kFloor = -200.0f;  // exponents of 2 from here down give 0, and stay finite in products

struct LogitsParams {
  const void* z;
  long long ld;
  int tokens, vocab, top, mark;
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

// Elements of a 16-byte vector.
template <bool kFp32>
struct Cells {
  using T = std::conditional_t<kFp32, float, __nv_bfloat16>;
  static constexpr int kEach = kFp32 ? 4 : 8;
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

// Value above, column counted down below: larger keys come first, equal logits by column.
typedef unsigned long long Key;
__device__ __forceinline__ Key make_key(const LogitsParams& P, float x, int column) {
  return (static_cast<Key>(ordered(x)) << P.index_bits) | static_cast<unsigned>(P.vocab - 1 - column);
}

// Running statistics in powers of 2: y = z scale2, reference m = the largest y, rounded,
// S and E against it, E in units of log2.  All of a row's differences are formed as one
// fused z scale2 - m, so that the rounding of m cancels.
struct Sums {
  float m, s, e;
};

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

struct Shared {
  Key list[kList];
  Key kept_keys[kMaxTop];
  int count;        // candidates appended, more than kList where some found no room
  int kept;
  Sums sums[kWarps];
  Sums all;
};

// Sum over the block.
__device__ __forceinline__ int block_total(int n, int* scratch) {
  n = __reduce_add_sync(0xFFFFFFFFu, n);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = n;
  __syncthreads();
  int t = 0;
#pragma unroll
  for (int i = 0; i < kWarps; ++i) t += scratch[i];
  return t;
}

// Largest key that at least `top` of the block's keys reach, by bisection; `count_from`
// counts a thread's keys not below its argument.
template <typename Count>
__device__ __forceinline__ Key best_from(int top, Key lo, Key hi, int* scratch, Count count_from) {
  // at least `top` keys reach lo, fewer reach hi
  while (hi - lo > 1) {
    const Key mid = lo + (hi - lo) / 2;
    const int n = block_total(count_from(mid), scratch);
    if (n >= top) {
      lo = mid;
      if (n == top) break;
    } else {
      hi = mid;
    }
  }
  return lo;
}

// Keeps the `top` largest of list[0, n), in any order.  All threads call.
__device__ __noinline__ void keep_best(const LogitsParams& P, Shared& sh, int n, int* scratch) {
  Key mine[kList / kThreads];
#pragma unroll
  for (int i = 0; i < kList / kThreads; ++i) {
    const int at = i * kThreads + static_cast<int>(threadIdx.x);
    mine[i] = at < n ? sh.list[at] : 0;
  }
  const Key from = best_from(P.top, 0, 1ull << (32 + P.index_bits), scratch, [&](Key k) {
    int c = 0;
#pragma unroll
    for (int i = 0; i < kList / kThreads; ++i) c += mine[i] >= k;
    return c;
  });
  __syncthreads();
  if (threadIdx.x == 0) sh.count = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kList / kThreads; ++i) {
    const int at = i * kThreads + static_cast<int>(threadIdx.x);
    if (at < n && mine[i] >= from) sh.list[atomicAdd(&sh.count, 1)] = mine[i];
  }
  __syncthreads();
}

// Where a tile has more candidates than the list holds (many equal logits, or a row that
// ascends): of the list only what came before this tile counts, and the tile's elements
// are read again.
template <bool kFp32>
__device__ __noinline__ void keep_best_of_tile(const LogitsParams& P, Shared& sh, const typename Cells<kFp32>::T* row, int shift,
                                               int v0, int end, int* scratch) {
  const int from = max(0, v0 * Cells<kFp32>::kEach - shift);
  const int to = min(P.vocab, min(end, v0 + kTileVectors) * Cells<kFp32>::kEach - shift);
  const Key columns = (1ull << P.index_bits) - 1;
  int earlier = 0;
  for (int i = threadIdx.x; i < kList; i += kThreads) earlier += P.vocab - 1 - static_cast<int>(sh.list[i] & columns) < from;
  earlier = block_total(earlier, scratch);
  auto each = [&](auto&& visit) {
    for (int i = threadIdx.x; i < earlier; i += kThreads) visit(sh.list[i]);
#pragma unroll 4
    for (int c = from + static_cast<int>(threadIdx.x); c < to; c += kThreads) visit(make_key(P, static_cast<float>(row[c]), c));
  };
  const Key best = best_from(P.top, 0, 1ull << (32 + P.index_bits), scratch, [&](Key k) {
    int n = 0;
    each([&](Key x) { n += x >= k; });
    return n;
  });
  __syncthreads();
  if (threadIdx.x == 0) sh.count = 0;
  __syncthreads();
  each([&](Key x) {
    if (x >= best) sh.kept_keys[atomicAdd(&sh.count, 1)] = x;
  });
  __syncthreads();
  for (int i = threadIdx.x; i < P.top; i += kThreads) sh.list[i] = sh.kept_keys[i];
  __syncthreads();
}

// The smallest value among the list's first n keys, as a float.
__device__ __forceinline__ float lowest(const LogitsParams& P, const Shared& sh, int n, int* scratch) {
  uint32_t low = 0xFFFFFFFFu;
  for (int i = threadIdx.x; i < n; i += kThreads) low = min(low, static_cast<uint32_t>(sh.list[i] >> P.index_bits));
  low = __reduce_min_sync(0xFFFFFFFFu, low);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = static_cast<int>(low);
  __syncthreads();
  low = 0xFFFFFFFFu;
#pragma unroll
  for (int i = 0; i < kWarps; ++i) low = min(low, static_cast<uint32_t>(scratch[i]));
  return unordered(low);
}

template <bool kFp32, bool kTop>
__global__ void __launch_bounds__(kThreads, 4) logprob_kernel(const __grid_constant__ LogitsParams P) {
  using C = Cells<kFp32>;
  constexpr int kEach = C::kEach;
  extern __shared__ __align__(16) unsigned char raw[];
  Shared& sh = *reinterpret_cast<Shared*>(raw);
  __shared__ int scratch[kWarps];
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
  if (kTop) {
    if (tid == 0) sh.count = 0;
    __syncthreads();
  }

  const int shift = static_cast<int>((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(typename C::T));
  const int vectors = static_cast<int>((static_cast<long long>(shift) + P.vocab + kEach - 1) / kEach);
  const int begin = static_cast<int>(static_cast<long long>(vectors) * part / parts);
  const int end = static_cast<int>(static_cast<long long>(vectors) * (part + 1) / parts);

  Sums a = {-INFINITY, 0.f, 0.f};
  float threshold = -INFINITY;
  bool first = true;
  uint4 next[kVectors];
#pragma unroll
  for (int i = 0; i < kVectors; ++i) next[i] = load_vector<kFp32>(row, P.vocab, shift, begin + i * kThreads + tid, end);
  for (int v0 = begin; v0 < end; v0 += kTileVectors) {
    uint4 v[kVectors];
#pragma unroll
    for (int i = 0; i < kVectors; ++i) v[i] = next[i];
    if (v0 + kTileVectors < end) {
#pragma unroll
      for (int i = 0; i < kVectors; ++i)
        next[i] = load_vector<kFp32>(row, P.vocab, shift, v0 + kTileVectors + i * kThreads + tid, end);
    }
    float top_of[kVectors], most = -INFINITY;
#pragma unroll
    for (int i = 0; i < kVectors; ++i) {
      float x = C::value(v[i], 0);
#pragma unroll
      for (int e = 1; e + 1 < kEach; e += 2) x = max3(x, C::value(v[i], e), C::value(v[i], e + 1));
      top_of[i] = fmaxf(x, C::value(v[i], kEach - 1));
      most = fmaxf(most, top_of[i]);
    }
    const float reference = most * P.scale2;
    if (reference > a.m) rescale(a, reference);
    const float base = a.m == -INFINITY ? 0.f : -a.m;
    float s[2] = {0.f, 0.f}, w[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kVectors; ++i)
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const float d = max_nan(fmaf(C::value(v[i], e), P.scale2, base), kFloor);
        const float p = ex2(d);
        s[e & 1] += p;
        w[e & 1] = fmaf(p, d, w[e & 1]);
      }
    a.s += s[0] + s[1];
    a.e += w[0] + w[1];

    if constexpr (kTop) {
      const int here = min(end - v0, kTileVectors);
      if (first && here >= P.top) {
        // the top-th largest of the threads' maxima, to 16 bits: as many elements reach it
        const uint32_t mine = ordered(most) >> 16;
        uint32_t lo = 0;
        const bool some = tid < here;
#pragma unroll 1
        for (uint32_t b = 0x8000u; b > 0; b >>= 1)
          if (__syncthreads_count(some && mine >= (lo | b)) >= P.top) lo |= b;
        threshold = unordered(max(lo << 16, 0x007FFFFFu));
      }
      int last = -1;
      const bool all = first && !(threshold > -INFINITY);
#pragma unroll
      for (int i = 0; i < kVectors; ++i) {
        const int index = v0 + i * kThreads + tid;
        if ((top_of[i] > threshold || (first && top_of[i] == threshold) || all) && index < end) {
          const int column0 = index * kEach - shift;
#pragma unroll
          for (int e = 0; e < kEach; ++e) {
            const float x = C::value(v[i], e);
            const int column = column0 + e;
            if ((x > threshold || (first && x == threshold) || all) && column >= 0 && column < P.vocab) {
              last = atomicAdd(&sh.count, 1);
              if (last < kList) sh.list[last] = make_key(P, x, column);
            }
          }
        }
      }
      // positions are given out one by one: one past the mark is seen by the thread that got it
      if (__syncthreads_or(last >= P.mark)) {
        const int n = sh.count;
        if (n > kList) {
          keep_best_of_tile<kFp32>(P, sh, row, shift, v0, end, scratch);
        } else {
          keep_best(P, sh, n, scratch);
        }
        threshold = lowest(P, sh, P.top, scratch);
        __syncthreads();
      }
      first = false;
    }
  }

  // statistics: warp, block, cluster
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const Sums b = {__shfl_xor_sync(0xFFFFFFFFu, a.m, o), __shfl_xor_sync(0xFFFFFFFFu, a.s, o),
                    __shfl_xor_sync(0xFFFFFFFFu, a.e, o)};
    a = join(a, b);
  }
  if (lane == 0) sh.sums[warp] = a;
  if (kTop) {
    __syncthreads();
    const int n = sh.count;
    __syncthreads();
    if (n > P.top) keep_best(P, sh, n, scratch);
  }
  __syncthreads();
  if (tid == 0) {
    a = sh.sums[0];
    for (int i = 1; i < kWarps; ++i) a = join(a, sh.sums[i]);
    sh.all = a;
    sh.kept = kTop ? sh.count : 0;
  }
  __syncthreads();
  if (parts > 1) {
    ptx::cluster_sync_all();
    if (part == 0) {
      // the other blocks' lists behind this one's, their sums into this one's
      int n = sh.kept;
      for (int r = 1; r < parts; ++r) {
        const uint32_t theirs = ptx::map_to_cta(ptx::smem_u32(raw), static_cast<uint32_t>(r));
        auto word = [&](size_t at) {
          uint32_t x;
          asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(x) : "r"(theirs + static_cast<uint32_t>(at)));
          return x;
        };
        if (tid == 0) {
          const Sums b = {__uint_as_float(word(offsetof(Shared, all))), __uint_as_float(word(offsetof(Shared, all) + 4)),
                          __uint_as_float(word(offsetof(Shared, all) + 8))};
          sh.all = join(sh.all, b);
        }
        if (kTop) {
          const int more = static_cast<int>(word(offsetof(Shared, kept)));
          for (int i = tid; i < more; i += kThreads) {
            const Key lo = word(8 * static_cast<size_t>(i)), hi = word(8 * static_cast<size_t>(i) + 4);
            sh.list[n + i] = lo | (hi << 32);
          }
          n += more;
        }
      }
      __syncthreads();
      if (kTop) {
        if (n > P.top) keep_best(P, sh, n, scratch);
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
  if (kTop && tid < P.top) {
    const Key mine = sh.list[tid];
    int place = 0;
    for (int i = 0; i < P.top; ++i) place += sh.list[i] > mine;
    const float z = unordered(static_cast<uint32_t>(mine >> P.index_bits));
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
  const bool nothing = !counts || lse == -INFINITY;
  const float c0 = -(r + h * entropy) * P.scale, c1 = -h * P.scale;
  const int target = static_cast<int>(y);
  const float at_target = r * P.scale;
  const bool vec = (reinterpret_cast<uintptr_t>(out - shift) & 15) == 0;
#pragma unroll
  for (int i = 0; i < kVectors; ++i) {
    const int index = v0 + i * kThreads + tid, at = index * kEach - shift;
    if (index >= vectors) continue;
    float g[kEach];
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      g[e] = 0.f;
      if (!nothing) {
        const float log_q = max_nan(fmaf(C::value(v[i], e), P.scale, -lse), kFloor);
        g[e] = ex2(log_q * kLog2e) * fmaf(c1, log_q, c0);
        if (at + e == target) g[e] += at_target;
      }
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

// Blocks that share a row: enough for a few on every SM, each with a tile at least.
int parts_for(int tokens, long long vectors, int sms) {
  int parts = 1;
  while (parts < kMaxCluster && static_cast<long long>(tokens) * parts * 2 <= 4ll * sms && vectors >= 2ll * parts * kTileVectors / 2) parts *= 2;
  return parts;
}

template <bool kFp32, bool kTop>
cudaError_t launch(const LogitsParams& P, int rows, int parts, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(parts), static_cast<unsigned>(rows));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = sizeof(Shared);
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = static_cast<unsigned>(parts);
  attr.val.clusterDim.y = 1;
  attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, logprob_kernel<kFp32, kTop>, P);
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
    P.mark = 8 * a->top < kList ? (8 * a->top > 256 ? 8 * a->top : 256) : kList;
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
