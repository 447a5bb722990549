// Row kernels around the products of the LM-head losses: which tokens count and
// their rows gathered (prepare), the softmax statistics joined into losses and
// gradient coefficients (finalise), partial dX joined (dx).  All of them are short
// streaming kernels.
#include <cuda_bf16.h>

#include "head_codes.cuh"
#include "ptx.cuh"

namespace muon {
namespace head {

namespace {

constexpr int kRowThreads = 256;
constexpr int kRowWarps = kRowThreads / 32;
constexpr float kLn2 = 0.693147180559945309f;

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  return v;
}

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
  return v;
}

// Sum over a block of kWarps warps in a fixed order; every thread gets it.
template <int kWarps = kRowWarps, typename T>
__device__ __forceinline__ T block_sum(T v, T* scratch) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
  __syncthreads();
  T s = scratch[0];
#pragma unroll
  for (int i = 1; i < kWarps; ++i) s += scratch[i];
  return s;
}

__device__ __forceinline__ float teacher_logit(const RowParams& R, int t, int k) {
  const long long at = static_cast<long long>(t) * R.ld_z + k;
  return R.z_fp32 ? static_cast<const float*>(R.z)[at] : __bfloat162float(static_cast<const __nv_bfloat16*>(R.z)[at]);
}

__device__ __forceinline__ bool in_vocab(const RowParams& R, int64_t id) { return id >= 0 && id < R.vocab; }

// Distillation: a token counts if one of its entries has an index in the
// vocabulary and a logit above minus infinity (a NaN counts, and shows).
__global__ void __launch_bounds__(kRowThreads) flags_kernel(const RowParams R) {
  const int t = blockIdx.x * kRowWarps + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (t < R.tokens) {
    bool any = false;
    for (int k = lane; k < R.top; k += 32)
      any |= in_vocab(R, R.ids_in[static_cast<long long>(t) * R.ld_ids + k]) && !(teacher_logit(R, t, k) == -INFINITY);
    any = __any_sync(0xFFFFFFFFu, any);
    if (lane == 0) R.flags[t] = any;
  }
}

// Token t counts?  flags: where distillation finds its answer.
template <bool kDistill>
__device__ __forceinline__ bool counts(const RowParams& R, const unsigned char* flags, int t) {
  return kDistill ? flags[t] != 0 : in_vocab(R, R.ids_in[static_cast<long long>(t) * R.ld_ids]);
}


// Many tokens: how many count in every run of kRowThreads, for prepare_kernel.
template <bool kDistill>
__global__ void __launch_bounds__(kRowThreads) count_kernel(const RowParams R) {
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  const int t = blockIdx.x * kRowThreads + threadIdx.x;
  const int n = __syncthreads_count(t < R.tokens && counts<kDistill>(R, R.flags, t));
  if (threadIdx.x == 0) R.run_counts[blockIdx.x] = n;
}

// Copy of a head whose rows TMA cannot address (16-byte aligned rows) into rows that it
// can, by block `block` of `blocks`; one warp per row.
__device__ __forceinline__ void pack_rows(const RowParams& R, int block, int blocks) {
  const int lane = threadIdx.x & 31;
  const long long step = static_cast<long long>(blocks) * kRowWarps;
  for (long long r = static_cast<long long>(block) * kRowWarps + (threadIdx.x >> 5); r < R.vocab; r += step) {
    const unsigned short* s = reinterpret_cast<const unsigned short*>(R.pack_from + r * R.ld_pack);
    uint32_t* d = reinterpret_cast<uint32_t*>(R.pack_to + r * R.ld_w);
    for (int c = lane * 2; c < R.dim; c += 64) {
      const uint32_t lo = s[c], hi = c + 1 < R.dim ? s[c + 1] : 0u;
      d[c >> 1] = lo | (hi << 16);
    }
  }
}

__global__ void __launch_bounds__(kRowThreads) pack_kernel(const RowParams R) { pack_rows(R, blockIdx.x, gridDim.x); }

// Gathers the rows of the tokens that count, in token order, so that masked
// tokens cost nothing in the products and whatever they hold reaches no sum.
// Every block counts the tokens before its own by itself (8 bytes a token out of
// L2) instead of waiting for a scan; with many tokens it adds up the counts of whole runs.  Distillation: the teacher's entries become
// probabilities, sorted by index, with the number of entries below every
// 256-column tile, so that an epilogue finds its entries without a search.
template <bool kDistill>
__global__ void __launch_bounds__(kRowThreads) prepare_kernel(const RowParams R) {
  __shared__ int s_int[kRowWarps];
  __shared__ float s_f[kRowWarps];
  __shared__ int s_id[kDistill ? kRowWarps : 1][kMaxTop];
  __shared__ int s_sorted[kDistill ? kRowWarps : 1][kMaxTop];
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int blocks = static_cast<int>(gridDim.x) - R.pack_blocks;  // the last ones copy the head
  if (static_cast<int>(blockIdx.x) >= blocks) {
    pack_rows(R, static_cast<int>(blockIdx.x) - blocks, R.pack_blocks);
    return;
  }
  const int first = blockIdx.x * kRowWarps;
  const unsigned char* flags = R.flags;

  int before = 0, total = 0;
  float wsum = 0.f;
  const bool sum_weights = blockIdx.x == 0 && R.weight != nullptr;
  if (R.run_counts == nullptr) {
    for (int t = tid; t < R.tokens; t += kRowThreads) {
      const bool c = counts<kDistill>(R, flags, t);
      total += c;
      before += c && t < first;
      if (sum_weights && c) wsum += R.weight[t];
    }
  } else {
    const int runs = (R.tokens + kRowThreads - 1) / kRowThreads, mine = first / kRowThreads;
    for (int i = tid; i < runs; i += kRowThreads) {
      const int n = R.run_counts[i];
      total += n;
      if (i < mine) before += n;
    }
    const int t = mine * kRowThreads + tid;
    before += t < first && counts<kDistill>(R, flags, t);
    if (sum_weights)
      for (int u = tid; u < R.tokens; u += kRowThreads)
        if (counts<kDistill>(R, flags, u)) wsum += R.weight[u];
  }
  total = block_sum(total, s_int);
  before = block_sum(before, s_int);
  if (sum_weights) wsum = block_sum(wsum, s_f);
  if (blockIdx.x == 0 && tid == 0) {
    const float norm = R.weight != nullptr ? wsum : static_cast<float>(total);
    R.ctrl->status = 0;
    R.ctrl->n_valid = total;
    R.ctrl->ticket = 0;
    R.ctrl->coef = !R.mean ? R.scale : (norm == 0.f ? 0.f : R.scale / norm);
    R.ctrl->kept = R.keeps;
  }

  const int t = first + warp;
  const bool mine = t < R.tokens && counts<kDistill>(R, flags, t);
  const int peer = first + lane;
  const unsigned ahead = __ballot_sync(0xFFFFFFFFu, lane < warp && peer < R.tokens && counts<kDistill>(R, flags, peer));
  const int pos = before + __popc(ahead);
  if (t < R.tokens && lane == 0) {
    if (mine) {
      R.row_of[pos] = t;
    } else if (R.loss != nullptr) {
      R.loss[t] = 0.f;
      if (R.lse != nullptr) R.lse[t] = 0.f;
      if (R.entropy != nullptr) R.entropy[t] = 0.f;
    }
  }
  if (t < R.tokens && !mine && R.dx != nullptr) {
    const long long at = static_cast<long long>(t) * R.ld_dx;
    for (int c = lane; c < R.dim; c += 32) {
      if (R.dx_fp32) static_cast<float*>(R.dx)[at + c] = 0.f;
      else static_cast<__nv_bfloat16*>(R.dx)[at + c] = __float2bfloat16_rn(0.f);
    }
  }
  if (mine) {
    const __nv_bfloat16* src = R.x + static_cast<long long>(t) * R.ld_x;
    __nv_bfloat16* dst = R.xc + static_cast<long long>(pos) * R.ld_xc;
    int done = 0;
    if (R.x_vec) {
      done = R.dim & ~7;
      for (int c = lane * 8; c < done; c += 256)
        *reinterpret_cast<uint4*>(dst + c) = __ldg(reinterpret_cast<const uint4*>(src + c));
    }
    for (int c = done + lane; c < R.dim; c += 32) dst[c] = src[c];

    if (!kDistill) {
      if (lane == 0) R.ids[pos] = static_cast<int>(R.ids_in[static_cast<long long>(t) * R.ld_ids]);
    } else {
      constexpr int kPer = kMaxTop / 32;
      const int K = R.top;
      int id[kPer];
      float z[kPer], p[kPer];
      float zmax = -INFINITY;
      bool bad = false;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int k = lane + 32 * i;
        id[i] = kNoId;
        z[i] = -INFINITY;
        if (k < K) {
          const int64_t raw = R.ids_in[static_cast<long long>(t) * R.ld_ids + k];
          if (in_vocab(R, raw)) {
            id[i] = static_cast<int>(raw);
            z[i] = teacher_logit(R, t, k) * R.inv_t;
            bad |= z[i] != z[i];
          }
          s_id[warp][k] = id[i];
        }
        zmax = fmaxf(zmax, z[i]);
      }
      zmax = warp_max(zmax);
      bad = __any_sync(0xFFFFFFFFu, bad);
      const float ref = R.teacher_lse != nullptr ? R.teacher_lse[t] : zmax;
      float psum = 0.f;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        p[i] = id[i] == kNoId ? 0.f : expf(z[i] - ref);
        psum += p[i];
      }
      psum = warp_sum(psum);
      float log_norm = ref;  // log p = z - log_norm
      if (R.teacher_lse == nullptr) {
        log_norm = ref + logf(psum);
        const float inv = 1.0f / psum;
#pragma unroll
        for (int i = 0; i < kPer; ++i) p[i] *= inv;
        psum = bad ? NAN : 1.0f;
      }
      float h = 0.f;
#pragma unroll
      for (int i = 0; i < kPer; ++i) h += p[i] > 0.f ? p[i] * (z[i] - log_norm) : (p[i] == 0.f ? 0.f : p[i]);
      h = warp_sum(h);
      __syncwarp();
      // place of an entry = how many come before it by (index, position)
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int k = lane + 32 * i;
        if (k < K) {
          int place = 0;
          for (int j = 0; j < K; ++j) {
            const int other = s_id[warp][j];
            place += other < id[i] || (other == id[i] && j < k);
          }
          s_sorted[warp][place] = id[i];
          R.ids[static_cast<long long>(pos) * K + place] = id[i];
          R.p[static_cast<long long>(pos) * K + place] = p[i];
        }
      }
      __syncwarp();
      if (lane == 0) {
        R.row_h[pos] = h;
        R.row_c[pos] = psum;
      }
      for (int tile = lane; tile < R.n_starts; tile += 32) {
        const long long bound = static_cast<long long>(tile) * kTileN;
        int lo = 0, hi = K;
        while (lo < hi) {
          const int mid = (lo + hi) >> 1;
          if (s_sorted[warp][mid] < bound) lo = mid + 1;
          else hi = mid;
        }
        // the last boundary lies past the vocabulary: entries that do not count stay above it
        R.starts[static_cast<long long>(pos) * R.n_starts + tile] = static_cast<unsigned char>(lo);
      }
    }
  }
  // zero rows up to the next K block of dW's product
  const int rows = min(R.tokens, (total + kBK - 1) / kBK * kBK);
  for (int r = total + blockIdx.x * kRowWarps + warp; r < rows; r += blocks * kRowWarps)
    for (int c = lane * 8; c < R.dim; c += 256)  // ld_xc is a multiple of 8
      *reinterpret_cast<uint4*>(R.xc + static_cast<long long>(r) * R.ld_xc + c) = make_uint4(0u, 0u, 0u, 0u);
}

// Entries with at least this share of the distribution get their logits again in
// plain fp32: at most 16 a token, two or three in practice.  The rounding of the
// others' logits reaches the loss through a sixteenth or less of the mass, about
// what fp32 sums leave anyway; recomputing every entry would read top rows of w a
// token (1 GB for 4096 tokens, 64 entries and 2048 columns).
constexpr float kExactMass = 1.0f / 16.0f;

// x . w in fp32 by one warp; both rows 16-byte aligned.  Every lane gets the sum.
__device__ __forceinline__ float warp_dot(const __nv_bfloat16* x, const __nv_bfloat16* w, int dim, int lane) {
  float a = 0.f, b = 0.f;
  const int whole = dim & ~7;
  for (int c = lane * 8; c < whole; c += 256) {
    const uint4 u = *reinterpret_cast<const uint4*>(x + c), v = __ldg(reinterpret_cast<const uint4*>(w + c));
    const uint32_t uu[4] = {u.x, u.y, u.z, u.w}, vv[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      a = fmaf(__uint_as_float(uu[e] << 16), __uint_as_float(vv[e] << 16), a);
      b = fmaf(__uint_as_float(uu[e] & 0xFFFF0000u), __uint_as_float(vv[e] & 0xFFFF0000u), b);
    }
  }
  if (whole + lane < dim) a = fmaf(__bfloat162float(x[whole + lane]), __bfloat162float(w[whole + lane]), a);
  return warp_sum(a + b);
}

// v as power of two times a fraction in [1, 2); 0, subnormal, infinite and NaN stay as they
// are, with fraction 1.
__device__ __forceinline__ float fraction_of(float v, float& power) {
  const uint32_t bits = __float_as_uint(v), exponent = bits & 0x7F800000u;
  const bool normal = exponent != 0u && exponent != 0x7F800000u;
  power = normal ? __uint_as_float(bits & 0xFF800000u) : v;
  return normal ? __uint_as_float((bits & 0x007FFFFFu) | 0x3F800000u) : 1.0f;
}

// Joins a token's statistics over the vocabulary and forms, with l the scaled
// logits, lse their log-sum-exp, p the sparse target distribution, c = sum p:
//   loss = sum p log p - sum p (l - lse) + z_loss lse^2
//   gradient of the raw logit: g a (c' q - p),  c' = c + 2 z_loss lse
// row_q holds (g a c', log2-domain lse), entry_g the gradient at the entries, both
// without the fraction of the factor that all tokens share, coef * logit_scale: in the
// bf16 gradients of logits that fraction would be rounded with every -g a (1 - q) of a
// q near 0 in the same way, and all of dX and dW come out up to 2^-8 too large or too
// small.  The sums of dX and dW are multiplied with it in fp32 (Ctrl::rest).
// Exponents are taken from one fused multiply-add on the raw logit, so that a
// large logit costs a single rounding.
//
// One block per row; where there are few rows, gridDim.y blocks per row, each joining
// the statistics by itself in the same order.  kConvert: the block then turns its
// share of the first stored piece's codes into gradients.
//
// kInPlace: few tokens, rows are tokens and nothing came before the statistics.  What
// prepare_kernel does for more tokens is done here for one row, before the wait for
// the statistics, while they run.
//
// kFusedTiles: tiles a warp converts at a time, two with few rows (four: 482 us in place
// of 466 at 100 x 2048 x 163840), four with many.
template <bool kDistill, bool kConvert, int kThreads, bool kInPlace, int kFusedTiles>
__global__ void __launch_bounds__(kThreads) finalise_kernel(const RowParams R, const ConvertParams C) {
  constexpr int kWarps = kThreads / 32;
  __shared__ float s_f[kWarps];
  __shared__ float s_max[kWarps];
  __shared__ int s_id[kMaxTop];
  __shared__ float s_p[kMaxTop], s_raw[kMaxTop], s_exact[kMaxTop], s_g[kMaxTop];
  __shared__ bool s_last;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int row = blockIdx.x;
  const bool writes = blockIdx.y == 0;
  const int runs = kConvert ? (C.tiles + kFusedTiles - 1) / kFusedTiles : 0;
  const int run0 = static_cast<int>(blockIdx.y) * kWarps + warp, run_step = static_cast<int>(gridDim.y) * kWarps;
  const int K = kDistill ? R.top : 1;
  const long long at = static_cast<long long>(row) * K;
  int my_id = kNoId, t = row;
  float my_p = 1.0f, my_raw = 0.f, row_c = 1.0f, row_h = 0.f, coef = 0.f;
  bool counted = true;
  int source = tid;  // entry of the caller's list that thread `tid` < K holds
  // The logits that carry the loss, again as plain fp32 dot products, for the softmax
  // sum to hold them in place of the tensor cores' values: the tensor cores truncate at
  // every step of 16 products, which shifts a logit of 15 over 2048 columns by about
  // 1e-5.
  unsigned heavy[kDistill ? kMaxTop / 32 : 1];  // entries with their own dot product
  auto dots = [&]() {
    int nth = 0;
#pragma unroll
    for (int i = 0; i < (kDistill ? kMaxTop / 32 : 1); ++i) {
      heavy[i] = __ballot_sync(0xFFFFFFFFu, 32 * i + lane < K && s_p[32 * i + lane] >= kExactMass);
      for (unsigned todo = heavy[i]; todo; todo &= todo - 1, ++nth)
        if (nth % kWarps == warp) {
          const int e = 32 * i + __ffs(todo) - 1;
          const float exact = warp_dot(kInPlace ? R.x + row * R.ld_x : R.xc + row * R.ld_xc,
                                       R.w + static_cast<long long>(s_id[e]) * R.ld_w, R.dim, lane);
          if (lane == 0) s_exact[e] = exact;
        }
    }
  };
  if constexpr (kInPlace) {
    ptx::grid_launch_dependents();
    __shared__ unsigned char s_flags[kInPlaceRows];
    __shared__ int s_raw_id[kMaxTop], s_source[kMaxTop];
    const bool known = tid < R.tokens;  // at most kThreads tokens
    if (kDistill) {
      s_flags[tid] = 0;
      __syncthreads();
      for (int i = tid; i < R.tokens * K; i += kThreads) {
        const int r = i / K, k = i - r * K;
        if (in_vocab(R, R.ids_in[static_cast<long long>(r) * R.ld_ids + k]) && !(teacher_logit(R, r, k) == -INFINITY))
          s_flags[r] = 1;
      }
      __syncthreads();
    }
    const bool c = known && counts<kDistill>(R, s_flags, tid);
    const float norm = block_sum<kWarps>(c ? (R.weight != nullptr ? R.weight[tid] : 1.0f) : 0.f, s_f);
    coef = !R.mean ? R.scale : (norm == 0.f ? 0.f : R.scale / norm);
    counted = counts<kDistill>(R, s_flags, row);
    if (kConvert && writes) {  // operand of dW's product, and which rows of dX stay 0
      if (tid == 0) R.row_of[row] = counted ? row : -1;
      const uint4* src = reinterpret_cast<const uint4*>(R.x + row * R.ld_x);
      uint4* dst = reinterpret_cast<uint4*>(R.xc + row * R.ld_xc);
      const int whole = R.dim >> 3;
      for (int i = tid; i < whole; i += kThreads) dst[i] = counted ? src[i] : make_uint4(0u, 0u, 0u, 0u);
      const int i = whole * 8 + tid;
      if (i < R.dim) R.xc[row * R.ld_xc + i] = counted ? R.x[row * R.ld_x + i] : __float2bfloat16_rn(0.f);
    }
    if (!kDistill) {
      if (tid == 0 && counted) {
        my_id = static_cast<int>(R.ids_in[static_cast<long long>(row) * R.ld_ids]);
        s_id[0] = my_id;
        s_p[0] = 1.0f;
      }
      __syncthreads();
    } else if (counted) {
      float z = -INFINITY;
      int id = kNoId;
      if (tid < K) {
        const int64_t raw = R.ids_in[static_cast<long long>(row) * R.ld_ids + tid];
        if (in_vocab(R, raw)) {
          id = static_cast<int>(raw);
          z = teacher_logit(R, row, tid) * R.inv_t;
        }
        s_raw_id[tid] = id;
      }
      const float wm = warp_max(z);
      if (lane == 0) s_max[warp] = wm;
      __syncthreads();
      float ref = s_max[0];
#pragma unroll
      for (int i = 1; i < kWarps; ++i) ref = fmaxf(ref, s_max[i]);
      if (R.teacher_lse != nullptr) ref = R.teacher_lse[row];
      float p = id == kNoId ? 0.f : expf(z - ref);
      row_c = block_sum<kWarps>(p, s_f);
      float log_norm = ref;
      if (R.teacher_lse == nullptr) {
        log_norm = ref + logf(row_c);
        p *= 1.0f / row_c;
        row_c = row_c == row_c ? 1.0f : row_c;  // a NaN among the logits shows
      }
      row_h = block_sum<kWarps>(p > 0.f ? p * (z - log_norm) : (p == 0.f ? 0.f : p), s_f);
      if (tid < K) {  // place of an entry = how many come before it by (index, position)
        int place = 0;
        for (int j = 0; j < K; ++j) {
          const int other = s_raw_id[j];
          place += other < id || (other == id && j < tid);
        }
        s_id[place] = id;
        s_p[place] = p;
        s_source[place] = tid;
      }
      __syncthreads();
      if (tid < K) {
        my_id = s_id[tid];
        my_p = s_p[tid];
        source = s_source[tid];
      }
    }
    if (counted) dots();
  }
  ptx::grid_dependency_wait();
  if (!kInPlace) ptx::grid_launch_dependents();
  // Everything whose address is known is asked for at once (rows past the tokens that
  // count hold no news, but they are there), so that one memory latency covers it.
  // Of the statistics four a thread, the others in the loop below: with 2, 4, 5 and 10 the
  // calls take the same time at every vocabulary tried, from 2000 to 163840 entries.
  constexpr int kAhead = 4;
  const float2* st = R.stats + static_cast<long long>(row) * R.stats_ld;
  float2 ahead[kAhead];
  Codes<kFusedTiles> codes;
  if (row < R.tokens) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      ahead[i] = tid + i * kThreads < R.stats_n ? st[tid + i * kThreads] : make_float2(-INFINITY, 0.f);
    if (tid < K) {
      my_raw = R.entry_logit[at + source];
      if (!kInPlace) {
        my_id = R.ids[at + tid];
        if (kDistill) my_p = R.p[at + tid];
      }
    }
    if (!kInPlace) {
      t = R.row_of[row];
      if (kDistill) {
        row_c = R.row_c[row];
        row_h = R.row_h[row];
      }
    }
    if (kConvert && run0 < runs) load_codes(C, row, run0 * kFusedTiles, lane, codes);
  }
  const int n_valid = kInPlace ? R.tokens : R.ctrl->n_valid;
  if (!kInPlace) coef = R.ctrl->coef;
  float power;
  const float rest = fraction_of(coef * R.logit_scale, power);
  if (row == 0 && writes && tid == 0) R.ctrl->rest = rest;
  if (row < n_valid && counted) {
    if (tid < K) {
      if (!kInPlace) {
        s_id[tid] = my_id;
        s_p[tid] = my_id == kNoId ? 0.f : my_p;
      }
      s_raw[tid] = my_id == kNoId ? 0.f : my_raw;
    }
    float m = -INFINITY, s = 0.f;
    auto join = [&](float2 v) {
      const float mx = fmaxf(m, v.x);
      const float base = mx == -INFINITY ? 0.f : mx;
      s = s * exp2f(m - base) + v.y * exp2f(v.x - base);
      m = mx;
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i) join(ahead[i]);
    for (int i = tid + kAhead * kThreads; i < R.stats_n; i += kThreads) join(st[i]);
    const float wm = warp_max(m);
    if (lane == 0) s_max[warp] = wm;
    __syncthreads();
    if (!kInPlace) dots();
    float mx = s_max[0];
#pragma unroll
    for (int i = 1; i < kWarps; ++i) mx = fmaxf(mx, s_max[i]);
    const float base = mx == -INFINITY ? 0.f : mx;
    s = block_sum<kWarps>(s * exp2f(m - base), s_f);
#pragma unroll
    for (int i = 0; i < (kDistill ? kMaxTop / 32 : 1); ++i)
      for (unsigned todo = heavy[i]; todo; todo &= todo - 1) {
        const int e = 32 * i + __ffs(todo) - 1;
        bool again = false;  // an index listed more than once is one logit
        for (int j = e - 1; j >= 0 && s_id[j] == s_id[e]; --j) again |= s_p[j] >= kExactMass;
        if (!again) s += exp2f(fmaf(s_exact[e], R.scale2, -base)) - exp2f(fmaf(s_raw[e], R.scale2, -base));
      }
    const float lse2 = base + log2f(s);
    const float lse = lse2 * kLn2;
    const float weight = R.weight != nullptr ? R.weight[t] : 1.0f;
    const float g = coef * weight, ga = weight * power;
    const float cq = row_c + 2.0f * R.z_loss * lse;
    float ce = 0.f;
    if (tid < K && s_id[tid] != kNoId) {
      const float p = s_p[tid];
      const float lq2 = fmaf(p >= kExactMass ? s_exact[tid] : s_raw[tid], R.scale2, -lse2);
      ce = p == 0.f ? 0.f : -p * lq2 * kLn2;
      // an index listed more than once: its entries share the gradient of the one logit
      float pj = p;
      for (int j = tid - 1; j >= 0 && s_id[j] == s_id[tid]; --j) pj += s_p[j];
      for (int j = tid + 1; j < K && s_id[j] == s_id[tid]; ++j) pj += s_p[j];
      s_g[tid] = ga * (cq * exp2f(lq2) - pj);
      if (!kInPlace && writes) R.entry_g[at + tid] = s_g[tid];
    }
    ce = block_sum<kWarps>(ce, s_f);  // a barrier, too: s_g is complete
    const float2 rq = make_float2(ga * cq, lse2);
    if (writes && tid == 0) {
      const float loss = ce + row_h + R.z_loss * lse * lse;
      R.loss[t] = loss;
      if (R.lse != nullptr) R.lse[t] = lse;
      if (!kInPlace) R.row_q[row] = rq;
      R.row_l[row] = g * loss;
    }
    if (kConvert)
      for (int r = run0; r < runs; r += run_step) {
        if (r != run0) load_codes(C, row, r * kFusedTiles, lane, codes);
        convert_codes(C, row, r * kFusedTiles, rq, s_id, s_g, lane, codes);
      }
  } else if (row < min(R.tokens, (n_valid + kBK - 1) / kBK * kBK)) {
    if (kInPlace && writes && tid == 0) {
      R.loss[row] = 0.f;
      if (R.lse != nullptr) R.lse[row] = 0.f;
      R.row_l[row] = 0.f;
    }
    if (kConvert)
      for (int r = run0; r < runs; r += run_step) clear_row<kFusedTiles>(C, row, r * kFusedTiles, lane);
  }
  if (R.total == nullptr || !writes) return;
  // no gradients: the last row's block adds the tokens up, always in the same order
  if (tid == 0) {
    __threadfence();
    s_last = atomicAdd(&R.ctrl->ticket, 1u) == gridDim.x - 1;
  }
  __syncthreads();
  if (s_last) {
    __threadfence();
    float sum = 0.f;
    for (int i = tid; i < n_valid; i += kThreads) sum += __ldcg(R.row_l + i);
    sum = block_sum<kWarps>(sum, s_f);
    if (tid == 0) *R.total = sum;
  }
}

// Log probability, entropy and log-sum-exp of one token from its statistics, all in units
// of log2: y = l log2(e), M a row's largest y, S = sum 2^(y - M), E = sum (y - M) 2^(y - M),
//   logprob = ln 2 (y_target - M - log2 S),  entropy = ln 2 (log2 S - E / S)
// The target's logit is formed again as a plain fp32 sum and takes the tensor cores' place in
// S and E, as in finalise_kernel.  One block a row; kInPlace: rows are tokens.
template <bool kInPlace, bool kEntropy>
__global__ void __launch_bounds__(kRowThreads) logprob_kernel(const RowParams R) {
  __shared__ float s_f[kRowWarps], s_max[kRowWarps];
  __shared__ float s_exact;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, row = blockIdx.x;
  int t = row, id = 0;
  if (kInPlace) {
    ptx::grid_launch_dependents();
    const int64_t raw = R.ids_in[static_cast<long long>(row) * R.ld_ids];
    if (!in_vocab(R, raw)) {
      if (tid == 0) {
        R.loss[row] = 0.f;
        if (R.lse != nullptr) R.lse[row] = 0.f;
        if (kEntropy) R.entropy[row] = 0.f;
      }
      // nothing of the product is needed, but a grid that did not wait could end before it,
      // and what comes next in the stream take the workspace while it is written to
      ptx::grid_dependency_wait();
      return;
    }
    id = static_cast<int>(raw);
  } else {
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    if (row >= R.ctrl->n_valid) return;
    t = R.row_of[row];
    id = R.ids[row];
  }
  if (warp == 0) {
    const float exact = warp_dot(kInPlace ? R.x + static_cast<long long>(row) * R.ld_x : R.xc + static_cast<long long>(row) * R.ld_xc,
                                 R.w + static_cast<long long>(id) * R.ld_w, R.dim, lane);
    if (lane == 0) s_exact = exact;
  }
  if (kInPlace) ptx::grid_dependency_wait();
  const long long at = static_cast<long long>(row) * R.stats_ld;
  float m = -INFINITY, s = 0.f, e = 0.f;
#pragma unroll 4
  for (int i = tid; i < R.stats_n; i += kRowThreads) {
    const float2 v = R.stats[at + i];
    const float ve = kEntropy ? R.stats_e[at + i] : 0.f;
    const float mx = fmaxf(m, v.x);
    const float dm = m == mx ? 0.f : fmaxf(m - mx, -200.f), dv = v.x == mx ? 0.f : fmaxf(v.x - mx, -200.f);
    const float fm = exp2f(dm), fv = exp2f(dv);
    if (kEntropy) e = fm * fmaf(dm, s, e) + fv * fmaf(dv, v.y, ve);
    s = s * fm + v.y * fv;
    m = mx;
  }
  const float wm = warp_max(m);
  if (lane == 0) s_max[warp] = wm;
  __syncthreads();
  float mx = s_max[0];
#pragma unroll
  for (int i = 1; i < kRowWarps; ++i) mx = fmaxf(mx, s_max[i]);
  const float d = m == mx ? 0.f : fmaxf(m - mx, -200.f), f = exp2f(d);
  if (kEntropy) e = block_sum(f * fmaf(d, s, e), s_f);
  s = block_sum(s * f, s_f);
  if (tid != 0) return;
  const float y = fmaf(s_exact, R.scale2, -mx);
  const float was = fmaf(R.entry_logit[row], R.scale2, -mx);
  const float p = exp2f(y), p_was = exp2f(was);
  s += p - p_was;
  const float log2_s = log2f(s);
  R.loss[t] = (y - log2_s) * kLn2;
  if (R.lse != nullptr) R.lse[t] = fmaf(mx, kLn2, log2_s * kLn2);
  if (kEntropy) {
    e += (p > 0.f ? p * y : p) - (p_was > 0.f ? p_was * was : p_was);
    R.entropy[t] = (log2_s - e / s) * kLn2;
  }
}

// What the gradient of a logit is formed from, for upstream gradients r of a token's log
// probability and h of its entropy H, a the logit scale:
//   g_j = a ( r [j = y] - q (r + h H + h ln 2 log2 q) )
// row_q = (coefficient of q, log2 of the softmax denominator), row_b = that of q log2 q,
// entry_g = g at the target.  All of them lack the fraction of the first token's a r, which
// is every token's where all share one coefficient: in bf16 it would be rounded with every
// r (1 - q) of a q near 0 in the same way (see finalise_kernel; Ctrl::rest).
//
// A warp a token.  With a forward pass that kept its logits nothing else comes before the
// products, and this pass also clears the rows of dX of the tokens that do not count.
__global__ void __launch_bounds__(kRowThreads) logprob_grad_kernel(const RowParams R) {
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  const int row = blockIdx.x * kRowWarps + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  int n_valid = R.kept != nullptr ? R.kept->n_valid : R.ctrl->n_valid;
  if (R.kept != nullptr) {
    // nothing kept, or of another call (other sizes, another scale, a knob turned in
    // between): no gradient, and a status
    const Kept a = R.kept->kept, b = R.keeps;
    const bool other = a.tokens != b.tokens || a.dim != b.dim || a.vocab != b.vocab || a.packed != b.packed ||
                       a.piece_tiles != b.piece_tiles || a.stored != b.stored || !(a.scale2 == b.scale2);
    if (other) n_valid = 0;
    if (row == 0 && lane == 0) {
      R.ctrl->n_valid = n_valid;
      R.ctrl->status = other ? -1 : R.kept->status;
    }
    if (R.dx != nullptr && row < R.tokens && (other || !in_vocab(R, R.ids_in[row]))) {
      const long long at = static_cast<long long>(row) * R.ld_dx;
      for (int c = lane; c < R.dim; c += 32) {
        if (R.dx_fp32) static_cast<float*>(R.dx)[at + c] = 0.f;
        else static_cast<__nv_bfloat16*>(R.dx)[at + c] = __float2bfloat16_rn(0.f);
      }
    }
  }
  if (lane != 0) return;
  if (n_valid == 0 && row == 0) R.ctrl->rest = 1.0f;
  if (row >= n_valid) return;
  const int first = R.row_of[0], t = R.row_of[row];
  float power;
  const float r0 = R.g_logprob != nullptr ? R.g_logprob[first] : 0.f;
  const float rest = fraction_of((r0 != 0.f ? r0 : R.g_entropy != nullptr ? R.g_entropy[first] : 0.f) * R.logit_scale, power);
  if (row == 0) R.ctrl->rest = rest;
  const float scale = R.logit_scale / rest;
  const float r = R.g_logprob != nullptr ? R.g_logprob[t] * scale : 0.f, h = R.g_entropy != nullptr ? R.g_entropy[t] * scale : 0.f;
  const float entropy = R.g_entropy != nullptr ? R.entropy_in[t] : 0.f;
  const float log_q = R.logprob_in[t], q = expf(log_q);
  R.row_q[row] = make_float2(-fmaf(h, entropy, r), R.lse_in[t] * (1.0f / kLn2));
  R.row_b[row] = -h * kLn2;
  R.entry_g[row] = r * -expm1f(log_q) - (q > 0.f ? h * q * (log_q + entropy) : 0.f);
}

// The first piece's codes into gradients; the others' are converted beside the products.
__global__ void __launch_bounds__(kRowThreads) convert_log_kernel(const RowParams R, const ConvertParams C) {
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  convert_piece<true>(C, R.ctrl->n_valid, R.tokens, static_cast<int>(blockIdx.x) * kRowWarps + (threadIdx.x >> 5),
                      static_cast<int>(gridDim.x) * kRowWarps, threadIdx.x & 31);
}

// dX of the tokens that count, in token order: the partial sums joined, always in the
// same order.  Four columns a thread, or, kWays > 1, kWays neighbouring lanes that
// take a stretch of the runs each: with the many runs of a small launch one memory
// latency instead of several (13 us -> 3 for 60 x 512 x 50000).  (Rows of dX written by
// the last product's epilogue itself, 64 bytes at a time and to scattered tokens,
// cost that launch 120 us at 8192 x 2048; this pass costs 28.)
template <int kWays>
__global__ void __launch_bounds__(kRowThreads) dx_kernel(const RowParams R) {
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  const int per_row = (R.dim + 3) >> 2;
  const long long thread = static_cast<long long>(blockIdx.x) * kRowThreads + threadIdx.x;
  // lanes 0..31/kWays - 1 of a warp hold neighbouring columns, the next as many the next way
  constexpr int kGroups = 32 / kWays;
  const int lane = threadIdx.x & 31;
  const long long i = (thread >> 5) * kGroups + lane % kGroups;
  const int way = lane / kGroups;
  const int row = static_cast<int>(i / per_row);
  const bool mine = row < (R.in_place ? R.tokens : R.ctrl->n_valid);
  const int c = static_cast<int>(i - static_cast<long long>(row) * per_row) * 4;
  float v[4] = {};
  int t = 0;
  if (mine) {
    t = R.row_of[row];
    const int s0 = R.splits * way / kWays, s1 = R.splits * (way + 1) / kWays;
    const float* src = R.part + static_cast<long long>(row) * R.part_ld + c + s0 * R.part_stride;
#pragma unroll 8
    for (int s = s0; s < s1; ++s, src += R.part_stride) {
      const float4 a = *reinterpret_cast<const float4*>(src);
      v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w;
    }
  }
  const float rest = R.ctrl->rest;
#pragma unroll
  for (int o = kGroups; o < 32; o <<= 1)
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] += __shfl_xor_sync(0xFFFFFFFFu, v[e], o);
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] *= rest;
  if (!mine || way != 0) return;
  if (t < 0) {  // a masked token among rows that are tokens: 0 whatever w holds
    t = row;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = 0.f;
  }
  const long long off = static_cast<long long>(t) * R.ld_dx + c;
  const bool whole = R.dx_vec && c + 4 <= R.dim;
  if (R.dx_fp32) {
    float* d = static_cast<float*>(R.dx) + off;
    if (whole) {
      *reinterpret_cast<float4*>(d) = make_float4(v[0], v[1], v[2], v[3]);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (c + e < R.dim) d[e] = v[e];
    }
  } else {
    __nv_bfloat16* d = static_cast<__nv_bfloat16*>(R.dx) + off;
    if (whole) {
      __nv_bfloat162 h[2] = {__floats2bfloat162_rn(v[0], v[1]), __floats2bfloat162_rn(v[2], v[3])};
      *reinterpret_cast<uint2*>(d) = *reinterpret_cast<const uint2*>(h);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (c + e < R.dim) d[e] = __float2bfloat16_rn(v[e]);
    }
  }
}

template <typename... Args>
cudaError_t launch_of(int threads, void (*kernel)(Args...), dim3 blocks, bool overlap, cudaStream_t stream, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = blocks;
  cfg.blockDim = dim3(static_cast<unsigned>(threads), 1, 1);
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = overlap ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <typename... Args>
cudaError_t launch(void (*kernel)(Args...), dim3 blocks, bool overlap, cudaStream_t stream, Args... args) {
  return launch_of(kRowThreads, kernel, blocks, overlap, stream, args...);
}

unsigned row_blocks(int tokens) { return tokens > 0 ? static_cast<unsigned>((tokens + kRowWarps - 1) / kRowWarps) : 1u; }

}  // namespace

cudaError_t launch_flags(const RowParams& R, cudaStream_t stream) {
  return launch(flags_kernel, dim3(row_blocks(R.tokens)), false, stream, R);
}

cudaError_t launch_count(const RowParams& R, bool overlap, cudaStream_t stream) {
  return launch(R.z != nullptr ? count_kernel<true> : count_kernel<false>,
                dim3(static_cast<unsigned>((R.tokens + kRowThreads - 1) / kRowThreads)), overlap, stream, R);
}

cudaError_t launch_prepare(const RowParams& R, bool overlap, cudaStream_t stream) {
  return launch(R.z != nullptr ? prepare_kernel<true> : prepare_kernel<false>, dim3(row_blocks(R.tokens) + static_cast<unsigned>(R.pack_blocks)),
                overlap, stream, R);
}

// Few rows: large blocks, several a row, to spread the conversion over the device.  More
// rows: small blocks, so that a thousand are in flight (40 us in place of 85 for 8192 rows
// without codes).  A conversion in a launch of its own is no faster at any size tried (375
// us in place of 374 at 1777 x 1792 x 32003, 11.13 ms in place of 11.10 at 8192 x 2048 x
// 163840) and slower at 500 x 1024 x 13000 (66 in place of 64).
template <int kThreads, bool kConvert, bool kInPlace, int kFusedTiles>
cudaError_t finalise_with(const RowParams& R, const ConvertParams& C, dim3 grid, cudaStream_t stream) {
  return launch_of(kThreads, R.z != nullptr ? finalise_kernel<true, kConvert, kThreads, kInPlace, kFusedTiles>
                                            : finalise_kernel<false, kConvert, kThreads, kInPlace, kFusedTiles>,
                   grid, true, stream, R, C);
}

cudaError_t launch_finalise(const RowParams& R, const ConvertParams& C, int sms, cudaStream_t stream) {
  const int rows = R.tokens > 0 ? R.tokens : 1;
  if (C.g != nullptr && R.tokens < kFusedRows) {
    // blocks for three on every SM
    const int runs = (C.tiles + 1) / 2;
    const int most = (runs + kRowWarps - 1) / kRowWarps, want = (3 * sms + rows - 1) / rows;
    const dim3 grid(static_cast<unsigned>(rows), static_cast<unsigned>(want < most ? want : most));
    return R.in_place ? finalise_with<256, true, true, 2>(R, C, grid, stream)
                      : finalise_with<256, true, false, 2>(R, C, grid, stream);
  }
  const dim3 grid(static_cast<unsigned>(rows));
  if (R.in_place) return finalise_with<256, false, true, 2>(R, C, grid, stream);
  return C.g != nullptr ? finalise_with<128, true, false, 4>(R, C, grid, stream)
                        : finalise_with<128, false, false, 2>(R, C, grid, stream);
}

cudaError_t launch_logprob(const RowParams& R, cudaStream_t stream) {
  const dim3 grid(static_cast<unsigned>(R.tokens));
  if (R.in_place) return launch(R.entropy != nullptr ? logprob_kernel<true, true> : logprob_kernel<true, false>, grid, true, stream, R);
  return launch(R.entropy != nullptr ? logprob_kernel<false, true> : logprob_kernel<false, false>, grid, true, stream, R);
}

cudaError_t launch_logprob_grad(const RowParams& R, cudaStream_t stream) {
  return launch(logprob_grad_kernel, dim3(row_blocks(R.tokens)), R.kept == nullptr, stream, R);
}

cudaError_t launch_convert_log(const RowParams& R, const ConvertParams& C, int sms, cudaStream_t stream) {
  const long long tasks = static_cast<long long>(R.tokens) * ((C.tiles + kConvertTiles - 1) / kConvertTiles);
  const long long most = 4ll * sms, want = (tasks + kRowWarps - 1) / kRowWarps;
  return launch(convert_log_kernel, dim3(static_cast<unsigned>(want < 1 ? 1 : want < most ? want : most)), true, stream, R, C);
}

cudaError_t launch_dx(const RowParams& R, cudaStream_t stream) {
  const int ways = R.splits >= 8 ? 8 : 1;
  const long long n = static_cast<long long>(R.tokens) * ((R.dim + 3) >> 2) * ways;
  const dim3 grid(static_cast<unsigned>((n + kRowThreads - 1) / kRowThreads));
  return launch(ways == 8 ? dx_kernel<8> : dx_kernel<1>, grid, true, stream, R);
}

cudaError_t launch_pack(const RowParams& R, cudaStream_t stream) {
  return launch(pack_kernel, dim3(static_cast<unsigned>(R.pack_blocks)), false, stream, R);
}

int pack_blocks(int vocab) {
  const int blocks = (vocab + kRowWarps - 1) / kRowWarps;
  return blocks < 4096 ? blocks : 4096;
}

}  // namespace head
}  // namespace muon
