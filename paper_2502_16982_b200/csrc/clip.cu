// Global gradient norm over many tensors, and clipping by it:
//   S = sum over tensors and elements of g^2,  norm = sqrt(S)
//   coef = min(1, max_norm / (norm + eps)),    g <- coef * g
// Two streaming kernels.  The norm reads every gradient once, the scaling reads and
// writes it once more and does nothing where coef is 1; muon_adamw_step_clipped
// multiplies by coef as it reads and needs no scaling pass.
//
// All tensors of a launch are cut into chunks of 32 KiB on 16-byte boundaries of
// their addresses, and a block finds a chunk's tensor by bisection of the chunk counts, so
// that many small tensors and a few large ones fill the device alike.  The descriptors travel as kernel parameters: nothing is
// allocated or copied.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstdio>

#include "../../include/muon.h"
#include "ptx.cuh"

namespace muon {
void set_last_error(const char* msg);
}

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kVectors = 8;  // 16-byte loads a thread has in flight
constexpr int kChunkVectors = kThreads * kVectors;

constexpr int kCtasPerSm = 6;
constexpr int kMaxBlocks = MUON_GRAD_NORM_WORKSPACE_BYTES / 8;  // partial sums
constexpr int kMaxTensors = 1024;  // of one launch: 28 bytes each, of 32764 bytes of parameters
constexpr int kSomeTensors = 384;
constexpr int kFewTensors = 64;    // fewer parameters take less time to pass

template <int kMost>
struct Tensors {
  const void* g[kMost];
  void* out[kMost];
  long long numel[kMost];
  unsigned chunks_to[kMost];  // chunks of this tensor and of those before it
  unsigned g_fp32[(kMost + 31) / 32], out_fp32[(kMost + 31) / 32];
  int count;
};

template <int kMost>
__device__ __forceinline__ bool bit(const unsigned (&mask)[kMost], int i) { return (mask[i >> 5] >> (i & 31)) & 1u; }

// One chunk of a tensor in units of 16-byte vectors from the aligned address at or
// below its start: elements [lo, hi) of the tensor's own, `shift` before element 0.
struct Chunk {
  int tensor;
  long long first;  // first vector
};

template <int kMost>
__device__ __forceinline__ Chunk find_chunk(const Tensors<kMost>& T, unsigned chunk) {
  int lo = 0, hi = T.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (T.chunks_to[mid] > chunk) hi = mid;
    else lo = mid + 1;
  }
  const unsigned before = lo > 0 ? T.chunks_to[lo - 1] : 0u;
  return Chunk{lo, static_cast<long long>(chunk - before) * kChunkVectors};
}

// Elements of a vector of one tensor: `at` is the index of the vector's first one, which
// lies below 0 or past the end at the tensor's edges.
template <typename Word>
struct Cells;
template <>
struct Cells<float> {
  static constexpr int kEach = 4;
  static __device__ __forceinline__ float value(const uint4& v, int e) {
    return __uint_as_float(e == 0 ? v.x : e == 1 ? v.y : e == 2 ? v.z : v.w);
  }
};
template <>
struct Cells<__nv_bfloat16> {
  static constexpr int kEach = 8;
  static __device__ __forceinline__ float value(const uint4& v, int e) {
    const uint32_t w = e < 2 ? v.x : e < 4 ? v.y : e < 6 ? v.z : v.w;
    return __uint_as_float(e & 1 ? w & 0xFFFF0000u : w << 16);
  }
};

// The thread's vectors of a chunk; what lies outside the tensor reads 0.  kReadOnly: nothing of
// the launch writes to the tensor (the path for such data must not be taken otherwise).
template <bool kReadOnly, typename T>
__device__ __forceinline__ void load_chunk(const T* g, long long numel, long long first, uint4 (&v)[kVectors]) {
  constexpr int kEach = Cells<T>::kEach;
  const int shift = static_cast<int>((reinterpret_cast<uintptr_t>(g) & 15) / sizeof(T));
#pragma unroll
  for (int i = 0; i < kVectors; ++i) {
    const long long at = (first + i * kThreads + threadIdx.x) * kEach - shift;
    v[i] = make_uint4(0u, 0u, 0u, 0u);
    if (at >= 0 && at + kEach <= numel) {
      const uint4* src = reinterpret_cast<const uint4*>(g + at);
      v[i] = kReadOnly ? __ldg(src) : *src;
    } else if (at < numel && at + kEach > 0) {
      uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
      for (int e = 0; e < kEach; ++e)
        if (at + e >= 0 && at + e < numel) {
          if constexpr (kEach == 4) w[e] = __float_as_uint(g[at + e]);
          else w[e >> 1] |= static_cast<uint32_t>(__bfloat16_as_ushort(g[at + e])) << (16 * (e & 1));
        }
      v[i] = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
}

// Squares of one chunk added up in fp32, at most 64 a thread, which the caller adds in
// fp64.  Where that sum leaves the range in which no square overflows or vanishes, the
// squares are formed again in fp64.
template <typename T>
__device__ __forceinline__ double chunk_squares(const uint4 (&v)[kVectors]) {
  constexpr int kEach = Cells<T>::kEach;
  float s[2] = {0.f, 0.f};
#pragma unroll
  for (int i = 0; i < kVectors; ++i)
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const float x = Cells<T>::value(v[i], e);
      s[e & 1] = fmaf(x, x, s[e & 1]);
    }
  const float sum = s[0] + s[1];
  if (sum >= 1e-24f && sum <= 1e38f) return static_cast<double>(sum);
  double d = 0.0;
#pragma unroll
  for (int i = 0; i < kVectors; ++i) {
    const uint4 u = v[i];
    if ((u.x | u.y | u.z | u.w) != 0u) {
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const double x = static_cast<double>(Cells<T>::value(u, e));
        d = fma(x, x, d);
      }
    }
  }
  return d;
}

// Sum over a block in a fixed order; thread 0 gets it.
__device__ __forceinline__ double block_sum(double sum) {
  __shared__ double s_sum[kWarps];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
  if ((threadIdx.x & 31) == 0) s_sum[threadIdx.x >> 5] = sum;
  __syncthreads();
  double t = s_sum[0];
  for (int i = 1; i < kWarps; ++i) t += s_sum[i];
  return t;
}

// A thread's squares of every gridDim.x-th chunk.
template <int kMost>
__device__ __forceinline__ double thread_squares(const Tensors<kMost>& T) {
  const unsigned chunks = T.count > 0 ? T.chunks_to[T.count - 1] : 0u;
  double sum = 0.0;
  for (unsigned c = blockIdx.x; c < chunks; c += gridDim.x) {
    const Chunk k = find_chunk(T, c);
    uint4 v[kVectors];
    if (bit(T.g_fp32, k.tensor)) {
      load_chunk<true>(static_cast<const float*>(T.g[k.tensor]), T.numel[k.tensor], k.first, v);
      sum += chunk_squares<float>(v);
    } else {
      load_chunk<true>(static_cast<const __nv_bfloat16*>(T.g[k.tensor]), T.numel[k.tensor], k.first, v);
      sum += chunk_squares<__nv_bfloat16>(v);
    }
  }
  return sum;
}

// One partial sum a block; blocks_before: partial sums that earlier launches of the call left.
template <int kMost>
__global__ void __launch_bounds__(kThreads) norm_kernel(const __grid_constant__ Tensors<kMost> T, double* partials,
                                                        int blocks_before) {
  const double sum = thread_squares(T);
  muon::ptx::grid_launch_dependents();
  double t = block_sum(sum);
  if (threadIdx.x == 0) {
    if (static_cast<int>(blockIdx.x) < blocks_before) t += partials[blockIdx.x];
    partials[blockIdx.x] = t;
  }
}

// NaN where the norm is not finite: nothing is clipped by it, and the steps that are given
// it leave everything as it is.
__device__ __forceinline__ float coefficient(double norm, double max_norm, double eps) {
  if (!isfinite(norm)) return __uint_as_float(0x7FC00000u);
  const double c = max_norm / (norm + eps);
  return c < 1.0 ? static_cast<float>(c) : 1.0f;  // 0 / 0 is no reason to clip
}

__device__ __forceinline__ void write_results(double sum, float max_norm, float eps, float* norm, float* coef) {
  const double n = sqrt(sum);
  if (norm != nullptr) *norm = static_cast<float>(n);
  if (coef != nullptr) *coef = coefficient(n, max_norm, eps);
}

__global__ void __launch_bounds__(kThreads) join_kernel(const double* partials, int count, float max_norm, float eps,
                                                        double* sum_sq, float* norm, float* coef) {
  muon::ptx::grid_dependency_wait();
  double sum = 0.0;
  for (int i = threadIdx.x; i < count; i += kThreads) sum += __ldcg(partials + i);
  const double t = block_sum(sum);
  if (threadIdx.x == 0) {
    if (sum_sq != nullptr) *sum_sq = t;
    write_results(t, max_norm, eps, norm, coef);
  }
}

// Both in one launch, for few chunks: one cluster, whose first block adds up the others' sums.
// (3 x 1408 + 65536 elements fp32: 3.4 us on the device either way, a call 4.5 us of the host's time, two
// launches 6.8.)
constexpr int kClusterBlocks = 8;
constexpr unsigned kClusterChunks = 64;
__global__ void __launch_bounds__(kThreads) norm_cluster_kernel(const __grid_constant__ Tensors<kFewTensors> T, float max_norm, float eps,
                                                                double* sum_sq, float* norm, float* coef) {
  __shared__ double s_all;
  const double mine = block_sum(thread_squares(T));
  if (threadIdx.x == 0) s_all = mine;
  muon::ptx::cluster_sync_all();
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    double t = mine;
    for (int r = 1; r < kClusterBlocks; ++r) {
      double theirs;
      asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(theirs) : "r"(muon::ptx::map_to_cta(muon::ptx::smem_u32(&s_all), r)));
      t += theirs;
    }
    if (sum_sq != nullptr) *sum_sq = t;
    write_results(t, max_norm, eps, norm, coef);
  }
  muon::ptx::cluster_sync_all();  // sums stay until they are read
}

template <typename T, typename Out>
__device__ __forceinline__ void scale_chunk(const T* g, Out* out, long long numel, long long first, float coef) {
  constexpr int kEach = Cells<T>::kEach;
  uint4 v[kVectors];
  load_chunk<false>(g, numel, first, v);
  const int shift = static_cast<int>((reinterpret_cast<uintptr_t>(g) & 15) / sizeof(T));
#pragma unroll
  for (int i = 0; i < kVectors; ++i) {
    const long long at = (first + i * kThreads + threadIdx.x) * kEach - shift;
    if (at >= numel || at + kEach <= 0) continue;
    constexpr int kOutBytes = kEach * static_cast<int>(sizeof(Out));
    const bool whole = at >= 0 && at + kEach <= numel && (reinterpret_cast<uintptr_t>(out + at) & (kOutBytes < 16 ? kOutBytes - 1 : 15)) == 0;
    if (whole) {
      uint32_t w[kOutBytes / 4];
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const float y = Cells<T>::value(v[i], e) * coef;
        if constexpr (sizeof(Out) == 4) {
          w[e] = __float_as_uint(y);
        } else {
          const uint32_t b = __bfloat16_as_ushort(__float2bfloat16_rn(y));
          w[e >> 1] = e & 1 ? w[e >> 1] | (b << 16) : b;
        }
      }
#pragma unroll
      for (int p = 0; p < kOutBytes / 16; ++p)
        __stcs(reinterpret_cast<uint4*>(out + at) + p, make_uint4(w[4 * p], w[4 * p + 1], w[4 * p + 2], w[4 * p + 3]));
      if constexpr (kOutBytes == 8) __stcs(reinterpret_cast<uint2*>(out + at), make_uint2(w[0], w[1]));
    } else {
#pragma unroll
      for (int e = 0; e < kEach; ++e)
        if (at + e >= 0 && at + e < numel) {
          const float y = Cells<T>::value(v[i], e) * coef;
          if constexpr (sizeof(Out) == 4) out[at + e] = y;
          else out[at + e] = __float2bfloat16_rn(y);
        }
    }
  }
}

// sum_sq: of all gradients that count for the norm, perhaps of several ranks.  One chunk a
// block, the last first: what the norm read last is still in L2.  (198 x 2883584 bf16 into
// other buffers: 334 us; with blocks that take every gridDim.x-th chunk, 6 an SM, 399.)
template <int kMost>
__global__ void __launch_bounds__(kThreads) scale_kernel(const __grid_constant__ Tensors<kMost> T, const double* sum_sq,
                                                         float max_norm, float eps, float* norm, float* coef_out) {
  __shared__ float s_coef;
  if (threadIdx.x == 0) {
    const double sum = *sum_sq;
    s_coef = coefficient(sqrt(sum), max_norm, eps);
    if (blockIdx.x == 0) write_results(sum, max_norm, eps, norm, coef_out);
  }
  __syncthreads();
  const float coef = s_coef == s_coef ? s_coef : 1.0f;
  const unsigned chunks = T.count > 0 ? T.chunks_to[T.count - 1] : 0u;
  if (blockIdx.x < chunks) {
    const Chunk k = find_chunk(T, chunks - 1 - blockIdx.x);
    const void* g = T.g[k.tensor];
    void* out = T.out[k.tensor];
    if (coef == 1.0f && out == g) return;
    const long long n = T.numel[k.tensor];
    const bool from32 = bit(T.g_fp32, k.tensor), to32 = bit(T.out_fp32, k.tensor);
    if (from32 && to32) scale_chunk(static_cast<const float*>(g), static_cast<float*>(out), n, k.first, coef);
    else if (from32) scale_chunk(static_cast<const float*>(g), static_cast<__nv_bfloat16*>(out), n, k.first, coef);
    else if (to32) scale_chunk(static_cast<const __nv_bfloat16*>(g), static_cast<float*>(out), n, k.first, coef);
    else scale_chunk(static_cast<const __nv_bfloat16*>(g), static_cast<__nv_bfloat16*>(out), n, k.first, coef);
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

#define CLIP_CUDA(call)                                                            \
  do {                                                                             \
    cudaError_t e_ = (call);                                                       \
    if (e_ != cudaSuccess) return fail(MUON_ERR_CUDA, cudaGetErrorString(e_));     \
  } while (0)

bool misaligned(const void* p, unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }
unsigned size_of(int dtype) { return dtype == MUON_DTYPE_FP32 ? 4u : 2u; }
bool known(int dtype) { return dtype == MUON_DTYPE_FP32 || dtype == MUON_DTYPE_BF16; }

int check(const muon_grad_tensor* t, int n, bool writes) {
  if (n < 0 || (n > 0 && !t)) return fail(MUON_ERR_INVALID_ARG, "tensors is null or n_tensors is negative");
  for (int i = 0; i < n; ++i) {
    if (t[i].numel < 0) return fail(MUON_ERR_INVALID_ARG, "numel is negative");
    if (t[i].numel >= (1ll << 42)) return fail(MUON_ERR_UNSUPPORTED, "2^42 elements or more in one tensor");
    if (!known(t[i].g_dtype) || (writes && t[i].out && !known(t[i].out_dtype)))
      return fail(MUON_ERR_UNSUPPORTED, "dtype must be bf16 or fp32");
    if (t[i].numel > 0 && !t[i].g) return fail(MUON_ERR_INVALID_ARG, "null gradient");
    if (misaligned(t[i].g, size_of(t[i].g_dtype)) || (writes && t[i].out && misaligned(t[i].out, size_of(t[i].out_dtype))))
      return fail(MUON_ERR_ALIGNMENT, "pointer not aligned to its element size");
    if (writes && t[i].numel > 0 && t[i].out == t[i].g && t[i].out_dtype != t[i].g_dtype)
      return fail(MUON_ERR_INVALID_ARG, "in place with another dtype");
  }
  return MUON_OK;
}

int check_limits(float max_norm, float eps) {
  if (!(max_norm >= 0.f)) return fail(MUON_ERR_INVALID_ARG, "max_norm must not be negative or NaN");
  if (!(eps >= 0.f) || !std::isfinite(eps)) return fail(MUON_ERR_INVALID_ARG, "eps must be finite and not negative");
  return MUON_OK;
}

// Descriptors of up to kMost tensors from t[first] on; returns how many of t were taken.
// Tensors without elements take no place.
template <int kMost>
int fill(const muon_grad_tensor* t, int first, int n, Tensors<kMost>* T) {
  int i = first;
  unsigned chunks = 0;
  T->count = 0;
  for (unsigned& m : T->g_fp32) m = 0;
  for (unsigned& m : T->out_fp32) m = 0;
  for (; i < n && T->count < kMost; ++i) {
    if (t[i].numel == 0) continue;
    const int k = T->count;
    const long long each = 16 / size_of(t[i].g_dtype);
    const long long shift = static_cast<long long>((reinterpret_cast<uintptr_t>(t[i].g) & 15) / size_of(t[i].g_dtype));
    const long long more = (t[i].numel + shift + each * kChunkVectors - 1) / (each * kChunkVectors);
    if (chunks + more > 0x7FFFFFFFll) break;  // chunk numbers are 32 bits; one tensor has fewer than 2^31
    T->g[k] = t[i].g;
    T->out[k] = t[i].out ? t[i].out : const_cast<void*>(t[i].g);
    T->numel[k] = t[i].numel;
    const bool out32 = (t[i].out ? t[i].out_dtype : t[i].g_dtype) == MUON_DTYPE_FP32;
    T->g_fp32[k >> 5] |= static_cast<unsigned>(t[i].g_dtype == MUON_DTYPE_FP32) << (k & 31);
    T->out_fp32[k >> 5] |= static_cast<unsigned>(out32) << (k & 31);
    chunks += static_cast<unsigned>(more);
    T->chunks_to[k] = chunks;
    T->count = k + 1;
  }
  return i - first;
}

int blocks_for(unsigned chunks, int sms) {
  const int most = sms * kCtasPerSm < kMaxBlocks ? sms * kCtasPerSm : kMaxBlocks;
  return chunks < static_cast<unsigned>(most) ? static_cast<int>(chunks) : most;
}

// Launches `each` over all tensors, up to kMost in one launch.
template <int kMost, typename Launch>
int for_launches(const muon_grad_tensor* t, int n, Launch each) {
  for (int first = 0; first < n;) {
    Tensors<kMost> T;
    first += fill(t, first, n, &T);
    if (T.count == 0) continue;
    each(T);
    CLIP_CUDA(cudaGetLastError());
  }
  return MUON_OK;
}

template <typename Launch>
int for_all(const muon_grad_tensor* t, int n, Launch each) {
  return n <= kFewTensors ? for_launches<kFewTensors>(t, n, each)
         : n <= kSomeTensors ? for_launches<kSomeTensors>(t, n, each) : for_launches<kMaxTensors>(t, n, each);
}

}  // namespace

extern "C" int muon_grad_norm(const muon_grad_tensor* tensors, int n_tensors, float max_norm, float eps, double* sum_sq,
                              float* norm, float* coef, void* workspace, size_t workspace_bytes, int device, void* stream_v) {
  int rc = check(tensors, n_tensors, false);
  if (rc == MUON_OK) rc = check_limits(max_norm, eps);
  if (rc != MUON_OK) return rc;
  if (!sum_sq && !norm && !coef) return fail(MUON_ERR_INVALID_ARG, "no output wanted");
  if (misaligned(sum_sq, 8) || misaligned(norm, 4) || misaligned(coef, 4))
    return fail(MUON_ERR_ALIGNMENT, "pointer not aligned to its element size");
  if (!workspace || workspace_bytes < MUON_GRAD_NORM_WORKSPACE_BYTES || misaligned(workspace, 8))
    return fail(MUON_ERR_WORKSPACE, "workspace: MUON_GRAD_NORM_WORKSPACE_BYTES, 8-byte aligned");
  DeviceGuard guard;
  CLIP_CUDA(guard.set(device));
  int sms = 0;
  CLIP_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device));
  cudaStream_t stream = static_cast<cudaStream_t>(stream_v);
  double* partials = static_cast<double*>(workspace);
  if (n_tensors <= kFewTensors) {
    Tensors<kFewTensors> T;
    if (fill(tensors, 0, n_tensors, &T) == n_tensors && (T.count == 0 || T.chunks_to[T.count - 1] <= kClusterChunks)) {
      cudaLaunchConfig_t cfg = {};
      cfg.gridDim = dim3(kClusterBlocks);
      cfg.blockDim = dim3(kThreads);
      cfg.stream = stream;
      cudaLaunchAttribute attr;
      attr.id = cudaLaunchAttributeClusterDimension;
      attr.val.clusterDim.x = kClusterBlocks;
      attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
      cfg.attrs = &attr;
      cfg.numAttrs = 1;
      CLIP_CUDA(cudaLaunchKernelEx(&cfg, norm_cluster_kernel, T, max_norm, eps, sum_sq, norm, coef));
      return MUON_OK;
    }
  }
  int blocks = 0;  // partial sums so far
  auto launch = [&](const auto& T) {
    const int b = blocks_for(T.chunks_to[T.count - 1], sms);
    norm_kernel<<<b, kThreads, 0, stream>>>(T, partials, blocks);
    blocks = b > blocks ? b : blocks;
  };
  rc = for_all(tensors, n_tensors, launch);
  if (rc != MUON_OK) return rc;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(1);
  cfg.blockDim = dim3(kThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = blocks > 0 ? 1 : 0;
  CLIP_CUDA(cudaLaunchKernelEx(&cfg, join_kernel, static_cast<const double*>(partials), blocks, max_norm, eps, sum_sq, norm, coef));
  return MUON_OK;
}

extern "C" int muon_clip_grads(const muon_grad_tensor* tensors, int n_tensors, const double* sum_sq, float max_norm, float eps,
                               float* norm, float* coef, int device, void* stream_v) {
  int rc = check(tensors, n_tensors, true);
  if (rc == MUON_OK) rc = check_limits(max_norm, eps);
  if (rc != MUON_OK) return rc;
  if (!sum_sq) return fail(MUON_ERR_INVALID_ARG, "sum_sq is null");
  if (misaligned(sum_sq, 8) || misaligned(norm, 4) || misaligned(coef, 4))
    return fail(MUON_ERR_ALIGNMENT, "pointer not aligned to its element size");
  DeviceGuard guard;
  CLIP_CUDA(guard.set(device));
  cudaStream_t stream = static_cast<cudaStream_t>(stream_v);
  bool wrote = false;  // norm and coef
  auto launch = [&](const auto& T) {
    scale_kernel<<<T.chunks_to[T.count - 1], kThreads, 0, stream>>>(T, sum_sq, max_norm, eps, wrote ? nullptr : norm,
                                                                                    wrote ? nullptr : coef);
    wrote = true;
  };
  rc = for_all(tensors, n_tensors, launch);
  if (rc != MUON_OK || wrote || (!norm && !coef)) return rc;
  Tensors<kFewTensors> none = {};
  scale_kernel<<<1, kThreads, 0, stream>>>(none, sum_sq, max_norm, eps, norm, coef);
  CLIP_CUDA(cudaGetLastError());
  return MUON_OK;
}
