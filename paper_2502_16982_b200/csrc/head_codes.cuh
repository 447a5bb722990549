// 16-bit codes of logits.  Where the workspace has room, the statistics pass keeps
// every logit as its distance below the largest one of its row in the same 64
// columns, in steps of 2^-11 on the log2 scale: code = round((max - y) 2^11), capped at
// 65535, y = scale2 * logit.  Decoding gives q within 2^-12 ln 2 = 1.7e-4, a
// twentieth of the bf16 rounding of the gradient that follows; what lies 2^-32
// or more below its tile's largest becomes 0.  The maximum's product with scale2 is
// rounded upwards, so that max - y is never negative (with the nearest value, a
// largest logit of some thousands can lie above it, and its code would wrap to 65535).
// The gradient of the logits is then a pass over the codes instead of a second
// product x w^T.
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

#include "head.h"

namespace muon {
namespace head {

constexpr float kCodeSteps = 2048.0f;
constexpr float kCodeMagic = 8388608.0f;  // 2^23: the low mantissa bits hold an integer
constexpr uint32_t kCodeMax = 65535u;

__device__ __forceinline__ float ex2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// `steps` = (max - y) kCodeSteps + kCodeMagic, rounded to a whole number by the
// addition; the code is in the low 16 bits of the result.  max - y >= 0.
__device__ __forceinline__ uint32_t clamp_code(float steps) {
  return __float_as_uint(fminf(steps, kCodeMagic + 65535.0f));
}

// Codes of up to kTiles 256-column tiles of one row -> bf16 gradient of the
// logits, in place, by one warp (8 columns a lane and tile, so that a tile is one
// coalesced 512-byte access).  rq: the row's coefficient of q and log2 softmax
// denominator; ids, entry_g: its sparse entries, ascending.
// kTiles: independent loads in flight.
constexpr int kConvertTiles = 8;

template <int kTiles>
struct Codes {
  uint4 v[kTiles];
};

__device__ __forceinline__ uint4* code_cell(const ConvertParams& C, int row, int tile0, int lane) {
  return reinterpret_cast<uint4*>(C.g + static_cast<long long>(row) * C.ld + tile0 * kTileN) + lane;
}

template <int kTiles>
__device__ __forceinline__ void load_codes(const ConvertParams& C, int row, int tile0, int lane, Codes<kTiles>& c) {
  const int tiles = min(kTiles, C.tiles - tile0);
  const uint4* cell = code_cell(C, row, tile0, lane);
#pragma unroll
  for (int i = 0; i < kTiles; ++i)
    if (i < tiles) c.v[i] = __ldcs(cell + i * 32);
}

template <int kTiles>
__device__ __forceinline__ void convert_codes(const ConvertParams& C, int row, int tile0, float2 rq, const int* ids,
                                              const float* entry_g, int lane, const Codes<kTiles>& c) {
  const int tiles = min(kTiles, C.tiles - tile0);
  uint4* cell = code_cell(C, row, tile0, lane);
  // lane i: what the i-th kStatN columns of the run add to the exponent
  float shift = 0.f;
  static_assert(kTiles * kUnits <= 32, "one lane per statistics entry");
  if (lane < kUnits * tiles)
    shift = C.stats[static_cast<long long>(row) * C.stats_ld + kUnits * (C.v_tile0 + tile0) + lane].x - rq.y;
  int next = 0, end = 1;
  if (C.top > 1 && C.starts == nullptr) {  // the list lies in shared memory: count
    const int lo = (C.v_tile0 + tile0) * kTileN, hi = lo + tiles * kTileN;
    end = 0;
    for (int k = 0; k < C.top; k += 32) {
      const int id = k + lane < C.top ? ids[k + lane] : kNoId;
      next += __popc(__ballot_sync(0xFFFFFFFFu, id < lo));
      end += __popc(__ballot_sync(0xFFFFFFFFu, id < hi));
    }
  } else if (C.top > 1) {
    const unsigned char* s = C.starts + static_cast<long long>(row) * C.n_starts + C.v_tile0 + tile0;
    next = s[0];
    end = s[tiles];
  }
  int id = next < end ? ids[next] - (C.v_tile0 + tile0) * kTileN : kNoId;
  if (id < 0) id = kNoId;
#pragma unroll
  for (int i = 0; i < kTiles; ++i) {
    if (i < tiles) {
      const float a = __shfl_sync(0xFFFFFFFFu, shift, kUnits * i + lane * 8 / kStatN);
      uint32_t w[4] = {c.v[i].x, c.v[i].y, c.v[i].z, c.v[i].w};
      float g[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t lo = w[e] & 0xFFFFu, hi = w[e] >> 16;
        const float dl = __uint_as_float(lo | 0x4B000000u) - kCodeMagic, dh = __uint_as_float(hi | 0x4B000000u) - kCodeMagic;
        g[2 * e] = rq.x * (lo == kCodeMax ? 0.f : ex2_fast(fmaf(dl, -1.0f / kCodeSteps, a)));
        g[2 * e + 1] = rq.x * (hi == kCodeMax ? 0.f : ex2_fast(fmaf(dh, -1.0f / kCodeSteps, a)));
      }
      // sparse entries of this tile (all lanes see the same list)
      while (id < (i + 1) * kTileN) {
        const float eg = entry_g[next];
        const int at = id - i * kTileN;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (at == lane * 8 + e) g[e] = eg;
        ++next;
        id = next < end ? ids[next] - (C.v_tile0 + tile0) * kTileN : kNoId;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        __nv_bfloat162 h = __floats2bfloat162_rn(g[2 * e], g[2 * e + 1]);
        w[e] = *reinterpret_cast<uint32_t*>(&h);
      }
      cell[i * 32] = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
}

// The same for the gradient of log probabilities, q (rq.x + rb log2 q), from codes that stay
// as they are: a caller may ask for it again.  One entry a row: the target.
template <int kTiles>
__device__ __forceinline__ void convert_log(const ConvertParams& C, int row, int tile0, int lane) {
  const int tiles = min(kTiles, C.tiles - tile0);
  const long long at = static_cast<long long>(row) * C.ld + static_cast<long long>(tile0) * kTileN;
  const uint4* src = reinterpret_cast<const uint4*>(C.codes + at) + lane;
  uint4* dst = reinterpret_cast<uint4*>(C.g + at) + lane;
  uint4 v[kTiles];
#pragma unroll
  for (int i = 0; i < kTiles; ++i)
    if (i < tiles) v[i] = __ldcs(src + i * 32);
  const float2 rq = C.row_q[row];
  const float rb = C.row_b[row];
  float shift = 0.f;
  static_assert(kTiles * kUnits <= 32, "one lane per statistics entry");
  if (lane < kUnits * tiles)
    shift = C.stats[static_cast<long long>(row) * C.stats_ld + kUnits * (C.v_tile0 + tile0) + lane].x - rq.y;
  const int target = C.ids[row] - (C.v_tile0 + tile0) * kTileN - lane * 8;  // from this lane's first column
  const float target_g = C.entry_g[row];
#pragma unroll
  for (int i = 0; i < kTiles; ++i) {
    if (i < tiles) {
      const float a = __shfl_sync(0xFFFFFFFFu, shift, kUnits * i + lane * 8 / kStatN);
      uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t lo = w[e] & 0xFFFFu, hi = w[e] >> 16;
        const float yl = fmaf(__uint_as_float(lo | 0x4B000000u) - kCodeMagic, -1.0f / kCodeSteps, a);
        const float yh = fmaf(__uint_as_float(hi | 0x4B000000u) - kCodeMagic, -1.0f / kCodeSteps, a);
        float gl = lo == kCodeMax ? 0.f : ex2_fast(yl) * fmaf(yl, rb, rq.x);
        float gh = hi == kCodeMax ? 0.f : ex2_fast(yh) * fmaf(yh, rb, rq.x);
        if (target == i * kTileN + 2 * e) gl = target_g;
        if (target == i * kTileN + 2 * e + 1) gh = target_g;
        const __nv_bfloat162 h = __floats2bfloat162_rn(gl, gh);
        w[e] = *reinterpret_cast<const uint32_t*>(&h);
      }
      dst[i * 32] = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
}

// A row past the tokens that count becomes zeros.
template <int kTiles>
__device__ __forceinline__ void clear_row(const ConvertParams& C, int row, int tile0, int lane) {
  const int tiles = min(kTiles, C.tiles - tile0);
  uint4* cell = code_cell(C, row, tile0, lane);
  for (int i = 0; i < tiles; ++i) cell[i * 32] = make_uint4(0u, 0u, 0u, 0u);
}

// All rows of a piece, dealt out to `warps` warps.
template <bool kLog = false>
__device__ __forceinline__ void convert_piece(const ConvertParams& C, int n_valid, int tokens, int warp, int warps, int lane) {
  const int runs = (C.tiles + kConvertTiles - 1) / kConvertTiles;
  const int rows = min(tokens, (n_valid + kBK - 1) / kBK * kBK);  // dW's product reads whole K blocks of rows
  const long long tasks = static_cast<long long>(rows) * runs;
  for (long long t = warp; t < tasks; t += warps) {
    const int row = static_cast<int>(t / runs);
    const int tile0 = static_cast<int>(t - static_cast<long long>(row) * runs) * kConvertTiles;
    const long long at = static_cast<long long>(row) * C.top;
    if (kLog && row < n_valid) {
      convert_log<kConvertTiles>(C, row, tile0, lane);
    } else if (row < n_valid) {
      Codes<kConvertTiles> c;
      load_codes(C, row, tile0, lane, c);
      convert_codes(C, row, tile0, C.row_q[row], C.ids + at, C.entry_g + at, lane, c);
    } else {
      clear_row<kConvertTiles>(C, row, tile0, lane);
    }
  }
}

}  // namespace head
}  // namespace muon
