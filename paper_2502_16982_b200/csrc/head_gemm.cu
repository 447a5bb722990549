// Products of the LM-head losses for sm_100a.  With hidden states x [T, D], head
// w [V, D], logits l = a x w^T, q = softmax(l) and a sparse target distribution p:
//
//   statistics  max and sum of exponentials of every token over every 256
//               columns of l, and l at the sparse entries (logits stay in TMEM)
//   gradient    G = g a (c q - p) for one piece of the vocabulary, in bf16
//   outputs     dX += G w(piece)  and  dW(piece) = G^T x, one launch
//
// One persistent, warp-specialised kernel on CTA pairs (tcgen05.mma
// cta_group::2, M = 256, N = 128 or 256), three instantiations by epilogue.
//   warp 0     TMA producer: this CTA's 128 rows of A and its half of B per K
//              block, into a ring of kStages; no multicast
//   warp 1     leader CTA only: UMMA issuer, two TMEM accumulator stages
//   warps 2-5  epilogue: lane = row of the tile, so that a row's maximum and sum
//              stay in one thread's registers
//   warps 6-9  outputs only: turn the next piece's codes (head_codes.cuh) into the
//              gradient of its logits while the tensor cores work on this piece
//
// Every wait is bounded (ptx::mbar_wait); on expiry the CTA records
// MUON_ERR_TIMEOUT, all roles drain and the kernel returns.
#include <cuda_bf16.h>

#include "head_codes.cuh"
#include "ptx.cuh"

namespace muon {
namespace head {

namespace {

constexpr int kConvertWarps = 4;
constexpr int threads_of(int mode) { return mode == kModeOut ? 192 + 32 * kConvertWarps : 192; }
constexpr int kStages = 6;
constexpr int kTileABytes = 128 * kBK * 2;
constexpr int kTileBBytes = 128 * kBK * 2;
constexpr int kStageBytes = kTileABytes + kTileBBytes;
constexpr int kEpiWarps = 4;
constexpr int kNumAcc = 2;
constexpr int kAccCols = 256;
constexpr int kTmemCols = kNumAcc * kAccCols;

struct Barriers {
  unsigned long long full[kStages];    // leader's copy is the live one
  unsigned long long empty[kStages];
  unsigned long long acc_full[kNumAcc];
  unsigned long long acc_empty[kNumAcc];  // leader's copy is the live one
  uint32_t tmem_base;
  int abort_flag;
};

constexpr int kSmemBytes = 1024 + kStages * kStageBytes + 512;
static_assert(sizeof(Barriers) <= 512 && kSmemBytes <= 232448, "exceeds the 227 KiB shared-memory limit");

__device__ __forceinline__ void report_timeout(const GemmParams& P) { atomicExch(&P.ctrl->status, -6); }

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&h);
}

__device__ __forceinline__ void st_global_32(void* dst, const uint32_t (&v)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst), "r"(v[0]), "r"(v[1]), "r"(v[2]),
               "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}

__device__ __forceinline__ void ld_global_32(const void* src, uint32_t (&v)[8]) {
  asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
               : "l"(src));
}

// Sizes of product `i` that depend on how many tokens count.
struct Shape {
  int m_tiles, n_tiles, k_blocks, splits, tiles;
};

__device__ __forceinline__ Shape shape_of(const GemmParams& P, int i, int n_valid) {
  const Product& p = P.prod[i];
  Shape s;
  s.m_tiles = p.m_tiles < 0 ? (n_valid + kTileM - 1) / kTileM : p.m_tiles;
  s.k_blocks = p.k_blocks < 0 ? (n_valid + kBK - 1) / kBK : p.k_blocks;
  s.n_tiles = p.n_tiles;
  s.splits = p.splits;
  s.tiles = s.m_tiles * s.n_tiles * s.splits;
  return s;
}

// One tile: which product, which 256 rows and n_tile columns, which run of K blocks.
struct Tile {
  int prod, mi, ni, split, kb0, kb1;
};

// Row tiles are walked in groups of `group` for each column tile (or the columns
// innermost, swap_order), one split after the other, so that the CTA pairs that
// run at the same time share operand tiles in L2.
__device__ __forceinline__ Tile locate(const GemmParams& P, const Shape& s0, const Shape& s1, int t) {
  Tile r;
  r.prod = t < s0.tiles ? 0 : 1;
  if (r.prod) t -= s0.tiles;
  const Shape& s = r.prod ? s1 : s0;
  const Product& p = P.prod[r.prod];
  const int per_split = s.m_tiles * s.n_tiles;
  r.split = t / per_split;
  t -= r.split * per_split;
  if (p.swap_order) {
    r.mi = t / s.n_tiles;
    r.ni = t - r.mi * s.n_tiles;
  } else {
    const int per_group = p.group * s.n_tiles;
    const int grp = t / per_group;
    t -= grp * per_group;
    const int rows = min(p.group, s.m_tiles - grp * p.group);
    r.ni = t / rows;
    r.mi = grp * p.group + (t - r.ni * rows);
  }
  r.kb0 = static_cast<int>(static_cast<long long>(s.k_blocks) * r.split / s.splits);
  r.kb1 = static_cast<int>(static_cast<long long>(s.k_blocks) * (r.split + 1) / s.splits);
  return r;
}

// Picks v[i] for a run-time i without putting v in local memory.
__device__ __forceinline__ float pick(const uint32_t (&v)[32], int i) {
  uint32_t r = v[0];
#pragma unroll
  for (int j = 1; j < 32; ++j) r = i == j ? v[j] : r;
  return __uint_as_float(r);
}

// The sparse entries of one row that fall into one 256-column tile.
struct Entries {
  int next, end;  // positions in the row's list
  int col;        // column of entry `next` within the tile, or past every column
  const int* ids;

  __device__ __forceinline__ void open(const GemmParams& P, int row, int tile_col0, bool row_ok) {
    next = end = 0;
    ids = P.ids + static_cast<long long>(row) * P.top;
    if (row_ok) {
      if (P.top == 1) {
        end = 1;
      } else {
        const unsigned char* s = P.starts + static_cast<long long>(row) * P.n_starts + tile_col0 / kTileN;
        next = s[0];
        end = s[1];
      }
    }
    fetch(tile_col0);
  }
  __device__ __forceinline__ void fetch(int tile_col0) {
    col = next < end ? ids[next] - tile_col0 : kNoId;
    if (col < 0 || col >= kTileN) col = kNoId;
  }
};

template <int kMode>
__global__ void __launch_bounds__(threads_of(kMode), 1) head_gemm_kernel(const __grid_constant__ GemmParams P) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~static_cast<uintptr_t>(1023));
  Barriers* bars = reinterpret_cast<Barriers*>(ring + kStages * kStageBytes);

  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  const uint32_t rank = ptx::cluster_ctarank();  // 0 = leader
  const int cluster = static_cast<int>(ptx::cluster_id_x());
  const int num_clusters = static_cast<int>(ptx::num_clusters_x());
  volatile int* abort_flag = &bars->abort_flag;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      ptx::mbar_init(ptx::smem_u32(&bars->full[s]), 1);
      ptx::mbar_init(ptx::smem_u32(&bars->empty[s]), 1);
    }
    for (int s = 0; s < kNumAcc; ++s) {
      ptx::mbar_init(ptx::smem_u32(&bars->acc_full[s]), 1);
      ptx::mbar_init(ptx::smem_u32(&bars->acc_empty[s]), 2 * kEpiWarps);
    }
    bars->abort_flag = 0;
    ptx::fence_barrier_init();
    for (int i = 0; i < P.n_prod; ++i) {
      ptx::prefetch_tensormap(&P.prod[i].map_a);
      ptx::prefetch_tensormap(&P.prod[i].map_b);
    }
  }
  if (warp == 1) {
    ptx::tmem_alloc_pair(ptx::smem_u32(&bars->tmem_base), kTmemCols);
    ptx::tmem_relinquish_pair();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::cluster_sync_all();  // both CTAs' barriers are initialised, both TMEM allocations done
  ptx::tc_fence_after();
  const uint32_t tmem_base = bars->tmem_base;
  // results of earlier kernels are needed from here on
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();

  const int n_valid = *reinterpret_cast<volatile int*>(&P.ctrl->n_valid);
  const Shape s0 = shape_of(P, 0, n_valid);
  Shape s1 = {0, 0, 0, 1, 0};
  if (kMode == kModeOut && P.n_prod == 2) s1 = shape_of(P, 1, n_valid);
  const int total_tiles = s0.tiles + s1.tiles;

  if (warp == 0) {
    // ------------------------------------------------------ TMA producer ----
    const bool elected = ptx::elect_one();
    uint32_t stage = 0, phase = 0;
    bool ok = true;
    const uint32_t ring_u32 = ptx::smem_u32(ring);
    const uint32_t full0 = ptx::smem_u32(&bars->full[0]);
    const uint32_t empty0 = ptx::smem_u32(&bars->empty[0]);
    const uint32_t leader_full0 = ptx::map_to_cta(full0, 0);
    for (int t = cluster; t < total_tiles && ok; t += num_clusters) {
      const Tile tl = locate(P, s0, s1, t);
      const Product& pr = P.prod[tl.prod];
      const int half_n = pr.n_tile >> 1;
      const int a_row = pr.a_m0 + tl.mi * kTileM + static_cast<int>(rank) * 128;
      const int b_row = pr.b_n0 + tl.ni * pr.n_tile + static_cast<int>(rank) * half_n;
      const uint32_t stage_tx = 2u * static_cast<uint32_t>(kTileABytes + half_n * 128);
      const bool a_mn = pr.a_mn != 0, b_mn = pr.b_mn != 0;
      for (int kb = tl.kb0; kb < tl.kb1; ++kb) {
        ok = ptx::mbar_wait(empty0 + stage * 8, phase ^ 1u, abort_flag);
        ok = __all_sync(0xFFFFFFFFu, ok);
        if (!ok) {
          if (elected) report_timeout(P);
          break;
        }
        if (elected) {
          const uint32_t leader_full = leader_full0 + stage * 8;
          const uint32_t sa = ring_u32 + stage * kStageBytes;
          const uint32_t sb = sa + kTileABytes;
          const int ka = pr.a_k0 + kb * kBK, kbb = pr.b_k0 + kb * kBK;
          if (rank == 0) ptx::mbar_arrive_expect_tx(full0 + stage * 8, stage_tx);
          if (!a_mn) {
            ptx::tma_load_3d_pair(sa, &pr.map_a, ka, a_row, 0, leader_full);
          } else {
            ptx::tma_load_3d_pair(sa, &pr.map_a, a_row, ka, 0, leader_full);
            ptx::tma_load_3d_pair(sa + 8192, &pr.map_a, a_row + 64, ka, 0, leader_full);
          }
          if (!b_mn) {
            ptx::tma_load_3d_pair(sb, &pr.map_b, kbb, b_row, 0, leader_full);
          } else {
            ptx::tma_load_3d_pair(sb, &pr.map_b, b_row, kbb, 0, leader_full);
            if (half_n == 128) ptx::tma_load_3d_pair(sb + 8192, &pr.map_b, b_row + 64, kbb, 0, leader_full);
          }
        }
        __syncwarp();
        if (++stage == kStages) {
          stage = 0;
          phase ^= 1u;
        }
      }
    }
    if (!ok) {
      for (int i = 0; i < 64; ++i) __nanosleep(1000);  // let copies in flight land
    }
  } else if (warp == 1) {
    // -------------------------------------------- UMMA issuer (leader CTA) ----
    if (rank == 0) {
      const bool elected = ptx::elect_one();
      uint32_t stage = 0, phase = 0;
      int acc = 0;
      uint32_t acc_phase = 0;
      bool ok = true;
      const uint32_t ring_enc = ptx::smem_u32(ring) >> 4;
      const uint32_t full0 = ptx::smem_u32(&bars->full[0]);
      const uint32_t empty0 = ptx::smem_u32(&bars->empty[0]);
      constexpr uint32_t kDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);  // SBO 1024, version 1, 128B swizzle
      constexpr uint32_t kLboK = (16u >> 4) << 16;
      constexpr uint32_t kLboMN = (8192u >> 4) << 16;  // next 64-element chunk of an MN-major operand
      for (int t = cluster; t < total_tiles && ok; t += num_clusters) {
        const Tile tl = locate(P, s0, s1, t);
        if (tl.kb0 == tl.kb1) continue;  // no token counts: the epilogue writes zeros by itself
        const Product& pr = P.prod[tl.prod];
        const bool a_mn = pr.a_mn != 0, b_mn = pr.b_mn != 0;
        ok = ptx::mbar_wait(ptx::smem_u32(&bars->acc_empty[acc]), acc_phase ^ 1u, abort_flag);
        ok = __all_sync(0xFFFFFFFFu, ok);
        if (!ok) {
          if (elected) report_timeout(P);
          break;
        }
        ptx::tc_fence_after();
        const uint32_t d_tmem = tmem_base + static_cast<uint32_t>(acc * kAccCols);
        const uint32_t idesc = ptx::make_idesc_bf16(256, pr.n_tile, a_mn ? 1 : 0, b_mn ? 1 : 0);
        const uint32_t a_fix = a_mn ? kLboMN : kLboK, b_fix = (b_mn ? kLboMN : kLboK) + (kTileABytes >> 4);
        const uint32_t a_step = a_mn ? (2048u >> 4) : (32u >> 4), b_step = b_mn ? (2048u >> 4) : (32u >> 4);
        uint32_t accumulate = 0;
#pragma unroll 1
        for (int kb = tl.kb0; kb < tl.kb1; ++kb) {
          ok = ptx::mbar_wait(full0 + stage * 8, phase, abort_flag);
          ok = __all_sync(0xFFFFFFFFu, ok);
          if (!ok) {
            if (elected) report_timeout(P);
            break;
          }
          ptx::tc_fence_after();
          const uint32_t enc = ring_enc + stage * (kStageBytes >> 4);
          const uint32_t a_lo = enc + a_fix, b_lo = enc + b_fix;
          if (elected) {
            ptx::umma_bf16_pair_lohi(d_tmem, a_lo, b_lo, kDescHi, idesc, accumulate);
            ptx::umma_bf16_pair_lohi(d_tmem, a_lo + a_step, b_lo + b_step, kDescHi, idesc, 1u);
            ptx::umma_bf16_pair_lohi(d_tmem, a_lo + 2 * a_step, b_lo + 2 * b_step, kDescHi, idesc, 1u);
            ptx::umma_bf16_pair_lohi(d_tmem, a_lo + 3 * a_step, b_lo + 3 * b_step, kDescHi, idesc, 1u);
            ptx::umma_commit_pair(empty0 + stage * 8, 3);
          }
          __syncwarp();
          accumulate = 1u;
          if (++stage == kStages) {
            stage = 0;
            phase ^= 1u;
          }
        }
        if (!ok) break;
        if (elected) ptx::umma_commit_pair(ptx::smem_u32(&bars->acc_full[acc]), 3);
        __syncwarp();
        if (++acc == kNumAcc) {
          acc = 0;
          acc_phase ^= 1u;
        }
      }
    }
  } else if (kMode == kModeOut && warp >= 6) {
    // ---------------------------------- codes of the next piece, meanwhile ----
    if (P.convert.g != nullptr)
      convert_piece(P.convert, n_valid, static_cast<int>(blockIdx.x) * kConvertWarps + warp - 6,
                    static_cast<int>(gridDim.x) * kConvertWarps, lane);
  } else {
    // ----------------------------------------------------------- epilogue ----
    const int q = warp & 3;  // TMEM lane quarter this warp may read
    int acc = 0;
    uint32_t acc_phase = 0;
    bool ok = true;
    for (int t = cluster; t < total_tiles && ok; t += num_clusters) {
      const Tile tl = locate(P, s0, s1, t);
      const int row = tl.mi * kTileM + static_cast<int>(rank) * 128 + q * 32 + lane;
      const bool have_acc = tl.kb0 != tl.kb1;
      if (have_acc) {
        ok = ptx::mbar_wait_relaxed(ptx::smem_u32(&bars->acc_full[acc]), acc_phase, abort_flag);
        ok = __all_sync(0xFFFFFFFFu, ok);
        if (!ok) {
          if (lane == 0) report_timeout(P);
          break;
        }
        ptx::tc_fence_after();
      }
      const uint32_t taddr = tmem_base + static_cast<uint32_t>(acc * kAccCols) + (static_cast<uint32_t>(q * 32) << 16);

      if (kMode == kModeStats) {
        const int c0 = tl.ni * kTileN;  // first vocabulary column of the tile
        const int limit = P.vocab - c0;
        const bool row_ok = row < n_valid;
        if (__any_sync(0xFFFFFFFFu, row_ok)) {
          Entries en;
          en.open(P, row, c0, row_ok);
          // the row's maximum over the tile first, then exponentials and codes against it
          float m = -INFINITY;
          {
            uint32_t va[32], vb[32];
            auto top_of = [&](const uint32_t (&v)[32], int c) {
              if (limit < c + 32) {
#pragma unroll
                for (int i = 0; i < 32; ++i)
                  if (c + i < limit) m = fmaxf(m, __uint_as_float(v[i]));
              } else {
                float a = __uint_as_float(v[0]), b = __uint_as_float(v[1]);
#pragma unroll
                for (int i = 2; i < 32; i += 2) {
                  a = fmaxf(a, __uint_as_float(v[i]));
                  b = fmaxf(b, __uint_as_float(v[i + 1]));
                }
                m = fmaxf(m, fmaxf(a, b));
              }
            };
            ptx::tmem_ld_32x32(taddr, va);
            ptx::tmem_ld_wait();
#pragma unroll 1
            for (int c = 0; c < kTileN; c += 64) {
              ptx::tmem_ld_32x32(taddr + c + 32, vb);
              top_of(va, c);
              ptx::tmem_ld_wait();
              if (c + 64 < kTileN) ptx::tmem_ld_32x32(taddr + c + 64, va);
              top_of(vb, c + 32);
              ptx::tmem_ld_wait();
            }
          }
          m *= P.scale2;
          const float base = m == -INFINITY ? 0.f : m;  // nothing but -inf
          unsigned short* crow = nullptr;
          if (tl.ni < P.code_tiles && row_ok) {
            const int piece = tl.ni / P.piece_tiles;
            crow = P.codes + piece * P.piece_stride + static_cast<long long>(row) * P.g_ld +
                   (tl.ni - piece * P.piece_tiles) * kTileN;
          }
          float s = 0.f;
          auto chunk = [&](uint32_t (&v)[32], int c) {
            // logits of entries that lie in these 32 columns
            while (__any_sync(0xFFFFFFFFu, en.col - c < 32)) {
              if (en.col - c < 32) {
                P.entry_logit[static_cast<long long>(row) * P.top + en.next] = pick(v, en.col - c);
                ++en.next;
                en.fetch(c0);
              }
            }
            if (limit < c + 32) {
#pragma unroll
              for (int i = 0; i < 32; ++i)
                if (c + i >= limit) v[i] = 0xFF800000u;  // -inf
            }
            float s0_ = 0.f, s1_ = 0.f, s2_ = 0.f, s3_ = 0.f;
#pragma unroll
            for (int i = 0; i < 32; i += 4) {
              const float y0 = fmaf(__uint_as_float(v[i]), P.scale2, -base);
              const float y1 = fmaf(__uint_as_float(v[i + 1]), P.scale2, -base);
              const float y2 = fmaf(__uint_as_float(v[i + 2]), P.scale2, -base);
              const float y3 = fmaf(__uint_as_float(v[i + 3]), P.scale2, -base);
              s0_ += ex2_fast(y0);
              s1_ += ex2_fast(y1);
              s2_ += ex2_fast(y2);
              s3_ += ex2_fast(y3);
              v[i >> 1] = __byte_perm(encode_logit(y0), encode_logit(y1), 0x5410);
              v[(i >> 1) + 1] = __byte_perm(encode_logit(y2), encode_logit(y3), 0x5410);
            }
            s += (s0_ + s1_) + (s2_ + s3_);
            if (crow != nullptr) {
              const uint32_t lo[8] = {v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]};
              const uint32_t hi[8] = {v[8], v[9], v[10], v[11], v[12], v[13], v[14], v[15]};
              st_global_32(crow + c, lo);
              st_global_32(crow + c + 16, hi);
            }
            __syncwarp();
          };
          uint32_t va[32], vb[32];
          ptx::tmem_ld_32x32(taddr, va);
          ptx::tmem_ld_wait();
#pragma unroll 1
          for (int c = 0; c < kTileN; c += 64) {
            ptx::tmem_ld_32x32(taddr + c + 32, vb);
            chunk(va, c);
            ptx::tmem_ld_wait();
            if (c + 64 < kTileN) ptx::tmem_ld_32x32(taddr + c + 64, va);
            chunk(vb, c + 32);
            ptx::tmem_ld_wait();
          }
          if (row_ok) P.stats[static_cast<long long>(row) * P.stats_ld + tl.ni] = make_float2(m, s);
        }
      } else if (kMode == kModeGrad) {
        const int g0 = tl.ni * kTileN;    // first column within the piece
        const int c0 = P.v0 + g0;         // and in the vocabulary
        const int limit = P.vocab - c0;
        const bool row_ok = row < n_valid;
        float2 rq = make_float2(0.f, 0.f);
        if (row_ok) rq = P.row_q[row];
        Entries en;
        en.open(P, row, c0, row_ok);
        __nv_bfloat16* grow = P.g + static_cast<long long>(row) * P.g_ld + g0;
        auto chunk = [&](uint32_t (&v)[32], int c) {
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            float y = rq.x * ex2_fast(fmaf(__uint_as_float(v[i]), P.scale2, -rq.y));
            v[i] = __float_as_uint(y);
          }
          if (!row_ok) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = 0u;
          }
          if (limit < c + 32) {
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (c + i >= limit) v[i] = 0u;
          }
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
              w[i] = pack2(__uint_as_float(v[16 * h + 2 * i]), __uint_as_float(v[16 * h + 2 * i + 1]));
            st_global_32(grow + c + 16 * h, w);
          }
          // the entries' gradients replace what was just written, by the same thread
          while (en.col - c < 32) {
            grow[en.col] = __float2bfloat16_rn(P.entry_g[static_cast<long long>(row) * P.top + en.next]);
            ++en.next;
            en.fetch(c0);
          }
          __syncwarp();
        };
        uint32_t va[32], vb[32];
        ptx::tmem_ld_32x32(taddr, va);
        ptx::tmem_ld_wait();
#pragma unroll 1
        for (int c = 0; c < kTileN; c += 64) {
          ptx::tmem_ld_32x32(taddr + c + 32, vb);
          chunk(va, c);
          ptx::tmem_ld_wait();
          if (c + 64 < kTileN) ptx::tmem_ld_32x32(taddr + c + 64, va);
          chunk(vb, c + 32);
          ptx::tmem_ld_wait();
        }
      } else {
        const int n_tile = P.prod[tl.prod].n_tile;
        const int c0 = tl.ni * n_tile;
        if (tl.prod == 0) {
          // partial dX, fp32
          float* prow = P.part + tl.split * P.part_stride + static_cast<long long>(row) * P.part_ld + c0;
          const bool row_ok = row < n_valid;
          const int limit = P.part_cols - c0;
#pragma unroll 1
          for (int c = 0; c < n_tile && c < limit; c += 32) {
            uint32_t v[32];
            ptx::tmem_ld_32x32(taddr + c, v);
            ptx::tmem_ld_wait();
            if (row_ok) {
#pragma unroll
              for (int h = 0; h < 4; ++h) {
                if (c + 8 * h < limit) {  // part_cols is a multiple of 8
                  uint32_t w[8];
                  if (P.part_add) {
                    ld_global_32(prow + c + 8 * h, w);
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                      w[i] = __float_as_uint(__uint_as_float(w[i]) + __uint_as_float(v[8 * h + i]));
                  } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[i] = v[8 * h + i];
                  }
                  st_global_32(prow + c + 8 * h, w);
                }
              }
            }
            __syncwarp();
          }
        } else {
          // dW rows of this vocabulary piece
          const bool row_ok = row < P.dw_rows;
          const int limit = P.dw_cols - c0;
          const long long off = static_cast<long long>(P.dw_row0 + row) * P.ld_dw + c0;
#pragma unroll 1
          for (int c = 0; c < n_tile && c < limit; c += 32) {
            uint32_t v[32];
            if (have_acc) {
              ptx::tmem_ld_32x32(taddr + c, v);
              ptx::tmem_ld_wait();
            } else {
#pragma unroll
              for (int i = 0; i < 32; ++i) v[i] = 0u;
            }
            if (row_ok) {
              if (P.dw_fp32) {
                float* d = static_cast<float*>(P.dw) + off + c;
                if (P.dw_vec == 32 && c + 32 <= limit) {
#pragma unroll
                  for (int h = 0; h < 4; ++h) {
                    uint32_t w[8];
                    if (P.dw_add) {
                      ld_global_32(d + 8 * h, w);
#pragma unroll
                      for (int i = 0; i < 8; ++i)
                        w[i] = __float_as_uint(__uint_as_float(w[i]) + __uint_as_float(v[8 * h + i]));
                    } else {
#pragma unroll
                      for (int i = 0; i < 8; ++i) w[i] = v[8 * h + i];
                    }
                    st_global_32(d + 8 * h, w);
                  }
                } else {
#pragma unroll
                  for (int i = 0; i < 32; ++i)
                    if (c + i < limit) d[i] = __uint_as_float(v[i]) + (P.dw_add ? d[i] : 0.f);
                }
              } else {
                __nv_bfloat16* d = static_cast<__nv_bfloat16*>(P.dw) + off + c;
                if (P.dw_add) {
#pragma unroll
                  for (int i = 0; i < 32; ++i)
                    if (c + i < limit) v[i] = __float_as_uint(__uint_as_float(v[i]) + __bfloat162float(d[i]));
                }
                if (P.dw_vec >= 16 && c + 32 <= limit) {
#pragma unroll
                  for (int h = 0; h < 2; ++h) {
                    uint32_t w[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                      w[i] = pack2(__uint_as_float(v[16 * h + 2 * i]), __uint_as_float(v[16 * h + 2 * i + 1]));
                    if (P.dw_vec == 32) {
                      st_global_32(d + 16 * h, w);
                    } else {
                      *reinterpret_cast<uint4*>(d + 16 * h) = make_uint4(w[0], w[1], w[2], w[3]);
                      *reinterpret_cast<uint4*>(d + 16 * h + 8) = make_uint4(w[4], w[5], w[6], w[7]);
                    }
                  }
                } else {
#pragma unroll
                  for (int i = 0; i < 32; ++i)
                    if (c + i < limit) d[i] = __float2bfloat16_rn(__uint_as_float(v[i]));
                }
              }
            }
            __syncwarp();
          }
        }
      }

      if (have_acc) {
        // accumulator fully read: hand the TMEM stage back to the leader's issuer
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive_cluster(ptx::map_to_cta(ptx::smem_u32(&bars->acc_empty[acc]), 0));
        if (++acc == kNumAcc) {
          acc = 0;
          acc_phase ^= 1u;
        }
      }
    }
  }

  // ---------------------------------------------------------------- teardown --
  ptx::tc_fence_before();
  __syncthreads();
  ptx::cluster_sync_all();  // the peer may still signal our barriers / read our tiles until here
  if (warp == 1) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc_pair(tmem_base, kTmemCols);
  }
}

template <int kMode>
cudaError_t configure_one() {
  return cudaFuncSetAttribute(head_gemm_kernel<kMode>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
}

template <int kMode>
cudaError_t launch_one(const GemmParams& P, unsigned clusters, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(2 * clusters, 1, 1);
  cfg.blockDim = dim3(threads_of(kMode), 1, 1);
  cfg.dynamicSmemBytes = kSmemBytes;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, head_gemm_kernel<kMode>, P);
}

}  // namespace

cudaError_t gemm_configure() {
  cudaError_t e = configure_one<kModeStats>();
  if (e == cudaSuccess) e = configure_one<kModeGrad>();
  if (e == cudaSuccess) e = configure_one<kModeOut>();
  return e;
}

// Largest number of co-resident CTA pairs (one CTA per SM).
cudaError_t gemm_max_clusters(int* out) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(2, 1, 1);
  cfg.blockDim = dim3(threads_of(kModeOut), 1, 1);
  cfg.dynamicSmemBytes = kSmemBytes;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = 2;
  attr.val.clusterDim.y = 1;
  attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaOccupancyMaxActiveClusters(out, head_gemm_kernel<kModeOut>, &cfg);
}

// `tiles`: an upper bound on the launch's tiles (every token counts).
cudaError_t launch_gemm(int mode, const GemmParams& P, long long tiles, int max_clusters, cudaStream_t stream) {
  if (tiles <= 0) return cudaSuccess;
  const unsigned clusters = static_cast<unsigned>(tiles < max_clusters ? tiles : max_clusters);
  if (mode == kModeStats) return launch_one<kModeStats>(P, clusters, stream);
  if (mode == kModeGrad) return launch_one<kModeGrad>(P, clusters, stream);
  return launch_one<kModeOut>(P, clusters, stream);
}

}  // namespace head
}  // namespace muon
