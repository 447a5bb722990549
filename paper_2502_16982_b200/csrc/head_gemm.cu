// Products of the LM-head losses for sm_100a.  With hidden states x [T, D], head
// w [V, D], logits l = a x w^T, q = softmax(l) and a sparse target distribution p:
//
//   statistics  max and sum of exponentials of every token over every 64 columns
//               of l, l at the sparse entries and, where they are kept, l as 16-bit
//               codes (head_codes.cuh)
//   gradient    G = g a (c q - p) for one piece of the vocabulary, in bf16
//   outputs     dX += G w(piece)  and  dW(piece) = G^T x, one launch; G lacks a factor
//               near 1 that all tokens share (Ctrl::rest), dW is given it here and dX
//               where its partial sums are joined
//
// One persistent, warp-specialised kernel on CTA pairs (tcgen05.mma
// cta_group::2, M = 256, N = 128 or 256), three instantiations by epilogue.
//   warp 0     TMA producer: this CTA's 128 rows of A and its half of B per K
//              block, into a ring of kStages; no multicast
//   warp 1     leader CTA only: UMMA issuer, two TMEM accumulator stages
//   epilogue   statistics and gradient: warps 2-17, a lane per row and 64 columns at
//              a time, so that a row's maximum and sum over them stay in one
//              thread's registers; outputs: warps 2-5
//   warps 6-9  outputs, several pieces: turn the next piece's codes (head_codes.cuh)
//              into the gradient of its logits while the tensor cores work on this
//              piece; with one piece they are four more epilogue warps
//
// Everything a tile stores goes through 4 KiB of shared memory per warp and leaves
// as a TMA store (or a TMA reduction, where dX or dW is added to): 32 rows by 128
// bytes at a time.
//
// Every wait is bounded (ptx::mbar_wait); on expiry the CTA records
// MUON_ERR_TIMEOUT, all roles drain and the kernel returns.
#include <cuda_bf16.h>

#include <type_traits>

#include "head_codes.cuh"
#include "ptx.cuh"

namespace muon {
namespace head {

namespace {

constexpr int kTileABytes = 128 * kBK * 2;
constexpr int kTileBBytes = 128 * kBK * 2;
constexpr int kStageBytes = kTileABytes + kTileBBytes;
constexpr int kNumAcc = 2;
constexpr int kAccCols = 256;
constexpr int kTmemCols = kNumAcc * kAccCols;
constexpr int kStageOut = 32 * 128;  // one warp's 32 rows x 128 bytes
// Shared memory is split between the operand ring and the staging of stores, six
// stages and 32 KiB or five stages and 64 KiB:
//   statistics  sixteen warps with one buffer each and five stages, or (kSpare) with half
//               a buffer and six stages.  896 us against 1015 at 8192 x 256 x 50000; but
//               165 us against 154 for 100 x 2048 x 163840, where w streams from memory
//   outputs     four warps with two buffers each and six stages beside four that
//               convert codes, or (kSpare) eight warps and five stages where nothing is
//               left to convert
template <int kMode, bool kSpare>
struct Config {
  static constexpr bool kDeep = kMode == kModeOut ? !kSpare : kSpare;
  static constexpr int kStages = kDeep ? 6 : 5;
  static constexpr int kStaging = (kDeep ? 8 : 16) * kStageOut;
  static constexpr int kEpiWarps = kMode == kModeOut ? (kSpare ? 8 : 4) : 16;
  static constexpr int kConvertWarps = kMode == kModeOut && !kSpare ? 4 : 0;
  static constexpr int kThreads = 64 + 32 * (kEpiWarps + kConvertWarps);
  static constexpr int kSmemBytes = 1024 + kStages * kStageBytes + kStaging + 512;
  static_assert(kSmemBytes <= 232448, "exceeds the 227 KiB shared-memory limit");
};
constexpr int kMaxStages = 6;

constexpr int kOutside = 1 << 30;  // a row coordinate past every tensor

struct Barriers {
  unsigned long long full[kMaxStages];    // leader's copy is the live one
  unsigned long long empty[kMaxStages];
  unsigned long long acc_full[kNumAcc];
  unsigned long long acc_empty[kNumAcc];  // leader's copy is the live one
  uint32_t tmem_base;
  int abort_flag;
};

static_assert(sizeof(Barriers) <= 512, "barrier block too large");

__device__ __forceinline__ void report_timeout(const GemmParams& P) { atomicExch(&P.ctrl->status, -6); }

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&h);
}

__device__ __forceinline__ void sts128(uint32_t addr, uint32_t w0, uint32_t w1, uint32_t w2, uint32_t w3) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(w0), "r"(w1), "r"(w2), "r"(w3) : "memory");
}

__device__ __forceinline__ void sts32(uint32_t addr, uint32_t w) {
  asm volatile("st.shared.b32 [%0], %1;" ::"r"(addr), "r"(w) : "memory");
}

__device__ __forceinline__ float lds32(uint32_t addr) {
  float y;
  asm volatile("ld.shared.b32 %0, [%1];" : "=f"(y) : "r"(addr));
  return y;
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

// Largest of three; a NaN shows.
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// Address of 16-byte chunk `c` of row `lane` in a 32-row staging buffer, 128-byte swizzle.
__device__ __forceinline__ uint32_t staged(uint32_t buf, int lane, int c) {
  return buf + static_cast<uint32_t>(lane * 128 + ((c ^ (lane & 7)) << 4));
}

// t / d for a tile number: a multiplication by the reciprocal, off by at most one
// below 2^24, put right by the remainder.
__device__ __forceinline__ int quotient(int t, int d, float reciprocal) {
  if (t >= (1 << 24)) return t / d;
  int q = static_cast<int>(static_cast<float>(t) * reciprocal);
  const int r = t - q * d;
  q += (r >= d) - (r < 0);
  return q;
}

// Sizes of product `i` that depend on how many tokens count.
struct Shape {
  int m_tiles, n_tiles, k_blocks, splits, tiles;
  float per_split, per_column;  // reciprocals of the tiles of a split and of a row (or group) of tiles
};

__device__ __forceinline__ Shape shape_of(const GemmParams& P, int i, int n_valid) {
  const Product& p = P.prod[i];
  Shape s;
  s.m_tiles = p.m_tiles < 0 ? (n_valid + kTileM - 1) / kTileM : p.m_tiles;
  s.k_blocks = p.k_blocks < 0 ? (n_valid + kBK - 1) / kBK : p.k_blocks;
  s.n_tiles = p.n_tiles;
  s.splits = p.splits;
  s.tiles = s.m_tiles * s.n_tiles * s.splits;
  s.per_split = __frcp_rn(static_cast<float>(max(1, s.m_tiles * s.n_tiles)));
  s.per_column = __frcp_rn(static_cast<float>(p.swap_order ? s.n_tiles : p.group * s.n_tiles));
  return s;
}

// One tile: which product, which 256 rows and n_tile columns, which run of K blocks.
struct Tile {
  int prod, mi, ni, split, kb0, kb1;
};

// Which tiles a CTA pair takes, one after the other.  Product 0's tiles are dealt out
// in turn.  Where that leaves some pairs with one more than others, product 1's go
// to the others first, `extra` each - dX has few long tiles, dW many short ones -
// and then to all in turn.
struct Deal {
  int pairs, pair;
  int mine0;  // this pair's tiles of product 0
  int more;   // pairs that have one more than the others
  int extra;
};

__device__ __forceinline__ Deal deal_out(const Shape& s0, const Shape& s1, int pair, int pairs) {
  Deal d;
  d.pairs = pairs;
  d.pair = pair;
  const int each = s0.tiles / pairs;
  d.more = s0.tiles - each * pairs;
  d.mine0 = each + (pair < d.more);
  d.extra = 0;
  if (s1.tiles > 0 && d.more > 0) {
    const int cost0 = (s0.k_blocks + s0.splits - 1) / s0.splits + kTileCost, cost1 = s1.k_blocks + kTileCost;
    d.extra = min((cost0 + cost1 / 2) / cost1, s1.tiles / (pairs - d.more));
  }
  return d;
}

// The pair's k-th tile; false past the last.  Row tiles are walked in groups of
// `group` for each column tile (or the columns innermost, swap_order), one split
// after the other, so that the CTA pairs that run at the same time share operand
// tiles in L2.
__device__ __forceinline__ bool locate(const GemmParams& P, const Shape& s0, const Shape& s1, const Deal& d, int k, Tile& r) {
  int t;
  if (k < d.mine0) {
    r.prod = 0;
    t = d.pair + k * d.pairs;
  } else {
    r.prod = 1;
    k -= d.mine0;
    const int few = d.pairs - d.more;
    if (d.pair >= d.more) {
      t = k < d.extra ? k * few + d.pair - d.more : d.extra * few + (k - d.extra) * d.pairs + d.pair;
    } else {
      t = d.extra * few + k * d.pairs + d.pair;
    }
    if (t >= s1.tiles) return false;
  }
  const Shape& s = r.prod ? s1 : s0;
  const Product& p = P.prod[r.prod];
  r.split = 0;
  r.kb0 = 0;
  r.kb1 = s.k_blocks;
  if (s.splits > 1) {  // at most 2^18 K blocks and 64 splits
    const int per_split = s.m_tiles * s.n_tiles;
    r.split = quotient(t, per_split, s.per_split);
    t -= r.split * per_split;
    r.kb0 = static_cast<int>(static_cast<unsigned>(s.k_blocks) * r.split / s.splits);
    r.kb1 = static_cast<int>(static_cast<unsigned>(s.k_blocks) * (r.split + 1) / s.splits);
  }
  if (p.swap_order) {
    r.mi = quotient(t, s.n_tiles, s.per_column);
    r.ni = t - r.mi * s.n_tiles;
  } else {
    const int per_group = p.group * s.n_tiles;
    const int grp = quotient(t, per_group, s.per_column);
    t -= grp * per_group;
    const int rows = min(p.group, s.m_tiles - grp * p.group);
    r.ni = quotient(t, rows, __frcp_rn(static_cast<float>(rows)));
    r.mi = grp * p.group + (t - r.ni * rows);
  }
  return true;
}

// Picks v[i] for a run-time i without putting v in local memory: halves by the bits of i.
__device__ __forceinline__ float pick(const uint32_t (&v)[kStatN], int i) {
  uint32_t r[kStatN / 2];
#pragma unroll
  for (int j = 0; j < kStatN / 2; ++j) r[j] = i & (kStatN / 2) ? v[j + kStatN / 2] : v[j];
#pragma unroll
  for (int half = kStatN / 4; half > 0; half >>= 1)
#pragma unroll
    for (int j = 0; j < half; ++j) r[j] = i & half ? r[j + half] : r[j];
  return __uint_as_float(r[0]);
}

// Where a row's sparse entries in one 256-column tile are found: asked for a tile
// ahead, so that the loads wait for nothing.
struct EntryHead {
  int a, b;  // one target per token: its index; else positions in the row's list
};

__device__ __forceinline__ EntryHead entry_head(const GemmParams& P, int row, int tile, bool row_ok) {
  EntryHead h = {kNoId, 0};
  if (P.top == 1) {
    if (row_ok) h.a = P.ids[row];
  } else {
    h.a = 0;
    if (row_ok) {
      const unsigned char* s = P.starts + static_cast<long long>(row) * P.n_starts + tile;
      h.a = s[0];
      h.b = s[1];
    }
  }
  return h;
}

// The sparse entries of one row in kStatN columns from col0 on.
struct Entries {
  int next, end;  // positions in the row's list
  int col;        // column of entry `next` from col0, or past every column
  const int* ids;

  __device__ __forceinline__ void open(const GemmParams& P, const EntryHead& h, int row, int col0) {
    if (P.top == 1) {
      next = 0;
      end = 1;
      col = h.a - col0;
      if (col < 0 || col >= kStatN) col = kNoId;
    } else {
      next = h.a;
      end = h.b;
      ids = P.ids + static_cast<long long>(row) * P.top;
      while (next < end && ids[next] < col0) ++next;
      fetch(col0);
    }
  }
  __device__ __forceinline__ void fetch(int col0) {
    col = next < end ? ids[next] - col0 : kNoId;
    if (col >= kStatN) col = kNoId;
  }
  __device__ __forceinline__ void pop(const GemmParams& P, int col0) {
    ++next;
    if (P.top == 1) col = kNoId;
    else fetch(col0);
  }
};

// The same from the caller's list, as it is: 64-bit indices in any order, few enough to
// look at all of a row's for every tile.  mask: entries that fall into `cols` columns
// from col0 on.
struct ListHead {
  int id;
  unsigned long long mask[2];
};

__device__ __forceinline__ int list_id(const GemmParams& P, int row, int k) {
  const int64_t id = P.ids64[row * P.ld_ids64 + k];
  return id >= 0 && id < P.vocab ? static_cast<int>(id) : kNoId;
}

__device__ __forceinline__ ListHead list_head(const GemmParams& P, int row, int col0, int cols, bool row_ok) {
  ListHead h = {kNoId, {0, 0}};
  if (row_ok) {
    if (P.top == 1) {
      h.id = list_id(P, row, 0);
    } else {
#pragma unroll 8
      for (int k = 0; k < P.top; ++k) {
        const unsigned long long in = static_cast<unsigned>(list_id(P, row, k) - col0) < static_cast<unsigned>(cols);
        h.mask[0] |= k < 64 ? in << k : 0;
        h.mask[1] |= k < 64 ? 0 : in << (k - 64);
      }
    }
  }
  return h;
}

struct ListEntries {
  int next, col;
  unsigned long long left[2];
  int row;

  __device__ __forceinline__ void open(const GemmParams& P, const ListHead& h, int r, int col0) {
    row = r;
    if (P.top == 1) {
      next = 0;
      col = h.id - col0;
      if (col < 0 || col >= kStatN) col = kNoId;
    } else {
      left[0] = h.mask[0];
      left[1] = h.mask[1];
      fetch(P, col0);
    }
  }
  __device__ __forceinline__ void fetch(const GemmParams& P, int col0) {
    col = kNoId;
    while (col == kNoId && (left[0] | left[1])) {
      if (left[0]) {
        next = __ffsll(static_cast<long long>(left[0])) - 1;
        left[0] &= left[0] - 1;
      } else {
        next = 63 + __ffsll(static_cast<long long>(left[1]));
        left[1] &= left[1] - 1;
      }
      const int c = list_id(P, row, next) - col0;
      if (c >= 0 && c < kStatN) col = c;
    }
  }
  __device__ __forceinline__ void pop(const GemmParams& P, int col0) {
    if (P.top == 1) col = kNoId;
    else fetch(P, col0);
  }
};

// The tokens' weighted losses added up, always in the same order, by one warp of the last
// CTA beside its other work.
__device__ __forceinline__ void add_losses(const GemmParams& P, int n_valid, int lane) {
  if (P.total == nullptr || blockIdx.x != gridDim.x - 1) return;
  float sum = 0.f;
  const int whole = n_valid & ~127;
#pragma unroll 8
  for (int i = lane * 4; i < whole; i += 128) {
    const float4 v = *reinterpret_cast<const float4*>(P.row_l + i);
    sum += (v.x + v.y) + (v.z + v.w);
  }
  for (int i = whole + lane; i < n_valid; i += 32) sum += P.row_l[i];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
  if (lane == 0) *P.total = sum;
}

// kList: the sparse entries come from the caller's list.
template <int kMode, bool kSpare, bool kList>
__global__ void __launch_bounds__(Config<kMode, kSpare>::kThreads, 1)
head_gemm_kernel(const __grid_constant__ GemmParams P) {
  using Cfg = Config<kMode, kSpare>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~static_cast<uintptr_t>(1023));
  constexpr int kStages = Cfg::kStages;
  constexpr int kRows = kSpare ? 16 : 32;  // logits: rows of a box that stores them
  uint8_t* staging = ring + kStages * kStageBytes;
  Barriers* bars = reinterpret_cast<Barriers*>(staging + Cfg::kStaging);

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
      // warps of both CTAs that read one accumulator
      ptx::mbar_init(ptx::smem_u32(&bars->acc_empty[s]), 2 * (kMode == kModeOut ? Cfg::kEpiWarps : (P.by_tile ? 8 : 16)));
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

  if (kList && blockIdx.x == 0 && threadIdx.x == 0) {  // first of the call's kernels
    P.ctrl->status = 0;
    P.ctrl->ticket = 0;
  }
  const int n_valid = kList || P.in_place ? P.tokens : *reinterpret_cast<volatile int*>(&P.ctrl->n_valid);
  const Shape s0 = shape_of(P, 0, n_valid);
  Shape s1 = {};
  if (kMode == kModeOut && P.n_prod == 2) s1 = shape_of(P, 1, n_valid);
  const Deal deal = deal_out(s0, s1, cluster, num_clusters);

  if (warp == 0) {
    // ------------------------------------------------------ TMA producer ----
    const bool elected = ptx::elect_one();
    uint32_t stage = 0, phase = 0;
    bool ok = true;
    const uint32_t ring_u32 = ptx::smem_u32(ring);
    const uint32_t full0 = ptx::smem_u32(&bars->full[0]);
    const uint32_t empty0 = ptx::smem_u32(&bars->empty[0]);
    const uint32_t leader_full0 = ptx::map_to_cta(full0, 0);
    Tile tl;
    for (int k = 0; ok && locate(P, s0, s1, deal, k, tl); ++k) {
      const Product& pr = P.prod[tl.prod];
      const int half_n = pr.n_tile >> 1;
      // rows past the tokens that count are asked for outside the tensor: zeros, without traffic
      const int m_row = tl.mi * kTileM + static_cast<int>(rank) * 128;
      const int a_row = pr.m_tiles < 0 && m_row >= n_valid ? kOutside : m_row;
      const int a_rows = pr.a_mn ? 128 : pr.a_rows;
      const int b_row = pr.b_n0 + tl.ni * pr.n_tile + static_cast<int>(rank) * half_n;
      const uint32_t stage_tx = 2u * static_cast<uint32_t>((a_rows + half_n) * 128);
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
          const int ka = kb * kBK, kbb = pr.b_k0 + kb * kBK;
          if (rank == 0) ptx::mbar_arrive_expect_tx(full0 + stage * 8, stage_tx);
          if (a_mn) {
            ptx::tma_load_3d_pair(sa, &pr.map_a, a_row, ka, pr.a_z, leader_full);
            ptx::tma_load_3d_pair(sa + 8192, &pr.map_a, a_row + 64, ka, pr.a_z, leader_full);
          } else {
            ptx::tma_load_3d_pair(sa, &pr.map_a, ka, a_row, pr.a_z, leader_full);
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
      Tile tl;
      for (int k = 0; ok && locate(P, s0, s1, deal, k, tl); ++k) {
        if (tl.kb0 == tl.kb1) continue;  // no token counts: the epilogue writes zeros by itself
        const Product& pr = P.prod[tl.prod];
        const bool a_mn = pr.a_mn != 0, b_mn = pr.b_mn != 0;
        ok = ptx::mbar_wait<true>(ptx::smem_u32(&bars->acc_empty[acc]), acc_phase ^ 1u, abort_flag);
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
  } else if (warp >= 2 + Cfg::kEpiWarps) {
    // ---------------------------------- codes of the next piece, meanwhile ----
    const int convert = warp - 2 - Cfg::kEpiWarps;
    if (P.convert.g != nullptr)
      convert_piece(P.convert, n_valid, P.tokens, static_cast<int>(blockIdx.x) * Cfg::kConvertWarps + convert,
                    static_cast<int>(gridDim.x) * Cfg::kConvertWarps, lane);
    if (convert == 0) add_losses(P, n_valid, lane);
  } else {
    // ----------------------------------------------------------- epilogue ----
    const int q = warp & 3;  // TMEM lane quarter this warp may read
    const uint32_t tmem_row = tmem_base + (static_cast<uint32_t>(q * 32) << 16);
    bool ok = true;
    auto wait_acc = [&](int acc, uint32_t acc_phase) {
      ok = ptx::mbar_wait_relaxed(ptx::smem_u32(&bars->acc_full[acc]), acc_phase, abort_flag);
      ok = __all_sync(0xFFFFFFFFu, ok);
      if (!ok && lane == 0) report_timeout(P);
      if (ok) ptx::tc_fence_after();
    };
    // accumulator fully read: hand the TMEM stage back to the leader's issuer
    auto release = [&](int acc) {
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0)
        ptx::mbar_arrive_cluster_relaxed(ptx::map_to_cta(ptx::smem_u32(&bars->acc_empty[acc]), 0));
    };
    if constexpr (kMode != kModeOut) {
      // Four groups of four warps, a unit of work being 64 columns of a warp's 32 rows:
      // all that a thread needs of its row then stays in registers.  Each group takes
      // one unit of every tile or, where a pair has several tiles, two units of every
      // other tile, so that the groups' waits and arithmetic overlap (a tile's
      // accumulator is read and handed back at once in either case).  With two groups
      // the schedulers issued in 45 % of the cycles, waiting for latencies.
      const int group = (warp - 2) >> 2;
      const bool by_tile = P.by_tile != 0;
      const int step = by_tile ? 2 : 1;
      const int unit0 = by_tile ? (group & 1) * 2 : group, unit1 = by_tile ? unit0 + 2 : unit0 + 1;
      const uint32_t buf = ptx::smem_u32(staging + (warp - 2) * (kStageOut * kRows / 32));
      const int row_in = static_cast<int>(rank) * 128 + q * 32;
      const uint64_t scale = pair(P.scale2, P.scale2);
      Tile tl;
      int k = by_tile ? group >> 1 : 0;
      bool more = locate(P, s0, s1, deal, k, tl);
      using Head = std::conditional_t<kList, ListHead, EntryHead>;
      using List = std::conditional_t<kList, ListEntries, Entries>;
      Head head = {};
      float2 rq = make_float2(0.f, 0.f);
      const int first_tile = kMode == kModeGrad ? P.v0 / kTileN : 0;
      auto ask = [&](const Tile& t, Head& h, float2& r) {
        const int row = t.mi * kTileM + row_in + lane;
        if constexpr (kList) h = list_head(P, row, t.ni * kTileN + unit0 * kStatN, (unit1 - unit0) * kStatN, row < n_valid);
        else h = entry_head(P, row, first_tile + t.ni, row < n_valid);
        if (kMode == kModeGrad) r = row < n_valid ? P.row_q[row] : make_float2(0.f, 0.f);
      };
      if (more) ask(tl, head, rq);
      while (more) {
        Tile tl_next;
        Head head_next = {};
        float2 rq_next = make_float2(0.f, 0.f);
        more = locate(P, s0, s1, deal, k + step, tl_next);
        if (more) ask(tl_next, head_next, rq_next);
        const int row0 = tl.mi * kTileM + row_in;
        const int row = row0 + lane;
        const bool row_ok = row < n_valid;
        const int c0 = (first_tile + tl.ni) * kTileN;  // first vocabulary column of the tile
        const int acc = k & 1;
        wait_acc(acc, static_cast<uint32_t>(k >> 1) & 1u);
        if (!ok) break;
        // nothing is asked of the statistics of rows past the tokens that count
        const bool idle = kMode == kModeStats && row0 >= n_valid;
        const bool codes = kMode == kModeStats && tl.ni < P.code_tiles;
        if (idle) release(acc);
#pragma unroll 1
        for (int unit = unit0; unit < unit1 && !idle; ++unit) {
          const int col0 = c0 + unit * kStatN;
          const int limit = P.vocab - col0;  // columns of the unit in the vocabulary
          uint32_t v[kStatN];
          ptx::tmem_ld_32x64(tmem_row + static_cast<uint32_t>(acc * kAccCols + unit * kStatN), v);
          List en;
          en.open(P, head, row, col0);
          ptx::tmem_ld_wait();
          if (unit + 1 == unit1) release(acc);
          float m = -INFINITY, base = 0.f;
          if (kMode == kModeStats) {
            // logits of the sparse entries
            while (__any_sync(0xFFFFFFFFu, en.col < kStatN)) {
              if (en.col < kStatN) {
                P.entry_logit[static_cast<long long>(row) * P.top + en.next] = pick(v, en.col);
                en.pop(P, col0);
              }
            }
            if (limit < kStatN) {
#pragma unroll
              for (int j = 0; j < kStatN; ++j)
                if (j >= limit) v[j] = 0xFF800000u;  // -inf
            }
            // the row's maximum first, then exponentials and codes against it
            float a = __uint_as_float(v[0]), b = __uint_as_float(v[1]);
#pragma unroll
            for (int j = 2; j < kStatN - 2; j += 4) {
              a = max3(a, __uint_as_float(v[j]), __uint_as_float(v[j + 1]));
              b = max3(b, __uint_as_float(v[j + 2]), __uint_as_float(v[j + 3]));
            }
            // rounded up: no exponent below comes out positive, which a code could not hold
            m = __fmul_ru(max3(max3(a, __uint_as_float(v[kStatN - 2]), __uint_as_float(v[kStatN - 1])), b, b), P.scale2);
            base = m == -INFINITY ? 0.f : m;  // nothing but -inf
          }
          const uint64_t shift = kMode == kModeStats ? pair(-base, -base) : pair(-rq.y, -rq.y);
          auto work = [&](auto store) {
            constexpr bool kStore = decltype(store)::value;
            const uint64_t steps = pair(-kCodeSteps, -kCodeSteps), magic = pair(kCodeMagic, kCodeMagic);
            uint64_t sum[2] = {0, 0};  // pairs of zeros
#pragma unroll
            for (int j = 0; j < kStatN; j += 2) {
              const uint64_t y = fma2(pair(__uint_as_float(v[j]), __uint_as_float(v[j + 1])), scale, shift);
              float y0, y1;
              unpair(y, y0, y1);
              y0 = ex2_fast(y0);
              y1 = ex2_fast(y1);
              if (kMode == kModeStats) {
                sum[(j >> 1) & 1] = add2(sum[(j >> 1) & 1], pair(y0, y1));
                if (kStore) {
                  float d0, d1;
                  unpair(fma2(y, steps, magic), d0, d1);
                  v[j >> 1] = __byte_perm(clamp_code(d0), clamp_code(d1), 0x5410);
                }
              } else {
                v[j >> 1] = row_ok ? pack2(rq.x * y0, rq.x * y1) : 0u;
              }
            }
            if (kMode == kModeStats && row_ok) {
              float s0_, s1_;
              unpair(add2(sum[0], sum[1]), s0_, s1_);
              P.stats[static_cast<long long>(row) * P.stats_ld + tl.ni * kUnits + unit] = make_float2(m, s0_ + s1_);
            }
          };
          if (kMode == kModeGrad || codes) {
            work(std::true_type{});
            if (kMode == kModeGrad && limit < kStatN) {  // columns past the vocabulary
#pragma unroll
              for (int j = 0; j < kStatN / 2; ++j)
                v[j] &= (2 * j < limit ? 0x0000FFFFu : 0u) | (2 * j + 1 < limit ? 0xFFFF0000u : 0u);
            }
            const int piece = kMode == kModeStats ? tl.ni / P.piece_tiles : 0;
            const int x = (tl.ni - piece * P.piece_tiles) * kTileN + unit * kStatN;
#pragma unroll 1
            for (int r = 0; r < 32 && row0 + r < P.tokens; r += kRows) {
              if (lane == 0) ptx::tma_store_wait_read();  // the previous store has left the buffer
              __syncwarp();
              if ((lane & (32 - kRows)) == r) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                  sts128(staged(buf, lane & (kRows - 1), i), v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
                if (kMode == kModeGrad) {
                  // the entries' gradients replace what the same thread just wrote
                  while (en.col < kStatN) {
                    const __nv_bfloat16 e = __float2bfloat16_rn(P.entry_g[static_cast<long long>(row) * P.top + en.next]);
                    asm volatile("st.shared.b16 [%0], %1;" ::"r"(staged(buf, lane & (kRows - 1), en.col >> 3) + 2u * (en.col & 7)),
                                 "h"(*reinterpret_cast<const unsigned short*>(&e))
                                 : "memory");
                    en.pop(P, col0);
                  }
                }
              }
              ptx::fence_proxy_async_smem();
              __syncwarp();
              if (lane == 0) {
                ptx::tma_store_3d(&P.map_g, x, row0 + r, piece, buf);
                ptx::tma_store_commit();
              }
            }
          } else {
            work(std::false_type{});
          }
        }
        tl = tl_next;
        head = head_next;
        rq = rq_next;
        k += step;
      }
    } else {
      if (kSpare && warp == 2) add_losses(P, n_valid, lane);
      int acc = 0;
      uint32_t acc_phase = 0;
      int turn = 0;  // staging buffer last used
      const float rest = *reinterpret_cast<volatile float*>(&P.ctrl->rest);
      Tile tl;
      for (int k = 0; ok && locate(P, s0, s1, deal, k, tl); ++k) {
        const int row0 = tl.mi * kTileM + static_cast<int>(rank) * 128 + q * 32;
        const bool have_acc = tl.kb0 != tl.kb1;
        if (have_acc) {
          wait_acc(acc, acc_phase);
          if (!ok) break;
        }
        const uint32_t taddr = tmem_row + static_cast<uint32_t>(acc * kAccCols);
        const uint32_t buf0 = ptx::smem_u32(staging + (warp - 2) * 2 * kStageOut);
        const bool is_dx = tl.prod == 0;
        const int n_tile = P.prod[tl.prod].n_tile;
        const int c0 = tl.ni * n_tile;
        // eight warps take half of the columns each
        const int from = kSpare ? (warp - 2) / 4 * (n_tile / 2) : 0;
        const int limit = min(kSpare ? from + n_tile / 2 : n_tile, (is_dx ? P.part_cols : P.dw_cols) - c0);
        const bool rows_ok = is_dx ? row0 < n_valid : row0 < P.dw_rows;
        // two buffers in turn: the store before last has been read
        auto next_buffer = [&]() {
          if (lane == 0) ptx::tma_store_wait_read_all_but_one();
          __syncwarp();
          turn ^= 1;
          return buf0 + static_cast<uint32_t>(turn * kStageOut);
        };
        auto send = [&](uint32_t buf, const CUtensorMap* map, int x, int y, int z, bool add) {
          ptx::fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) {
            if (add) ptx::tma_reduce_add_3d(map, x, y, z, buf);
            else ptx::tma_store_3d(map, x, y, z, buf);
            ptx::tma_store_commit();
          }
        };
        const float factor = is_dx ? 1.0f : rest;
        auto scaled = [&](uint32_t v) { return __uint_as_float(v) * factor; };
        auto load = [&](uint32_t (&v)[32], int c) {
          if (have_acc) {
            ptx::tmem_ld_32x32(taddr + c, v);
          } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = 0u;
          }
        };
        if (rows_ok && (is_dx || (P.dw_fp32 && P.dw_tma))) {
          const CUtensorMap* map = is_dx ? &P.map_part : &P.map_dw;
          const int y = is_dx ? row0 : P.dw_row0 + row0, z = is_dx ? tl.split : 0;
          const bool add = is_dx ? P.part_add != 0 : P.dw_add != 0;
#pragma unroll 1
          for (int c = from; c < limit; c += 32) {
            uint32_t v[32];
            load(v, c);
            ptx::tmem_ld_wait();
            const uint32_t buf = next_buffer();
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(scaled(v[i]));
#pragma unroll
            for (int i = 0; i < 8; ++i) sts128(staged(buf, lane, i), v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
            send(buf, map, c0 + c, y, z, add);
          }
        } else if (rows_ok && P.dw_tma) {
#pragma unroll 1
          for (int c = from; c < limit; c += 64) {
            uint32_t v[32], u[32];
            load(v, c);
            load(u, c + 32);
            ptx::tmem_ld_wait();
            const uint32_t buf = next_buffer();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              uint32_t w[4], z[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                w[e] = pack2(scaled(v[8 * i + 2 * e]), scaled(v[8 * i + 2 * e + 1]));
                z[e] = pack2(scaled(u[8 * i + 2 * e]), scaled(u[8 * i + 2 * e + 1]));
              }
              sts128(staged(buf, lane, i), w[0], w[1], w[2], w[3]);
              sts128(staged(buf, lane, i + 4), z[0], z[1], z[2], z[3]);
            }
            send(buf, &P.map_dw, c0 + c, P.dw_row0 + row0, 0, false);
          }
        } else if (rows_ok) {
          // rows TMA cannot address, or sums into bf16: through shared memory, so that
          // a warp's accesses run along a row
#pragma unroll 1
          for (int c = from; c < limit; c += 32) {
            uint32_t v[32];
            load(v, c);
            ptx::tmem_ld_wait();
            if (lane == 0) ptx::tma_store_wait_read();
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 32; ++i)
              sts32(buf0 + 4u * (lane * 32 + (i ^ lane)), __float_as_uint(scaled(v[i])));
            __syncwarp();
            const int rows = min(32, P.dw_rows - row0);
            if (c + lane < limit) {
              long long off = static_cast<long long>(P.dw_row0 + row0) * P.ld_dw + c0 + c + lane;
#pragma unroll 4
              for (int r = 0; r < rows; ++r, off += P.ld_dw) {
                const float y = lds32(buf0 + 4u * (r * 32 + (lane ^ r)));
                if (P.dw_fp32) {
                  float* d = static_cast<float*>(P.dw) + off;
                  *d = P.dw_add ? *d + y : y;
                } else {
                  __nv_bfloat16* d = static_cast<__nv_bfloat16*>(P.dw) + off;
                  *d = __float2bfloat16_rn(P.dw_add ? __bfloat162float(*d) + y : y);
                }
              }
            }
            __syncwarp();
          }
        }
        if (have_acc) {
          release(acc);
          if (++acc == kNumAcc) {
            acc = 0;
            acc_phase ^= 1u;
          }
        }
      }
    }
    if (lane == 0) ptx::tma_store_wait_all();
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

template <int kMode, bool kSpare = false, bool kList = false>
cudaError_t configure_one() {
  return cudaFuncSetAttribute(head_gemm_kernel<kMode, kSpare, kList>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              Config<kMode, kSpare>::kSmemBytes);
}

template <int kMode, bool kSpare = false, bool kList = false>
cudaError_t launch_one(const GemmParams& P, unsigned clusters, bool overlap, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(2 * clusters, 1, 1);
  cfg.blockDim = dim3(Config<kMode, kSpare>::kThreads, 1, 1);
  cfg.dynamicSmemBytes = Config<kMode, kSpare>::kSmemBytes;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = overlap ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, head_gemm_kernel<kMode, kSpare, kList>, P);
}

}  // namespace

cudaError_t gemm_configure() {
  cudaError_t e = configure_one<kModeStats>();
  if (e == cudaSuccess) e = configure_one<kModeStats, true>();
  if (e == cudaSuccess) e = configure_one<kModeStats, true, true>();
  if (e == cudaSuccess) e = configure_one<kModeGrad>();
  if (e == cudaSuccess) e = configure_one<kModeOut>();
  if (e == cudaSuccess) e = configure_one<kModeOut, true>();
  return e;
}

// Largest number of co-resident CTA pairs (one CTA per SM).
cudaError_t gemm_max_clusters(int* out) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(2, 1, 1);
  cfg.blockDim = dim3(Config<kModeOut, false>::kThreads, 1, 1);
  cfg.dynamicSmemBytes = Config<kModeOut, false>::kSmemBytes;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = 2;
  attr.val.clusterDim.y = 1;
  attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaOccupancyMaxActiveClusters(out, head_gemm_kernel<kModeOut, false, false>, &cfg);
}

// Rows of a box in which the statistics' codes are stored: one row tile reads w from
// memory once, more share it in L2.
int stats_rows(int tokens) { return tokens <= kTileM ? 16 : 32; }

// `tiles`: an upper bound on the launch's tiles (every token counts).  overlap: an earlier
// kernel of the call is what it waits for.
cudaError_t launch_gemm(int mode, const GemmParams& P, long long tiles, int max_clusters, bool overlap, cudaStream_t stream) {
  if (tiles <= 0) return cudaSuccess;
  const unsigned clusters = static_cast<unsigned>(tiles < max_clusters ? tiles : max_clusters);
  if (mode == kModeStats) {
    if (P.ids64 != nullptr) return launch_one<kModeStats, true, true>(P, clusters, overlap, stream);
    return stats_rows(P.tokens) == 16 ? launch_one<kModeStats, true>(P, clusters, overlap, stream)
                                      : launch_one<kModeStats>(P, clusters, overlap, stream);
  }
  if (mode == kModeGrad) return launch_one<kModeGrad>(P, clusters, overlap, stream);
  return P.spare ? launch_one<kModeOut, true>(P, clusters, overlap, stream)
                 : launch_one<kModeOut>(P, clusters, overlap, stream);
}

}  // namespace head
}  // namespace muon
