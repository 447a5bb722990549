// Structures shared by the host side and the kernels of the losses at the LM
// head (softmax cross entropy, distillation from a teacher's top logits).
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace muon {
namespace head {

constexpr int kTileM = 256;   // output rows of a CTA pair's tile (128 per CTA)
constexpr int kTileN = 256;   // widest output tile
constexpr int kStatN = 64;    // vocabulary columns of one statistics entry: what an epilogue thread holds of a row
constexpr int kUnits = kTileN / kStatN;
constexpr int kBK = 64;       // K elements per pipeline stage (128 bytes of bf16)
constexpr int kTileCost = 6;  // K blocks that a tile's epilogue and start are worth, to the plan and to the dealing of tiles
// Fewer tokens than this are finalised by several blocks a row, whose conversion spreads
// over the device: two a SM, and more than are ever left in place.  (Whole calls, us, with
// and without: 90 and 100 for 290 x 512 x 50000, 256 and 271 for 290 x 1024 x 100000; 131
// and 130 for 400 x 2048 x 20000, 133 and 131 for 600 x 512 x 50000.)
constexpr int kFusedRows = 296;
// From here on the tokens that count are counted in runs of 256 first, a launch more.  (Whole
// calls, us, with and without, x 64 x 2000: 30.7 and 30.9 for 1000 tokens, 146 and 169 for
// 16384, 533 and 878 for 65536.)
constexpr int kManyTokens = 16384;
// Most tokens whose rows are not gathered (one thread of a block looks at each), and most of
// a teacher's entries in all: every block looks at all of them.  (Whole calls, us, in place
// and gathered, x 256 x 4096: 24.6 and 32.7 for 20 tokens with 16 entries, 41.0 and 40.9 for
// 100 with 32, 54 and 49 for 100 with 64, 92 and 68 for 250 with 128.)
constexpr int kInPlaceRows = 256;
constexpr int kInPlaceEntries = 4096;
static_assert(kInPlaceRows < kFusedRows, "rows in place are converted by the finalisation of few tokens");
constexpr long long kHeadInCache = 96ll << 20;   // bytes of w that do, between its two readings
constexpr int kMaxTop = 128;  // sparse target entries of one token
constexpr int kNoId = 0x7FFFFFFF;  // sorted after every vocabulary index: an entry that does not count

// Control block at the start of the workspace.
struct Ctrl {
  int status;      // 0 or MUON_ERR_TIMEOUT
  int n_valid;     // tokens that count
  unsigned ticket; // blocks of the finalisation that are done
  float coef;      // scale, divided by the sum of the weights where a mean is asked for
  float rest;      // what dX and dW are still to be multiplied with, see finalise_kernel
};

// One product of a launch: D[m][n] = sum_k A[m][k] B[n][k].
struct Product {
  CUtensorMap map_a, map_b;
  int a_mn, b_mn;    // operand stored with M (N) contiguous instead of K
  int a_rows;        // rows of a box of operand A (K contiguous): 128, or what few tokens need
  int n_tile;        // 128 or 256
  int m_tiles;       // row tiles of 256; -1: from the number of tokens that count
  int n_tiles;
  int k_blocks;      // K blocks of 64 in all; -1: from the number of tokens that count
  int splits;        // the K blocks are cut into this many runs, each its own tile
  int a_z;           // third coordinate of operand A (buffer of the vocabulary piece)
  int b_k0;          // first K coordinate of operand B (vocabulary piece in W)
  int b_n0;          // first row of operand B
  int group;         // row tiles that are walked together for each column tile
  int swap_order;    // walk the column tiles innermost
};

// A piece of the vocabulary whose logits are kept as codes (head_codes.cuh), to be
// turned into the bf16 gradient of the logits in place.
struct ConvertParams {
  __nv_bfloat16* g;  // [token][ld]; NULL: nothing to convert
  long long ld;
  int tiles;         // 256-column tiles of the piece
  int v_tile0;       // its first tile in the vocabulary
  const float2* row_q;
  const float2* stats;
  int stats_ld;
  int top;
  const int* ids;
  const float* entry_g;
  const unsigned char* starts;
  int n_starts;
};

enum { kModeStats = 0, kModeGrad = 1, kModeOut = 2 };

struct GemmParams {
  Product prod[2];
  int n_prod;
  int by_tile;  // statistics, gradient: see the epilogue
  int spare;    // outputs: nothing to convert, see Config
  Ctrl* ctrl;

  int tokens;
  // Few tokens: the statistics run on x as it is, before anything else, every token a
  // row, and find the sparse entries in the caller's list; otherwise ids64 is NULL
  const int64_t* ids64;  // [token][top], row stride ld_ids64
  long long ld_ids64;
  int in_place;          // rows are tokens (few tokens), not the gathered ones

  // statistics and gradient of the logits
  int vocab;          // columns of the whole problem
  int v0;             // first vocabulary column of this launch
  float scale2;       // logit scale * log2(e)
  int top;            // sparse entries per token; 1: one target
  const int* ids;     // [token][top], ascending within a row
  const unsigned char* starts;  // [token][n_starts]: entries below each 256-column tile (top > 1)
  int n_starts;
  float* entry_logit; // [token][top] raw logit of each entry
  float2* stats;      // [token][stats_ld]: maximum and sum of exponentials per kStatN columns
  int stats_ld;
  const float2* row_q;   // [token]: coefficient of q, log2 of the softmax denominator
  const float* entry_g;  // [token][top]: gradient of the logit at the entry
  // Piece buffers [buffer][token][piece columns], box {64, stats_rows} or
  // {64, 32}: where the
  // gradient of one piece's logits is stored, or the codes of the logits of the
  // first `code_tiles` tiles, in pieces of piece_tiles tiles.
  CUtensorMap map_g;
  int code_tiles, piece_tiles;
  // outputs: the next piece's codes are converted while the products run, and the
  // tokens' weighted losses added up
  ConvertParams convert;
  const float* row_l;
  float* total;       // NULL: not here

  // product 0 of kModeOut: partial dX, fp32 [split][token][cols], box {32, 32}
  CUtensorMap map_part;
  int part_cols;
  int part_add;       // add to what an earlier piece left
  // product 1 of kModeOut: dW, box {64, 32} bf16 or {32, 32} fp32
  CUtensorMap map_dw;
  void* dw;
  long long ld_dw;
  int dw_fp32, dw_add, dw_tma;  // dw_tma: tiles leave through map_dw, else element by element
  int dw_row0, dw_rows, dw_cols;
};

struct RowParams {
  Ctrl* ctrl;
  int tokens, dim, vocab;
  const __nv_bfloat16* x;
  long long ld_x;
  const __nv_bfloat16* w;  // head with 16-byte aligned rows
  long long ld_w;
  // where the caller's has none: the copy that w points to, and what it is made from
  __nv_bfloat16* pack_to;
  const __nv_bfloat16* pack_from;
  long long ld_pack;
  int pack_blocks;
  __nv_bfloat16* xc;     // [token][ld_xc] rows of the tokens that count, then zeros to the next K block
  long long ld_xc;
  int x_vec;             // rows can be copied in 16-byte pieces
  int in_place;          // few tokens: rows are tokens, nothing is gathered
  const int64_t* ids_in; // [tokens][top]
  long long ld_ids;
  const void* z;         // teacher logits [tokens][top], NULL: one target per token
  long long ld_z;
  int z_fp32;
  const float* teacher_lse;
  float inv_t;           // 1 / temperature
  int top;
  const float* weight;
  float scale;
  int mean;
  unsigned char* flags;  // [tokens] token counts (distillation)
  int* run_counts;       // many tokens: how many count in every run of 256, else NULL
  int* row_of;           // [row]: its token; in_place: the row itself or, masked, -1
  int* ids;              // [token][top]
  float* p;              // [token][top]
  float* row_h;          // [token]: sum p log p
  float* row_c;          // [token]: sum p
  unsigned char* starts;
  int n_starts;
  float* entry_logit;
  float2* stats;
  int stats_ld, stats_n;
  float scale2;          // logit scale * log2(e)
  float logit_scale;
  float z_loss;
  float2* row_q;
  float* entry_g;
  float* row_l;          // [token]: coefficient * loss
  float* loss;           // [tokens]
  float* lse;            // [tokens] or NULL
  float* total;          // [1] or NULL
  // dX: rows of tokens that do not count become zeros
  void* dx;
  long long ld_dx;
  int dx_fp32, dx_vec;
  const float* part;     // partial dX of each run of K blocks
  long long part_ld, part_stride;
  int splits;
};

cudaError_t gemm_configure();
cudaError_t gemm_max_clusters(int* out);
int stats_rows(int tokens);
cudaError_t launch_gemm(int mode, const GemmParams& P, long long tiles, int max_clusters, bool overlap,
                        cudaStream_t stream);

cudaError_t launch_flags(const RowParams& R, cudaStream_t stream);
cudaError_t launch_count(const RowParams& R, bool overlap, cudaStream_t stream);
cudaError_t launch_prepare(const RowParams& R, bool after_flags, cudaStream_t stream);
cudaError_t launch_finalise(const RowParams& R, const ConvertParams& C, int sms, cudaStream_t stream);
cudaError_t launch_dx(const RowParams& R, cudaStream_t stream);
cudaError_t launch_pack(const RowParams& R, cudaStream_t stream);
int pack_blocks(int vocab);

}  // namespace head
}  // namespace muon
