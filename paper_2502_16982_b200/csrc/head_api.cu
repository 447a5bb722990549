// Host side of the LM-head losses and of the log probabilities at the head: argument
// checks, the plan (vocabulary pieces, splits, workspace layout) and the launch sequence.
#include <cuda.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "../../include/muon.h"
#include "head.h"

namespace muon {
void set_last_error(const char* msg);
}

namespace {

using namespace muon::head;

int fail(int code, const char* fmt, ...) {
  char buf[256];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  muon::set_last_error(buf);
  return code;
}

long long round_up(long long v, long long to) { return (v + to - 1) / to * to; }

// Bytes of logit gradients (bf16) that one vocabulary piece takes, at most, and of
// the pieces together whose logits are kept as codes in the workspace that
// muon_head_workspace_bytes asks for, their statistics (a sixteenth) included.
constexpr long long kPieceBytes = 1ll << 28;
constexpr long long kCodeBytes = 3ll << 30;
long long g_piece_bytes = kPieceBytes;
int g_codes = 0;
// Bytes of partial dX that splitting its long axis may take.
constexpr long long kPartBytes = 1ll << 28;

// What a call computes: a loss, with or without its gradients; log probabilities; or the
// gradients of log probabilities that an earlier call computed.
enum Kind { kLoss, kLogprob, kLogprobGrad };

struct Plan {
  Kind kind;
  int tokens, rows, m_tiles, dim, vocab, top;  // rows: tokens, at least 1
  bool want_dx, want_dw, grads, distill, pack, in_place;
  int v_tiles;               // 256-column tiles of the vocabulary
  int piece_tiles, n_pieces;
  int n_stored, n_buffers;   // pieces kept as codes; piece buffers in the workspace
  int splits, dx_n_tile, dx_n_tiles;
  long long ld_xc, ld_wc, part_ld, part_stride;
  size_t ctrl, xc, wc, flags, run_counts, row_of, ids, p, row_h, row_c, starts, entry_logit, entry_g, stats, stats_e, row_q, row_b, row_l, g,
      part, bytes, least;
};

// How many runs the K blocks of dX's tiles are cut into.  dX has few tiles with
// a long axis (the vocabulary piece), dW many with a short one; the launch deals
// them out evenly (head_gemm.cu).  The number with the smallest load of the fullest
// CTA pair is taken, a tile counted as its K blocks plus kTileCost for its
// epilogue, dX's long tiles a quarter dearer where a pair waits for them alone -
// three times as dear with one row tile, whose w comes from memory and is not shared,
// so that all pairs should read - and `split_cost` for each partial sum that is joined.
// Measured at 1024 x 2560 x 65536 (1 split chosen): 769 us with 1, 799 with 2, 837
// with 4; at 1 x 512 x 8192: 39 us with 8, 35 with 16 and with 32.
int choose_splits(int m_tiles, int n_tiles, int dx_kb, long long dw_tiles, int dw_kb, int pairs, int most, double split_cost) {
  const long long dx_tiles = static_cast<long long>(m_tiles) * n_tiles;
  const double wait = m_tiles == 1 ? 3.0 : 1.25;
  int best = 1;
  double best_load = -1;
  for (int s = 1; s <= most; ++s) {
    if (s > 1 && dx_kb / s < 4) break;
    const long long nx = dx_tiles * s;
    const int cx = (dx_kb + s - 1) / s + kTileCost, cw = dw_kb + kTileCost;
    const double even = (static_cast<double>(nx) * cx + static_cast<double>(dw_tiles) * cw) / pairs + (dw_tiles ? cw / 2 : 0);
    const double fullest = wait * static_cast<double>((nx + pairs - 1) / pairs) * cx;
    double load = even > fullest ? even : fullest;
    load += s * split_cost;
    if (best_load < 0 || load < best_load) {
      best_load = load;
      best = s;
    }
  }
  return best;
}

// Codes or a second product x w^T?  The second product costs 2 dim FLOPs for every
// logit, the codes 2 bytes written and 4 bytes of conversion, and in a short call a
// launch more against one fewer.  Measured, second product against codes, us: 4718 and
// 3932 for 8192 x 1024 x 100000, 2711 and 2633 at 512 columns, 2442 and 2488 at 384;
// 55.0 and 55.0 for 2000 x 256 x 5000, 47.0 and 43.0 for 500 x 256 x 13000; 85 and 80 for
// 100 x 64 x 163840, whose tokens are not gathered.
constexpr int kCodesDim = 448;
constexpr long long kFewCodes = 20ll << 20;
bool want_codes(int tokens, int dim, int vocab) {
  if (g_codes != 0) return g_codes == 2;
  return dim >= kCodesDim || tokens <= kInPlaceRows || 2ll * tokens * vocab <= kFewCodes;
}

// `room`: bytes of workspace to plan for; 0 plans for as many as are useful.
int make_plan(const muon_head_args* a, int top, bool distill, int pairs, size_t room, Plan* P, Kind kind = kLoss,
              bool entropy = false, bool keep = false) {
  P->kind = kind;
  P->tokens = a->tokens;
  P->dim = a->dim;
  P->vocab = a->vocab;
  P->top = top;
  P->distill = distill;
  P->rows = a->tokens > 0 ? a->tokens : 1;
  P->m_tiles = (a->tokens + kTileM - 1) / kTileM;
  P->want_dx = a->dx != nullptr && a->tokens > 0;
  P->want_dw = a->dw != nullptr;
  P->grads = P->want_dx || P->want_dw;
  P->pack = (reinterpret_cast<uintptr_t>(a->w) & 15) != 0 || (a->ld_w & 7) != 0;
  P->v_tiles = static_cast<int>((static_cast<long long>(a->vocab) + kTileN - 1) / kTileN);
  P->ld_xc = round_up(a->dim, 8);
  P->ld_wc = round_up(a->dim, 8);
  P->part_ld = round_up(a->dim, 8);
  P->part_stride = P->rows * P->part_ld;

  long long tiles = g_piece_bytes / (2ll * P->rows * kTileN);
  if (tiles < 1) tiles = 1;
  if (tiles > P->v_tiles) tiles = P->v_tiles;
  P->n_pieces = static_cast<int>((P->v_tiles + tiles - 1) / tiles);
  P->piece_tiles = (P->v_tiles + P->n_pieces - 1) / P->n_pieces;
  P->n_pieces = (P->v_tiles + P->piece_tiles - 1) / P->piece_tiles;

  P->dx_n_tile = a->dim <= 128 ? 128 : 256;
  P->dx_n_tiles = (a->dim + P->dx_n_tile - 1) / P->dx_n_tile;
  P->splits = 1;
  if (P->want_dx) {
    long long most = kPartBytes / (P->part_stride * 4);
    most = most < 1 ? 1 : (most > 64 ? 64 : most);
    // a partial sum costs its bytes (1.7 MB in the time of a K block, 0.27 us) once a call
    // and its place in the loop that joins them
    const double split_cost = 1.0 + static_cast<double>(P->part_stride) * 4 / 1.7e6 / P->n_pieces;
    P->splits = choose_splits(P->m_tiles, P->dx_n_tiles, P->piece_tiles * (kTileN / kBK),
                              P->want_dw ? static_cast<long long>(P->piece_tiles) * P->dx_n_tiles : 0,
                              (P->tokens + kBK - 1) / kBK, pairs, static_cast<int>(most), split_cost);
  }

  const size_t rows = static_cast<size_t>(P->rows), entries = rows * top;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off = static_cast<size_t>(round_up(static_cast<long long>(off + bytes), 1024));
    return at;
  };
  P->ctrl = take(sizeof(Ctrl));
  // `keep` of a gradient: what the forward pass kept is not formed again
  const bool gather = !(kind == kLogprobGrad && keep);
  P->xc = take(gather ? rows * P->ld_xc * 2 : 0);
  P->row_of = take(gather ? rows * 4 : 0);
  P->run_counts = take(gather && P->tokens >= kManyTokens ? (rows / 256 + 1) * 4 : 0);
  P->ids = take(gather ? entries * 4 : 0);
  // the gradient of log probabilities starts from what an earlier call left with the caller
  const size_t units = kind == kLogprobGrad ? 0 : rows * P->v_tiles * kUnits;
  P->entry_logit = take(entries * 4);
  P->entry_g = take(entries * 4);
  P->stats = take(units * sizeof(float2));
  P->row_q = take(rows * sizeof(float2));
  P->row_b = take(kind == kLogprobGrad ? rows * 4 : 0);
  P->row_l = take(rows * 4);
  P->flags = P->p = P->row_h = P->row_c = P->starts = P->wc = P->g = P->part = 0;
  if (distill) {
    P->flags = take(rows);
    P->p = take(entries * 4);
    P->row_h = take(rows * 4);
    P->row_c = take(rows * 4);
    P->starts = take(rows * (P->v_tiles + 1));
  }
  if (P->pack && gather) P->wc = take(static_cast<size_t>(a->vocab) * P->ld_wc * 2);
  // Where no second piece is kept as codes nothing reads the statistics after the
  // finalisation, and partial dX may lie in their place.
  const size_t part_bytes = P->want_dx ? static_cast<size_t>(P->splits) * P->part_stride * 4 : 0;
  const size_t stats_bytes = units * sizeof(float2);
  const bool share = part_bytes > 0 && stats_bytes >= part_bytes;
  const size_t apart = static_cast<size_t>(round_up(static_cast<long long>(part_bytes), 1024));
  P->n_stored = P->n_buffers = 0;
  const long long one = static_cast<long long>(rows) * P->piece_tiles * kTileN * 2;
  if (kind == kLogprob && keep && want_codes(P->tokens, P->dim, P->vocab)) {
    const long long fit = (kCodeBytes - static_cast<long long>(stats_bytes)) / one;
    P->n_stored = static_cast<int>(fit < 0 ? 0 : (fit > P->n_pieces ? P->n_pieces : fit));
    P->n_buffers = P->n_stored;
    P->g = take(static_cast<size_t>(one) * P->n_stored);
  }
  P->stats_e = take(entropy ? units * 4 : 0);  // behind what is kept
  P->least = off;
  if (P->grads) {
    // two in turn, where codes that stay are converted while the products of the other run
    P->n_buffers = kind == kLogprobGrad && keep && P->n_pieces > 1 ? 2 : 1;
    if (kind == kLoss && want_codes(P->tokens, P->dim, P->vocab)) {
      long long fit = (room ? static_cast<long long>(room) - static_cast<long long>(off + apart)
                            : kCodeBytes - static_cast<long long>(stats_bytes)) / one;
      P->n_buffers = static_cast<int>(fit < 1 ? 1 : (fit > P->n_pieces ? P->n_pieces : fit));
      P->n_stored = P->n_buffers;
    }
    P->least = off + (share ? 0 : apart) + static_cast<size_t>(round_up(one * (kind == kLogprobGrad ? P->n_buffers : 1), 1024));
    if (part_bytes) P->part = share && P->n_stored <= 1 ? P->stats : take(part_bytes);
    P->g = take(static_cast<size_t>(one) * P->n_buffers);
  }
  // few tokens with rows that TMA can address, and nothing but codes between the passes
  P->in_place = a->tokens > 0 && a->tokens <= kInPlaceRows && static_cast<long long>(a->tokens) * top <= kInPlaceEntries &&
                (reinterpret_cast<uintptr_t>(a->x) & 15) == 0 && (a->ld_x & 7) == 0 &&
                (!P->grads || (P->n_pieces == 1 && P->n_stored == 1)) && !keep;
  P->bytes = off;
  return MUON_OK;
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_fn() {
  static EncodeTiledFn fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess)
      p = nullptr;
    return reinterpret_cast<EncodeTiledFn>(p);
  }();
  return fn;
}

// bf16 or fp32 matrices [count][rows][cols] with row pitch ld, one behind the
// other, 128-byte swizzled boxes of 128 bytes x box_rows.
int encode(CUtensorMap* out, const void* base, long long count, long long rows, long long cols, long long ld,
           int box_rows, bool fp32 = false) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return fail(MUON_ERR_CUDA, "cuTensorMapEncodeTiled entry point not available");
  const cuuint64_t pitch = static_cast<cuuint64_t>(ld) * (fp32 ? 4 : 2);
  cuuint64_t dims[3] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows), static_cast<cuuint64_t>(count)};
  cuuint64_t strides[2] = {pitch, pitch * static_cast<cuuint64_t>(rows)};
  cuuint32_t box[3] = {fp32 ? 32u : 64u, static_cast<cuuint32_t>(box_rows), 1};
  cuuint32_t estr[3] = {1, 1, 1};
  CUresult r = fn(out, fp32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3,
                  const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) return fail(MUON_ERR_CUDA, "cuTensorMapEncodeTiled failed with CUresult %d", static_cast<int>(r));
  return MUON_OK;
}

// CTA pairs that fit the device, looked up once per device.
int device_pairs(int device, int* out) {
  constexpr int kMaxDevices = 64;
  static int cached[kMaxDevices] = {};
  if (device < 0 || device >= kMaxDevices) return fail(MUON_ERR_INVALID_ARG, "device ordinal %d", device);
  if (cached[device] == 0) {
    cudaError_t e = gemm_configure();
    int n = 0;
    if (e == cudaSuccess) e = gemm_max_clusters(&n);
    if (e != cudaSuccess) return fail(MUON_ERR_CUDA, "%s", cudaGetErrorString(e));
    if (n < 1) return fail(MUON_ERR_CUDA, "no CTA pair fits the device");
    cached[device] = n;
  }
  *out = cached[device];
  return MUON_OK;
}

// Pairs assumed where the workspace is sized: the plan must not depend on the device.
constexpr int kPlanPairs = 74;

bool misaligned(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }

int check(const muon_head_args* a, int top, bool need_ptrs) {
  if (!a) return fail(MUON_ERR_INVALID_ARG, "args is null");
  if (a->tokens < 0 || a->dim <= 0 || a->vocab <= 0)
    return fail(MUON_ERR_INVALID_ARG, "tokens must not be negative, dim and vocab must be positive");
  if (a->tokens > (1 << 24) || a->dim > (1 << 20) || a->vocab > (1 << 24))
    return fail(MUON_ERR_UNSUPPORTED, "more than 2^24 tokens, 2^24 vocabulary entries or 2^20 dimensions");
  if (top < 1 || top > kMaxTop) return fail(MUON_ERR_UNSUPPORTED, "1 to %d teacher entries per token", kMaxTop);
  if (a->x_dtype != MUON_DTYPE_BF16 || a->w_dtype != MUON_DTYPE_BF16)
    return fail(MUON_ERR_UNSUPPORTED, "x and w must be bf16 (fp32 weights: pass their bf16 copy)");
  if ((a->dx_dtype != MUON_DTYPE_BF16 && a->dx_dtype != MUON_DTYPE_FP32) ||
      (a->dw_dtype != MUON_DTYPE_BF16 && a->dw_dtype != MUON_DTYPE_FP32))
    return fail(MUON_ERR_UNSUPPORTED, "gradients must be bf16 or fp32");
  if (!need_ptrs) return MUON_OK;
  if (!a->w || (a->tokens > 0 && (!a->x || !a->loss))) return fail(MUON_ERR_INVALID_ARG, "x, w or loss is null");
  if (a->ld_w < a->dim || (a->tokens > 0 && a->ld_x < a->dim) || (a->dx && a->tokens > 0 && a->ld_dx < a->dim) ||
      (a->dw && a->ld_dw < a->dim))
    return fail(MUON_ERR_INVALID_ARG, "a row stride is smaller than dim");
  if (!std::isfinite(a->scale) || !std::isfinite(a->logit_scale) || !(a->logit_scale > 0.f))
    return fail(MUON_ERR_INVALID_ARG, "scale must be finite, logit_scale finite and positive");
  if (misaligned(a->x, 2) || misaligned(a->w, 2) || misaligned(a->weight, 4) || misaligned(a->loss, 4) ||
      misaligned(a->lse, 4) || misaligned(a->total, 4) || misaligned(a->dx, a->dx_dtype == MUON_DTYPE_FP32 ? 4 : 2) ||
      misaligned(a->dw, a->dw_dtype == MUON_DTYPE_FP32 ? 4 : 2))
    return fail(MUON_ERR_ALIGNMENT, "pointer not aligned to its element size");
  return MUON_OK;
}

// logit_scale / temperature, and the same times log2(e) for exponents of 2.
float logit_scale_of(const muon_head_args* a, const muon_head_teacher* t) {
  return t ? a->logit_scale / t->temperature : a->logit_scale;
}
float scale2_of(float logit_scale) { return static_cast<float>(logit_scale * 1.4426950408889634); }

// As numbers that fp32 holds: with 0 or infinity in their place every row would be NaN.
int check_scale(const muon_head_args* a, const muon_head_teacher* t) {
  const float scale2 = scale2_of(logit_scale_of(a, t));
  if (!std::isfinite(scale2) || scale2 == 0.f || (t && !std::isfinite(1.0f / t->temperature)))
    return fail(MUON_ERR_INVALID_ARG, "logit_scale / temperature: 0 or infinite in fp32");
  return MUON_OK;
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

#define HEAD_CUDA(call)                                                              \
  do {                                                                               \
    cudaError_t e_ = (call);                                                         \
    if (e_ != cudaSuccess) return fail(MUON_ERR_CUDA, "%s", cudaGetErrorString(e_)); \
  } while (0)
#define HEAD_TRY(call)             \
  do {                             \
    int rc_ = (call);              \
    if (rc_ != MUON_OK) return rc_; \
  } while (0)

// l, d: log probabilities, and their gradients; NULL for a loss.
int run(const muon_head_args* a, const muon_head_teacher* t, const int64_t* targets, float z_loss, const muon_logprob_args* l,
        const muon_logprob_grads* d, void* workspace, size_t workspace_bytes, int device, cudaStream_t stream) {
  const bool distill = t != nullptr;
  const int top = distill ? t->top : 1;
  const Kind kind = d ? kLogprobGrad : l ? kLogprob : kLoss;
  const bool entropy = kind == kLogprob && l->entropy, keep = l && (d ? d->kept != nullptr : l->keep != 0);
  Plan P, K = {};  // K: of the forward pass that kept its logits
  HEAD_TRY(make_plan(a, top, distill, kPlanPairs, workspace_bytes ? workspace_bytes : 1, &P, kind, entropy, keep));
  if (!workspace || workspace_bytes < P.least || misaligned(workspace, 1024))
    return fail(MUON_ERR_WORKSPACE, "workspace: need at least %zu bytes, 1024-byte aligned", P.least);
  char* ws = static_cast<char*>(workspace);
  char* kept = nullptr;
  if (d && keep) {
    muon_head_args forward = *a;
    forward.dx = forward.dw = nullptr;
    HEAD_TRY(make_plan(&forward, 1, false, kPlanPairs, 1, &K, kLogprob, false, true));
    if (d->kept_bytes < K.least || misaligned(d->kept, 1024))
      return fail(MUON_ERR_WORKSPACE, "kept: need the workspace of the forward pass, %zu bytes", K.least);
    kept = static_cast<char*>(const_cast<void*>(d->kept));  // only read
    if (kept < ws + P.bytes && ws < kept + K.least) return fail(MUON_ERR_WORKSPACE, "workspace and kept overlap");
  }
  DeviceGuard guard;
  HEAD_CUDA(guard.set(device));
  int pairs = 0;
  HEAD_TRY(device_pairs(device, &pairs));

  const void* w = a->w;
  long long ld_w = a->ld_w;
  if (P.pack) {
    w = kept ? kept + K.wc : ws + P.wc;
    ld_w = P.ld_wc;
  }
  const float logit_scale = logit_scale_of(a, t);

  RowParams R = {};
  R.ctrl = reinterpret_cast<Ctrl*>(ws + P.ctrl);
  R.tokens = P.tokens;
  R.dim = P.dim;
  R.vocab = P.vocab;
  R.x = static_cast<const __nv_bfloat16*>(a->x);
  R.ld_x = a->ld_x;
  R.w = static_cast<const __nv_bfloat16*>(w);
  R.ld_w = ld_w;
  R.xc = reinterpret_cast<__nv_bfloat16*>(ws + P.xc);
  R.ld_xc = P.ld_xc;
  R.x_vec = !misaligned(a->x, 16) && (a->ld_x & 7) == 0;
  R.ids_in = distill ? t->top_ids : targets;
  R.ld_ids = distill ? t->ld_ids : 1;
  R.z = distill ? t->top_logits : nullptr;
  R.ld_z = distill ? t->ld_logits : 0;
  R.z_fp32 = distill && t->logits_dtype == MUON_DTYPE_FP32;
  R.teacher_lse = distill ? t->teacher_lse : nullptr;
  R.inv_t = distill ? 1.0f / t->temperature : 1.0f;
  R.top = top;
  R.weight = a->weight;
  R.scale = a->scale;
  R.mean = a->mean;
  R.flags = nullptr;
  R.row_of = reinterpret_cast<int*>(ws + P.row_of);
  R.ids = reinterpret_cast<int*>(ws + P.ids);
  R.p = reinterpret_cast<float*>(ws + P.p);
  R.row_h = reinterpret_cast<float*>(ws + P.row_h);
  R.row_c = reinterpret_cast<float*>(ws + P.row_c);
  R.starts = reinterpret_cast<unsigned char*>(ws + P.starts);
  R.n_starts = P.v_tiles + 1;
  R.entry_logit = reinterpret_cast<float*>(ws + P.entry_logit);
  R.stats = reinterpret_cast<float2*>(ws + P.stats);
  R.stats_ld = R.stats_n = kUnits * P.v_tiles;
  R.scale2 = scale2_of(logit_scale);
  R.logit_scale = logit_scale;
  R.z_loss = z_loss;
  R.row_q = reinterpret_cast<float2*>(ws + P.row_q);
  R.entry_g = reinterpret_cast<float*>(ws + P.entry_g);
  R.row_l = reinterpret_cast<float*>(ws + P.row_l);
  R.loss = a->loss;
  R.lse = a->lse;
  R.total = a->total;
  if (l) {
    R.row_b = reinterpret_cast<float*>(ws + P.row_b);
    if (keep) {
      const Plan& F = d ? K : P;
      R.keeps = Kept{F.tokens, F.dim, F.vocab, F.pack, F.piece_tiles, F.n_stored, R.scale2};
    }
    if (d) {
      R.logprob_in = l->logprob;
      R.entropy_in = l->entropy;
      R.lse_in = l->lse;
      R.g_logprob = d->g_logprob;
      R.g_entropy = d->g_entropy;
      R.loss = R.lse = nullptr;
      if (kept) {
        R.kept = reinterpret_cast<const Ctrl*>(kept + K.ctrl);
        R.xc = reinterpret_cast<__nv_bfloat16*>(kept + K.xc);
        R.row_of = reinterpret_cast<int*>(kept + K.row_of);
        R.ids = reinterpret_cast<int*>(kept + K.ids);
        R.stats = reinterpret_cast<float2*>(kept + K.stats);
      }
    } else if (entropy) {
      R.entropy = l->entropy;
      R.stats_e = reinterpret_cast<const float*>(ws + P.stats_e);
    }
  }
  R.dx = P.want_dx ? a->dx : nullptr;
  R.ld_dx = a->ld_dx;
  R.dx_fp32 = a->dx_dtype == MUON_DTYPE_FP32;
  R.dx_vec = !misaligned(a->dx, 16) && (a->ld_dx & (R.dx_fp32 ? 3 : 7)) == 0;
  R.part = reinterpret_cast<const float*>(ws + P.part);
  R.part_ld = P.part_ld;
  R.part_stride = P.part_stride;
  R.splits = P.splits;

  GemmParams S = {};
  S.n_prod = 1;
  S.ctrl = R.ctrl;
  S.tokens = P.tokens;
  S.vocab = P.vocab;
  S.scale2 = R.scale2;
  S.top = top;
  S.ids = R.ids;
  S.starts = R.starts;
  S.n_starts = R.n_starts;
  S.entry_logit = R.entry_logit;
  S.stats = R.stats;
  S.stats_ld = R.stats_ld;
  S.row_q = R.row_q;
  S.entry_g = R.entry_g;
  if (entropy) S.stats_e = reinterpret_cast<float*>(ws + P.stats_e);
  if (d) S.row_b = R.row_b;
  __nv_bfloat16* const g = reinterpret_cast<__nv_bfloat16*>(ws + P.g);
  const long long g_ld = static_cast<long long>(P.piece_tiles) * kTileN;
  S.piece_tiles = P.piece_tiles;
  auto tiles_of = [&](int piece) {
    const int left = P.v_tiles - piece * P.piece_tiles;
    return left < P.piece_tiles ? left : P.piece_tiles;
  };
  S.code_tiles = P.n_stored * P.piece_tiles < P.v_tiles ? P.n_stored * P.piece_tiles : P.v_tiles;
  if (P.n_buffers > 0) HEAD_TRY(encode(&S.map_g, g, P.n_buffers, P.rows, g_ld, g_ld, stats_rows(P.tokens)));
  // Fewer than 32 tokens: boxes of operand A that hold no more rows than there are; what a
  // slot holds past them reaches only rows of the accumulator that nothing reads.  (A box of
  // 128 rows over a tensor of fewer than 32 made the statistics of 10 x 2048 x 163840 take
  // 172 us in place of 117, the whole call of 20 rows 403 in place of 373; from 32 rows on
  // the whole box is as fast.)
  const int a_rows = P.rows < 32 ? static_cast<int>(round_up(P.rows, 8)) : 128;
  Product& L = S.prod[0];  // logits: tokens x vocabulary
  L.a_rows = a_rows;
  if (P.in_place) {
    S.ids64 = R.ids_in;
    S.ld_ids64 = R.ld_ids;
    S.in_place = 1;
    R.in_place = 1;
    HEAD_TRY(encode(&L.map_a, a->x, 1, P.rows, P.dim, a->ld_x, a_rows));
  } else {
    HEAD_TRY(encode(&L.map_a, R.xc, 1, P.rows, P.dim, P.ld_xc, a_rows));
  }
  HEAD_TRY(encode(&L.map_b, w, 1, P.vocab, P.dim, ld_w, 128));
  L.n_tile = kTileN;
  L.m_tiles = -1;
  L.n_tiles = P.v_tiles;
  L.k_blocks = (P.dim + kBK - 1) / kBK;
  L.splits = 1;
  L.group = 16;  // 16 row tiles of x (16 MB at 2048 columns) stay in L2 while w streams past

  GemmParams O = S;
  if (P.grads) {
    O.n_prod = 0;
    Product& X = O.prod[0];  // dX: tokens x dim, over the vocabulary piece
    X = Product{};
    X.a_rows = a_rows;
    HEAD_TRY(encode(&X.map_a, g, P.n_buffers, P.rows, g_ld, g_ld, a_rows));
    HEAD_TRY(encode(&X.map_b, w, 1, P.vocab, P.dim, ld_w, 64));
    X.b_mn = 1;
    X.n_tile = P.dx_n_tile;
    X.m_tiles = P.want_dx ? -1 : 0;
    X.n_tiles = P.dx_n_tiles;
    X.splits = P.splits;
    X.swap_order = 1;
    Product& W = O.prod[1];  // dW: vocabulary piece x dim, over the tokens
    W = Product{};
    HEAD_TRY(encode(&W.map_a, g, P.n_buffers, P.rows, g_ld, g_ld, 64));
    HEAD_TRY(encode(&W.map_b, R.xc, 1, P.rows, P.dim, P.ld_xc, 64));
    W.a_mn = W.b_mn = 1;
    W.n_tile = P.dx_n_tile;
    W.n_tiles = P.dx_n_tiles;
    W.k_blocks = -1;
    W.splits = 1;
    W.swap_order = 1;
    O.n_prod = P.want_dw ? 2 : 1;
    O.part_cols = static_cast<int>(P.part_ld);
    if (P.want_dx)
      HEAD_TRY(encode(&O.map_part, ws + P.part, P.splits, P.rows, P.part_ld, P.part_ld, 32, true));
    O.dw = a->dw;
    O.ld_dw = a->ld_dw;
    O.dw_fp32 = a->dw_dtype == MUON_DTYPE_FP32;
    O.dw_add = a->dw_accumulate != 0;
    O.dw_cols = P.dim;
    const long long pitch = a->ld_dw * (O.dw_fp32 ? 4 : 2);
    O.dw_tma = P.want_dw && !misaligned(a->dw, 16) && (pitch & 15) == 0 && (O.dw_fp32 || !O.dw_add);
    if (O.dw_tma) HEAD_TRY(encode(&O.map_dw, a->dw, 1, P.vocab, P.dim, a->ld_dw, 32, O.dw_fp32 != 0));
  }

  if (P.pack && !kept) {
    R.pack_to = reinterpret_cast<__nv_bfloat16*>(ws + P.wc);
    R.pack_from = static_cast<const __nv_bfloat16*>(a->w);
    R.ld_pack = a->ld_w;
    R.pack_blocks = pack_blocks(P.vocab);
    if (P.in_place) HEAD_CUDA(launch_pack(R, stream));
  }
  if (!P.in_place && !kept) {
    const bool flags = distill && P.tokens > 0;
    if (flags) {
      R.flags = reinterpret_cast<unsigned char*>(ws + P.flags);
      HEAD_CUDA(launch_flags(R, stream));
    }
    const bool many = P.tokens >= kManyTokens;
    if (many) {
      R.run_counts = reinterpret_cast<int*>(ws + P.run_counts);
      HEAD_CUDA(launch_count(R, flags, stream));
    }
    HEAD_CUDA(launch_prepare(R, flags || many, stream));
  }
  const long long m_tiles = P.m_tiles;
  // more tiles than CTA pairs: the epilogue's warps share them out instead of their columns
  S.by_tile = m_tiles * P.v_tiles > pairs;
  if (!d) HEAD_CUDA(launch_gemm(kModeStats, S, m_tiles * P.v_tiles, pairs, !P.in_place, stream));
  if (kind == kLogprob) {
    if (P.tokens > 0) HEAD_CUDA(launch_logprob(R, stream));
    return MUON_OK;
  }
  ConvertParams C = {};
  C.ld = g_ld;
  C.row_q = R.row_q;
  C.stats = R.stats;
  C.stats_ld = R.stats_ld;
  C.top = top;
  C.ids = R.ids;
  C.entry_g = R.entry_g;
  C.starts = P.in_place ? nullptr : R.starts;
  C.n_starts = R.n_starts;
  // of log probabilities: kept codes, into the buffer that the piece's products read
  const int n_kept = kept ? K.n_stored : 0;
  auto log_codes_of = [&](int piece) {
    ConvertParams D = C;
    const long long one = P.rows * g_ld;
    D.codes = reinterpret_cast<const __nv_bfloat16*>(kept + K.g) + piece * one;
    D.row_b = R.row_b;
    D.g = g + (piece % P.n_buffers) * one;
    D.tiles = tiles_of(piece);
    D.v_tile0 = piece * P.piece_tiles;
    return D;
  };
  auto codes_of = [&](int piece) {
    ConvertParams D = C;
    if (piece < P.n_stored) D.g = g + static_cast<long long>(piece) * P.rows * g_ld;
    D.tiles = tiles_of(piece);
    D.v_tile0 = piece * P.piece_tiles;
    return D;
  };
  if (P.grads) R.total = nullptr;  // the products' launch adds the losses up beside its work
  if (d) {
    HEAD_CUDA(launch_logprob_grad(R, stream));
    if (n_kept > 0) HEAD_CUDA(launch_convert_log(R, log_codes_of(0), 2 * pairs, stream));
  } else HEAD_CUDA(launch_finalise(R, codes_of(0), 2 * pairs, stream));
  if (P.grads) {
    for (int i = 0; i < P.n_pieces; ++i) {
      // stored pieces lie in a buffer each, the others use the first one after them
      const bool stored = d ? i < n_kept : i < P.n_stored;
      const int buffer = d ? i % P.n_buffers : stored ? i : 0;
      const int tiles = tiles_of(i);
      const int v0 = i * P.piece_tiles * kTileN;
      const int cols = P.vocab - v0 < tiles * kTileN ? P.vocab - v0 : tiles * kTileN;
      if (!stored) {
        S.v0 = v0;
        // the launch stores into the first buffer of its map
        HEAD_TRY(encode(&S.map_g, g + buffer * P.rows * g_ld, 1, P.rows, g_ld, g_ld, 32));
        L.b_n0 = v0;
        L.n_tiles = tiles;
        S.by_tile = m_tiles * tiles > pairs;
        HEAD_CUDA(launch_gemm(kModeGrad, S, m_tiles * tiles, pairs, true, stream));
      }
      O.convert = i + 1 < n_kept ? log_codes_of(i + 1) : i + 1 < P.n_stored ? codes_of(i + 1) : ConvertParams{};
      O.prod[0].a_z = O.prod[1].a_z = buffer;
      O.prod[0].k_blocks = (cols + kBK - 1) / kBK;
      O.prod[0].b_k0 = v0;
      O.part_add = i > 0;
      // Four epilogue warps more (whole calls, us, with and without).  Where dW leaves element
      // by element: 37 and 42 for 333 x 203 x 5003, 86 and 90 for 4000 tokens of it, 212 and
      // 288 for 100 x 2047 x 20000, 296 and 379 for 1000 tokens of it.  Else for one row tile of
      // half a CTA pair or less with its products out of L2, x 512 x 50000: 51.1 and 53.2 for
      // 10 tokens, 56.9 and 58.2 for 60, 62.1 and 63.3 for 128, 65.9 and 65.8 for 150, 72.3
      // and 71.5 for 200, 109.6 and 107.1 for 400; 24.8 and 26.6 for 1 x 512 x 8192.  With w
      // out of memory 217 and 210 for 250 x 1024 x 100000.
      O.spare = P.n_pieces == 1 && ((P.want_dw && !O.dw_tma) || (P.tokens <= kTileM / 2 && 2ll * P.vocab * P.dim <= kHeadInCache));
      O.row_l = R.row_l;
      O.total = i == 0 ? a->total : nullptr;
      O.prod[1].m_tiles = tiles;
      O.dw_row0 = v0;
      O.dw_rows = cols;
      const long long out_tiles = (P.want_dx ? m_tiles * P.dx_n_tiles * P.splits : 0) +
                                  (P.want_dw ? static_cast<long long>(tiles) * P.dx_n_tiles : 0);
      HEAD_CUDA(launch_gemm(kModeOut, O, out_tiles, pairs, true, stream));
    }
    if (P.want_dx) HEAD_CUDA(launch_dx(R, stream));
  }
  return MUON_OK;
}

// The same call as a loss: sizes, operands and gradients, for the checks and the plan.
muon_head_args as_head_args(const muon_logprob_args* l, const muon_logprob_grads* d) {
  muon_head_args a = {};
  a.tokens = l->tokens;
  a.dim = l->dim;
  a.vocab = l->vocab;
  a.x = l->x;
  a.w = l->w;
  a.ld_x = l->ld_x;
  a.ld_w = l->ld_w;
  a.x_dtype = l->x_dtype;
  a.w_dtype = l->w_dtype;
  a.scale = 1.0f;
  a.logit_scale = l->logit_scale;
  a.loss = l->logprob;
  a.lse = l->lse;
  if (d) {
    a.dx = d->dx;
    a.dw = d->dw;
    a.ld_dx = d->ld_dx;
    a.ld_dw = d->ld_dw;
    a.dx_dtype = d->dx_dtype;
    a.dw_dtype = d->dw_dtype;
    a.dw_accumulate = d->dw_accumulate;
  }
  return a;
}

}  // namespace

extern "C" int muon_head_logprob_workspace_bytes(const muon_logprob_args* l, const muon_logprob_grads* d, size_t* out_bytes) {
  if (!l || !out_bytes) return fail(MUON_ERR_INVALID_ARG, "args or out_bytes is null");
  const muon_head_args a = as_head_args(l, d);
  HEAD_TRY(check(&a, 1, false));
  Plan P;
  HEAD_TRY(make_plan(&a, 1, false, kPlanPairs, 0, &P, d ? kLogprobGrad : kLogprob, !d && l->entropy,
                     d ? d->kept != nullptr : l->keep != 0));
  *out_bytes = P.bytes;
  return MUON_OK;
}

static int check_logprob(const muon_logprob_args* l, const muon_head_args* a) {
  HEAD_TRY(check(a, 1, true));
  if (l->tokens > 0 && !l->targets) return fail(MUON_ERR_INVALID_ARG, "targets is null");
  if (misaligned(l->targets, 8) || misaligned(l->entropy, 4)) return fail(MUON_ERR_ALIGNMENT, "pointer not aligned to its element size");
  return check_scale(a, nullptr);
}

extern "C" int muon_head_logprob(const muon_logprob_args* l, void* workspace, size_t workspace_bytes, int device, void* stream) {
  if (!l) return fail(MUON_ERR_INVALID_ARG, "args is null");
  const muon_head_args a = as_head_args(l, nullptr);
  HEAD_TRY(check_logprob(l, &a));
  return run(&a, nullptr, l->targets, 0.f, l, nullptr, workspace, workspace_bytes, device, static_cast<cudaStream_t>(stream));
}

extern "C" int muon_head_logprob_grad(const muon_logprob_args* l, const muon_logprob_grads* d, void* workspace,
                                      size_t workspace_bytes, int device, void* stream) {
  if (!l || !d) return fail(MUON_ERR_INVALID_ARG, "args or grads is null");
  const muon_head_args a = as_head_args(l, d);
  HEAD_TRY(check_logprob(l, &a));
  if (!d->dx && !d->dw) return fail(MUON_ERR_INVALID_ARG, "no gradient wanted");
  if (misaligned(d->kept, 1024)) return fail(MUON_ERR_WORKSPACE, "kept is not 1024-byte aligned");
  if (l->tokens > 0 && (!l->lse || (d->g_entropy && !l->entropy)))
    return fail(MUON_ERR_INVALID_ARG, "the gradient needs lse, and entropy where g_entropy is given");
  if (misaligned(d->g_logprob, 4) || misaligned(d->g_entropy, 4))
    return fail(MUON_ERR_ALIGNMENT, "pointer not aligned to its element size");
  return run(&a, nullptr, l->targets, 0.f, l, d, workspace, workspace_bytes, device, static_cast<cudaStream_t>(stream));
}

extern "C" int muon_head_workspace_bytes(const muon_head_args* a, int top, size_t* out_bytes, size_t* least_bytes) {
  if (!out_bytes && !least_bytes) return fail(MUON_ERR_INVALID_ARG, "out_bytes and least_bytes are null");
  // top = 0: cross entropy
  HEAD_TRY(check(a, top > 0 ? top : (top == 0 ? 1 : top), false));
  Plan P;
  HEAD_TRY(make_plan(a, top > 0 ? top : 1, top > 0, kPlanPairs, 0, &P));
  if (out_bytes) *out_bytes = P.bytes;
  if (least_bytes) *least_bytes = P.least;
  return MUON_OK;
}

extern "C" size_t muon_debug_set_head_piece_bytes(size_t bytes) {
  const size_t before = static_cast<size_t>(g_piece_bytes);
  g_piece_bytes = bytes ? static_cast<long long>(bytes) : kPieceBytes;
  return before;
}

extern "C" int muon_debug_set_head_codes(int mode) {
  const int before = g_codes;
  if (mode >= 0 && mode <= 2) g_codes = mode;
  return before;
}

extern "C" int muon_head_xent(const muon_head_args* a, const int64_t* targets, float z_loss, void* workspace,
                              size_t workspace_bytes, int device, void* stream) {
  HEAD_TRY(check(a, 1, true));
  if (a->tokens > 0 && !targets) return fail(MUON_ERR_INVALID_ARG, "targets is null");
  if (misaligned(targets, 8)) return fail(MUON_ERR_ALIGNMENT, "targets not aligned to 8 bytes");
  if (!std::isfinite(z_loss)) return fail(MUON_ERR_INVALID_ARG, "z_loss must be finite");
  HEAD_TRY(check_scale(a, nullptr));
  return run(a, nullptr, targets, z_loss, nullptr, nullptr, workspace, workspace_bytes, device, static_cast<cudaStream_t>(stream));
}

extern "C" int muon_head_distill(const muon_head_args* a, const muon_head_teacher* t, void* workspace,
                                 size_t workspace_bytes, int device, void* stream) {
  if (!t) return fail(MUON_ERR_INVALID_ARG, "teacher is null");
  HEAD_TRY(check(a, t->top, true));
  if (a->tokens > 0 && (!t->top_ids || !t->top_logits)) return fail(MUON_ERR_INVALID_ARG, "top_ids or top_logits is null");
  if (a->tokens > 0 && (t->ld_ids < t->top || t->ld_logits < t->top))
    return fail(MUON_ERR_INVALID_ARG, "a row stride of the teacher's entries is smaller than top");
  if (t->logits_dtype != MUON_DTYPE_BF16 && t->logits_dtype != MUON_DTYPE_FP32)
    return fail(MUON_ERR_UNSUPPORTED, "top_logits must be bf16 or fp32");
  if (!std::isfinite(t->temperature) || !(t->temperature > 0.f))
    return fail(MUON_ERR_INVALID_ARG, "temperature must be finite and positive");
  HEAD_TRY(check_scale(a, t));
  if (misaligned(t->top_ids, 8) || misaligned(t->top_logits, t->logits_dtype == MUON_DTYPE_FP32 ? 4 : 2) ||
      misaligned(t->teacher_lse, 4))
    return fail(MUON_ERR_ALIGNMENT, "pointer not aligned to its element size");
  return run(a, t, nullptr, 0.f, nullptr, nullptr, workspace, workspace_bytes, device, static_cast<cudaStream_t>(stream));
}

extern "C" int muon_head_status(const void* workspace, int device, void* stream, int* device_status) {
  if (!workspace || !device_status) return fail(MUON_ERR_INVALID_ARG, "workspace or device_status is null");
  DeviceGuard guard;
  HEAD_CUDA(guard.set(device));
  Ctrl c;
  HEAD_CUDA(cudaMemcpyAsync(&c, workspace, sizeof(c), cudaMemcpyDeviceToHost, static_cast<cudaStream_t>(stream)));
  HEAD_CUDA(cudaStreamSynchronize(static_cast<cudaStream_t>(stream)));
  *device_status = c.status;
  return MUON_OK;
}
