// The head of a fine-tuning step: logits X W over the vocabulary and their softmax cross entropy with labels, or with a teacher's
// top logits, a piece of the vocabulary at a time and without keeping a logit; and the norm in front of it as a plan of its own.
// The forward is one product whose epilogue keeps softmax statistics; the backward forms a piece's logits again, leaves
// their gradient dz from the same epilogue (head_epilogue.cuh), and feeds it to dX += dz W^T and dW = X^T dz in one launch.
#include <math.h>
#include <stdlib.h>

#include <new>

#include "fbl_internal.h"
#include "k_head.h"

namespace {

inline cudaStream_t as_stream(void* s) { return reinterpret_cast<cudaStream_t>(s); }
inline bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & (FBL_ALIGN - 1)) != 0; }
inline int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

#define HEAD_CUDA(expr)                                 \
  do {                                                  \
    cudaError_t e__ = (expr);                           \
    if (e__ != cudaSuccess) {                           \
      fbl_note_cuda_error(e__, #expr);                  \
      return FBL_ERR_CUDA;                              \
    }                                                   \
  } while (0)
#define HEAD_STEP(expr) do { HEAD_CUDA(expr); p->launches++; } while (0)

// What the shared launchers read the token geometry, dtype, norm, SM count and knobs from: an attention-layer plan of the same
// batch, sequence and width (one head per tile column so that any d_model passes its checks).
int base_plan(int batch, int seq, int d_model, int dtype, int norm, float eps, fbl_plan** out) {
  fbl_layer_desc ld = {};
  ld.batch = batch; ld.seq = seq; ld.d_model = d_model; ld.head_dim = dtype == FBL_DTYPE_FP32 ? 32 : 64;
  ld.n_q_heads = ld.n_kv_heads = 1; ld.dtype = dtype; ld.norm = norm; ld.eps = eps;
  return fbl_plan_create(&ld, out);
}

// Columns of a piece.  Its logits' gradient is written once and read twice by the two products behind, and each piece costs two launches'
// start and end, some 13 us.  Pieces of half a Tflop and more are of 128 MB: 8192 x 4096 over 32000 columns, in three runs that the power cap's
// clock keeps 3 % apart, 7253 to 7263 us a step with 32 MB, 6938 to 6955 with 64 MB, 6789 to 6986 with 128 MB, 6764 to 7038 with 256 MB and 6732 to 6807
// with one piece of 524 MB, whose memory is not worth that.  Smaller ones are up to 256 MB: 2048 x 768 over 50257 columns, a third without a
// loss, 352 us in one piece of 206 MB, 365 in two, 377 in three, 394 in four, 438 in six.
int64_t piece_columns(int64_t n_pad, int d_model, int e) {
  int64_t piece = ((int64_t)128 << 20) / (n_pad * e);
  const int64_t enough = (int64_t)(0.5e12 / (6.0 * (double)n_pad * d_model));
  if (piece < enough) piece = enough < 2 * piece ? enough : 2 * piece;
  return piece > 2048 ? piece / HEAD_TILE * HEAD_TILE : 2048;
}

// The tensor core's additions round toward zero, so that a logit comes out smaller in magnitude: by 2.2e-8 of itself and 1.62e-8 more
// for each 16 columns where the terms have one sign (2.1e-6 at 2048 columns, 4.2e-6 at 4096: logits of tokens that the hidden state
// points at), by 0.7 to 0.95 of that where they do not.  That is ten times what fp32 sums lose, and all one way, so it would stay in
// the mean loss; logits are scaled up by it (mean loss off by 2.5e-6 at 4096 columns without).
double logit_lift(int d_model) { return 2.2e-8 + 1.6e-8 * (d_model / 16); }

}  // namespace

// Products at the targets are formed again in 64 bits (exact_products) for up to so many rows and entries, which an SM's blocks hold at
// once.  Of more tokens the errors that this takes out average out against the losses' size (2.9e-7 of their norm at 256 tokens
// of 2048 over 32000 columns; one token's over 128256 was off by up to 3.0e-6 of itself).
constexpr int EXACT_ROWS = 64, EXACT_ENTRIES = 1024;

// Up to so many rows, half of a tile of 128, dz comes in two parts, the second below the first (head_epilogue.cuh): the rows are there
// anyway, and what it costs is writing and reading dz twice (us a step, 50 tokens of 768 over 50257 columns 88 -> 90).
constexpr int SECOND_ROWS = 64;

struct fbl_head_plan {
  fbl_head_desc d;
  fbl_plan* base;
  int64_t n_pad;
  int cols;                     // vocabulary in whole tiles: columns of the logits
  int64_t w_rows;               // stored rows of W
  int top_k, tiles;             // entries a row; partials of the softmax statistics
  int logits_tile, grad_tile;   // HeadEpi.tile of the two passes
  int piece, pieces, slices[2]; // columns of a piece; pieces; areas that dX's reduction is cut into, alone and beside dW
  int second;                   // few rows: where they lie again, for dz's second part (0: nowhere)
  int64_t x_rows;               // rows of the products
  float scale;                  // from a product to a logit times log2 e
  size_t sv_ids, sv_y, sv_count, sv_constant, sv_row_of, sv_pos, sv_n, sv_k, sv_sum, sv_total, sv_x, saved_bytes;
  bool exact;                   // products at the targets formed again in 64 bits
  size_t sf_part, sf_z, sf_blocks, sf_exact, scratch_fwd_bytes;
  size_t sb_raise, sb_dz, sb_acc, scratch_bwd_bytes;
  mutable int64_t launches;
};
struct fbl_norm_plan {
  fbl_norm_desc d;
  fbl_plan* base;
  mutable int64_t launches;
};

namespace {

HeadRows rows_of(const fbl_head_plan* p, const void* saved) {
  char* sv = (char*)saved;
  HeadRows R;
  R.rows = p->n_pad;
  R.ids = (int32_t*)(sv + p->sv_ids); R.count = (int32_t*)(sv + p->sv_count);
  R.y = (float*)(sv + p->sv_y); R.constant = (float*)(sv + p->sv_constant);
  R.row_of = (int32_t*)(sv + p->sv_row_of); R.pos = (int32_t*)(sv + p->sv_pos); R.n = (int32_t*)(sv + p->sv_n);
  R.k = (float*)(sv + p->sv_k); R.sum = (float*)(sv + p->sv_sum);
  R.total = (float*)(sv + p->sv_total);
  R.x = sv + p->sv_x; R.x_rows = p->x_rows; R.second = p->second;
  return R;
}

HeadEpi epilogue_of(const fbl_head_plan* p, const HeadRows& R, int col0) {
  HeadEpi h = {};
  h.ids = R.ids; h.count = R.count; h.row_of = R.row_of; h.n = R.n; h.y = R.y; h.rows = R.rows;
  h.vocab = p->d.vocab; h.col0 = col0; h.top_k = p->top_k; h.scale = p->scale;
  h.k = R.k; h.sum = R.sum;
  h.inv_tau = 1.f / p->d.temperature;
  h.second = p->second;
  return h;
}

// Where the weights of vocabulary columns from col0 on begin.
const char* weights_at(const fbl_head_plan* p, const void* W, int col0) {
  return (const char*)W + (p->d.vocab_rows ? (int64_t)col0 * 128 : (int64_t)col0 * p->d.d_model * p->base->e);
}

// Rows of W, of those from column col0 of the vocabulary on, that a piece of `cols` columns has (one value for all but the last piece).
int64_t piece_rows(const fbl_head_plan* p, int col0, int cols) {
  const int64_t left = p->w_rows - col0;
  return p->d.vocab_rows ? (left < cols ? left : cols) : 0;
}

// The products behind a piece of dz but for addresses: a token-axis reduction, dz^T X [vocab, d_model] or X^T dz, and dz W^T.
GemmArgs dw_product(const fbl_head_plan* p, int cols) {
  GemmArgs g = {};
  const int n = (int)p->x_rows, D = p->d.d_model;
  g.dyn = p->second ? 0 : 2;
  g.n_terms = 1;
  if (p->d.vocab_rows) { g.m = cols; g.n = D; }
  else { g.m = D; g.n = cols; }
  g.t[0] = {nullptr, n, 1, nullptr, n, 0, n, 0};
  g.c_rpad = p->w_rows;
  return g;
}
GemmArgs dx_product(const fbl_head_plan* p, int cols) {
  GemmArgs g = {};
  g.dyn = 1;
  g.n_terms = 1;
  g.m = (int)p->x_rows; g.n = p->d.d_model;
  g.t[0] = {nullptr, p->x_rows, 0, nullptr, p->w_rows, p->d.vocab_rows ? 0 : 1, cols, 0};
  g.c_rpad = p->x_rows;
  return g;
}

// Logits of columns col0 .. col0 + cols - 1: X [tokens with a loss, d_model] times W's piece.
GemmArgs logits_product(const fbl_head_plan* p, const HeadRows& R, const void* W, int col0, int cols) {
  GemmArgs g = {};
  g.rows = R.n + 1; g.dyn = 1;
  g.m = (int)p->x_rows; g.n = cols; g.n_terms = 1;
  g.t[0] = {R.x, p->x_rows, 0, weights_at(p, W, col0), p->w_rows, p->d.vocab_rows, p->d.d_model, piece_rows(p, col0, cols)};
  g.b_static = 1;
  g.c_rpad = p->x_rows;
  g.seq = p->d.seq; g.t_pad = p->base->t_pad;
  return g;
}

int run_products(const fbl_head_plan* p, GemmArgs* gs, int count, int32_t* status, cudaStream_t st) {
  if (p->d.dtype == FBL_DTYPE_FP32) HEAD_CUDA(launch_gemm_tc_f32_head(p->base, gs, count, status, st));
  else HEAD_CUDA(launch_gemm_tc_head(p->base, gs, count, status, st));
  p->launches++;
  return FBL_OK;
}
#define HEAD_RUN(expr) do { const int rc__ = (expr); if (rc__ != FBL_OK) return rc__; } while (0)

HeadExact exact_of(const fbl_head_plan* p, const void* W, char* sf) {
  HeadExact e = {};
  if (p->exact) e.z = (double*)(sf + p->sf_exact);
  e.W = W; e.w_rows = p->w_rows; e.vocab_rows = p->d.vocab_rows; e.d_model = p->d.d_model; e.top_k = p->top_k;
  e.unlift = 1.0 / (1.0 + logit_lift(p->d.d_model));
  return e;
}

int forward(const fbl_head_plan* p, const void* W, float* loss, float* total, const HeadRows& R, char* sf, cudaStream_t st) {
  int32_t* status = (int32_t*)sf;
  float2* part = (float2*)(sf + p->sf_part);
  float* z_at = (float*)(sf + p->sf_z);
  GemmArgs g = logits_product(p, R, W, 0, p->cols);
  g.epi = 6;
  g.head = epilogue_of(p, R, 0);
  g.head.part = part; g.head.tiles = p->tiles; g.head.z_at = z_at;
  g.head.tile = p->logits_tile;
  HEAD_RUN(run_products(p, &g, 1, status, st));
  HEAD_STEP(launch_head_combine(part, p->tiles, z_at, R, p->scale, loss, total, (double2*)(sf + p->sf_blocks), p->d.seq, p->base->t_pad,
                                exact_of(p, W, sf), status, st));
  return FBL_OK;
}

bool forward_args_ok(const fbl_head_plan* p, const void* X, const void* W, const float* loss, const float* total, const void* saved, const void* scratch) {
  return p && X && W && loss && total && saved && scratch;
}

}  // namespace

extern "C" {

int fbl_head_plan_create(const fbl_head_desc* desc, fbl_head_plan** out) {
  if (!desc || !out) return FBL_ERR_INVALID_ARG;
  *out = nullptr;
  const fbl_head_desc& d = *desc;
  if (d.vocab <= 0 || d.top_k < 0 || (d.vocab_rows != 0 && d.vocab_rows != 1)) return FBL_ERR_INVALID_ARG;
  if (!(d.temperature > 0.f) || isinf(d.temperature) || isinf(1.5f / d.temperature)) return FBL_ERR_INVALID_ARG;
  if (d.top_k == 0 && d.temperature != 1.f) return FBL_ERR_INVALID_ARG;
  if (d.vocab > 1 << 20 || d.top_k > HEAD_MAX_TOP) return FBL_ERR_UNSUPPORTED_SHAPE;
  if (d.batch <= 0 || d.seq <= 0) return FBL_ERR_INVALID_ARG;
  if ((int64_t)d.batch * up(d.seq, 8) > 1 << 22) return FBL_ERR_UNSUPPORTED_SHAPE;
  fbl_plan* base = nullptr;
  const int rc = base_plan(d.batch, d.seq, d.d_model, d.dtype, FBL_NORM_RMSNORM, 0.f, &base);
  if (rc != FBL_OK) return rc;
  fbl_head_plan* p = new (std::nothrow) fbl_head_plan();
  if (!p) { fbl_plan_destroy(base); return FBL_ERR_INVALID_ARG; }
  p->d = d; p->base = base; p->n_pad = base->n_pad; p->launches = 0;
  const bool bf16 = d.dtype == FBL_DTYPE_BF16;
  p->second = bf16 && p->n_pad <= SECOND_ROWS ? (int)p->n_pad : 0;
  p->x_rows = p->second ? 2 * p->n_pad : p->n_pad;
  p->cols = (int)up(d.vocab, base->tw);
  p->w_rows = d.vocab_rows ? up(d.vocab, 8) : d.d_model;
  p->top_k = d.top_k ? d.top_k : 1;
  int width = HEAD_TILE_F32;
  p->grad_tile = getenv("FBL_HEAD_TILE") ? atoi(getenv("FBL_HEAD_TILE")) : -1;                                               // tuning / test knob
  p->logits_tile = bf16 ? gemm_tc_logits_tile(base, p->x_rows, p->cols, d.d_model, p->grad_tile, &width) : 0;
  if (p->grad_tile >= 0) p->grad_tile = p->logits_tile;
  p->tiles = (p->cols + width - 1) / width;
  p->scale = (float)(1.4426950408889634 / (double)d.temperature * (1.0 + (bf16 ? logit_lift(d.d_model) : 0.0)));

  // pieces of about one size, in whole tiles
  int64_t piece = piece_columns(p->n_pad, d.d_model, base->e);
  if (getenv("FBL_HEAD_PIECE") && atoi(getenv("FBL_HEAD_PIECE")) > 0) piece = up(atoi(getenv("FBL_HEAD_PIECE")), HEAD_TILE);   // tuning / test knob
  p->pieces = (int)((p->cols + piece - 1) / piece);
  p->piece = (int)up((p->cols + p->pieces - 1) / p->pieces, HEAD_TILE);
  p->pieces = (p->cols + p->piece - 1) / p->piece;
  if (p->piece > p->cols) p->piece = p->cols;

  // dX reduces over a piece of the vocabulary: cut it where that balances the SMs, beside dW, which reduces over the tokens, or, bf16, alone
  // (frozen heads, us a step with the slices that go with dW, with their own, and with the best of 1 to 64: 50 tokens of 768 over 50257 columns 72,
  // 66, 65; 10 of 2048 over 128256 268, 261, 260; 200 of 1024 over 32000 75, 77, 75; 4096 of 64 over 32000 218, 208, 208.  fp32, whose model of a
  // launch takes areas for dearer than they are: 231 tokens of 512 over 32000 217, 252, 206; 40 of 768 over 30011 147, 165, 137)
  for (int beside = 0; beside < 2; ++beside) {
    GemmArgs gs[2] = {dw_product(p, p->piece), dx_product(p, p->piece)};
    const int kb = (p->piece + 63) / 64;
    int want = 1;
    if (bf16) {
      const GemmShape dw = {gs[0].m, gs[0].n, (gs[0].t[0].k + 63) / 64, 0};
      want = gemm_tc_choose_own_slices(base->sm_count, beside ? &dw : nullptr, {gs[1].m, gs[1].n, kb, 1});
    } else {
      want = gemm_tc_f32_choose_areas(base, gs, 2);
    }
    if (getenv("FBL_HEAD_SLICES") && atoi(getenv("FBL_HEAD_SLICES")) > 0) want = atoi(getenv("FBL_HEAD_SLICES"));               // likewise
    if (want > kb) want = kb;
    const int per = (kb + want - 1) / want;                                                                                   // none empty
    p->slices[beside] = (kb + per - 1) / per;
  }

  const size_t n = (size_t)p->n_pad;
  auto take = [](size_t& o, size_t bytes) { const size_t at = o; o += fbl_align_up(bytes, FBL_ALIGN); return at; };
  size_t o = 0;
  p->sv_ids = take(o, n * p->top_k * 4);
  p->sv_y = take(o, n * p->top_k * 4);
  p->sv_count = take(o, n * 4);
  p->sv_constant = take(o, n * 4);
  p->sv_row_of = take(o, n * 4);
  p->sv_pos = take(o, n * 4);
  p->sv_n = take(o, 8);
  p->sv_k = take(o, n * 4);
  p->sv_sum = take(o, n * 4);
  p->sv_total = take(o, 8);
  p->sv_x = take(o, (size_t)p->x_rows * d.d_model * base->e);
  p->saved_bytes = o;
  const size_t piece_bytes = (size_t)p->x_rows * p->piece * base->e;
  o = FBL_ALIGN;                // status word
  p->sf_part = take(o, n * p->tiles * sizeof(float2));
  p->sf_z = take(o, n * p->top_k * 4);
  p->sf_blocks = take(o, n / 8 * sizeof(double2));
  p->exact = bf16 && p->n_pad <= EXACT_ROWS && p->n_pad * p->top_k <= EXACT_ENTRIES;
  p->sf_exact = take(o, p->exact ? n * p->top_k * 8 : 0);
  p->scratch_fwd_bytes = o;
  o = FBL_ALIGN;
  p->sb_raise = take(o, 4);
  p->sb_dz = take(o, piece_bytes);
  p->sb_acc = take(o, (size_t)p->x_rows * d.d_model * 4 * (p->slices[0] > p->slices[1] ? p->slices[0] : p->slices[1]));
  p->scratch_bwd_bytes = o;
  *out = p;
  return FBL_OK;
}

void fbl_head_plan_destroy(fbl_head_plan* plan) {
  if (!plan) return;
  fbl_plan_destroy(plan->base);
  delete plan;
}

int64_t fbl_head_launch_count(const fbl_head_plan* plan) { return plan ? plan->launches + plan->base->launches : -1; }

static bool head_shape(const fbl_head_plan* p, int id, int64_t* outer, int64_t* rows, int64_t* rows_pad, int* cols) {
  const fbl_head_desc& d = p->d;
  if (id == FBL_HT_X) { *outer = d.batch; *rows = d.seq; *rows_pad = p->base->t_pad; *cols = d.d_model; return true; }
  if (id != FBL_HT_W) return false;
  *outer = 1;
  *rows = d.vocab_rows ? d.vocab : d.d_model;
  *rows_pad = p->w_rows;
  *cols = d.vocab_rows ? d.d_model : p->cols;
  return true;
}

int fbl_head_tensor_bytes(const fbl_head_plan* plan, int matrix_id, size_t* bytes) {
  int64_t outer, rows, rows_pad; int cols;
  if (!plan || !bytes || !head_shape(plan, matrix_id, &outer, &rows, &rows_pad, &cols)) return FBL_ERR_INVALID_ARG;
  *bytes = (size_t)(outer * rows_pad) * cols * plan->base->e;
  return FBL_OK;
}

int fbl_head_workspace_bytes(const fbl_head_plan* plan, size_t* saved, size_t* scratch_fwd, size_t* scratch_bwd) {
  if (!plan) return FBL_ERR_INVALID_ARG;
  if (saved) *saved = plan->saved_bytes;
  if (scratch_fwd) *scratch_fwd = plan->scratch_fwd_bytes;
  if (scratch_bwd) *scratch_bwd = plan->scratch_bwd_bytes;
  return FBL_OK;
}

// Row-major weights [d_model, vocab] have rows of `vocab` elements, tiles whole columns: the last tiles' columns past the
// vocabulary are zero, which launch_pack does not do.
static int head_pack_common(const fbl_head_plan* p, int id, const void* src, void* dst, void* stream, int unpack) {
  int64_t outer, rows, rows_pad; int cols;
  if (!p || !src || !dst || !head_shape(p, id, &outer, &rows, &rows_pad, &cols)) return FBL_ERR_INVALID_ARG;
  if (misaligned(unpack ? src : dst)) return FBL_ERR_MISALIGNED;
  if (id == FBL_HT_W && !p->d.vocab_rows && p->d.vocab != cols)
    HEAD_CUDA(launch_pack_columns(p->d.dtype, unpack, src, dst, rows, p->d.vocab, cols, as_stream(stream)));
  else
    HEAD_CUDA(launch_pack(p->d.dtype, unpack, src, dst, outer, rows, rows_pad, cols, as_stream(stream)));
  return FBL_OK;
}
int fbl_head_pack(const fbl_head_plan* plan, int id, const void* rowmajor_dev, void* tiled_dev, void* stream) {
  return head_pack_common(plan, id, rowmajor_dev, tiled_dev, stream, 0);
}
int fbl_head_unpack(const fbl_head_plan* plan, int id, const void* tiled_dev, void* rowmajor_dev, void* stream) {
  return head_pack_common(plan, id, tiled_dev, rowmajor_dev, stream, 1);
}

int fbl_head_status_poll(const fbl_head_plan* plan, const void* scratch, int32_t* device_status) {
  if (!plan) return FBL_ERR_INVALID_ARG;
  return fbl_status_poll(plan->base, scratch, device_status);
}

int fbl_head_xent_fwd(const fbl_head_plan* p, const void* X, const void* W, const int32_t* targets, float* loss, float* total, void* saved,
                      void* scratch, void* stream) {
  if (!forward_args_ok(p, X, W, loss, total, saved, scratch) || !targets || p->d.top_k) return FBL_ERR_INVALID_ARG;
  const void* ptrs[] = {X, W, saved, scratch};
  for (const void* q : ptrs) if (misaligned(q)) return FBL_ERR_MISALIGNED;
  cudaStream_t st = as_stream(stream);
  const HeadRows R = rows_of(p, saved);
  char* sf = (char*)scratch;
  HEAD_STEP(launch_head_rows(p->d.dtype, targets, R, p->d.seq, p->base->t_pad, p->d.vocab, X, p->d.d_model, exact_of(p, W, sf), (int32_t*)sf, st));
  return forward(p, W, loss, total, R, sf, st);
}

int fbl_head_distill_fwd(const fbl_head_plan* p, const void* X, const void* W, const int32_t* top_ids, const float* top_logits, float* loss,
                         float* total, void* saved, void* scratch, void* stream) {
  if (!forward_args_ok(p, X, W, loss, total, saved, scratch) || !top_ids || !top_logits || !p->d.top_k) return FBL_ERR_INVALID_ARG;
  const void* ptrs[] = {X, W, saved, scratch};
  for (const void* q : ptrs) if (misaligned(q)) return FBL_ERR_MISALIGNED;
  cudaStream_t st = as_stream(stream);
  const HeadRows R = rows_of(p, saved);
  char* sf = (char*)scratch;
  HEAD_STEP(launch_teacher_entries(top_ids, top_logits, p->d.top_k, p->d.temperature, R, p->d.seq, p->base->t_pad, p->d.vocab, (int32_t*)sf, st));
  HEAD_STEP(launch_head_rows(p->d.dtype, nullptr, R, p->d.seq, p->base->t_pad, p->d.vocab, X, p->d.d_model, exact_of(p, W, sf), (int32_t*)sf, st));
  return forward(p, W, loss, total, R, sf, st);
}

int fbl_head_bwd(const fbl_head_plan* p, const void* X, const void* W, const float* dloss, const void* saved, void* dX, void* dW, void* scratch,
                 void* stream) {
  if (!p || !X || !W || !saved || !scratch || (!dX && !dW)) return FBL_ERR_INVALID_ARG;      // (X's rows with a loss are in `saved`)
  const void* ptrs[] = {X, W, saved, scratch, dX, dW};
  for (const void* q : ptrs) if (misaligned(q)) return FBL_ERR_MISALIGNED;
  cudaStream_t st = as_stream(stream);
  const HeadRows R = rows_of(p, saved);
  char* sc = (char*)scratch;
  int32_t* status = (int32_t*)sc;
  void* dz = sc + p->sb_dz;
  float* acc = (float*)(sc + p->sb_acc);
  const bool bf16 = p->d.dtype == FBL_DTYPE_BF16;
  const int D = p->d.d_model;
  const int slices = p->slices[dW != nullptr];
  const float inv_tau = 1.f / p->d.temperature;
  // what the products of a bf16 dz are divided by: the mean's number of tokens and temperature, or what weights were multiplied by (of few
  // rows, whose dz comes in two parts, they are not)
  float* raise = bf16 && dloss && !p->second ? (float*)(sc + p->sb_raise) : nullptr;
  const float* over = dloss ? raise : R.total + 1;
  const float alpha = dloss ? 1.f : inv_tau;
  if (raise) HEAD_STEP(launch_head_weights(dloss, R, p->d.seq, p->base->t_pad, inv_tau, raise, st));
  for (int col0 = 0; col0 < p->cols; col0 += p->piece) {
    const int cols = p->cols - col0 < p->piece ? p->cols - col0 : p->piece;
    {
      GemmArgs g = logits_product(p, R, W, col0, cols);
      g.c = dz;
      g.reset_status = col0 == 0;
      g.epi = 7;
      g.head = epilogue_of(p, R, col0);
      g.head.dloss = dloss; g.head.raise = raise;
      g.head.tile = p->grad_tile;
      if (!bf16) g.head.over = over;
      HEAD_RUN(run_products(p, &g, 1, status, st));
    }
    GemmArgs gs[2];
    int count = 0;
    if (dW) {
      GemmArgs& g = gs[count++];
      g = dw_product(p, cols);
      g.rows = R.n + 1;
      g.t[0].a = p->d.vocab_rows ? dz : R.x;
      g.t[0].b = p->d.vocab_rows ? R.x : dz;
      g.c_rows = piece_rows(p, col0, cols);
      g.c = (void*)weights_at(p, dW, col0);
      if (bf16) { g.over = over; g.alpha = alpha; }
    }
    if (dX) {
      GemmArgs& g = gs[count++];
      g = dx_product(p, cols);
      g.rows = R.n + 1;
      g.t[0].a = dz;
      g.t[0].b = weights_at(p, W, col0);
      g.t[0].b_rows = piece_rows(p, col0, cols);
      g.c = g.acc = acc;
      g.ksplit = slices; g.acc_mode = col0 == 0 ? 1 : 2;
    }
    HEAD_RUN(run_products(p, gs, count, status, st));
  }
  if (dX) HEAD_STEP(launch_head_scatter(p->d.dtype, p->base->sm_count, acc, slices, R, D, bf16 ? over : nullptr, alpha, dX, st));
  return FBL_OK;
}

int fbl_norm_plan_create(const fbl_norm_desc* desc, fbl_norm_plan** out) {
  if (!desc || !out) return FBL_ERR_INVALID_ARG;
  *out = nullptr;
  fbl_plan* base = nullptr;
  const int rc = base_plan(desc->batch, desc->seq, desc->d_model, desc->dtype, desc->norm, desc->eps, &base);
  if (rc != FBL_OK) return rc;
  fbl_norm_plan* p = new (std::nothrow) fbl_norm_plan();
  if (!p) { fbl_plan_destroy(base); return FBL_ERR_INVALID_ARG; }
  p->d = *desc; p->base = base; p->launches = 0;
  *out = p;
  return FBL_OK;
}

void fbl_norm_plan_destroy(fbl_norm_plan* plan) {
  if (!plan) return;
  fbl_plan_destroy(plan->base);
  delete plan;
}

int64_t fbl_norm_launch_count(const fbl_norm_plan* plan) { return plan ? plan->launches + plan->base->launches : -1; }

int fbl_norm_tensor_bytes(const fbl_norm_plan* plan, size_t* bytes) {
  if (!plan || !bytes) return FBL_ERR_INVALID_ARG;
  *bytes = (size_t)plan->base->n_pad * plan->d.d_model * plan->base->e;
  return FBL_OK;
}

int fbl_norm_workspace_bytes(const fbl_norm_plan* plan, size_t* saved, size_t* scratch_fwd, size_t* scratch_bwd) {
  if (!plan) return FBL_ERR_INVALID_ARG;
  if (saved) *saved = fbl_align_up((size_t)plan->base->n_pad * 2 * sizeof(float), FBL_ALIGN);
  if (scratch_fwd) *scratch_fwd = FBL_ALIGN;
  // at most two blocks an SM, each with a row of dgamma and one of dbeta
  if (scratch_bwd) *scratch_bwd = FBL_ALIGN + fbl_align_up((size_t)plan->base->sm_count * 4 * plan->d.d_model * sizeof(float), FBL_ALIGN);
  return FBL_OK;
}

static int norm_pack_common(const fbl_norm_plan* p, const void* src, void* dst, void* stream, int unpack) {
  if (!p || !src || !dst) return FBL_ERR_INVALID_ARG;
  if (misaligned(unpack ? src : dst)) return FBL_ERR_MISALIGNED;
  HEAD_CUDA(launch_pack(p->d.dtype, unpack, src, dst, p->d.batch, p->d.seq, p->base->t_pad, p->d.d_model, as_stream(stream)));
  return FBL_OK;
}
int fbl_norm_pack(const fbl_norm_plan* plan, const void* rowmajor_dev, void* tiled_dev, void* stream) {
  return norm_pack_common(plan, rowmajor_dev, tiled_dev, stream, 0);
}
int fbl_norm_unpack(const fbl_norm_plan* plan, const void* tiled_dev, void* rowmajor_dev, void* stream) {
  return norm_pack_common(plan, tiled_dev, rowmajor_dev, stream, 1);
}

int fbl_norm_fwd(const fbl_norm_plan* p, const void* X, const float* gamma, const float* beta, void* Y, void* saved, void* scratch, void* stream) {
  if (!p || !X || !gamma || !Y || !saved || !scratch) return FBL_ERR_INVALID_ARG;
  if (p->d.norm == FBL_NORM_LAYERNORM && !beta) return FBL_ERR_INVALID_ARG;
  const void* ptrs[] = {X, Y, saved, scratch};
  for (const void* q : ptrs) if (misaligned(q)) return FBL_ERR_MISALIGNED;
  HEAD_STEP(launch_norm_op_fwd(p->base, X, gamma, beta, Y, (float*)saved, as_stream(stream)));
  return FBL_OK;
}

int fbl_norm_bwd(const fbl_norm_plan* p, const void* dY, const void* X, const float* gamma, const void* saved, void* dX, float* dgamma, float* dbeta,
                 void* scratch, void* stream) {
  if (!p || !dY || !X || !gamma || !saved || !dX || !scratch) return FBL_ERR_INVALID_ARG;
  // both vectors' gradients or, with the norm's parameters frozen, neither
  if (p->d.norm == FBL_NORM_LAYERNORM ? !dgamma != !dbeta : dbeta != nullptr) return FBL_ERR_INVALID_ARG;
  const void* ptrs[] = {dY, X, saved, dX, scratch};
  for (const void* q : ptrs) if (misaligned(q)) return FBL_ERR_MISALIGNED;
  HEAD_CUDA(launch_norm_bwd(p->base, dY, X, nullptr, (const float*)saved, gamma, dX, dgamma, dbeta, (float*)((char*)scratch + FBL_ALIGN),
                            (int32_t*)scratch, as_stream(stream)));
  return FBL_OK;
}

}  // extern "C"
