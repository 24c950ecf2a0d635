// Launchers of the kernels around the head's products (k_head.cu).
#pragma once
#include "fbl_internal.h"

constexpr int HEAD_MAX_TOP = 128;       // teacher logits a token
constexpr int HEAD_TICKET = 32;         // word of the status word's block in which head_combine_kernel counts its blocks

// What the forward keeps of the padded token rows, in `saved`.  The products run over the rows that carry a loss, in their order.
struct HeadRows {
  int64_t rows;
  int32_t *ids, *count;       // entries, see HeadEpi (count 0: no loss)
  int32_t *row_of, *pos;      // the products' rows' token rows, and the other way round (-1: none)
  int32_t* n;                 // [2] rows with a loss, the same and at least 1
  float *y, *constant;        // constant: sum of y log y
  float *k, *sum;             // softmax statistics
  float* total;               // [2] loss, counted tokens
  void* x;                    // the products' rows of X, zeros behind them to whole tiles
  int64_t x_rows;             // how many it has
  int second;                 // where the same rows lie again (0: nowhere)
};

// Products at the targets formed again in 64 bits by the kernel that brings the rows together (bf16, few of them): z [entry][row] null: not.
struct HeadExact {
  double* z;
  const void* W;
  int64_t w_rows;
  int vocab_rows, d_model, top_k;
  double unlift;              // what the other products come out as, over what they are
};

// Labels, or what teacher_entries has left in `count`, to positions; the rows of X with a loss to R.x.
cudaError_t launch_head_rows(int dtype, const int32_t* targets, const HeadRows& R, int seq, int t_pad, int vocab, const void* X, int d_model,
                             const HeadExact& exact, int32_t* status, cudaStream_t st);
cudaError_t launch_teacher_entries(const int32_t* ids, const float* logits, int top_k, float temperature, const HeadRows& R, int seq, int t_pad,
                                   int vocab, int32_t* status, cudaStream_t st);
cudaError_t launch_head_combine(const float2* part, int tiles, const float* z_at, const HeadRows& R, float scale, float* loss, float* total,
                                double2* block_sums, int seq, int t_pad, const HeadExact& exact, int32_t* status, cudaStream_t st);
// raise: 1 to 2, by which weights of losses are multiplied in dz and what comes of dz is divided again (see the kernel)
cudaError_t launch_head_weights(const float* dloss, const HeadRows& R, int seq, int t_pad, float inv_tau, float* raise, cudaStream_t st);
// dX from the areas' sums, times alpha / max(*over, 1) where `over` is not null
cudaError_t launch_head_scatter(int dtype, int sm_count, const float* acc, int areas, const HeadRows& R, int d_model, const float* over, float alpha,
                                void* dX, cudaStream_t st);
// [rows][cols] <-> tiles of [rows][padded], for a number of columns that is not whole tiles
cudaError_t launch_pack_columns(int dtype, int unpack, const void* src, void* dst, int64_t rows, int cols, int padded, cudaStream_t st);
