// The vocabulary's softmax in the epilogue of the head's products, bf16 and fp32: logits leave the accumulator as softmax statistics (forward)
// or as the gradient of their cross entropy (backward), so that no logit reaches memory.
//
// With z the product x.w of a token and a vocabulary column and c = log2 e / temperature,
//   forward   k = max z,  s = sum of 2^(c (z - k))  over a tile's columns, and z itself at the row's targets
//   backward  dz = (g / s) 2^(c (z - k)) - g y,  g = the loss's gradient / temperature, y the target probability of the column
//             (bf16: g = 1 for the mean loss, whose 1 / (tokens x temperature) the two products behind are scaled by: with it in dz every
//             token's target would be rounded the same way, and dX and dW come out too large or too small by up to 2^-9; weights that the
//             caller gives are multiplied by a common factor of 1 to 2 for the same reason, head_weights_kernel)
// k and s are a whole row's by then (head_combine_kernel).  Logits only ever enter as distances from the row's largest: a target that
// holds all of its row's probability gives log s = log 1 exactly, and logits of any size have a loss.  Sums are fp32; dz is
// rounded to the storage type, as an operand of the two products that consume it (bf16: half a step of 2^-8 of each value, as
// large as the rounding of the results; up to 64 rows, half of a tile, its other half takes what that loses, with the same rows of X, so that
// the gradients of few tokens are as near as their own rounding: 3.5e-3 of their norm -> 1.7e-3).
//
// What bounds a tile's epilogue is the exponential unit: 256 columns of 32 rows a warp, a lane's 256 exponentials at 8 clocks a
// warp instruction are 2048 clocks, beside some 1200 issued instructions; the products of the next tile take 640 clocks per 64 columns
// of the reduction, so from 256 columns of d_model on they hide it.
//
// A row's targets are looked up by position: entries come sorted, a binary search before the accumulator is complete finds the
// tile's first one, and a warp looks at a panel's entries only where one of its rows has some (one label a row: one panel in
// vocab / 2048; 64 teacher logits over 128 thousand columns: two panels in three).
#pragma once
#include "fbl_internal.h"
#include "tc_common.cuh"

namespace headepi {

constexpr int NONE = 0x7fffffff;

// The row's entries from column `col` on.  What is read first goes out together: each step that waits for the one before costs a tile of
// a short reduction some 700 clocks.
struct Entries {
  const int32_t* ids;
  long long rows;
  int at, count, next;
  __device__ __forceinline__ Entries() : ids(nullptr), rows(0), at(0), count(0), next(NONE) {}
  __device__ __forceinline__ Entries(const HeadEpi& H, int row, int count_, int first, int col) : ids(H.ids + row), rows(H.rows), at(0), count(count_) {
    if (H.top_k == 1) {                         // `first`: the row's first id, if it has one
      at = count > 0 && first < col;
      next = at < count ? first : NONE;
      return;
    }
    for (int end = count; at < end;) {
      const int mid = (at + end) / 2;
      if (ids[mid * rows] < col) at = mid + 1;
      else end = mid;
    }
    fetch();
  }
  __device__ __forceinline__ void fetch() { next = at < count ? ids[at * rows] : NONE; }
  __device__ __forceinline__ void advance() { ++at; fetch(); }
};

// v[i] of registers, i in 0..63: six halvings.
__device__ __forceinline__ uint32_t pick(const uint32_t (&v)[64], int i) {
  uint32_t w[32];
#pragma unroll
  for (int j = 0; j < 32; ++j) w[j] = i & 32 ? v[j + 32] : v[j];
#pragma unroll
  for (int n = 16; n > 0; n /= 2)
#pragma unroll
    for (int j = 0; j < n; ++j) w[j] = i & n ? w[j + n] : w[j];
  return w[0];
}

template <typename Acc>
__device__ __forceinline__ void load_panel(Acc acc, int pn, uint32_t (&v)[64]) {
  acc.load(pn * 64, *reinterpret_cast<uint32_t(*)[32]>(&v[0]));
  acc.load(pn * 64 + 32, *reinterpret_cast<uint32_t(*)[32]>(&v[32]));
  acc.wait();
}

// What a lane knows of its product's row m, and of the columns from `col` on; GRAD: for the backward.
template <bool GRAD>
struct Row {
  Entries e;
  int row, count;
  bool low;                   // a row's second: what dz loses by its rounding
  bool live;                  // rows behind the last token's are zero: the reduction over tokens ends inside a k-block
  float g, gs, k;
  __device__ __forceinline__ Row() : row(0), count(0), low(false), live(false), g(0.f), gs(0.f), k(0.f) {}
  __device__ __forceinline__ Row(const HeadEpi& H, int m, int col, int seq, int t_pad) : low(H.second && m >= H.second), g(0.f), gs(0.f), k(0.f) {
    if (low) m -= H.second;
    const int n = __ldcg(H.n), at = H.row_of[min((long long)m, H.rows - 1)];
    live = m < n && (GRAD || !low);
    // (bounded by what the buffers were made for: both lie in the caller's memory)
    row = live ? (int)min((uint32_t)at, (uint32_t)H.rows - 1u) : 0;
    const int entries = H.count[row], first = H.ids[row];
    float scale = H.inv_tau, sum = 1.f;
    if (GRAD) {
      const int b = row / t_pad, t = row - b * t_pad;
      if (H.dloss) {
        scale *= t < seq ? H.dloss[(long long)b * seq + t] : 0.f;
        if (H.raise) scale *= __ldcg(H.raise);
      } else scale = H.over ? scale / fmaxf(*H.over, 1.f) : 1.f;
      k = H.k[row];
      sum = H.sum[row];
    }
    count = live ? min(entries, H.top_k) : 0;
    e = Entries(H, row, count, first, col);
    if (GRAD && count > 0) {
      g = scale;
      gs = g / sum;
    } else if (GRAD) {
      k = 0.f;
      gs = count < 0 ? __int_as_float(0x7fffffff) : 0.f;
    }
  }
};

// 64 columns of logits, those from `col` of the vocabulary on, join the row's (k, s); products at its targets are noted.
__device__ __forceinline__ void stats64(const HeadEpi& H, Row<false>& R, uint32_t (&v)[64], int col, float& k, float& s) {
  if (col + 64 > H.vocab) {                               // columns that only pad the weights to whole tiles
#pragma unroll
    for (int j = 0; j < 64; ++j) v[j] = col + j < H.vocab ? v[j] : 0xff800000u;
  }
  while (__any_sync(0xffffffffu, R.e.next < col + 64)) {
    if (R.e.next < col + 64) {
      H.z_at[R.e.at * H.rows + R.row] = __uint_as_float(pick(v, R.e.next - col));
      R.e.advance();
    }
  }
  float top[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) top[i] = fmaxf(__uint_as_float(v[i]), __uint_as_float(v[4 + i]));
#pragma unroll
  for (int j = 8; j < 64; j += 8)
#pragma unroll
    for (int i = 0; i < 4; ++i) top[i] = tc::fmax3(top[i], __uint_as_float(v[j + i]), __uint_as_float(v[j + 4 + i]));
  const float was = k;
  k = fmaxf(k, tc::fmax3(top[0], top[1], fmaxf(top[2], top[3])));
  const float from = k == -INFINITY ? 0.f : k;            // so far nothing but -inf, whose distances from one another are NaN and not a sum of 0
  const float2 mk = make_float2(-from, -from), c2 = make_float2(H.scale, H.scale);
  float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
  for (int j = 0; j < 64; j += 2) {
    const float2 x = __fmul2_rn(__fadd2_rn(make_float2(__uint_as_float(v[j]), __uint_as_float(v[j + 1])), mk), c2);
    sum[j / 2 % 2] = __fadd2_rn(sum[j / 2 % 2], make_float2(tc::fast_exp2(x.x), tc::fast_exp2(x.y)));
  }
  sum[0] = __fadd2_rn(sum[0], sum[1]);
  s = s * tc::fast_exp2((was - from) * H.scale) + (sum[0].x + sum[0].y);
}

// 64 columns of logits become their gradient.
__device__ __forceinline__ void grad64(const HeadEpi& H, Row<true>& R, uint32_t (&v)[64], int col) {
  const float2 c2 = make_float2(H.scale, H.scale), mk = make_float2(-R.k, -R.k), gs2 = make_float2(R.gs, R.gs);
#pragma unroll
  for (int j = 0; j < 64; j += 2) {
    const float2 x = __fmul2_rn(__fadd2_rn(make_float2(__uint_as_float(v[j]), __uint_as_float(v[j + 1])), mk), c2);
    const float2 d = __fmul2_rn(make_float2(tc::fast_exp2(x.x), tc::fast_exp2(x.y)), gs2);
    v[j] = __float_as_uint(d.x);
    v[j + 1] = __float_as_uint(d.y);
  }
  while (__any_sync(0xffffffffu, R.e.next < col + 64)) {
    const bool mine = R.e.next < col + 64;
    const int j0 = mine ? R.e.next - col : -1;
    const float gy = mine ? R.g * H.y[R.e.at * H.rows + R.row] : 0.f;
#pragma unroll
    for (int j = 0; j < 64; ++j)
      if (j == j0) v[j] = __float_as_uint(__uint_as_float(v[j]) - gy);
    if (mine) R.e.advance();
  }
  if (col + 64 > H.vocab) {
#pragma unroll
    for (int j = 0; j < 64; ++j) v[j] = col + j < H.vocab ? v[j] : 0u;
  }
}

}  // namespace headepi

// SETS: 2: two of four warps, each with half of the tile's columns (a partial of the statistics is a set's); 3: two that take a tile each.
template <int BN, int SETS, typename Acc, typename Wait>
__device__ __forceinline__ bool head_stats_tile(const HeadEpi& H, int seq, int t_pad, int m0, int n0, int q, Acc acc, Wait wait) {
  constexpr int WIDTH = SETS == 2 ? BN / 2 : BN;
  const int m = m0 + q * 32 + threadIdx.x % 32, first = SETS != 2 ? 0 : ((int)threadIdx.x / 32 - 2) / 4 * WIDTH;
  headepi::Row<false> R(H, m, n0 + first, seq, t_pad);
  if (!wait()) return false;
  tc::tc_fence_after();
  float k = -INFINITY, s = 0.f;
#pragma unroll 1
  for (int c = first; c < first + WIDTH && n0 + c < H.vocab; c += 64) {
    uint32_t v[64];
    headepi::load_panel(acc, c / 64, v);
    headepi::stats64(H, R, v, n0 + c, k, s);
  }
  if (R.live && n0 + first < H.vocab) H.part[(long long)R.row * H.tiles + (n0 + first) / WIDTH] = make_float2(k, s);
  return true;
}

template <int BN, int SETS, typename Problem, typename Acc, typename Wait>
__device__ __forceinline__ bool head_grad_tile(const HeadEpi& H, const Problem& P, int m0, int n0, int q, Acc acc, uint32_t stg0, int& pc, Wait wait) {
  constexpr int WIDTH = SETS == 2 ? BN / 2 : BN;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, first = SETS != 2 ? 0 : (warp - 2) / 4 * WIDTH;
  headepi::Row<true> R(H, m0 + q * 32 + lane, H.col0 + n0 + first, P.seq, P.t_pad);
  if (!wait()) return false;
  tc::tc_fence_after();
#pragma unroll 1
  for (int c = first; c < first + WIDTH; c += 64) {
    const int n = n0 + c;
    if (n >= P.n) break;
    uint32_t v[64];
    headepi::load_panel(acc, c / 64, v);
    headepi::grad64(H, R, v, H.col0 + n);
    if (R.low) {
#pragma unroll
      for (int j = 0; j < 64; ++j) {
        const float f = __uint_as_float(v[j]);
        v[j] = __float_as_uint(f - __bfloat162float(__float2bfloat16_rn(f)));
      }
    }
    uint32_t ow[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) ow[j] = R.count ? tc::pack_bf16(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1])) : 0u;
    // as in epilogue_tile: the staging tile's last store has been read
    const uint32_t stg = stg0 + (SETS >= 2 ? (uint32_t)(warp - 2) : (uint32_t)(q * 2 + (pc & 1))) * 4096u;
    if (SETS >= 2 && lane == 0) tc::bulk_wait_group_read0();
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 8; ++j) tc::sts4(stg + lane * 128 + (((uint32_t)j ^ (uint32_t)(lane & 7)) * 16), &ow[4 * j]);
    tc::fence_proxy_async();
    __syncwarp();
    if (lane == 0) {
      tc::tma_store_3d(&P.tc, stg, 0, m0 + q * 32, n / 64);
      tc::bulk_commit_group();
      if (SETS == 1) tc::bulk_wait_group_read1();
    }
    ++pc;
  }
  return true;
}
