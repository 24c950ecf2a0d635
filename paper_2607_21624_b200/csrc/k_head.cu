// Around the head's products: targets made ready, softmax statistics joined into losses, and the passes over logits that fp32
// storage takes instead of the bf16 products' epilogues (head_epilogue.cuh has the formulas).
#include <math.h>

#include <type_traits>

#include "fbl_internal.h"
#include "k_head.h"
#include "pdl.cuh"
#include "tc_common.cuh"

namespace {

constexpr float LN2 = 0.69314718055994531f;

// What head_combine_kernel counts its blocks in, reset with the pass's status word.
__device__ __forceinline__ void start_pass(int32_t* status) {
  if (blockIdx.x == 0 && threadIdx.x == 0) status[0] = status[FBL_EARLY_COLSUM] = status[FBL_EARLY_ROUND] = status[HEAD_TICKET] = 0;
}

// Rows of tokens with a loss are brought together, so that the products behind spend nothing on the others (prompts and padding
// are a fifth to a half of a fine-tuning batch), and what those rows hold does not matter.  Block b has `per` rows from b * per on: it
// counts the tokens with a loss in front of them, then gives its own their positions and copies them.  Every block reads all
// labels in front of it, blocks x rows / 2 of them in all: `per` grows with the rows, so that this stays a small part of the
// copying.  TARGETS: labels make entries of probability 1 here; labels below zero carry no loss, labels past the vocabulary make it
// NaN.  Otherwise `count` has been filled.
constexpr int ROWS_THREADS = 256;
template <bool TARGETS>
__global__ void __launch_bounds__(ROWS_THREADS) head_rows_kernel(const int32_t* __restrict__ targets, HeadRows R, int seq, int t_pad, int vocab, int per,
                                                                 const uint4* __restrict__ X, uint4* __restrict__ Xc, int panels, int32_t* status) {
  __shared__ int s_warp[ROWS_THREADS / 32], s_pos[ROWS_THREADS];
  pdl_launch_dependents();
  pdl_wait();
  if (TARGETS) start_pass(status);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int first = blockIdx.x * per, end = min(first + per, (int)R.rows);
  auto block_sum = [&](int v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    __syncthreads();
    if (lane == 0) s_warp[warp] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < ROWS_THREADS / 32; ++w) v += s_warp[w];
    return v;
  };
  int before = 0;
  if (TARGETS) {                // labels have no padding between sequences
    const int b = first / t_pad, ahead = b * seq + min(first - b * t_pad, seq);
#pragma unroll 8
    for (int i = threadIdx.x; i < ahead; i += ROWS_THREADS) before += targets[i] >= 0;
  } else {
#pragma unroll 8
    for (int i = threadIdx.x; i < first; i += ROWS_THREADS) before += R.count[i] != 0;
  }
  before = block_sum(before);
  for (int r0 = first; r0 < end; r0 += ROWS_THREADS) {
    const int row = r0 + (int)threadIdx.x;
    bool counted = false;
    if (row < end) {
      if (TARGETS) {
        const int b = row / t_pad, t = row - b * t_pad;
        const int id = t < seq ? targets[b * seq + t] : -1;
        counted = id >= 0;
        R.count[row] = id < 0 ? 0 : id < vocab ? 1 : -1;
        R.constant[row] = id < vocab ? 0.f : NAN;
        R.ids[row] = id;
        R.y[row] = 1.f;
      } else {
        counted = R.count[row] != 0;
      }
    }
    const uint32_t mask = __ballot_sync(0xffffffffu, counted);
    const int total = block_sum(lane == 0 ? __popc(mask) : 0);          // (leaves the warps' counts in s_warp)
    int pos = before + __popc(mask & ((1u << lane) - 1));
    for (int w = 0; w < warp; ++w) pos += s_warp[w];
    if (!counted) pos = -1;
    if (row < end) R.pos[row] = pos;
    if (counted) R.row_of[pos] = row;
    s_pos[threadIdx.x] = pos;
    __syncthreads();
    // eight threads to a row's 128 bytes of a panel
    const int rows = min(ROWS_THREADS, end - r0), vecs = rows * 8;
#pragma unroll 8
    for (int i = threadIdx.x; i < panels * vecs; i += ROWS_THREADS) {
      const int p = i / vecs, rest = i - p * vecs, to = s_pos[rest / 8];
      if (to >= 0) Xc[((int64_t)p * R.rows + to) * 8 + rest % 8] = X[((int64_t)p * R.rows + r0) * 8 + rest];
    }
    before += total;
  }
  if (end < (int)R.rows) return;
  // the last block: how many there are, and zeros behind them up to a whole tile (a reduction over tokens ends inside a k-block)
  if (threadIdx.x == 0) { R.n[0] = before; R.n[1] = max(before, 1); }
  const int stop = min((int)R.rows, (max(before, 1) + 127) / 128 * 128), vecs = (stop - before) * 8;
  for (int i = threadIdx.x; i < panels * vecs; i += ROWS_THREADS) {
    const int p = i / vecs;
    Xc[((int64_t)p * R.rows + before) * 8 + (i - p * vecs)] = make_uint4(0u, 0u, 0u, 0u);
  }
}

// The same rows once more, for the backward.
__global__ void __launch_bounds__(256) head_gather_kernel(HeadRows R, const uint4* __restrict__ X, uint4* __restrict__ Xc, int all_panels, int32_t* status) {
  pdl_launch_dependents();
  pdl_wait();
  start_pass(status);
  const int c = blockIdx.x * 32 + threadIdx.x / 8, p0 = blockIdx.y * 8, panels = min(8, all_panels - p0);
  const int n = R.n[0], stop = (R.n[1] + 127) / 128 * 128;
  if (c >= min((int64_t)stop, R.rows)) return;
  const int row = c < n ? R.row_of[c] : -1;
  uint4 v[8];
#pragma unroll
  for (int p = 0; p < 8; ++p)
    if (p < panels) v[p] = row >= 0 ? X[((int64_t)(p0 + p) * R.rows + row) * 8 + threadIdx.x % 8] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
  for (int p = 0; p < 8; ++p)
    if (p < panels) Xc[((int64_t)(p0 + p) * R.rows + c) * 8 + threadIdx.x % 8] = v[p];
}

// A teacher's top logits: their softmax over the ids given, ids given twice added up, sorted by id.  A warp has a row, a lane up
// to four of its entries; every entry is compared with every other (K^2 broadcasts from shared memory: 4096 rows of 64 take about
// the time that their 2 MB take to arrive).  Additions go in the order of the entries.  Ids below zero are not there, a row without
// any, or whose logits are all -inf, carries no loss; ids past the vocabulary and logits of NaN or +inf make it NaN.
constexpr int ENTRY_WARPS = 8;
__global__ void __launch_bounds__(32 * ENTRY_WARPS) teacher_entries_kernel(const int32_t* __restrict__ ids, const float* __restrict__ logits,
                                                                           int top_k, float temperature, HeadRows R, int seq, int t_pad,
                                                                           int vocab, int32_t* status) {
  constexpr int PER = HEAD_MAX_TOP / 32;
  __shared__ int s_id[ENTRY_WARPS][HEAD_MAX_TOP];
  __shared__ float s_p[ENTRY_WARPS][HEAD_MAX_TOP];
  pdl_launch_dependents();
  pdl_wait();
  start_pass(status);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int row = blockIdx.x * ENTRY_WARPS + warp;
  if (row >= R.rows) return;
  const int b = row / t_pad, t = row - b * t_pad;
  const int64_t at = ((int64_t)b * seq + t) * top_k;
  int id[PER];
  float p[PER], top = -INFINITY;
  bool bad = false;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int e = j * 32 + lane;
    id[j] = t < seq && e < top_k ? ids[at + e] : -1;
    p[j] = id[j] >= 0 ? logits[at + e] / temperature : -INFINITY;
    bad = bad || id[j] >= vocab || p[j] != p[j];
    top = fmaxf(top, p[j]);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  bad = __any_sync(0xffffffffu, bad) || top == INFINITY;
  if (bad || top == -INFINITY) {
    if (lane == 0) { R.count[row] = bad ? -1 : 0; R.constant[row] = bad ? NAN : 0.f; }
    return;
  }
  float sum = 0.f;
#pragma unroll
  for (int j = 0; j < PER; ++j) { p[j] = expf(p[j] - top); sum += p[j]; }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int e = j * 32 + lane;
    p[j] /= sum;
    s_id[warp][e] = id[j];
    s_p[warp][e] = p[j];
  }
  __syncwarp();
  // an id's first entry takes the probability of all of them
  bool first[PER];
  float y[PER];
#pragma unroll
  for (int j = 0; j < PER; ++j) { first[j] = id[j] >= 0; y[j] = 0.f; }
  for (int e = 0; e < top_k; ++e) {
    const int other = s_id[warp][e];
    const float q = s_p[warp][e];
#pragma unroll
    for (int j = 0; j < PER; ++j)
      if (other == id[j]) { y[j] += q; first[j] = first[j] && e >= j * 32 + lane; }
  }
  __syncwarp();
#pragma unroll
  for (int j = 0; j < PER; ++j)
    if (!first[j]) s_id[warp][j * 32 + lane] = headk::NONE;
  __syncwarp();
  int rank[PER] = {}, count = 0;
  float constant = 0.f;
  for (int e = 0; e < top_k; ++e) {
    const int other = s_id[warp][e];
    count += other != headk::NONE;
#pragma unroll
    for (int j = 0; j < PER; ++j) rank[j] += other < id[j];
  }
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    if (!first[j]) continue;
    R.ids[(int64_t)rank[j] * R.rows + row] = id[j];
    R.y[(int64_t)rank[j] * R.rows + row] = y[j];
    if (y[j] > 0.f) constant = fmaf(y[j], logf(y[j]), constant);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) constant += __shfl_xor_sync(0xffffffffu, constant, o);
  if (lane == 0) { R.count[row] = count; R.constant[row] = constant; }
}

// (k, s) stands for s 2^k.
__device__ __forceinline__ void join(float& k, float& s, float k2, float s2) {
  const float top = fmaxf(k, k2);
  s = (k == top ? s : s * exp2f(k - top)) + (k2 == top ? s2 : s2 * exp2f(k2 - top));
  k = top;
}

// A block has eight rows, thirty-two threads to each, which share the row's partials and its entries; all joins and sums go in a
// fixed order.  loss = sum of y (log y - logit) + log of the sum of exp(logit).  The block that ends last adds the blocks' sums up.
// What bounds it is reading the partials, 8 bytes a row and tile; eight rows of a tile are one 64-byte piece.
__global__ void __launch_bounds__(256) head_combine_kernel(const float2* __restrict__ part, int tiles, const float* __restrict__ z_at,
                                                           HeadRows R, float scale, float* __restrict__ loss, float* __restrict__ total,
                                                           float* __restrict__ block_sums, int seq, int t_pad, int32_t* status) {
  __shared__ float s_k[32][8], s_s[32][8], s_y[32][8];
  __shared__ float s_loss[8];
  __shared__ double s_sum[256], s_count[256];
  __shared__ int s_last;
  pdl_launch_dependents();
  pdl_wait();
  const int r = threadIdx.x % 8, slice = threadIdx.x / 8, row = blockIdx.x * 8 + r;      // rows come in eights
  float k = -INFINITY, s = 0.f;
  const int pos = R.pos[row];
  int tile = pos < 0 ? tiles : slice;       // rows without a loss have no partials
  for (; tile + 96 < tiles; tile += 128) {
    float2 v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = part[(int64_t)(tile + 32 * u) * R.rows + pos];
#pragma unroll
    for (int u = 0; u < 4; ++u) join(k, s, v[u].x, v[u].y);
  }
  for (; tile < tiles; tile += 32) {
    const float2 v = part[(int64_t)tile * R.rows + pos];
    join(k, s, v.x, v.y);
  }
  s_k[slice][r] = k;
  s_s[slice][r] = s;
  __syncthreads();
  for (int n = 16; n > 0; n /= 2) {
    if (slice < n) join(s_k[slice][r], s_s[slice][r], s_k[slice + n][r], s_s[slice + n][r]);
    __syncthreads();
  }
  k = s_k[0][r];
  s = s_s[0][r];
  const int count = R.count[row];
  float toward = 0.f;                       // sum of y (k - c z)
  for (int e = slice; e < count; e += 32) {
    const float y = R.y[(int64_t)e * R.rows + row];
    if (y != 0.f) toward = fmaf(y, -fmaf(z_at[(int64_t)e * R.rows + row], scale, -k), toward);
  }
  s_y[slice][r] = toward;
  __syncthreads();
  for (int n = 16; n > 0; n /= 2) {
    if (slice < n) s_y[slice][r] += s_y[slice + n][r];
    __syncthreads();
  }
  if (slice == 0) {
    const float l = count == 0 ? 0.f : count < 0 ? NAN : fmaf(LN2, s_y[0][r], logf(s)) + R.constant[row];
    const int b = row / t_pad, t = row - b * t_pad;
    if (t < seq) loss[(int64_t)b * seq + t] = l;
    R.k[row] = k;
    R.sum[row] = s;
    s_loss[r] = l;
    s_y[0][r] = count != 0 ? 1.f : 0.f;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    float l = 0.f, n = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) { l += s_loss[i]; n += s_y[0][i]; }
    block_sums[2 * blockIdx.x] = l;
    block_sums[2 * blockIdx.x + 1] = n;
    __threadfence();
    s_last = atomicAdd(status + HEAD_TICKET, 1) == (int)gridDim.x - 1;
  }
  __syncthreads();
  if (!s_last) return;
  __threadfence();
  double l = 0.0, n = 0.0;
  for (int i = threadIdx.x; i < (int)gridDim.x; i += 256) {
    const float2 v = __ldcg(reinterpret_cast<const float2*>(block_sums) + i);
    l += v.x;
    n += v.y;
  }
  s_sum[threadIdx.x] = l;
  s_count[threadIdx.x] = n;
  __syncthreads();
  for (int m = 128; m > 0; m /= 2) {
    if ((int)threadIdx.x < m) { s_sum[threadIdx.x] += s_sum[threadIdx.x + m]; s_count[threadIdx.x] += s_count[threadIdx.x + m]; }
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    total[0] = R.total[0] = (float)s_sum[0];
    total[1] = R.total[1] = (float)s_count[0];
  }
}

// fp32 storage: the logits of a piece of the vocabulary are in memory, [panel of 32 columns][product's row][32].  A block has 32 rows and
// HEAD_TILE columns, eight threads to a row with 16 bytes each: one pass over the logits, bound by memory.
constexpr int F32_PANELS = HEAD_TILE / 32;

__global__ void __launch_bounds__(256) head_stats_f32_kernel(const float* __restrict__ z, HeadRows R, int vocab, int col0, float scale,
                                                             float2* __restrict__ part, float* __restrict__ z_at) {
  pdl_launch_dependents();
  pdl_wait();
  const int c = blockIdx.x * 32 + threadIdx.x / 8, l8 = threadIdx.x % 8;
  const int n0 = blockIdx.y * HEAD_TILE;
  const bool live = c < R.n[0];
  float k = -INFINITY, s = 0.f;
  float4 v[F32_PANELS];
#pragma unroll
  for (int p = 0; p < F32_PANELS; ++p) {
    const int n = n0 + p * 32 + l8 * 4;
    v[p] = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
    if (!live || col0 + n >= vocab) continue;
    v[p] = *reinterpret_cast<const float4*>(z + rt_off<32>(R.rows, c, n));
    if (col0 + n + 1 >= vocab) v[p].y = -INFINITY;
    if (col0 + n + 2 >= vocab) v[p].z = -INFINITY;
    if (col0 + n + 3 >= vocab) v[p].w = -INFINITY;
  }
#pragma unroll
  for (int p = 0; p < F32_PANELS; ++p) k = fmaxf(k, fmaxf(fmaxf(v[p].x, v[p].y), fmaxf(v[p].z, v[p].w)));
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) k = fmaxf(k, __shfl_xor_sync(0xffffffffu, k, o));
  k *= scale;
#pragma unroll
  for (int p = 0; p < F32_PANELS; ++p)
    s += (exp2f(fmaf(v[p].x, scale, -k)) + exp2f(fmaf(v[p].y, scale, -k))) + (exp2f(fmaf(v[p].z, scale, -k)) + exp2f(fmaf(v[p].w, scale, -k)));
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (!live) return;
  if (l8 == 0) part[(int64_t)((col0 + n0) / HEAD_TILE) * R.rows + c] = make_float2(k, s);
  const int row = R.row_of[c], count = R.count[row];
  for (int e = l8; e < count; e += 8) {
    const int n = R.ids[(int64_t)e * R.rows + row] - col0;
    if (n >= n0 && n < n0 + HEAD_TILE) z_at[(int64_t)e * R.rows + row] = z[rt_off<32>(R.rows, c, n)];
  }
}

// dz over z, in place; zeros behind the last row with a loss, up to a whole tile.
__global__ void __launch_bounds__(256) head_grad_f32_kernel(float* __restrict__ z, HeadRows R, const float* __restrict__ dloss, int vocab,
                                                            int col0, int cols, float scale, float inv_tau, int seq, int t_pad) {
  pdl_launch_dependents();
  pdl_wait();
  const int c = blockIdx.x * 32 + threadIdx.x / 8, l8 = threadIdx.x % 8;
  const int n0 = blockIdx.y * HEAD_TILE;
  const bool live = c < min(R.rows, (int64_t)(R.n[1] + 127) / 128 * 128);
  const int row = c < R.n[0] ? R.row_of[c] : -1;
  int count = 0;
  float g = 0.f, gs = 0.f, k = 0.f;
  if (live) {
    count = row >= 0 ? R.count[row] : 0;
    if (count > 0) {
      const int b = row / t_pad, t = row - b * t_pad;
      g = (dloss ? dloss[(int64_t)b * seq + t] : 1.f / R.total[1]) * inv_tau;
      k = R.k[row];
      gs = g / R.sum[row];
    } else if (count < 0) {
      gs = NAN;
    }
#pragma unroll
    for (int p = 0; p < F32_PANELS; ++p) {
      const int n = n0 + p * 32 + l8 * 4;
      if (n >= cols) break;
      float4* at = reinterpret_cast<float4*>(z + rt_off<32>(R.rows, c, n));
      const float4 v = *at;
      float d[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) d[i] = count && col0 + n + i < vocab ? exp2f(fmaf(d[i], scale, -k)) * gs : 0.f;
      *at = make_float4(d[0], d[1], d[2], d[3]);
    }
  }
  __syncthreads();
  for (int e = l8; e < count; e += 8) {           // distinct ids: no two threads meet
    const int n = R.ids[(int64_t)e * R.rows + row] - col0;
    if (n >= n0 && n < min(n0 + HEAD_TILE, cols)) z[rt_off<32>(R.rows, c, n)] -= g * R.y[(int64_t)e * R.rows + row];
  }
}

// dX: the areas' sums, in their order, times alpha / max(*over, 1) where `over` is not null, at the tokens' own rows, and zeros at the
// rows without a loss.  Four consecutive columns a thread; bound by memory.
template <typename T>
__global__ void __launch_bounds__(256) head_scatter_kernel(const float* __restrict__ acc, int areas, HeadRows R, int64_t n, const float* __restrict__ over,
                                                           float alpha, T* __restrict__ dX) {
  constexpr int TW = tile_w_of<T>::value;
  pdl_launch_dependents();
  pdl_wait();
  const float a = over ? alpha / fmaxf(*over, 1.f) : 1.f;
  for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < n; i += (int64_t)gridDim.x * 1024) {
    const int64_t line = i / TW, panel = line / R.rows;
    const int pos = R.pos[line - panel * R.rows];
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (pos >= 0) {
      const float* from = acc + (panel * R.rows + pos) * TW + i % TW;
#pragma unroll 8
      for (int k = 0; k < areas; ++k) {
        const float4 v = __ldcg(reinterpret_cast<const float4*>(from + k * n));
        s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
      }
    }
    if constexpr (sizeof(T) == 2) {
      uint2 o;
      o.x = tc::pack_bf16(s.x * a, s.y * a);
      o.y = tc::pack_bf16(s.z * a, s.w * a);
      *reinterpret_cast<uint2*>(dX + i) = o;
    } else {
      *reinterpret_cast<float4*>(dX + i) = s;
    }
  }
}

// Pack and unpack of a matrix whose columns are not whole tiles: [rows][cols] and [panel][row][128 bytes] with zeros past the last.
template <typename T, bool PACK>
__global__ void __launch_bounds__(256) pack_columns_kernel(const T* __restrict__ src, T* __restrict__ dst, int64_t rows, int cols, int64_t n) {
  constexpr int TW = tile_w_of<T>::value;
  pdl_wait();                   // no early trigger: the kernel behind may request weights before it waits
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t line = i / TW, r = line % rows;
    const int64_t c = line / rows * TW + i % TW;
    if (PACK) dst[i] = c < cols ? src[r * cols + c] : from_f<T>(0.f);
    else if (c < cols) dst[r * cols + c] = src[i];
  }
}

}  // namespace

cudaError_t launch_pack_columns(int dtype, int unpack, const void* src, void* dst, int64_t rows, int cols, int padded, cudaStream_t st) {
  const int64_t n = rows * padded;
  const dim3 grid((unsigned)min((int64_t)148 * 16, (n + 255) / 256));
  auto go = [&](auto kernel, auto* t) {
    using T = std::remove_pointer_t<decltype(t)>;
    return launch_pdl(kernel, grid, dim3(256), 0, st, (const T*)src, (T*)dst, rows, cols, n);
  };
  if (dtype == FBL_DTYPE_FP32) return unpack ? go(pack_columns_kernel<float, false>, (float*)0) : go(pack_columns_kernel<float, true>, (float*)0);
  return unpack ? go(pack_columns_kernel<__nv_bfloat16, false>, (__nv_bfloat16*)0) : go(pack_columns_kernel<__nv_bfloat16, true>, (__nv_bfloat16*)0);
}
cudaError_t launch_head_rows(int dtype, const int32_t* targets, const HeadRows& R, int seq, int t_pad, int vocab, const void* X, void* Xc, int d_model,
                             int32_t* status, cudaStream_t st) {
  const int panels = d_model / (dtype == FBL_DTYPE_FP32 ? 32 : 64);
  const int64_t per = R.rows <= 32 * 1024 ? 32 : (R.rows / 1024 + 31) / 32 * 32;
  return launch_pdl(targets ? head_rows_kernel<true> : head_rows_kernel<false>, dim3((unsigned)((R.rows + per - 1) / per)), dim3(ROWS_THREADS), 0, st,
                    targets, R, seq, t_pad, vocab, (int)per, (const uint4*)X, (uint4*)Xc, panels, status);
}
cudaError_t launch_head_gather(int dtype, const HeadRows& R, const void* X, void* Xc, int d_model, int32_t* status, cudaStream_t st) {
  const int panels = d_model / (dtype == FBL_DTYPE_FP32 ? 32 : 64);
  return launch_pdl(head_gather_kernel, dim3((unsigned)((R.rows + 31) / 32), (unsigned)((panels + 7) / 8)), dim3(256), 0, st, R, (const uint4*)X,
                    (uint4*)Xc, panels, status);
}
cudaError_t launch_teacher_entries(const int32_t* ids, const float* logits, int top_k, float temperature, const HeadRows& R, int seq, int t_pad,
                                   int vocab, int32_t* status, cudaStream_t st) {
  return launch_pdl(teacher_entries_kernel, dim3((unsigned)((R.rows + ENTRY_WARPS - 1) / ENTRY_WARPS)), dim3(32 * ENTRY_WARPS), 0, st, ids, logits,
                    top_k, temperature, R, seq, t_pad, vocab, status);
}
cudaError_t launch_head_combine(const float2* part, int tiles, const float* z_at, const HeadRows& R, float scale, float* loss, float* total,
                                float* block_sums, int seq, int t_pad, int32_t* status, cudaStream_t st) {
  return launch_pdl(head_combine_kernel, dim3((unsigned)(R.rows / 8)), dim3(256), 0, st, part, tiles, z_at, R, scale, loss, total, block_sums, seq,
                    t_pad, status);
}
cudaError_t launch_head_stats_f32(const float* z, const HeadRows& R, int vocab, int col0, int cols, float scale, float2* part, float* z_at,
                                  cudaStream_t st) {
  return launch_pdl(head_stats_f32_kernel, dim3((unsigned)((R.rows + 31) / 32), (unsigned)((cols + HEAD_TILE - 1) / HEAD_TILE)), dim3(256), 0, st, z, R,
                    vocab, col0, scale, part, z_at);
}
cudaError_t launch_head_grad_f32(float* z, const HeadRows& R, const float* dloss, int vocab, int col0, int cols, float scale, float inv_tau, int seq,
                                 int t_pad, cudaStream_t st) {
  return launch_pdl(head_grad_f32_kernel, dim3((unsigned)((R.rows + 31) / 32), (unsigned)((cols + HEAD_TILE - 1) / HEAD_TILE)), dim3(256), 0, st, z, R,
                    dloss, vocab, col0, cols, scale, inv_tau, seq, t_pad);
}
cudaError_t launch_head_scatter(int dtype, int sm_count, const float* acc, int areas, const HeadRows& R, int d_model, const float* over, float alpha,
                                void* dX, cudaStream_t st) {
  const int64_t n = R.rows * d_model;
  const dim3 grid((unsigned)min((int64_t)sm_count * 8, (n / 4 + 255) / 256));
  if (dtype == FBL_DTYPE_FP32) return launch_pdl(head_scatter_kernel<float>, grid, dim3(256), 0, st, acc, areas, R, n, over, alpha, (float*)dX);
  return launch_pdl(head_scatter_kernel<__nv_bfloat16>, grid, dim3(256), 0, st, acc, areas, R, n, over, alpha, (__nv_bfloat16*)dX);
}
