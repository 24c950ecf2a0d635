// Around the head's products: targets made ready and rows brought together, softmax statistics joined into losses, dX's areas added
// up and taken back to their rows (head_epilogue.cuh has the formulas).
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

// A block forms an entry's product again, of bf16 values exactly and summed in 64 bits.  The tensor core's own sums are off by some 2^-23
// of themselves, either way, which over many tokens averages out and of a few is what their losses are off by (one token of 2048 over
// 128256 columns, twenty draws: up to 4.2e-6, 3.0e-6 of the loss, and with this 4.7e-7, 2.5e-7 of it).  It hides beside the rows' copies: a thread's loads are all on their way at once (a warp for an entry,
// 5 tokens of 3392 with weights by columns: 8 us more).
template <bool TARGETS>
__device__ __forceinline__ void exact_products(const HeadExact& E, const int32_t* __restrict__ targets, const HeadRows& R, int seq, int t_pad, int vocab,
                                               const uint4* __restrict__ X, int first, int step) {
  constexpr int U = 2;
  __shared__ double s_sum[8];
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  for (int64_t i = first; i < R.rows * E.top_k; i += step) {
    const int row = (int)(i % R.rows), e = (int)(i / R.rows), b = row / t_pad, t = row - b * t_pad;
    const int id = TARGETS ? (t < seq ? targets[b * seq + t] : -1) : e < R.count[row] ? R.ids[i] : -1;
    if (id < 0 || id >= vocab) continue;       // the block's threads alike
    const __nv_bfloat16* W = (const __nv_bfloat16*)E.W;
    double sum = 0.0;
    for (int v0 = threadIdx.x; v0 < E.d_model / 8; v0 += 256 * U) {
      uint4 x[U];
      __align__(16) __nv_bfloat16 w[U][8];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int v = v0 + 256 * u;
        x[u] = make_uint4(0u, 0u, 0u, 0u);
        *reinterpret_cast<uint4*>(w[u]) = x[u];
        if (v >= E.d_model / 8) continue;
        x[u] = X[((int64_t)(v / 8) * R.rows + row) * 8 + v % 8];
        if (E.vocab_rows) {
          *reinterpret_cast<uint4*>(w[u]) = *reinterpret_cast<const uint4*>(W + ((int64_t)(v / 8) * E.w_rows + id) * 64 + v % 8 * 8);
        } else {
#pragma unroll
          for (int k = 0; k < 8; ++k) w[u][k] = W[((int64_t)(id / 64) * E.w_rows + v * 8 + k) * 64 + id % 64];
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const __nv_bfloat16* xs = reinterpret_cast<const __nv_bfloat16*>(&x[u]);
#pragma unroll
        for (int k = 0; k < 8; ++k) sum = fma((double)__bfloat162float(xs[k]), (double)__bfloat162float(w[u][k]), sum);
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) s_sum[warp] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
      double all = 0.0;
#pragma unroll
      for (int w = 0; w < 8; ++w) all += s_sum[w];
      E.z[i] = all;
    }
    __syncthreads();
  }
}

// Rows of tokens with a loss are brought together, so that the products behind spend nothing on the others (prompts and padding
// are a fifth to a half of a fine-tuning batch), and what those rows hold does not matter.  A block has `per` rows from its first on
// and eight column panels of X: it counts the tokens with a loss in front of them, then gives its own their positions and copies
// them, 32 rows at a time.  Every block reads all labels in front of it (rows x blocks / 2 of them in all, from L2: 33 MB of reads for
// 8192 x 4096, beside a copy of 134 MB; `per` grows with the rows), and loads its rows of X before it knows where they go: what a
// short pass waits for here is a chain of memory latencies.  TARGETS: labels make entries of probability 1; labels below zero carry
// no loss, labels past the vocabulary make it NaN.  Otherwise `count` has been filled.
constexpr int ROWS_PANELS = 8;
template <bool TARGETS>
__global__ void __launch_bounds__(256) head_rows_kernel(const int32_t* __restrict__ targets, HeadRows R, int seq, int t_pad, int vocab, int per,
                                                        const uint4* __restrict__ X, uint4* __restrict__ Xc, int all_panels, const HeadExact exact, int32_t* status) {
  __shared__ int s_before[8], s_pos[32], s_count;
  pdl_wait();
  pdl_launch_dependents();      // after the wait: the product behind may ask for weights early, and what wrote them is complete then
  const int groups = (all_panels + ROWS_PANELS - 1) / ROWS_PANELS;
  if ((int)blockIdx.y >= groups) {             // the blocks behind those that copy
    exact_products<TARGETS>(exact, targets, R, seq, t_pad, vocab, X, (blockIdx.y - groups) * gridDim.x + blockIdx.x, (gridDim.y - groups) * gridDim.x);
    return;
  }
  const bool lead = blockIdx.y == 0;
  if (TARGETS && lead) start_pass(status);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, r = threadIdx.x / 8, vec = threadIdx.x % 8;
  const int first = blockIdx.x * per, end = min(first + per, (int)R.rows);
  const int p0 = blockIdx.y * ROWS_PANELS, panels = min(ROWS_PANELS, all_panels - p0);
  const uint4* from = X + (int64_t)p0 * R.rows * 8 + vec;
  uint4* to = Xc + (int64_t)p0 * R.x_rows * 8 + vec;
  const int64_t pitch = R.rows * 8, x_pitch = R.x_rows * 8;
  uint4 x[ROWS_PANELS];
  auto load = [&](int row) {
#pragma unroll
    for (int p = 0; p < ROWS_PANELS; ++p)
      if (p < panels && row < end) x[p] = from[p * pitch + (int64_t)row * 8];
  };
  load(first + r);
  int before = 0;
  if (TARGETS) {                // labels have no padding between sequences
    const int b = first / t_pad, ahead = b * seq + min(first - b * t_pad, seq);
#pragma unroll 4
    for (int i = threadIdx.x; i < ahead; i += 256) before += targets[i] >= 0;
  } else {
#pragma unroll 4
    for (int i = threadIdx.x; i < first; i += 256) before += R.count[i] != 0;
  }
  before = __reduce_add_sync(0xffffffffu, before);
  if (lane == 0) s_before[warp] = before;
  __syncthreads();
  before = 0;
#pragma unroll
  for (int w = 0; w < 8; ++w) before += s_before[w];
#pragma unroll 1
  for (int r0 = first; r0 < end; r0 += 32) {
    if (warp == 0) {
      const int row = r0 + lane;
      bool counted = false;
      if (row < end) {
        if (TARGETS) {
          const int b = row / t_pad, t = row - b * t_pad;
          const int id = t < seq ? targets[b * seq + t] : -1;
          counted = id >= 0;
          if (lead) {
            R.count[row] = id < 0 ? 0 : id < vocab ? 1 : -1;
            R.constant[row] = id < vocab ? 0.f : NAN;
            R.ids[row] = id;
            R.y[row] = 1.f;
          }
        } else {
          counted = R.count[row] != 0;
        }
      }
      const uint32_t mask = __ballot_sync(0xffffffffu, counted);
      const int pos = counted ? before + __popc(mask & ((1u << lane) - 1)) : -1;
      if (lead && row < end) {
        R.pos[row] = pos;
        if (counted) R.row_of[pos] = row;
      }
      s_pos[lane] = pos;
      if (lane == 0) s_count = __popc(mask);
    }
    __syncthreads();
    const int pos = s_pos[r];
    if (pos >= 0) {
#pragma unroll
      for (int p = 0; p < ROWS_PANELS; ++p) {
        if (p >= panels) break;
        to[p * x_pitch + (int64_t)pos * 8] = x[p];
        if (R.second) to[p * x_pitch + (int64_t)(pos + R.second) * 8] = x[p];
      }
    }
    before += s_count;
    if (r0 + 32 < end) load(r0 + 32 + r);
    __syncthreads();
  }
  if (end < (int)R.rows) return;
  // the last rows' blocks: how many there are, and zeros behind them up to a whole tile (a reduction over tokens ends inside a k-block)
  if (lead && threadIdx.x == 0) { R.n[0] = before; R.n[1] = max(before, 1); }
  const int stop = R.second ? R.second : min((int)R.x_rows, (max(before, 1) + 127) / 128 * 128);
  for (int c = before + r; c < stop; c += 32)
    for (int p = 0; p < panels; ++p) {
      to[p * x_pitch + (int64_t)c * 8] = make_uint4(0u, 0u, 0u, 0u);
      if (R.second) to[p * x_pitch + (int64_t)(c + R.second) * 8] = make_uint4(0u, 0u, 0u, 0u);
    }
}

// A teacher's top logits: their softmax over the ids given, ids given twice added up, sorted by id.  A warp has a row, a lane every
// 32nd of its entries (PER of them, as top_k needs): keys of an id and the entry's place are sorted in registers by exchanges, so
// that equal ids are neighbours, in the order of the list, and are added up in it.  Ids below zero are not there, a row without
// any, or whose logits are all -inf, carries no loss; ids past the vocabulary and logits of NaN or +inf make it NaN.  The block's
// eight rows leave through shared memory, eight values of an entry to a 32-byte sector.  Bound by instructions.  (Every entry compared
// with every other, and a warp storing its own row's: 24.5 us for 4096 rows of 64.)
constexpr int ENTRY_WARPS = 8;
template <int PER>
__global__ void __launch_bounds__(32 * ENTRY_WARPS) teacher_entries_kernel(const int32_t* __restrict__ ids, const float* __restrict__ logits,
                                                                           int top_k, float temperature, HeadRows R, int seq, int t_pad,
                                                                           int vocab, int32_t* status) {
  constexpr int N = 32 * PER;
  constexpr uint32_t NO_KEY = 0xffffffffu;
  static_assert(HEAD_MAX_TOP <= 128, "a key is an id times 128 and a place");
  __shared__ float s_p[ENTRY_WARPS][N], s_y[N][ENTRY_WARPS];
  __shared__ uint32_t s_key[ENTRY_WARPS][N];
  __shared__ int s_id[N][ENTRY_WARPS], s_count[ENTRY_WARPS];
  pdl_launch_dependents();
  pdl_wait();
  start_pass(status);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int row = blockIdx.x * ENTRY_WARPS + warp;             // rows come in eights
  const int b = row / t_pad, t = row - b * t_pad;
  const int64_t at = ((int64_t)b * seq + t) * top_k;
  uint32_t key[PER];
  float p[PER], top = -INFINITY;
  bool bad = false;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int e = j * 32 + lane;
    const bool in = t < seq && e < top_k;
    const int id = in ? ids[at + e] : -1;
    const float z = in ? logits[at + e] : 0.f;
    key[j] = id >= 0 ? (uint32_t)id * 128u + (uint32_t)e : NO_KEY;
    p[j] = id >= 0 ? z : -INFINITY;
    bad = bad || id >= vocab || p[j] != p[j];
    top = fmaxf(top, p[j]);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  bad = __any_sync(0xffffffffu, bad) || top == INFINITY;
  int count = 0;
  float constant = 0.f;
  if (!bad && top > -INFINITY) {
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < PER; ++j) { p[j] = expf((p[j] - top) / temperature); sum += p[j]; }      // (a quotient alone may leave fp32, and is rounded at its own size)
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
#pragma unroll
    for (int j = 0; j < PER; ++j) s_p[warp][j * 32 + lane] = p[j] / sum;
    // bitonic sort: key number i is key[i / 32] of lane i % 32
#pragma unroll
    for (int size = 2; size <= N; size *= 2)
#pragma unroll
      for (int d = size / 2; d > 0; d /= 2) {
        if (d >= 32) {
#pragma unroll
          for (int j = 0; j < PER; ++j) {
            if (j & (d / 32)) continue;
            const bool up = ((j * 32) & size) == 0;
            const uint32_t lo = min(key[j], key[(j + d / 32) % PER]), hi = max(key[j], key[(j + d / 32) % PER]);
            key[j] = up ? lo : hi;
            key[(j + d / 32) % PER] = up ? hi : lo;
          }
        } else {
#pragma unroll
          for (int j = 0; j < PER; ++j) {
            const uint32_t other = __shfl_xor_sync(0xffffffffu, key[j], d);
            const bool up = ((j * 32 + lane) & size) == 0, low = (lane & d) == 0;
            key[j] = up == low ? min(key[j], other) : max(key[j], other);
          }
        }
      }
#pragma unroll
    for (int j = 0; j < PER; ++j) s_key[warp][j * 32 + lane] = key[j];
    __syncwarp();
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int i = j * 32 + lane;
      const uint32_t id = key[j] / 128u;
      const bool first = key[j] != NO_KEY && (i == 0 || s_key[warp][i - 1] / 128u != id);
      const uint32_t firsts = __ballot_sync(0xffffffffu, first);
      if (first) {                                             // takes the probability of the id's other places, too
        float y = s_p[warp][key[j] % 128u];
        for (int n = i + 1; n < N && s_key[warp][n] != NO_KEY && s_key[warp][n] / 128u == id; ++n) y += s_p[warp][s_key[warp][n] % 128u];
        const int rank = count + __popc(firsts & ((1u << lane) - 1));
        s_id[rank][warp] = (int)id;
        s_y[rank][warp] = y;
        if (y > 0.f) constant = fmaf(y, logf(y), constant);
      }
      count += __popc(firsts);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) constant += __shfl_xor_sync(0xffffffffu, constant, o);
  }
  if (lane == 0) {
    R.count[row] = bad ? -1 : count;
    R.constant[row] = bad ? NAN : constant;
    s_count[warp] = count;
  }
  __syncthreads();
  const int r = threadIdx.x % ENTRY_WARPS, mine = s_count[r];
  for (int e = threadIdx.x / ENTRY_WARPS; e < mine; e += 32) {
    R.ids[(int64_t)e * R.rows + blockIdx.x * ENTRY_WARPS + r] = s_id[e][r];
    R.y[(int64_t)e * R.rows + blockIdx.x * ENTRY_WARPS + r] = s_y[e][r];
  }
}

// s 2^(c k) in units of 2^(c top), where k is at most top; nothing where nothing has been added up (k = -inf: of two such, -inf - -inf
// is NaN).
__device__ __forceinline__ float scaled(float k, float s, float top, float c) { return k == top ? s : s * exp2f((k - top) * c); }

// A warp has a row at a time: its lanes share the row's partials, which lie behind each other, and its entries; all joins and sums go in
// a fixed order.  loss = sum of y (log y - logit) + log of the sum of exp(logit).  What bounds it is latency, so all that a row needs is
// asked for at once (of rows without a loss, too, whose partials are nothing), and up to 64 rows are one block's, which adds its
// losses up itself; of several blocks the one that ends last does, two latencies later.
constexpr int COMBINE_FEW = 64;
template <bool EXACT>
__global__ void __launch_bounds__(1024) head_combine_kernel(const float2* __restrict__ part, int tiles, const float* __restrict__ z_at,
                                                            HeadRows R, float scale, float* __restrict__ loss, float* __restrict__ total,
                                                            double2* __restrict__ block_sums, int seq, int t_pad, const HeadExact exact, int32_t* status) {
  constexpr int U = 8;
  __shared__ double s_sum[32], s_count[32];
  __shared__ int s_last;
  pdl_launch_dependents();
  pdl_wait();
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, warps = blockDim.x / 32;
  double sum = 0.0, counted = 0.0;
  for (int row = blockIdx.x * warps + warp; row < R.rows; row += gridDim.x * warps) {
    const float2* mine = part + (int64_t)row * tiles;
    float2 v[U];
    auto load = [&](int t0) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int t = t0 + 32 * u + lane;
        v[u] = t < tiles ? __ldcg(mine + t) : make_float2(-INFINITY, 0.f);
      }
    };
    load(0);
    const float y0 = R.y[row], z0 = __ldcg(z_at + row), constant = R.constant[row];      // entry 0, which lane 0 takes
    const double x0 = EXACT ? __ldcg(exact.z + row) : 0.0;
    const int count = R.count[row];
    float l = 0.f;
    if (count != 0) {
      float k = -INFINITY, s = 0.f;
#pragma unroll 1
      for (int t0 = 0;;) {
        float top = v[0].x, some = 0.f;                        // the largest first: the exponentials then do not wait for one another
#pragma unroll
        for (int u = 1; u < U; ++u) top = fmaxf(top, v[u].x);
#pragma unroll
        for (int u = 0; u < U; ++u) some += scaled(v[u].x, v[u].y, top, scale);
        const float both = fmaxf(k, top);
        s = scaled(k, s, both, scale) + scaled(top, some, both, scale);
        k = both;
        if ((t0 += 32 * U) >= tiles) break;
        load(t0);
      }
      float top = k;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      s = scaled(k, s, top, scale);
      k = top;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      float toward = 0.f, more = 0.f;       // sum of y c (k - z); what s lacks, or has too much of, at the targets
      for (int e = lane; e < count; e += 32) {
        const float y = e ? R.y[(int64_t)e * R.rows + row] : y0, z = e ? __ldcg(z_at + (int64_t)e * R.rows + row) : z0;
        if (y != 0.f) toward = fmaf(y, (k - z) * scale, toward);
        if (EXACT) {
          const double x = e ? __ldcg(exact.z + (int64_t)e * R.rows + row) : x0;
          const float off = (float)(x * exact.unlift - (double)z) * scale;
          if (fabsf(off) < 1.f) {           // (of infinities, none)
            toward = fmaf(-y, off, toward);
            more = fmaf(exp2f((z - k) * scale), expm1f(LN2 * off), more);
          }
        }
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) toward += __shfl_xor_sync(0xffffffffu, toward, o);
      l = fmaf(LN2, toward, logf(s)) + constant;
      if (EXACT) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) more += __shfl_xor_sync(0xffffffffu, more, o);
        l += log1pf(more / s);
      }
      if (count < 0) l = NAN;
      if (lane == 0) { R.k[row] = k; R.sum[row] = s; }
      sum += l;
      counted += 1.0;
    }
    const int b = row / t_pad, t = row - b * t_pad;
    if (lane == 0 && t < seq) loss[(int64_t)b * seq + t] = l;
  }
  if (lane == 0) { s_sum[warp] = sum; s_count[warp] = counted; }
  __syncthreads();
  auto whole = [&](double& a, double& n) {                     // by thread 0
    a = n = 0.0;
    for (int w = 0; w < warps; ++w) { a += s_sum[w]; n += s_count[w]; }
  };
  auto publish = [&](double a, double n) {
    total[0] = R.total[0] = (float)a;
    total[1] = R.total[1] = (float)n;
  };
  if (threadIdx.x == 0) {
    double a, n;
    whole(a, n);
    if (gridDim.x == 1) {
      publish(a, n);
    } else {
      block_sums[blockIdx.x] = make_double2(a, n);
      __threadfence();
      s_last = atomicAdd(status + HEAD_TICKET, 1) == (int)gridDim.x - 1;
    }
  }
  if (gridDim.x == 1) return;
  __syncthreads();
  if (!s_last) return;
  __threadfence();
  double a = 0.0, n = 0.0;
#pragma unroll 4
  for (int i = threadIdx.x; i < (int)gridDim.x; i += blockDim.x) {
    const double2 v = __ldcg(block_sums + i);
    a += v.x;
    n += v.y;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    a += __shfl_xor_sync(0xffffffffu, a, o);
    n += __shfl_xor_sync(0xffffffffu, n, o);
  }
  if (lane == 0) { s_sum[warp] = a; s_count[warp] = n; }
  __syncthreads();
  if (threadIdx.x == 0) {
    whole(a, n);
    publish(a, n);
  }
}

// Losses of equal weight -- 1 / tokens given as weights, a loss scale, weights of 0 and 1 / tokens -- put one factor into dz, and where a
// target's probability is small its entry is that factor, which bf16 rounds the same way in every token: dX and dW come out too large or too small by
// up to 2^-9 (1/788: by 0.2 %).  So the largest weight of a token with a loss is made a power of two, by a factor of 1 to 2 that the products'
// epilogues take out again in fp32, and equal weights round as a mean's 1 does.  One block, since a maximum of a few thousand weights is a
// handful of memory latencies (a launch of its own all the same: 2048 tokens of 768 over 50257 columns 458 -> 462 us a step).
__global__ void __launch_bounds__(1024) head_weights_kernel(const float* __restrict__ dloss, HeadRows R, int seq, int t_pad, float inv_tau, float* __restrict__ raise) {
  __shared__ float s_top[32];
  pdl_wait();
  pdl_launch_dependents();      // after the wait: the product behind may ask for weights early, and what wrote them is complete then
  float top = 0.f;
#pragma unroll 8
  for (int row = threadIdx.x; row < (int)R.rows; row += 1024) {
    const int b = row / t_pad, t = row - b * t_pad;
    const float w = t < seq ? fabsf(dloss[(int64_t)b * seq + t]) : 0.f;
    if (R.count[row] != 0 && w < INFINITY) top = fmaxf(top, w);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  if (threadIdx.x % 32 == 0) s_top[threadIdx.x / 32] = top;
  __syncthreads();
  if (threadIdx.x >= 32) return;
  top = s_top[threadIdx.x];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  if (threadIdx.x) return;
  top *= inv_tau;
  int e;
  const float m = frexpf(top, &e);                             // in [1/2, 1)
  *raise = top > 0.f && top < 0x1p127f ? 1.f / m : 1.f;
}

// dX: the areas' sums (of a row and its second, where there are such) times alpha / max(*over, 1) where `over` is not null, at the tokens' own rows, and zeros at the rows without a
// loss.  A warp has 128 consecutive bytes of sums: with GROUPS = 4 its quarters take every fourth area each and are added up in
// that order (few elements and many areas: 56 x 768 of 24 areas), with 1 four pieces of 128 bytes.  Bound by memory.
template <typename T, int GROUPS, bool SECOND>
__global__ void __launch_bounds__(256) head_scatter_kernel(const float* __restrict__ acc, int areas, int64_t area, HeadRows R, int64_t n,
                                                           const float* __restrict__ over, float alpha, T* __restrict__ dX) {
  constexpr int TW = tile_w_of<T>::value;
  pdl_launch_dependents();
  pdl_wait();
  const float a = over ? alpha / fmaxf(*over, 1.f) : 1.f;
  const int lane = threadIdx.x % 32, group = GROUPS == 1 ? 0 : lane / 8;
  constexpr int64_t per_warp = GROUPS == 1 ? 128 : 32;
  const int64_t warps = (int64_t)gridDim.x * 8;
  for (int64_t i0 = ((int64_t)blockIdx.x * 8 + threadIdx.x / 32) * per_warp; i0 < n; i0 += warps * per_warp) {
    const int64_t i = i0 + (GROUPS == 1 ? lane : lane % 8) * 4;
    const int64_t line = i / TW, panel = line / R.rows;
    const int pos = R.pos[line - panel * R.rows];
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (pos >= 0 && pos < R.rows) {
      const float* from = acc + (panel * R.x_rows + pos) * TW + i % TW;
#pragma unroll 8
      for (int k = group; k < areas; k += GROUPS) {
        const float4 v = __ldcg(reinterpret_cast<const float4*>(from + k * area));
        s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        if (SECOND) {
          const float4 u = __ldcg(reinterpret_cast<const float4*>(from + k * area + R.second * TW));
          s.x += u.x; s.y += u.y; s.z += u.z; s.w += u.w;
        }
      }
    }
    if (GROUPS > 1) {
#pragma unroll
      for (int o = 8; o < 32; o *= 2) {
        s.x += __shfl_xor_sync(0xffffffffu, s.x, o); s.y += __shfl_xor_sync(0xffffffffu, s.y, o);
        s.z += __shfl_xor_sync(0xffffffffu, s.z, o); s.w += __shfl_xor_sync(0xffffffffu, s.w, o);
      }
      if (group) continue;
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
cudaError_t launch_head_rows(int dtype, const int32_t* targets, const HeadRows& R, int seq, int t_pad, int vocab, const void* X, int d_model,
                             const HeadExact& exact, int32_t* status, cudaStream_t st) {
  const int panels = d_model / (dtype == FBL_DTYPE_FP32 ? 32 : 64);
  const int64_t per = R.rows <= 32 * 1024 ? 32 : (R.rows / 1024 + 31) / 32 * 32;
  dim3 grid((unsigned)((R.rows + per - 1) / per), (unsigned)((panels + ROWS_PANELS - 1) / ROWS_PANELS));
  if (exact.z) grid.y += (unsigned)((R.rows * exact.top_k + grid.x - 1) / grid.x);       // a block for each
  return launch_pdl(targets ? head_rows_kernel<true> : head_rows_kernel<false>, grid, dim3(256), 0, st,
                    targets, R, seq, t_pad, vocab, (int)per, (const uint4*)X, (uint4*)R.x, panels, exact, status);
}
cudaError_t launch_teacher_entries(const int32_t* ids, const float* logits, int top_k, float temperature, const HeadRows& R, int seq, int t_pad,
                                   int vocab, int32_t* status, cudaStream_t st) {
  auto kernel = top_k <= 32 ? teacher_entries_kernel<1> : top_k <= 64 ? teacher_entries_kernel<2> : teacher_entries_kernel<4>;
  return launch_pdl(kernel, dim3((unsigned)(R.rows / ENTRY_WARPS)), dim3(32 * ENTRY_WARPS), 0, st, ids, logits, top_k, temperature, R, seq, t_pad,
                    vocab, status);
}
cudaError_t launch_head_combine(const float2* part, int tiles, const float* z_at, const HeadRows& R, float scale, float* loss, float* total,
                                double2* block_sums, int seq, int t_pad, const HeadExact& exact, int32_t* status, cudaStream_t st) {
  const bool few = R.rows <= COMBINE_FEW;
  const unsigned threads = !few ? 256 : (unsigned)(R.rows <= 32 ? R.rows * 32 : R.rows / 8 * 128);       // a warp has a row, or two
  return launch_pdl(exact.z ? head_combine_kernel<true> : head_combine_kernel<false>, dim3(few ? 1u : (unsigned)(R.rows / 8)), dim3(threads), 0, st,
                    part, tiles, z_at, R, scale, loss, total, block_sums, seq, t_pad, exact, status);
}
cudaError_t launch_head_weights(const float* dloss, const HeadRows& R, int seq, int t_pad, float inv_tau, float* raise, cudaStream_t st) {
  return launch_pdl(head_weights_kernel, dim3(1), dim3(1024), 0, st, dloss, R, seq, t_pad, inv_tau, raise);
}
cudaError_t launch_head_scatter(int dtype, int sm_count, const float* acc, int areas, const HeadRows& R, int d_model, const float* over, float alpha,
                                void* dX, cudaStream_t st) {
  const int64_t n = R.rows * d_model;                        // whole tiles: a multiple of 256 bytes of sums
  const bool spread = areas >= 4 && n <= (int64_t)sm_count * 8 * 1024;
  const dim3 grid((unsigned)min((int64_t)sm_count * 8, (n + (spread ? 255 : 1023)) / (spread ? 256 : 1024)));
  auto go = [&](auto kernel, auto* t) { return launch_pdl(kernel, grid, dim3(256), 0, st, acc, areas, R.x_rows * d_model, R, n, over, alpha, t); };
  if (dtype == FBL_DTYPE_FP32) return spread ? go(head_scatter_kernel<float, 4, false>, (float*)dX) : go(head_scatter_kernel<float, 1, false>, (float*)dX);
  if (R.second) return spread ? go(head_scatter_kernel<__nv_bfloat16, 4, true>, (__nv_bfloat16*)dX) : go(head_scatter_kernel<__nv_bfloat16, 1, true>, (__nv_bfloat16*)dX);
  return spread ? go(head_scatter_kernel<__nv_bfloat16, 4, false>, (__nv_bfloat16*)dX) : go(head_scatter_kernel<__nv_bfloat16, 1, false>, (__nv_bfloat16*)dX);
}
