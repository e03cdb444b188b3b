// Cross entropy of a linear layer's logits, and its gradients, without all of them in memory.
// For a row x_i with label y_i in [0, V) and the table W [V][C]:
//
//   z_v = x_i . W_v + b_v,  lse_i = log sum exp z_v,  loss_i = lse_i - z_{y_i}
//   dz_v = w_i (exp(z_v - lse_i) - [v = y_i])
//   dx_i = sum over v of dz_v W_v,  dW_v = sum over i of dz_v x_i,  db_v = sum of dz_v
//
// Rows whose label is outside of [0, V) are padding.  A first pass over the labels
// lists the others; where any is left out, the rows of x that count are packed, so
// that padding costs no products and whatever it holds reaches no sum.  How many they
// are stays on the device: workgroups past them end at once.
//
// Forward: one product over all of V whose epilogue takes every row's maximum and sum
// of exponentials over the tile's columns and the label's logit; a second launch joins
// the tiles.  Nothing of size rows x V is written, but for few logits (`cut_logits`).
//
// Gradients: for a piece of rows at a time dz [rows][V] (bf16, rounded once from fp32, or
// fp32), and the products dz W and dz^T x over it; db from the unrounded dz, summed
// over 64 rows or a tile's, then over these.  A piece is at most 2^30 (bf16) or 2^28
// (fp32) elements of dz, so most calls have one; with more, dW is summed over them in
// fp32.  dz comes
// - in the backward, from the logits again, in the epilogue of their product;
// - in the step, from what its forward kept of the piece: bf16 without db, the
//   exponentials relative to the maximum of their tile's columns, in fp16 times 2^15
//   (off by 2^-11 of their value, 2^-40 of the tile's largest at the small end: next to
//   the rounding of dz to bf16, nothing); fp32, or with db, the logits in fp32.  One pass
//   over them gives dz.  For short rows in bf16 the product is cheaper than that pass
//   (`keeps`).
// dz in bf16 is off by less the nearer it is below a power of two: with row weights it is
// formed times a factor in [1, 2] that makes the largest one a power of two, which the sums
// over it undo (624 rows of weights 0.8e-3 to 2.4e-3: gradients off by
// 0.0022 in place of 0.0025, of which 0.0016 is their own rounding).
// The rounding of dz is mostly that of the rows' labels: at random over many rows, all of the
// gradient over few (7 rows: 0.0028 of it, 0.0017 with two terms).  Up to kFine rows of
// bf16 dz is two terms, the rounded one and the rest, and multiplied twice: as twice the
// rows for dx, which reads W once, one step of K more for dW.  Steps, us with two terms / one:
// 7 x 448 x 3,456 45 / 41, 64 x 4,096 x 32,000 302 / 265, 16 x 4,096 x 131,072 980 / 898.
//
// Few logits of long rows (some tiles of them, which would leave most CUs idle) are one
// product cut along C and joined in the workspace, at most 2^21 of them in fp32; all
// passes start from there (`cut_logits`).
//
// 16 rows of 4,096 over 131,072 classes in bf16: 192 us, the table read at 6.2 TB/s in 174.
// Loss and gradients of 4,096 such rows: 11.3 ms, three products at 1.12 to 1.22
// PFLOP/s, the power limit, and 0.4 ms for dz.  67,040 rows of 128 over 10,475 classes, loss:
// 634 us; gradients: 1,342 us; logits to dz 650 (exponentials and stores beside short products),
// dx 410 and dW 275 from reading dz.
#include <algorithm>
#include <mutex>

#include "dense.h"
#include "dense_epilogue.h"

namespace shc {

using namespace dense;

namespace {

constexpr int64_t kFine = 64;  // rows of bf16 whose dz is two terms
constexpr float kLog2e = 1.44269504088896340736f;
constexpr int kLabels = 4;  // a thread's
constexpr int kLabelsPerBlock = 256 * kLabels;

__device__ __forceinline__ int64_t label_at(const void* labels, int id64, int64_t stride,
                                            int64_t i) {
  return id64 ? static_cast<const int64_t*>(labels)[i * stride]
              : (int64_t)static_cast<const int32_t*>(labels)[i * stride];
}

struct Labels {
  const void* p;
  int id64;
  int64_t stride;
  int32_t V;
  __device__ __forceinline__ int64_t get(int64_t i) const { return label_at(p, id64, stride, i); }
  __device__ __forceinline__ bool live(int64_t i) const {
    const int64_t y = get(i);
    return y >= 0 && y < V;
  }
  // the thread's labels of a block, all loads under way at once; -1 past the last
  __device__ __forceinline__ void get_block(int64_t i0, int64_t n, int (&y)[kLabels]) const {
    int64_t x[kLabels];
#pragma unroll
    for (int q = 0; q < kLabels; ++q) x[q] = get(i0 + q * 256 < n ? i0 + q * 256 : n - 1);
#pragma unroll
    for (int q = 0; q < kLabels; ++q)
      y[q] = i0 + q * 256 < n && x[q] >= 0 && x[q] < V ? (int)x[q] : -1;
  }
};

// The largest finite weight, without its sign, of the thread's live rows (0 without any).
__device__ __forceinline__ float most_weight(const float* weight, int64_t i0,
                                             const int (&y)[kLabels]) {
  float m = 0.f;
#pragma unroll
  for (int q = 0; q < kLabels; ++q)
    if (y[q] >= 0) {
      const float w = fabsf(weight[i0 + q * 256]);
      m = w < __builtin_inff() ? fmaxf(m, w) : m;
    }
  return rowops::lanes_reduce<64>(m, rowops::MaxOp{});
}

// Live rows of every block of labels, and their largest weight (`weight` not NULL).
__global__ __launch_bounds__(256) void count_labels_kernel(Labels l, int64_t n, int32_t* counts,
                                                           const float* weight, float* most) {
  __shared__ int total;
  __shared__ float top[4];
  if (threadIdx.x == 0) total = 0;
  __syncthreads();
  int y[kLabels], c = 0;
  l.get_block((int64_t)blockIdx.x * kLabelsPerBlock + threadIdx.x, n, y);
#pragma unroll
  for (int q = 0; q < kLabels; ++q) c += __popcll(__ballot(y[q] >= 0));
  if ((threadIdx.x & 63) == 0) atomicAdd(&total, c);  // whole numbers: any order
  if (weight != nullptr) {
    const float m = most_weight(weight, (int64_t)blockIdx.x * kLabelsPerBlock + threadIdx.x, y);
    if ((threadIdx.x & 63) == 0) top[threadIdx.x >> 6] = m;
  }
  __syncthreads();
  if (threadIdx.x == 0) counts[blockIdx.x] = total;
  if (threadIdx.x == 0 && weight != nullptr)
    most[blockIdx.x] = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
}

// What the epilogues need of the live rows, in their order.
struct LiveRows {
  int32_t* idx;
  int32_t* label;
  float* weight;
  float* lse;
};

// The live rows in ascending order, their number, and the results of the others.  scale (NULL:
// not asked for): what dz in bf16 is multiplied by, so that the largest weight becomes a power
// of two, and what undoes it (1 where there is no such weight).
__global__ __launch_bounds__(256) void list_rows_kernel(
    Labels l, int64_t n, const int32_t* __restrict__ counts, LiveRows rows, int32_t* count,
    const float* __restrict__ weight, const float* __restrict__ lse_in, float* __restrict__ loss,
    float* __restrict__ lse, const float* __restrict__ most, float* scale) {
  __shared__ int wave[kLabels][4], before[4];
  __shared__ float top[4];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int64_t i0 = (int64_t)blockIdx.x * kLabelsPerBlock + threadIdx.x;
  uint64_t mask[kLabels];
  int y[kLabels];
  l.get_block(i0, n, y);
#pragma unroll
  for (int q = 0; q < kLabels; ++q) {
    mask[q] = __ballot(y[q] >= 0);
    if (lane == 0) wave[q][w] = __popcll(mask[q]);
  }
  int c = 0;
  for (int b = threadIdx.x; b < (int)blockIdx.x; b += 256) c += counts[b];
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) c += __shfl_xor(c, d, 64);
  if (lane == 0) before[w] = c;
  const bool last = blockIdx.x == gridDim.x - 1;
  if (last && scale != nullptr) {
    float m = most_weight(weight, i0, y);
    for (int b = threadIdx.x; b < (int)blockIdx.x; b += 256) m = fmaxf(m, most[b]);
    m = rowops::lanes_reduce<64>(m, rowops::MaxOp{});
    if (lane == 0) top[w] = m;
  }
  __syncthreads();
  if (last && scale != nullptr && threadIdx.x == 0) {
    const float m = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
    const uint32_t bits = __float_as_uint(m);
    // m is f 2^e, f in [1, 2): times 2 / f
    const float f = __uint_as_float((bits & 0x7FFFFFu) | 0x3F800000u);
    const bool normal = m >= 0x1p-126f && m < 0x1p126f;
    scale[0] = normal ? 2.f / f : 1.f;
    scale[1] = normal ? f * 0.5f : 1.f;
  }
  int base = before[0] + before[1] + before[2] + before[3];
#pragma unroll
  for (int q = 0; q < kLabels; ++q) {
    const int64_t i = i0 + q * 256;
    int at = base + __popcll(mask[q] & ((1ull << lane) - 1));
    for (int p = 0; p < w; ++p) at += wave[q][p];
    if (y[q] >= 0) {
      rows.idx[at] = (int32_t)i;
      rows.label[at] = y[q];
      rows.weight[at] = weight != nullptr ? weight[i] : 1.f;
      if (lse_in != nullptr) rows.lse[at] = lse_in[i];
    } else if (i < n) {
      if (loss != nullptr) loss[i] = 0.f;
      if (lse != nullptr) lse[i] = 0.f;
    }
    base += wave[q][0] + wave[q][1] + wave[q][2] + wave[q][3];
  }
  if (last && threadIdx.x == 0) *count = base;
}

struct Logits {
  Operand A, B;       // rows of x from row0 on, the table
  int64_t rows, C;    // rows of the piece, channels
  const int32_t* count;
  int64_t row0, full;
  const float* bias;
  int V;
  LiveRows live;  // of the piece
  int tm, tn;
  // statistics
  float2* parts;  // [tn][rows]: maximum and sum over a tile's columns
  float* at_label;
  void* kept;  // [rows][width]
  // gradient
  void* dz;
  int64_t ld_dz;
  int64_t low;  // bf16: elements from dz to its second term, 0 without one
  const float* scale;  // of dz, or NULL
  int width;
  float* sums;  // [tm * WM][V] or NULL
};

// 8 values of dz, in bf16 with what the rounding leaves.  Not of what is not finite, where
// that would be a NaN.
template <bool BF16>
__device__ __forceinline__ void put_dz(void* dz, int64_t low, int64_t row, int64_t ld, int v,
                                       int width, const float (&z)[8]) {
  put8<BF16>(dz, row, ld, v, width, z);
  if constexpr (BF16)
    if (low != 0) {
      float t[8];
      rowops::Row<uint16_t>::widen(rowops::Row<uint16_t>::narrow(z), t);
#pragma unroll
      for (int e = 0; e < 8; ++e) t[e] = __builtin_isfinite(t[e]) ? z[e] - t[e] : 0.f;
      put8<true>(static_cast<uint16_t*>(dz) + low, row, ld, v, width, t);
    }
}

// The logits of a tile: M rows are live.  False where none is.
template <class S, Mode MODE>
__device__ __forceinline__ bool logits_tile(Logits& a, Tile<S, true, true, MODE>& tile,
                                            int64_t* m0, int64_t* n0, int64_t* M, int* tn,
                                            char* smem) {
  *M = a.A.extent = rows_left(a.count, a.row0, a.rows);
  int tm;
  if (!tile_of(blockIdx.x, (int)((*M + S::BM - 1) / S::BM), a.tn, &tm, tn)) return false;
  *m0 = (int64_t)tm * S::BM, *n0 = (int64_t)*tn * S::BN;
  if (a.A.alt != nullptr && *a.count != a.full) a.A.p = a.A.alt, a.A.ld = a.A.alt_ld;
  tile.run(a.A, a.B, *M, a.V, a.C, *m0, *n0, 0, (int)((a.C + BK - 1) / BK), smem);
  return true;
}

// What is added to the products of 8 columns: the bias, -inf past the last.
__device__ __forceinline__ void load_bias(float (&b)[8], const float* bias, int64_t col, int V) {
#pragma unroll
  for (int e = 0; e < 8; ++e) b[e] = col + e < V ? 0.f : -__builtin_inff();
  if (bias != nullptr) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (col + e < V) b[e] = bias[col + e];
  }
}

// e^(z - by) of N logits in place.  The difference comes first: z log2(e) - by log2(e) in
// one multiplication and addition is off by half a step of by log2(e), a factor of 2^2 at
// 1e8 (masks of a large finite number) and past fp32 at 1e10, also where z is `by` itself.
template <int N>
__device__ __forceinline__ void exps_less(float (&z)[N], float by) {
#pragma unroll
  for (int e = 0; e < N; ++e) z[e] = __builtin_amdgcn_exp2f((z[e] - by) * kLog2e);
}

// dz of N logits, y the label less the first one's column.  lse = -inf: a row of nothing
// but -inf, whose probabilities are 0.
template <int N>
__device__ __forceinline__ void grad_of(float (&z)[N], int y, float lse, float w) {
  if (lse == -__builtin_inff()) {
#pragma unroll
    for (int e = 0; e < N; ++e) z[e] = 0.f;
  } else {
    exps_less(z, lse);
  }
  if (y >= 0 && y < N) {
#pragma unroll
    for (int e = 0; e < N; ++e) z[e] = y == e ? z[e] - 1.f : z[e];
  }
#pragma unroll
  for (int e = 0; e < N; ++e) z[e] *= w;
}

// (m, s) with s = sum of e^(z - m): a maximum of -inf stands for 0 in the differences, so
// that a row of nothing but -inf has s = 0, and a NaN stays in s whatever its maximum.
__device__ __forceinline__ float finite_or_0(float m) { return m == -__builtin_inff() ? 0.f : m; }
__device__ __forceinline__ float2 join(float2 a, float2 b) {
  const float m = fmaxf(a.x, b.x), f = finite_or_0(m);
  return float2{m, a.y * __builtin_amdgcn_exp2f((a.x - f) * kLog2e) +
                       b.y * __builtin_amdgcn_exp2f((b.x - f) * kLog2e)};
}

// What the forward of a step keeps of the logits.
enum Keep { kNothing, kExps, kLogits };
constexpr float kExpScale = 32768.f;

template <class S, Mode MODE, Keep KEEP>
__global__ __launch_bounds__(S::THREADS) void logit_stats_kernel(Logits a) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  Tile<S, true, true, MODE> tile;
  int64_t m0, n0, M;
  int tn;
  if (!logits_tile<S, MODE>(a, tile, &m0, &n0, &M, &tn, smem)) return;
  // per row and 64 columns, behind what the tile passes its sums through
  constexpr int BLOCKS = S::BN / 64;
  static_assert(S::NW * 8192 + (2 * BLOCKS + 1) * S::BM * 4 <= S::template lds<MODE>(),
                "fits the tile's LDS");
  float* most = reinterpret_cast<float*>(smem + S::NW * 8192);  // [BLOCKS][BM]
  float* sums = most + BLOCKS * S::BM;
  int32_t* label = reinterpret_cast<int32_t*>(sums + BLOCKS * S::BM);  // [BM]
  for (int r = threadIdx.x; r < S::BM; r += S::THREADS)
    label[r] = m0 + r < M ? a.live.label[m0 + r] : -1;
  __syncthreads();
  const bool first = (threadIdx.x & 7) == 0;
  float bias[8];
  load_bias(bias, a.bias, tile.col_of(n0), a.V);
  tile.each(m0, n0, smem, [&](int64_t row, int64_t col, float (&z)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) z[e] += bias[e];
    float m = z[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) m = fmaxf(m, z[e]);
    m = rowops::lanes_reduce<8>(m, rowops::MaxOp{});
    if (first) most[(int)(col - n0) / 64 * S::BM + (int)(row - m0)] = m;
    const int y = label[(int)(row - m0)] - (int)col;
    if (y >= 0 && y < 8) {
      float at = z[0];
#pragma unroll
      for (int e = 1; e < 8; ++e) at = y == e ? z[e] : at;
      a.at_label[row] = at;
    }
  });
  __syncthreads();
  const auto row_most = [&](int r) {
    float m = most[r];
#pragma unroll
    for (int b = 1; b < BLOCKS; ++b) m = fmaxf(m, most[b * S::BM + r]);
    return m;
  };
  tile.each(m0, n0, smem, [&](int64_t row, int64_t col, float (&z)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) z[e] += bias[e];
    const bool store = row < M && col < a.width;
    if constexpr (KEEP == kLogits)
      if (store)
        rowops::store_channels<8>(static_cast<float*>(a.kept) + row * a.width, (int)(col / 8),
                                  a.width, z);
    exps_less(z, finite_or_0(row_most((int)(row - m0))));
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) s += z[e];
    s = rowops::lanes_reduce<8>(s, rowops::AddOp{});
    if (first) sums[(int)(col - n0) / 64 * S::BM + (int)(row - m0)] = s;
    if constexpr (KEEP == kExps) {
      typedef _Float16 half8 __attribute__((ext_vector_type(8)));
      half8 x;
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = (_Float16)(z[e] * kExpScale);
      if (store)
        *reinterpret_cast<half8*>(static_cast<_Float16*>(a.kept) + row * a.width + col) = x;
    }
  });
  __syncthreads();
  for (int r = threadIdx.x; r < S::BM && m0 + r < M; r += S::THREADS) {
    float s = sums[r];
#pragma unroll
    for (int b = 1; b < BLOCKS; ++b) s += sums[b * S::BM + r];
    a.parts[(int64_t)tn * a.rows + m0 + r] = float2{row_most(r), s};
  }
}

// dz of the live rows from what was kept: 64 rows by 512 columns to a workgroup, 16 rows
// of 8 columns to a thread.  Bound by HBM: 3,891 rows of 131,072 exponentials in 400 us,
// 5.1 TB/s read and written.
struct FromKept {
  const void* kept;
  int64_t rows;
  const int32_t* count;
  int64_t row0;
  const float2* parts;
  int tile;  // columns of a tile of parts
  int V;
  const float* bias;  // what the logits lack, or NULL
  LiveRows live;
  void* dz;
  int64_t low;  // as Logits'
  const float* scale;
  int width, dz_width;
  float* sums;  // [ceil(rows / 64)][V] or NULL
};
template <bool BF16, Keep KEEP>
__global__ __launch_bounds__(256) void from_kept_kernel(FromKept a) {
  __shared__ float part[3][64 * 8];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int64_t live = rows_left(a.count, a.row0, a.rows);
  const int64_t r0 = (int64_t)blockIdx.x * 64;
  if (r0 >= live) return;
  const int64_t r1 = r0 + 64 < live ? r0 + 64 : live;
  const int v = blockIdx.y * 64 + lane, col = 8 * v;
  const int V = a.V;
  const float scale = a.scale != nullptr ? *a.scale : 1.f;
  float sum[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) sum[e] = 0.f;
  if (col < a.dz_width) {
#pragma unroll 2
    for (int64_t row = r0 + w; row < r1; row += 4) {
      const float lse = a.live.lse[row], wt = a.live.weight[row] * scale;
      const int y = a.live.label[row] - col;
      float z[8];
      if constexpr (KEEP == kExps) {
        typedef _Float16 half8 __attribute__((ext_vector_type(8)));
        const half8 x = *reinterpret_cast<const half8*>(static_cast<const _Float16*>(a.kept) +
                                                        row * a.width + col);
        // a tile of nothing but -inf has probability 0, unless the row is a NaN
        const float m = a.parts[(int64_t)(col / a.tile) * a.rows + row].x;
        const float f = m == -__builtin_inff() && lse == lse
                            ? 0.f
                            : __builtin_amdgcn_exp2f((m - lse) * kLog2e) * (1.f / kExpScale);
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = (float)x[e] * f;
        if (y >= 0 && y < 8) {
#pragma unroll
          for (int e = 0; e < 8; ++e) z[e] = y == e ? z[e] - 1.f : z[e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] *= wt;
      } else {
        rowops::load_channels<8>(static_cast<const float*>(a.kept) + row * a.width, v, a.width, z);
        if (a.bias != nullptr) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (col + e < V) z[e] += a.bias[col + e];
        }
        grad_of(z, y, lse, wt);
      }
      if (col + 8 > V) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (col + e >= V) z[e] = 0.f;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[e] += z[e];
      put_dz<BF16>(a.dz, a.low, row, a.dz_width, v, a.dz_width, z);
    }
  }
  if (a.sums == nullptr) return;
  if (w > 0)
#pragma unroll
    for (int e = 0; e < 8; ++e) part[w - 1][e * 64 + lane] = sum[e];
  __syncthreads();
  if (w > 0 || col >= V) return;
#pragma unroll
  for (int q = 0; q < 3; ++q)
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] += part[q][e * 64 + lane];
  rowops::store_channels<8>(a.sums + (int64_t)blockIdx.x * V, v, V, sum);
}

// 16 rows to a workgroup, 16 threads to a row.
__global__ __launch_bounds__(256) void join_stats_kernel(const float2* parts, int tiles,
                                                         int64_t rows, const int32_t* count,
                                                         int64_t row0, LiveRows rows_live,
                                                         const float* at_label, float* loss,
                                                         float* lse) {
  __shared__ float2 part[16][16];
  const int r = threadIdx.x & 15, p = threadIdx.x >> 4;
  const int64_t row = (int64_t)blockIdx.x * 16 + r;
  const int64_t live = rows_left(count, row0, rows);
  if ((int64_t)blockIdx.x * 16 >= live) return;
  float2 t = {-__builtin_inff(), 0.f};
  if (row < live)
#pragma unroll 4
    for (int q = p; q < tiles; q += 16) t = join(t, parts[(int64_t)q * rows + row]);
  part[p][r] = t;
  __syncthreads();
  if (p != 0 || row >= live) return;
  for (int q = 1; q < 16; ++q) t = join(t, part[q][r]);
  const float l = t.x + __logf(t.y), z = at_label[row];
  const int64_t to = rows_live.idx[row];
  rows_live.lse[row] = l;
  if (lse != nullptr) lse[to] = l;
  // a label on a logit of -inf, in a row of nothing but -inf too
  if (loss != nullptr) loss[to] = z == -__builtin_inff() && l == l ? -z : l - z;
}

// Statistics of the live rows from their logits less the bias, a workgroup to a row.
__global__ __launch_bounds__(256) void row_stats_kernel(const float* logits, int V,
                                                        const int32_t* count, const float* bias,
                                                        LiveRows live, float* loss, float* lse) {
  __shared__ float2 part[4];
  const int64_t row = blockIdx.x;
  if (row >= *count) return;
  const float* z = logits + row * V;
  float2 t = {-__builtin_inff(), 0.f};
#pragma unroll 4
  for (int v = threadIdx.x; v < V; v += 256)
    t = join(t, float2{z[v] + (bias != nullptr ? bias[v] : 0.f), 1.f});
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1)
    t = join(t, float2{__shfl_xor(t.x, d, 64), __shfl_xor(t.y, d, 64)});
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = t;
  __syncthreads();
  if (threadIdx.x != 0) return;
  for (int w = 1; w < 4; ++w) t = join(t, part[w]);
  const int y = live.label[row];
  const float at = z[y] + (bias != nullptr ? bias[y] : 0.f), l = t.x + __logf(t.y);
  const int64_t to = live.idx[row];
  live.lse[row] = l;
  if (lse != nullptr) lse[to] = l;
  if (loss != nullptr) loss[to] = at == -__builtin_inff() && l == l ? -at : l - at;
}

template <class S, Mode MODE>
__global__ __launch_bounds__(S::THREADS) void logit_grad_kernel(Logits a) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  Tile<S, true, true, MODE> tile;
  int64_t m0, n0, M;
  int tn;
  if (!logits_tile<S, MODE>(a, tile, &m0, &n0, &M, &tn, smem)) return;
  // the rows' label, lse and weight, behind what the tile passes its sums through
  static_assert(S::NW * 8192 + 3 * S::BM * 4 <= S::template lds<MODE>(),
                "fits the tile's LDS");
  int32_t* label = reinterpret_cast<int32_t*>(smem + S::NW * 8192);
  float* lse = reinterpret_cast<float*>(label + S::BM);
  float* weight = lse + S::BM;
  const float scale = a.scale != nullptr ? *a.scale : 1.f;
  for (int r = threadIdx.x; r < S::BM; r += S::THREADS)
    if (m0 + r < M) {
      label[r] = a.live.label[m0 + r];
      lse[r] = a.live.lse[m0 + r];
      weight[r] = a.live.weight[m0 + r] * scale;
    }
  __syncthreads();
  float sum[8], bias[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) sum[e] = 0.f;
  load_bias(bias, a.bias, tile.col_of(n0), a.V);
  tile.each(m0, n0, smem, [&](int64_t row, int64_t col, float (&z)[8]) {
    if (row >= M) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) z[e] += bias[e];
    const int r = (int)(row - m0);
    grad_of(z, label[r] - (int)col, lse[r], weight[r]);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] += z[e];
    if (col < a.width)
      put_dz<MODE == kPlain>(a.dz, a.low, row, a.ld_dz, (int)(col / 8), a.width, z);
  });
  if (a.sums == nullptr) return;
  // over the wavefront's rows: the lane's, then the lanes' of the same columns
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int64_t part = m0 / S::BM * S::WM + w / S::WN;
#pragma unroll
  for (int e = 0; e < 8; ++e) sum[e] = rowops::groups_sum<8>(sum[e]);
  const int64_t col = n0 + (w % S::WN) * 64 + lane * 8;
  if (lane < 8 && col < a.V)
    rowops::store_channels<8>(a.sums + part * a.V, (int)(col / 8), a.V, sum);
}

// Column sums over the parts of the live rows, in order, added to what the pieces
// before gave (`first` 0) or to what db holds (`accumulate`).
__global__ __launch_bounds__(1024) void join_sums_kernel(const float* sums, int rows_per_part,
                                                         int64_t rows, const int32_t* count,
                                                         int64_t row0, int V, int add, const float* scale,
                                                         float* db) {
  __shared__ float part[16][64];
  const int x = threadIdx.x & 63, y = threadIdx.x >> 6;
  const int64_t c = (int64_t)blockIdx.x * 64 + x;
  const int64_t parts =
      (rows_left(count, row0, rows) + rows_per_part - 1) / rows_per_part;
  const int64_t per = (parts + 15) / 16, p0 = y * per, p1 = p0 + per < parts ? p0 + per : parts;
  float s = 0.f;
  if (c < V)
    for (int64_t p = p0; p < p1; ++p) s += sums[p * V + c];
  part[y][x] = s;
  __syncthreads();
  if (y != 0 || c >= V) return;
  for (int q = 1; q < 16; ++q) s += part[q][x];
  if (scale != nullptr) s *= *scale;
  db[c] = add ? db[c] + s : s;
}

// The gradient of rows of padding: zeros.
template <typename T>
__global__ __launch_bounds__(256) void zero_rows_kernel(Labels l, int64_t n, const int32_t* count,
                                                        T* dx, int64_t ld, int C) {
  using namespace rowops;
  if (*count == n) return;
  const int lane = threadIdx.x & 63;
  for (int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); i < n;
       i += (int64_t)gridDim.x * 4) {
    if (l.live(i)) continue;
    for (int v = lane; v * Row<T>::N < C; v += 64) store_vec<T>(dx + i * ld, v, C, i32x4{0, 0, 0, 0});
  }
}

struct Layout {
  int64_t width, rows, pieces;  // columns of dz, rows and number of the pieces
  size_t idx, label, weight, lse, count, counts, most, scale, x, W, logits, parts, at_label, kept, dz, dz32,
      sums, acc, partials, partial_bytes, total;
};

// Logits that are one product, cut along C, where that is faster by more than the launch
// that it costs: 5 us.  Rows x C x V, us cut / whole: bf16 16 x 4,096 x 512 25.5 / 42.4, 200 x
// 2,048 x 300 24.1 / 28.9, 1 x 4,096 x 1,000 22.3 / 31.3; fp32 31.1 / 157.5, 33.6 / 59.0,
// 28.7 / 153.0.
constexpr int64_t kMostCut = (int64_t)1 << 21;
bool cut_logits(int64_t n, int32_t C, int32_t V, Mode mode) {
  if (n > kMostCut / V) return false;
  double whole, cut;
  plan_product(n, V, C, mode, true, 0, true, &whole);
  const Plan plan = plan_product(n, V, C, mode, true, partial_bytes(n, V, C), false, &cut);
  return plan.parts > 1 && cut + 5.0 < whole;
}

// Whether the step keeps the logits or their exponentials, or forms them twice.  8,192
// rows by 16,384 classes, us kept / twice at C = 128, 256, 512, 1,024: bf16 without db
// 419 / 403, 474 / 483, 643 / 692, 935 / 1,108; bf16 with db, which keeps four bytes of a
// logit, 629 / 497 at 256, 767 / 706, 1,055 / 1,124; fp32 1,336 / 1,467, 1,797 / 2,090,
// 2,827 / 3,428, 5,112 / 6,442.  Below these widths a step's bits are those of a forward
// and a backward pass, also where 4% would be had (fp32 1,200 / 1,258 at 64).
bool keeps(int32_t C, bool bf16, bool db) { return C >= (!bf16 ? 128 : db ? 768 : 256); }

Layout layout(int64_t n, int32_t C, int32_t V, bool bf16, bool aligned, XentPass pass) {
  Layout w{};
  size_t at = 0;
  const auto take = [&](size_t bytes) {
    const size_t here = at;
    at += align256(bytes);
    return here;
  };
  w.width = packed_width(V);
  // 2^27 and 2^25 in their place: 67,040 x 10,475 of bf16 1,412 us instead of 1,305, 777 x
  // 50,021 of fp32 1,822 instead of 1,464
  const int64_t most = (int64_t)1 << (bf16 ? 30 : 28);
  w.rows = std::min<int64_t>(n, std::max<int64_t>(256, most / w.width / 256 * 256));
  w.pieces = n == 0 ? 0 : (n + w.rows - 1) / w.rows;
  w.idx = take((size_t)n * 4);
  w.label = take((size_t)n * 4);
  w.weight = take((size_t)n * 4);
  w.lse = take((size_t)n * 4);
  w.count = take(4);
  w.counts = take((size_t)((n + kLabelsPerBlock - 1) / kLabelsPerBlock) * 4);
  w.most = take((size_t)((n + kLabelsPerBlock - 1) / kLabelsPerBlock) * 4);
  w.scale = take(8);
  w.x = take(packed_bytes(n, C, !bf16));
  w.W = take(bf16 && aligned && C % 8 == 0 ? 0 : packed_bytes(V, C, !bf16));
  const int64_t cut_rows = std::min<int64_t>(n, kMostCut / V);
  w.logits = take((size_t)cut_rows * V * 4);
  w.partial_bytes = partial_bytes(cut_rows, V, C);
  if (pass != XentPass::kBackward) {
    w.parts = take((size_t)((V + 127) / 128) * n * 8);
    w.at_label = take((size_t)n * 4);
  }
  if (pass != XentPass::kForward) {
    // kept fp32 logits become dz where they are; bf16 exponentials too (a step without db)
    const bool kept = pass == XentPass::kStep && keeps(C, bf16, true);
    // two terms of up to kFine rows, and no less for more rows
    const int64_t dz_rows = bf16 ? std::max(w.rows, std::min(2 * n, 2 * kFine)) : w.rows;
    w.dz = take(packed_bytes(dz_rows, V, !bf16));
    w.dz32 = take(bf16 ? 0 : (size_t)w.rows * V * 4);
    w.kept = take(bf16 && kept ? (size_t)w.rows * w.width * 4 : 0);
    w.sums = take((size_t)(w.rows / 32 + 4) * V * 4);  // 32 rows to a part at least
    w.acc = take(w.pieces > 1 ? (size_t)V * C * 4 : 0);
    w.partial_bytes = std::max(w.partial_bytes,
                               std::max(partial_bytes(w.rows, C, V), partial_bytes(V, C, w.rows)));
    if (bf16)  // dx of dz's two terms
      w.partial_bytes = std::max(w.partial_bytes, (size_t)(std::min(n, kFine) * C) * 8);
  }
  w.partials = take(w.partial_bytes);
  w.total = at;
  return w;
}

char* byte(void* ws, size_t at) { return static_cast<char*>(ws) + at; }

#define SHC_LAUNCH(...)                    \
  do {                                     \
    const hipError_t _e = (__VA_ARGS__);   \
    if (_e != hipSuccess) return _e;       \
  } while (0)

enum class Logit { kStats, kStatsExps, kStatsLogits, kGrad };
template <class S, Mode MODE, Logit WHAT>
hipError_t run_logits(const Logits& a, hipStream_t stream) {
  constexpr Keep keep = WHAT == Logit::kStatsExps     ? kExps
                        : WHAT == Logit::kStatsLogits ? kLogits
                                                      : kNothing;
  void (*kern)(Logits);
  if constexpr (WHAT == Logit::kGrad)
    kern = logit_grad_kernel<S, MODE>;
  else
    kern = logit_stats_kernel<S, MODE, keep>;
  constexpr int lds = S::template lds<MODE>();
  static std::once_flag once;
  static hipError_t attr = hipSuccess;
  std::call_once(once, [&] {
    attr = hipFuncSetAttribute(reinterpret_cast<const void*>(kern),
                               hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  });
  if (attr != hipSuccess) return attr;
  kern<<<a.tm * a.tn, S::THREADS, lds, stream>>>(a);
  return hipGetLastError();
}

// `kind` receives the tile that was taken.
template <Logit WHAT>
hipError_t launch_logits(Logits a, bool bf16, TileKind* kind, hipStream_t stream) {
  const bool direct = !bf16 && a.full <= kFewRows;
  const TileKind k =
      plan_product(a.rows, a.V, a.C, direct ? kDirect : bf16 ? kPlain : kSplit, true, 0, true)
          .kind;
  *kind = k;
  const int64_t tm = (a.rows + tile_m(k) - 1) / tile_m(k);
  const int64_t tn = (a.V + tile_n(k) - 1) / tile_n(k);
  if (tm * tn >= kMostTiles) return hipErrorInvalidConfiguration;
  a.tm = (int)tm, a.tn = (int)tn;
  return with_tile(k, [&](auto shape) {
    using S = decltype(shape);
    if constexpr (WHAT != Logit::kStatsExps && S::BM == 32)
      if (direct) return run_logits<S, kDirect, WHAT>(a, stream);
    if constexpr (WHAT != Logit::kStatsExps && S::BM <= 128)
      if (!bf16) return run_logits<S, kSplit, WHAT>(a, stream);
    return bf16 ? run_logits<S, kPlain, WHAT>(a, stream) : hipErrorInvalidValue;
  });
}

template <bool BF16, Keep KEEP>
hipError_t launch_from_kept(const FromKept& a, hipStream_t stream) {
  const dim3 grid((unsigned)((a.rows + 63) / 64), (a.dz_width + 511) / 512);
  from_kept_kernel<BF16, KEEP><<<grid, 256, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

bool xent_aligned(const XentArgs& a) { return !a.bf16 || direct(a.W, a.ldw, 8); }

size_t xent_workspace_bytes(int64_t n, int32_t C, int32_t V, bool bf16, bool aligned,
                            XentPass pass) {
  return layout(n, C, V, bf16, aligned, pass).total;
}

hipError_t launch_xent(const XentArgs& a, XentPass pass, hipStream_t stream) {
  const Layout w = layout(a.n, a.C, a.V, a.bf16, xent_aligned(a), pass);
  // a step without gradients is a forward pass
  const bool grads = pass != XentPass::kForward &&
                     (a.dx != nullptr || a.dW != nullptr || a.db != nullptr);
  if (pass == XentPass::kBackward && !grads) return hipSuccess;
  const Labels labels{a.labels, a.id64, a.label_stride, a.V};
  int32_t* idx = reinterpret_cast<int32_t*>(byte(a.ws, w.idx));
  const auto live_from = [&](int64_t row0) {
    return LiveRows{idx + row0, reinterpret_cast<int32_t*>(byte(a.ws, w.label)) + row0,
                    reinterpret_cast<float*>(byte(a.ws, w.weight)) + row0,
                    reinterpret_cast<float*>(byte(a.ws, w.lse)) + row0};
  };
  int32_t* count = reinterpret_cast<int32_t*>(byte(a.ws, w.count));
  if (a.n == 0) {  // the parameters' gradients of no rows
    if (grads && !a.accumulate) {
      if (a.db != nullptr) SHC_LAUNCH(launch_sum_rows(nullptr, 0, 0, a.V, 0, a.db, stream));
      if (a.dW != nullptr) {
        Product p{};
        p.split = !a.bf16;
        p.M = a.V, p.N = a.C;
        p.store.out = a.dW, p.store.ld_out = a.lddW;
        SHC_LAUNCH(launch_product(p, stream));
      }
    }
    return hipSuccess;
  }
  // 1. the live rows
  const int blocks = (int)((a.n + kLabelsPerBlock - 1) / kLabelsPerBlock);
  int32_t* counts = reinterpret_cast<int32_t*>(byte(a.ws, w.counts));
  float* most = reinterpret_cast<float*>(byte(a.ws, w.most));
  float* scale = a.bf16 && grads && a.weight != nullptr
                     ? reinterpret_cast<float*>(byte(a.ws, w.scale))
                     : nullptr;
  if (blocks > 1) {
    count_labels_kernel<<<blocks, 256, 0, stream>>>(labels, a.n, counts,
                                                    scale != nullptr ? a.weight : nullptr, most);
    SHC_LAUNCH(hipGetLastError());
  }
  const bool back = pass == XentPass::kBackward;
  list_rows_kernel<<<blocks, 256, 0, stream>>>(
      labels, a.n, counts, live_from(0), count, a.weight, back ? a.lse : nullptr,
      back ? nullptr : a.loss, pass == XentPass::kForward ? a.lse : nullptr, most, scale);
  SHC_LAUNCH(hipGetLastError());
  const bool as_is = a.bf16 && direct(a.x, a.ldx, a.C);
  const int64_t xwidth = packed_width(a.C);
  uint16_t* xs = reinterpret_cast<uint16_t*>(byte(a.ws, w.x));
  SHC_LAUNCH(launch_pack(Pack{a.x, a.ldx, a.n, a.n, a.C, !a.bf16, idx, count, 0,
                              as_is ? a.n : -1, xs}, stream));
  // rows of x from row0 on, along the rows or across
  const auto x_of = [&](int64_t row0, int64_t rows, bool along) {
    Operand o{};
    o.ld = as_is ? a.ldx : xwidth;
    o.p = as_is ? static_cast<const uint16_t*>(a.x) + row0 * a.ldx : xs + row0 * xwidth;
    if (as_is) o.alt = xs + row0 * xwidth, o.alt_ld = xwidth;
    const int64_t width = as_is ? a.C : xwidth;
    o.extent = along ? rows : width;
    o.k = along ? width : rows;
    o.plane = a.n * xwidth;
    if (!a.bf16) o.f32 = static_cast<const float*>(a.x), o.f32_ld = a.ldx, o.idx = idx + row0;
    return o;
  };
  // 2. the table
  const bool W_as_is = a.bf16 && direct(a.W, a.ldw, a.C);
  const int64_t Wwidth = W_as_is ? a.C : packed_width(a.C);
  const uint16_t* Wp = static_cast<const uint16_t*>(a.W);
  int64_t Wld = a.ldw;
  const bool few = !a.bf16 && a.n <= kFewRows;
  if (!W_as_is && !few) {
    uint16_t* to = reinterpret_cast<uint16_t*>(byte(a.ws, w.W));
    SHC_LAUNCH(launch_pack(Pack{a.W, a.ldw, a.V, a.V, a.C, !a.bf16, nullptr, nullptr, 0, -1, to},
                           stream));
    Wp = to, Wld = Wwidth;
  }
  const auto W_of = [&](bool along) {
    Operand o{};
    o.p = Wp, o.ld = Wld;
    o.extent = along ? a.V : Wwidth;
    o.k = along ? Wwidth : a.V;
    o.plane = (int64_t)a.V * Wwidth;
    if (!a.bf16) o.f32 = static_cast<const float*>(a.W), o.f32_ld = a.ldw;
    return o;
  };
  Logits g{};
  g.B = W_of(true);
  g.C = a.C;
  g.count = count, g.full = a.n;
  g.bias = a.bias;
  g.V = a.V;
  TileKind kind;
  g.parts = reinterpret_cast<float2*>(byte(a.ws, w.parts));
  g.at_label = reinterpret_cast<float*>(byte(a.ws, w.at_label));
  const auto join = [&](int64_t row0, int64_t rows) {
    join_stats_kernel<<<(int)((rows + 15) / 16), 256, 0, stream>>>(
        g.parts, (a.V + tile_n(kind) - 1) / tile_n(kind), rows, count, row0,
        live_from(row0), g.at_label, a.loss, pass == XentPass::kForward ? a.lse : nullptr);
    return hipGetLastError();
  };
  const bool products = a.dx != nullptr || a.dW != nullptr;
  const bool cut = cut_logits(a.n, a.C, a.V, few ? kDirect : a.bf16 ? kPlain : kSplit);
  if (cut) {
    Product p{};
    p.A = x_of(0, a.n, true), p.B = W_of(true);
    p.a_rows = p.b_rows = true;
    p.split = !a.bf16, p.direct = few;
    p.M = a.n, p.N = a.V, p.K = a.C;
    p.count = count, p.full = a.n;
    p.store.out32 = reinterpret_cast<float*>(byte(a.ws, w.logits));
    p.partials = reinterpret_cast<float*>(byte(a.ws, w.partials));
    p.partial_bytes = partial_bytes(a.n, a.V, a.C);
    SHC_LAUNCH(launch_product(p, stream));
    if (pass != XentPass::kBackward) {
      row_stats_kernel<<<(int)a.n, 256, 0, stream>>>(
          p.store.out32, a.V, count, a.bias, live_from(0), a.loss,
          pass == XentPass::kForward ? a.lse : nullptr);
      SHC_LAUNCH(hipGetLastError());
    }
  }
  const bool keep = !cut && pass == XentPass::kStep && keeps(a.C, a.bf16, a.db != nullptr) && grads;
  if (pass != XentPass::kBackward && !keep && !cut) {  // 3. statistics, loss and lse
    g.A = x_of(0, a.n, true);
    g.rows = a.n, g.row0 = 0, g.live = live_from(0);
    SHC_LAUNCH(launch_logits<Logit::kStats>(g, a.bf16, &kind, stream));
    SHC_LAUNCH(join(0, a.n));
  }
  if (!grads) return hipSuccess;
  // 4. gradients, a piece of the live rows at a time
  const int64_t dz_ld = a.bf16 ? w.width : a.V;
  const bool fine = a.bf16 && a.n <= kFine;
  const float* undo = scale != nullptr ? scale + 1 : nullptr;
  uint16_t* dz = reinterpret_cast<uint16_t*>(byte(a.ws, w.dz));
  float* acc = reinterpret_cast<float*>(byte(a.ws, w.acc));
  for (int64_t piece = 0; piece < w.pieces; ++piece) {
    const int64_t row0 = piece * w.rows, rows = std::min(w.rows, a.n - row0);
    g.A = x_of(row0, rows, true);
    g.rows = rows, g.row0 = row0, g.live = live_from(row0);
    g.dz = a.bf16 ? static_cast<void*>(dz) : byte(a.ws, w.dz32);
    g.ld_dz = dz_ld;
    g.low = fine ? rows * dz_ld : 0;
    g.scale = scale;
    g.width = (int)dz_ld;
    g.sums = a.db != nullptr ? reinterpret_cast<float*>(byte(a.ws, w.sums)) : nullptr;
    int per = 64;  // rows to a part of the sums
    if (keep || cut) {
      const bool exps = !cut && a.bf16 && a.db == nullptr;
      g.kept = cut ? byte(a.ws, w.logits) : a.bf16 && !exps ? byte(a.ws, w.kept) : g.dz;
      if (keep) {
        SHC_LAUNCH(exps ? launch_logits<Logit::kStatsExps>(g, a.bf16, &kind, stream)
                        : launch_logits<Logit::kStatsLogits>(g, a.bf16, &kind, stream));
        SHC_LAUNCH(join(row0, rows));
      }
      const FromKept f{g.kept,  rows,  count, row0, g.parts, cut ? 0 : tile_n(kind),
                       a.V,     cut ? a.bias : nullptr,     g.live,  g.dz,  g.low, scale,
                       cut ? a.V : (int)dz_ld, (int)dz_ld, g.sums};
      SHC_LAUNCH(exps     ? launch_from_kept<true, kExps>(f, stream)
                 : a.bf16 ? launch_from_kept<true, kLogits>(f, stream)
                          : launch_from_kept<false, kLogits>(f, stream));
    } else {
      SHC_LAUNCH(launch_logits<Logit::kGrad>(g, a.bf16, &kind, stream));
      per = kind == TileKind::k256 ? 128 : kind == TileKind::k128 ? 64 : 32;  // a wavefront's
    }
    if (a.db != nullptr) {
      join_sums_kernel<<<(a.V + 63) / 64, 1024, 0, stream>>>(g.sums, per, rows, count, row0, a.V,
                                                             piece > 0 || a.accumulate, undo, a.db);
      SHC_LAUNCH(hipGetLastError());
    }
    if (!products) continue;
    if (!a.bf16 && (!few || a.dW != nullptr))
      SHC_LAUNCH(launch_pack(Pack{g.dz, dz_ld, rows, rows, a.V, 1, nullptr, count, row0, -1, dz},
                             stream));
    Operand d{};
    d.p = dz, d.ld = w.width, d.plane = rows * w.width;
    if (!a.bf16) d.f32 = static_cast<const float*>(g.dz), d.f32_ld = dz_ld;
    Product p{};
    p.split = !a.bf16, p.a_low = fine;
    p.store.scale = undo;
    p.count = count, p.row0 = row0, p.full = a.n;
    p.partials = reinterpret_cast<float*>(byte(a.ws, w.partials));
    p.partial_bytes = w.partial_bytes;
    if (a.dx != nullptr) {
      p.A = d, p.A.extent = rows, p.A.k = w.width;
      p.B = W_of(false);
      p.direct = few;
      p.a_rows = true, p.b_rows = false;
      p.M = rows, p.N = a.C, p.K = a.V;
      p.store.out = a.dx, p.store.ld_out = a.lddx, p.store.to = idx + row0;
      SHC_LAUNCH(launch_product(p, stream));
    }
    if (a.dW != nullptr) {
      p.A = d, p.A.extent = w.width, p.A.k = rows;
      p.direct = false;
      p.B = x_of(row0, rows, false);
      p.a_rows = p.b_rows = false;
      p.M = a.V, p.N = a.C, p.K = rows;
      p.count_is_k = true;
      p.store = Store{};
      p.store.scale = undo;
      p.store.add32 = piece > 0 ? acc : nullptr;
      if (piece + 1 < w.pieces) {
        p.store.out32 = acc;
      } else {
        p.store.out = a.dW, p.store.ld_out = a.lddW;
        if (a.accumulate) p.store.res = a.dW, p.store.ld_res = a.lddW;
      }
      SHC_LAUNCH(launch_product(p, stream));
    }
  }
  if (a.dx != nullptr) {
    const int zero_blocks = (int)std::min<int64_t>((a.n + 3) / 4, 2048);
    if (a.bf16)
      zero_rows_kernel<uint16_t><<<zero_blocks, 256, 0, stream>>>(
          labels, a.n, count, static_cast<uint16_t*>(a.dx), a.lddx, a.C);
    else
      zero_rows_kernel<float><<<zero_blocks, 256, 0, stream>>>(
          labels, a.n, count, static_cast<float*>(a.dx), a.lddx, a.C);
    SHC_LAUNCH(hipGetLastError());
  }
  return hipSuccess;
}

}  // namespace shc
