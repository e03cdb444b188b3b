// Matrix products of the dense layers: D = A B^T over the tile of dense_tile.h, with
// bias, activation, residual, row scatter and rounding in the epilogue; and the packing
// of operands that the tile cannot read as they are.
//
// Which tile, and how many parts K is cut into, follows from the sizes by a model of
// the time, `plan_product`: rounds of workgroups over the CUs times the steps of one,
// plus what parts cost (their fp32 sums written and read back, a second launch).
//
// bf16 products, us by tile, 256 x 256, 128 x 128, 64 x 128, 32 x 128:
//   67,040 x   128 x   128     26.2    15.3    11.6    13.7
//   67,040 x 1,024 x   128     84.7    59.5    52.9    74.2
//   20,000 x   512 x   512     26.6    23.2    20.6    28.0
//   16,384 x 1,024 x 1,024     42.1    43.3    47.4    63.6
//    4,096 x 4,096 x 4,096      122     142     182     256
//    8,192 x 8,192 x 8,192      891   1,026   1,382   3,510
//       16 x 16,384 x 4,096    34.7    30.0    28.8    29.4  (K in 3 or 4 parts)
//        1 x 4,096 x 4,096             14.7    13.6    13.2  (in 6)
// Large ones are bound by the matrix cores at the power limit: 8,192 cubed at 1.10, 1.23
// and 1.26 PFLOP/s with rows x rows, rows x cols, cols x cols, 4,096 x 131,072 x 4,096 at 1.25 in
// any order; the matrix units are busy 0.62 to 0.66 of the time, LDS 0.24, without a
// conflict.  Split fp32, 4,096 cubed: 981, 1,141, 1,170 TFLOP/s of bf16, 164 to 195 of
// fp32, against 154 of a library's product on the fp32 matrix cores.
//
// Few rows are bound by reading the second operand: 16 rows by 16,384 x 4,096 in bf16 27
// us (5 TB/s) and 4.5 for joining the two parts of K.  fp32, us from memory / in three terms
// (which packs that operand first): 1 row through 4,096 x 4,096 25.7 / 52.0, 32 rows 27.2 /
// 52.5; 32 rows through 512 x 512 11.4 / 15.4, 1,024 x 16,384 22.7 / 51.5 (kFewRows).
#include <algorithm>
#include <mutex>

#include "dense.h"
#include "dense_epilogue.h"

namespace shc {
namespace dense {
namespace {

struct Args {
  Operand A, B;
  int64_t M, N, K;
  const int32_t* count;
  int64_t row0, full;
  int count_is_k, a_low;
  Store store;
  float* partials;
  int parts, tn;  // parts of K, columns of tiles
  int join;       // the sums go to partials
};

template <class S, bool AROWS, bool BROWS, Mode MODE>
__global__ __launch_bounds__(S::THREADS) void product_kernel(Args a) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  int64_t M = a.M, K = a.K;
  if (a.count != nullptr) {
    const int64_t left = rows_left(a.count, a.row0, a.count_is_k ? a.K : a.M);
    if (a.count_is_k)
      K = a.A.k = a.B.k = left;
    else
      M = a.A.extent = left;
    if (*a.count != a.full) {
      if (a.A.alt != nullptr) a.A.p = a.A.alt, a.A.ld = a.A.alt_ld;
      if (a.B.alt != nullptr) a.B.p = a.B.alt, a.B.ld = a.B.alt_ld;
    }
  }
  int tm, tn;
  if (!tile_of(blockIdx.x, (int)((M + S::BM - 1) / S::BM), a.tn, &tm, &tn)) return;
  const int64_t m0 = (int64_t)tm * S::BM, n0 = (int64_t)tn * S::BN;
  const int KT = (int)((K + BK - 1) / BK), per = (KT + a.parts - 1) / a.parts;
  const int t0 = min(KT, (int)blockIdx.y * per), t1 = min(KT, t0 + per);
  constexpr bool BF16 = MODE == kPlain;
  Tile<S, AROWS, BROWS, MODE> tile;
  const auto fetch = [&](int64_t row, int64_t col) {
    Fetched<BF16> g{};
    if (!a.join && row < M && col < a.N)
      g = fetch8<BF16>(a.store, row, (int)(col / 8), (int)a.N);
    return g;
  };
  // small tiles have registers to fetch what the store needs before the product
  Fetched<BF16> got[4];
  if constexpr (S::MB == 1) tile.fetch_block(m0, n0, 0, got, fetch);
  tile.run(a.A, a.B, M, a.N, K, m0, n0, t0, t1, smem);
  if constexpr (BF16 && !AROWS)
    if (a.a_low) {
      a.A.p += a.A.plane;
      tile.add(a.A, a.B, M, a.N, K, m0, n0, t0, t1, smem);
    }
  if (a.join) {
    float* to = a.partials + (int64_t)blockIdx.y * a.M * a.N;
    tile.each(m0, n0, smem, [&](int64_t row, int64_t col, const float (&v)[8]) {
      if (row < M && col < a.N)
        rowops::store_channels<8>(to + row * a.N, (int)(col / 8), (int)a.N, v);
    });
    return;
  }
  if constexpr (S::MB > 1) tile.fetch_block(m0, n0, 0, got, fetch);
  const float scale = scale_of(a.store);
  float bias[8];
  if (tile.col_of(n0) < a.N) bias8(a.store, (int)(tile.col_of(n0) / 8), (int)a.N, bias);
  tile.each(m0, n0, smem, got, fetch,
            [&](int64_t row, int64_t col, const float (&v)[8], const Fetched<BF16>& g) {
              if (row < M && col < a.N)
                store8<BF16>(a.store, row, (int)(col / 8), (int)a.N, v, scale, bias, g);
            });
}

// Sums the parts in order and stores: a thread to 8 columns of a row.  Bound by latency: 4
// us for 16 x 16,384 in two parts.
template <bool BF16>
__global__ __launch_bounds__(256) void join_kernel(const float* parts, int n, int64_t M, int N,
                                                   const int32_t* count, int64_t row0, Store st) {
  const int nv = (N + 7) / 8;
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = at / nv;
  if (row >= rows_left(count, row0, M)) return;
  const int v = (int)(at - row * nv);
  float sum[8], f[8], bias[8];
  bias8(st, v, N, bias);
  const Fetched<BF16> g = fetch8<BF16>(st, row, v, N);
  const float* from = parts + row * N;
  rowops::load_channels<8>(from, v, N, sum);
  for (int p = 1; p < n; ++p) {
    rowops::load_channels<8>(from + p * M * N, v, N, f);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] += f[e];
  }
  store8<BF16>(st, row, v, N, sum, scale_of(st), bias, g);
}

// 8 elements of a packed row to a thread.  Bound by HBM: 520 rows of 50,021 fp32 into
// three terms (104 MB read, 154 written) in 40 us, 6.5 TB/s; small ones by the launch.
template <typename T, bool SPLIT>
__global__ __launch_bounds__(256) void pack_kernel(Pack p, int width) {
  using namespace rowops;
  if (p.unless_full >= 0 && *p.count == p.unless_full) return;
  const int nv = width / 8;
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = at / nv;
  if (row >= rows_left(p.count, p.row0, p.n)) return;
  const int v = (int)(at - row * nv);
  const T* from = static_cast<const T*>(p.src) +
                  (p.idx != nullptr ? (int64_t)p.idx[row] : row) * p.ld;
  uint16_t* to = p.dst + row * width + 8 * v;
  if constexpr (!SPLIT) {
    i32x4 x = {0, 0, 0, 0};
    if (8 * v < p.C) x = load_vec<T>(from, v, p.C);
    *reinterpret_cast<i32x4*>(to) = x;
  } else {
    float x[8], t[8], r[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = 0.f;
    if (8 * v < p.C) load_channels<8>(from, v, p.C, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= kSplitScale;
    // each term is the nearest bf16 to what is left: 8 + 8 + 8 significand bits
    for (int term = 0; term < 3; ++term) {
      const i32x4 h = Row<uint16_t>::narrow(x);
      Row<uint16_t>::widen(h, t);
#pragma unroll
      for (int e = 0; e < 8; ++e) r[e] = x[e] - t[e], x[e] = r[e];
      *reinterpret_cast<i32x4*>(to + term * p.rows * width) = h;
    }
  }
}

// 64 columns to a workgroup, the rows to 16 wavefronts in turn: 5 us for 512 rows of 8,192.
__global__ __launch_bounds__(1024) void sum_rows_kernel(const float* parts, int64_t rows,
                                                        int64_t ld, int C, int accumulate,
                                                        float* out) {
  __shared__ float part[16][64];
  const int x = threadIdx.x & 63, y = threadIdx.x >> 6;
  const int c = blockIdx.x * 64 + x;
  const int64_t per = (rows + 15) / 16, r0 = y * per, r1 = r0 + per < rows ? r0 + per : rows;
  float s = 0.f;
  if (c < C)
    for (int64_t r = r0; r < r1; ++r) s += parts[r * ld + c];
  part[y][x] = s;
  __syncthreads();
  if (y != 0 || c >= C) return;
  for (int q = 1; q < 16; ++q) s += part[q][x];
  out[c] = accumulate ? out[c] + s : s;
}

// Bytes of parts at most.  From 512 tiles of 128 x 128 on a product fills the CUs without
// them; two parts of that are half of this.
constexpr int64_t kMostPartial = (int64_t)128 << 20;

template <class S, bool AROWS, bool BROWS, Mode MODE>
hipError_t run(const Args& a, int tiles, hipStream_t stream) {
  auto kern = product_kernel<S, AROWS, BROWS, MODE>;
  constexpr int lds = S::template lds<MODE>();
  static std::once_flag once;
  static hipError_t attr = hipSuccess;
  std::call_once(once, [&] {
    attr = hipFuncSetAttribute(reinterpret_cast<const void*>(kern),
                               hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  });
  if (attr != hipSuccess) return attr;
  kern<<<dim3(tiles, a.parts), S::THREADS, lds, stream>>>(a);
  return hipGetLastError();
}

template <class S, Mode MODE>
hipError_t run_orders(const Args& a, int tiles, bool ar, bool br, hipStream_t stream) {
  if constexpr (S::BM >= 128)  // a cols operand has 128 rows at least
    if (!ar && !br) return run<S, false, false, MODE>(a, tiles, stream);
  if (ar && br) return run<S, true, true, MODE>(a, tiles, stream);
  if (ar && !br) return run<S, true, false, MODE>(a, tiles, stream);
  return hipErrorInvalidValue;
}

}  // namespace

size_t partial_bytes(int64_t M, int64_t N, int64_t K) {
  // at most a part to two steps of K, and at most kMostPartial
  const int64_t parts = K / (2 * BK);
  if (parts <= 1) return 0;
  const int64_t mn = M * N * 4;
  return (size_t)(mn > kMostPartial / parts ? kMostPartial : mn * parts);
}

// Times in us, from the figures at the top.  A CU holds `slots` workgroups of a kind; a
// step of 64 of K takes `latency` or, of as many as are there, `work` each; a tile has
// `fixed` beside its steps.
Plan plan_product(int64_t M, int64_t N, int64_t K, Mode mode, bool few_rows,
                  size_t partial_bytes, bool logits, double* time, const Operand* reach) {
  struct Kind {
    TileKind kind;
    int slots;
    double latency, work, fixed, fixed_logits;
  };
  static constexpr Kind plain[] = {{TileKind::k256, 1, 1.8, 1.8, 14.0, 10.8},
                                   {TileKind::k128, 2, 0.7, 0.51, 5.2, 5.8},
                                   {TileKind::k64, 3, 0.6, 0.34, 2.8, 4.9},
                                   {TileKind::k32, 4, 0.5, 0.25, 2.5, 4.5}};
  static constexpr Kind terms[] = {{TileKind::k128, 1, 2.6, 2.8, 8.0, 8.0},
                                   {TileKind::k64, 1, 1.5, 2.0, 5.0, 6.0},
                                   {TileKind::k32, 1, 1.2, 1.6, 4.0, 5.0}};
  static constexpr Kind direct[] = {{TileKind::k32, 8, 1.9, 0.85, 3.0, 4.0}};
  constexpr int kCUs = 256;
  const int64_t KT = (K + BK - 1) / BK;
  Plan best{TileKind::k128, 1};
  double least = 1e300;
  const Kind* kinds = mode == kDirect ? direct : mode == kSplit ? terms : plain;
  for (int i = 0; i < (mode == kDirect ? 1 : mode == kSplit ? 3 : 4); ++i) {
    const Kind& k = kinds[i];
    if (!few_rows && tile_m(k.kind) < 128) continue;
    if (reach != nullptr && !in_reach(*reach, true, tile_m(k.kind))) continue;
    const int64_t tiles = ((M + tile_m(k.kind) - 1) / tile_m(k.kind)) *
                          ((N + tile_n(k.kind) - 1) / tile_n(k.kind));
    // few rows of tiles share what they read of B with few others: its bytes of a
    // step for every column come from memory, at 6.2 TB/s
    const int bytes = mode == kPlain ? 128 : mode == kSplit ? 384 : 256;
    const double read = (double)tile_n(k.kind) * bytes * kCUs / 6.2e6 /
                        (double)((M + tile_m(k.kind) - 1) / tile_m(k.kind));
    for (int parts = 1; parts <= 64; parts = parts < 4 ? parts + 1 : parts + parts / 2) {
      if (parts > 1 && (KT < 2 * parts || (double)parts * M * N * 4 > (double)partial_bytes)) break;
      const int64_t rounds = tiles * parts / (kCUs * k.slots);
      const int64_t rest = tiles * parts % (kCUs * k.slots);
      const double steps = (double)((KT + parts - 1) / parts);
      const auto round = [&](double here) {
        return steps * std::max(k.latency, here * std::max(k.work, read)) +
               (logits ? k.fixed_logits : k.fixed);
      };
      double t = rounds * round(k.slots);
      if (rest > 0)
        t += round(rest < kCUs ? (double)rest / kCUs : (double)((rest + kCUs - 1) / kCUs));
      if (parts > 1) t += 4.0 + (double)parts * M * N * 8 / 4e6;
      if (t < least) least = t, best = {k.kind, parts};
    }
  }
  if (time != nullptr) *time = least;
  return best;
}

// Rows of dz are as far apart as there are classes, up to 2^24: a tile of 64 of them is
// within reach, one of 128 up to 8,454,000 classes, one of 256 up to 4,210,000.
Plan plan_of(const Product& p) {
  const Mode mode = p.direct ? kDirect : p.split ? kSplit : kPlain;
  return plan_product(p.a_low && p.a_rows ? 2 * p.M : p.M, p.N, p.K, mode, p.a_rows,
                      p.partials != nullptr ? p.partial_bytes : 0, false, nullptr,
                      p.a_rows && !p.direct ? &p.A : nullptr);
}

hipError_t launch_product(const Product& p, hipStream_t stream) {
  if (p.M <= 0 || p.N <= 0) return hipSuccess;
  // two terms of A in rows: as many rows again, joined with the first as parts of K are
  const bool twice = p.a_low && p.a_rows;
  const int64_t M = twice ? 2 * p.M : p.M;
  if (twice && (p.partial_bytes < (size_t)M * p.N * 4 || p.A.plane != p.M * p.A.ld))
    return hipErrorInvalidValue;
  const Plan plan = plan_of(p);
  // direct products have offsets of 64 bits
  if (!p.direct && p.K > 0 &&
      (!in_reach(p.A, p.a_rows, tile_m(plan.kind)) || !in_reach(p.B, p.b_rows, tile_n(plan.kind))))
    return hipErrorInvalidValue;
  Args a;
  a.A = p.A, a.B = p.B;
  a.M = M, a.N = p.N, a.K = p.K;
  if (twice) a.A.extent = M;
  a.count = twice ? nullptr : p.count;
  a.row0 = p.row0, a.full = p.full, a.count_is_k = p.count_is_k, a.a_low = p.a_low;
  a.store = p.store;
  a.partials = p.partials;
  a.parts = plan.parts;
  a.join = plan.parts > 1 || twice;
  const int64_t tm = (M + tile_m(plan.kind) - 1) / tile_m(plan.kind);
  const int64_t tn = (p.N + tile_n(plan.kind) - 1) / tile_n(plan.kind);
  if (tm * tn >= kMostTiles) return hipErrorInvalidConfiguration;
  a.tn = (int)tn;
  const int tiles = (int)(tm * tn);
  hipError_t e = with_tile(plan.kind, [&](auto shape) {
    using S = decltype(shape);
    if constexpr (S::BM == 32)
      if (p.direct) return run_orders<S, kDirect>(a, tiles, p.a_rows, p.b_rows, stream);
    if constexpr (S::BM <= 128)
      if (p.split) return run_orders<S, kSplit>(a, tiles, p.a_rows, p.b_rows, stream);
    return p.split ? hipErrorInvalidValue
                   : run_orders<S, kPlain>(a, tiles, p.a_rows, p.b_rows, stream);
  });
  if (e != hipSuccess || !a.join) return e;
  const int parts = twice ? 2 * plan.parts : plan.parts;
  const int64_t threads = p.M * ((p.N + 7) / 8);
  const int blocks = (int)((threads + 255) / 256);
  const int32_t* rows = p.count_is_k ? nullptr : p.count;
  if (p.split)
    join_kernel<false><<<blocks, 256, 0, stream>>>(p.partials, parts, p.M, (int)p.N, rows,
                                                   p.row0, p.store);
  else
    join_kernel<true><<<blocks, 256, 0, stream>>>(p.partials, parts, p.M, (int)p.N, rows,
                                                  p.row0, p.store);
  return hipGetLastError();
}

hipError_t launch_pack(const Pack& p, hipStream_t stream) {
  const int width = (int)packed_width(p.C);
  const int64_t blocks = (p.n * (width / 8) + 255) / 256;
  if (blocks == 0) return hipSuccess;
  if (blocks >= (int64_t)1 << 24) {  // a launch has fewer than 2^32 threads
    Pack a = p, b = p;
    a.n = p.n / 2, b.n = p.n - a.n, b.row0 += a.n;
    if (p.idx != nullptr)
      b.idx += a.n;
    else
      b.src = static_cast<const char*>(p.src) + a.n * p.ld * (p.split ? 4 : 2);
    b.dst += a.n * width;
    const hipError_t e = launch_pack(a, stream);
    return e != hipSuccess ? e : launch_pack(b, stream);
  }
  if (p.split)
    pack_kernel<float, true><<<(int)blocks, 256, 0, stream>>>(p, width);
  else
    pack_kernel<uint16_t, false><<<(int)blocks, 256, 0, stream>>>(p, width);
  return hipGetLastError();
}

hipError_t launch_sum_rows(const float* parts, int64_t rows, int64_t ld, int32_t C, int accumulate,
                           float* out, hipStream_t stream) {
  sum_rows_kernel<<<(C + 63) / 64, 1024, 0, stream>>>(parts, rows, ld, C, accumulate, out);
  return hipGetLastError();
}

}  // namespace dense
}  // namespace shc
