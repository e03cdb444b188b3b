// Layer norm over the channels of a row, with weight and bias, and its
// gradient:
//
//   mu = sum(x) / C,  var = sum((x - mu)^2) / C,  rs = 1 / sqrt(var + eps)
//   y  = (x - mu) rs gamma + beta
//
//   h = (x - mu) rs,  g = dy gamma,
//   dx = rs (g - sum(g) / C - h sum(g h) / C)
//   dgamma = sum over rows of dy h,  dbeta = sum over rows of dy
//
// Both are bound by HBM: a row is read once into registers (G lanes hold NV
// 16-byte vectors each), reduced there, and written.  The variance is taken
// from the deviations of the values in registers, so a large mean costs no
// digits.  A group of lanes walks rows a grid apart with gamma (and beta, or
// the two column sums) in registers and the next row's vectors in flight.
//
// The column sums dgamma and dbeta: every thread sums its columns over its
// rows, the groups of a wavefront are added across its lanes and the wavefronts of
// a workgroup in LDS, every workgroup writes one partial row to the workspace, and a
// second launch adds the partial rows, all in a fixed order.  The number of
// workgroups follows the sizes alone, so results repeat bit for bit.
//
// Measured: forward, 4,099 rows of 5,001 fp32: 34.7 us, 4.7 TB/s; gradient, 16,384
// rows of 4,096 bf16: 81.4 us, 4.9 TB/s (78 and 5 in the second launch).
#include <algorithm>

#include "row_ops.h"

namespace shc {
namespace {

using namespace rowops;

template <typename T, int G, int NV>
__global__ __launch_bounds__(G > 256 ? G : 256) void layer_norm_kernel(
    const T* __restrict__ x, int64_t ldx, int64_t n, int C, const float* __restrict__ gamma,
    const float* __restrict__ beta, float eps, T* __restrict__ y, int64_t ldy,
    float* __restrict__ mean, float* __restrict__ rstd) {
  constexpr int N = Row<T>::N, BLOCK = G > 256 ? G : 256, R = BLOCK / G;
  __shared__ float part[G > 64 ? BLOCK / 64 : 1];
  const int lane = threadIdx.x % G;
  const int nvec = (C + N - 1) / N;
  const float inv_c = 1.0f / (float)C;
  // a group of more than a wavefront has LDS partials of its own
  float* my_part = G > 64 ? part + (threadIdx.x / G) * (G / 64) : part;

  float ga[NV][N], be[NV][N];
#pragma unroll
  for (int q = 0; q < NV; ++q) {
    const int v = q * G + lane;
#pragma unroll
    for (int e = 0; e < N; ++e) ga[q][e] = 1.f, be[q][e] = 0.f;
    if (v < nvec) {
      if (gamma != nullptr) load_channels<N>(gamma, v, C, ga[q]);
      if (beta != nullptr) load_channels<N>(beta, v, C, be[q]);
    }
  }
  const int64_t step = (int64_t)gridDim.x * R;
  int64_t row = (int64_t)blockIdx.x * R + threadIdx.x / G;
  i32x4 cur[NV];
  auto fetch = [&](int64_t r, i32x4* to) {
#pragma unroll
    for (int q = 0; q < NV; ++q) {
      const int v = q * G + lane;
      to[q] = v < nvec ? load_vec(x + r * ldx, v, C) : i32x4{};
    }
  };
  if (row < n) fetch(row, cur);
  // with a barrier in the reduction (R == 1) every thread of the workgroup has
  // the same row, so the loop's length is uniform
  for (; row < n; row += step) {
    i32x4 next[NV];
    if (row + step < n) fetch(row + step, next);
    float sum = 0.f;
#pragma unroll
    for (int q = 0; q < NV; ++q) {
      float f[N];
      Row<T>::widen(cur[q], f);
#pragma unroll
      for (int e = 0; e < N; ++e) sum += f[e];  // past the row's end: zeros
    }
    const float mu = group_reduce<G>(sum, AddOp{}, my_part) * inv_c;
    float sq = 0.f;
#pragma unroll
    for (int q = 0; q < NV; ++q) {
      const int left = C - (q * G + lane) * N;
      float f[N];
      Row<T>::widen(cur[q], f);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float d = f[e] - mu;
        if (e < left) sq = fmaf(d, d, sq);
      }
    }
    const float var = group_reduce<G>(sq, AddOp{}, my_part) * inv_c;
    const float rs = 1.0f / sqrtf(var + eps);
    if (lane == 0) {
      if (mean != nullptr) mean[row] = mu;
      if (rstd != nullptr) rstd[row] = rs;
    }
#pragma unroll
    for (int q = 0; q < NV; ++q) {
      const int v = q * G + lane;
      if (v < nvec) {
        float f[N];
        Row<T>::widen(cur[q], f);
#pragma unroll
        for (int e = 0; e < N; ++e) f[e] = fmaf((f[e] - mu) * rs, ga[q][e], be[q][e]);
        store_vec(y + row * ldy, v, C, Row<T>::narrow(f));
      }
    }
#pragma unroll
    for (int q = 0; q < NV; ++q) cur[q] = next[q];
  }
}

template <typename T, int G, int NV>
__global__ __launch_bounds__(G > 256 ? G : 256) void layer_norm_backward_kernel(
    const T* __restrict__ dy, int64_t lddy, const T* __restrict__ x, int64_t ldx, int64_t n,
    int C, const float* __restrict__ gamma, const float* __restrict__ mean,
    const float* __restrict__ rstd, T* __restrict__ dx, int64_t lddx, float* __restrict__ col) {
  constexpr int N = Row<T>::N, BLOCK = G > 256 ? G : 256, R = BLOCK / G;
  __shared__ float part[G > 64 ? BLOCK / 64 : 1];
  // column sums of the workgroup's wavefronts (R > 1), one's at a time
  __shared__ float cols[R > 1 ? 2 * G * NV * N : 1];
  const int lane = threadIdx.x % G;
  const int nvec = (C + N - 1) / N;
  const float inv_c = 1.0f / (float)C;
  float* my_part = G > 64 ? part + (threadIdx.x / G) * (G / 64) : part;

  float ga[NV][N], dg[NV][N], db[NV][N];
#pragma unroll
  for (int q = 0; q < NV; ++q) {
    const int v = q * G + lane;
#pragma unroll
    for (int e = 0; e < N; ++e) ga[q][e] = 1.f, dg[q][e] = 0.f, db[q][e] = 0.f;
    if (v < nvec && gamma != nullptr) load_channels<N>(gamma, v, C, ga[q]);
  }
  // the next row's vectors in flight, where the registers hold them
  constexpr bool AHEAD = !(G == 1024 && NV == 4);
  const int64_t step = (int64_t)gridDim.x * R;
  int64_t row = (int64_t)blockIdx.x * R + threadIdx.x / G;
  i32x4 cx[NV], cy[NV];
  float cmu = 0.f, crs = 0.f;
  auto fetch = [&](int64_t r, i32x4* tx, i32x4* ty, float* mu, float* rs) {
#pragma unroll
    for (int q = 0; q < NV; ++q) {
      const int v = q * G + lane;
      tx[q] = v < nvec ? load_vec(x + r * ldx, v, C) : i32x4{};
      ty[q] = v < nvec ? load_vec(dy + r * lddy, v, C) : i32x4{};
    }
    *mu = mean[r];
    *rs = rstd[r];
  };
  if (row < n) fetch(row, cx, cy, &cmu, &crs);
  for (; row < n; row += step) {
    i32x4 nx[NV], ny[NV];
    float nmu = 0.f, nrs = 0.f;
    if (AHEAD && row + step < n) fetch(row + step, nx, ny, &nmu, &nrs);
    float sg = 0.f, sgh = 0.f;  // past the row's end x = dy = 0
#pragma unroll
    for (int q = 0; q < NV; ++q) {
      float fx[N], fy[N];
      Row<T>::widen(cx[q], fx);
      Row<T>::widen(cy[q], fy);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float h = (fx[e] - cmu) * crs, g = fy[e] * ga[q][e];
        sg += g;
        sgh = fmaf(g, h, sgh);
        dg[q][e] = fmaf(fy[e], h, dg[q][e]);
        db[q][e] += fy[e];
      }
    }
    if (dx != nullptr) {
      // past the row's end h = -mean rstd: 0 times that is nothing unless it is past fp32
      // (a row of 1e37 throughout), when the sum is taken over the row's own channels
      if (__builtin_expect(!(fabsf(cmu * crs) < INFINITY), 0)) {
        sgh = 0.f;
#pragma unroll
        for (int q = 0; q < NV; ++q) {
          const int left = C - (q * G + lane) * N;
          float fx[N], fy[N];
          Row<T>::widen(cx[q], fx);
          Row<T>::widen(cy[q], fy);
#pragma unroll
          for (int e = 0; e < N; ++e)
            if (e < left) sgh = fmaf(fy[e] * ga[q][e], (fx[e] - cmu) * crs, sgh);
        }
      }
      const float mg = group_reduce<G>(sg, AddOp{}, my_part) * inv_c;
      const float mgh = group_reduce<G>(sgh, AddOp{}, my_part) * inv_c;
#pragma unroll
      for (int q = 0; q < NV; ++q) {
        const int v = q * G + lane;
        if (v < nvec) {
          float fx[N], fy[N];
          Row<T>::widen(cx[q], fx);
          Row<T>::widen(cy[q], fy);
#pragma unroll
          for (int e = 0; e < N; ++e) {
            const float h = (fx[e] - cmu) * crs;
            fx[e] = crs * (fmaf(fy[e], ga[q][e], -mg) - h * mgh);
          }
          store_vec(dx + row * lddx, v, C, Row<T>::narrow(fx));
        }
      }
    }
    if constexpr (AHEAD) {
#pragma unroll
      for (int q = 0; q < NV; ++q) cx[q] = nx[q], cy[q] = ny[q];
      cmu = nmu;
      crs = nrs;
    } else if (row + step < n) {
      fetch(row + step, cx, cy, &cmu, &crs);
    }
  }
  if (col == nullptr) return;
  // the sums of a wavefront's groups, then of the wavefronts, one after the other
  if constexpr (R > 1) {
    constexpr int WAVES = BLOCK / 64;
#pragma unroll
    for (int q = 0; q < NV; ++q)
#pragma unroll
      for (int e = 0; e < N; ++e) {
        dg[q][e] = groups_sum<G>(dg[q][e]);
        db[q][e] = groups_sum<G>(db[q][e]);
      }
    const int first = threadIdx.x & 63;  // the lanes of a wavefront's first group
    for (int w = 1; w < WAVES; ++w) {
      __syncthreads();
      if (threadIdx.x >> 6 == w && first < G) {
#pragma unroll
        for (int q = 0; q < NV; ++q)
#pragma unroll
          for (int e = 0; e < N; ++e) {
            cols[((q * N + e) * 2) * G + lane] = dg[q][e];
            cols[((q * N + e) * 2 + 1) * G + lane] = db[q][e];
          }
      }
      __syncthreads();
      if (threadIdx.x < G) {
#pragma unroll
        for (int q = 0; q < NV; ++q)
#pragma unroll
          for (int e = 0; e < N; ++e) {
            dg[q][e] += cols[((q * N + e) * 2) * G + lane];
            db[q][e] += cols[((q * N + e) * 2 + 1) * G + lane];
          }
      }
    }
  }
  if (threadIdx.x < G) {
    float* out = col + (int64_t)blockIdx.x * 2 * C;
#pragma unroll
    for (int q = 0; q < NV; ++q) {
      const int v = q * G + lane;
      if (v < nvec) {
        store_channels<N>(out, v, C, dg[q]);
        store_channels<N>(out + C, v, C, db[q]);
      }
    }
  }
}

// Adds `parts` partial rows of 2 C columns (dgamma, then dbeta): 16 lanes hold four
// columns each, 64 threads a column take the rows in turn, and their sums are added
// in two steps, all in a fixed order.
__global__ __launch_bounds__(1024) void column_sum_kernel(const float* __restrict__ col, int parts,
                                                          int C, int accumulate,
                                                          float* __restrict__ dgamma,
                                                          float* __restrict__ dbeta) {
  __shared__ f32x4 s[64][16];
  const int lane = threadIdx.x & 15, share = threadIdx.x >> 4;
  const int v = blockIdx.x * 16 + lane;
  float a[4] = {0.f, 0.f, 0.f, 0.f}, f[4];
  if (4 * v < 2 * C) {
#pragma unroll 8
    for (int p = share; p < parts; p += 64) {
      load_channels<4>(col + (int64_t)p * 2 * C, v, 2 * C, f);
#pragma unroll
      for (int e = 0; e < 4; ++e) a[e] += f[e];
    }
  }
  s[share][lane] = f32x4{a[0], a[1], a[2], a[3]};
  __syncthreads();
  if (share < 8) {
#pragma unroll
    for (int q = 1; q < 8; ++q)
#pragma unroll
      for (int e = 0; e < 4; ++e) a[e] += s[share + 8 * q][lane][e];
    s[share][lane] = f32x4{a[0], a[1], a[2], a[3]};  // read by no other until the barrier
  }
  __syncthreads();
  if (share != 0) return;
#pragma unroll
  for (int q = 1; q < 8; ++q)
#pragma unroll
    for (int e = 0; e < 4; ++e) a[e] += s[q][lane][e];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int at = 4 * v + e;
    float* out = at < C ? dgamma : dbeta;
    if (at >= 2 * C || out == nullptr) continue;
    out += at < C ? at : at - C;
    *out = accumulate ? *out + a[e] : a[e];
  }
}

// Calls f with the lanes of a row and the vectors a lane, as types, for rows of
// nvec vectors (up to 16,384 channels).  The lanes fit the row within a third: at
// 513 vectors (16,384 rows of 4,104 bf16) 256 lanes of three take 56 us forward and
// 90 backward, 512 of two 70 and 125.  A row in one wavefront needs no barrier,
// which the backward, with more registers a vector and fewer wavefronts, gains by
// up to 256 vectors (16,384 rows of 2,048: 46 us, 54 with 256 lanes), the forward up
// to 192 (of 2,048: 30, 27 with 256 lanes).  Short rows are bound by the steps that a
// group's lanes wait for: 200,000 rows of 64 bf16 take 10.6 and 20.4 us with 8 lanes,
// 14.9 and 24.5 with 16.
template <typename T, bool BACKWARD, typename F>
auto with_shape(int nvec, F&& f) {
  using std::integral_constant;
#define SHC_SHAPE(limit, g, v) \
  if (nvec <= limit) return f(integral_constant<int, g>{}, integral_constant<int, v>{})
  SHC_SHAPE(8, 8, 1);
  SHC_SHAPE(16, 16, 1);
  SHC_SHAPE(32, 32, 1);
  SHC_SHAPE(64, 64, 1);
  SHC_SHAPE(128, 64, 2);
  SHC_SHAPE(192, 64, 3);
  if constexpr (BACKWARD) {
    SHC_SHAPE(256, 64, 4);
  } else {
    SHC_SHAPE(256, 256, 1);
  }
  SHC_SHAPE(512, 256, 2);
  SHC_SHAPE(768, 256, 3);
  if constexpr (BACKWARD) {
    SHC_SHAPE(1024, 256, 4);
  } else {
    SHC_SHAPE(1024, 512, 2);
  }
  SHC_SHAPE(1536, 512, 3);
  if constexpr (sizeof(T) == 4) {
    SHC_SHAPE(2048, 1024, 2);
    return f(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
  } else {
    return f(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
  }
#undef SHC_SHAPE
}

template <typename T>
int vectors_of(int32_t C) {
  return (C + Row<T>::N - 1) / Row<T>::N;
}

// Workgroups of the row kernels, per_cu to a CU: enough to keep HBM busy, few
// enough that gamma is read once per many rows.
int norm_blocks(int64_t n, int G, int per_cu) {
  const int rows = G > 256 ? 1 : 256 / G;
  const int64_t need = (n + rows - 1) / rows;
  return (int)std::min<int64_t>(need, 256 * per_cu);
}
// Of the backward, whose workgroups write a partial row of column sums each: three to
// a CU for short rows (268,160 rows of 128 bf16: 45 us, 48 with two), two up to 256
// lanes (16,384 rows of 4,096: 80 us, 117 with one, 100 with four) and four rows or
// more each past one to a CU (700 rows of 8,192: 18.4 us, 22.2 without), and one for
// longer rows (1,110 rows of 9,280: 23.5 us, 32.4 with two; 12,000 of 16,384: 224, 242).
int backward_groups(int64_t n, int G) {
  if (G > 256) return norm_blocks(n, G, 1);
  const int blocks = norm_blocks(n, G, G <= 32 ? 3 : 2);
  return G < 256 ? blocks : (int)std::min<int64_t>(blocks, std::max<int64_t>(256, n / 4));
}

template <typename T>
int backward_blocks(int64_t n, int32_t C) {
  return with_shape<T, true>(vectors_of<T>(C), [&](auto g, auto) {
    return backward_groups(n, decltype(g)::value);
  });
}

template <typename T>
hipError_t norm(const void* x, int64_t ldx, int64_t n, int32_t C, const float* gamma,
                const float* beta, float eps, void* y, int64_t ldy, float* mean, float* rstd,
                hipStream_t stream) {
  return with_shape<T, false>(vectors_of<T>(C), [&](auto g, auto v) {
    constexpr int G = decltype(g)::value, NV = decltype(v)::value;
    layer_norm_kernel<T, G, NV><<<norm_blocks(n, G, 4), G > 256 ? G : 256, 0, stream>>>(
        static_cast<const T*>(x), ldx, n, C, gamma, beta, eps, static_cast<T*>(y), ldy, mean,
        rstd);
    return hipGetLastError();
  });
}

template <typename T>
hipError_t norm_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx, int64_t n,
                         int32_t C, const float* gamma, const float* mean, const float* rstd,
                         void* dx, int64_t lddx, float* col, hipStream_t stream) {
  return with_shape<T, true>(vectors_of<T>(C), [&](auto g, auto v) {
    constexpr int G = decltype(g)::value, NV = decltype(v)::value;
    layer_norm_backward_kernel<T, G, NV>
        <<<backward_groups(n, G), G > 256 ? G : 256, 0, stream>>>(
            static_cast<const T*>(dy), lddy, static_cast<const T*>(x), ldx, n, C, gamma, mean,
            rstd, static_cast<T*>(dx), lddx, col);
    return hipGetLastError();
  });
}

}  // namespace

size_t layer_norm_backward_workspace_bytes(int64_t n, int32_t C) {
  // the larger of the two dtypes' partial rows: the caller's dtype need not be known
  const int b = std::max(backward_blocks<float>(n, C), backward_blocks<uint16_t>(n, C));
  return (size_t)b * 2 * (size_t)C * sizeof(float);
}

hipError_t launch_layer_norm(const void* x, int64_t ldx, int64_t n, int32_t C, const float* gamma,
                             const float* beta, float eps, int is_bf16, void* y, int64_t ldy,
                             float* mean, float* rstd, hipStream_t stream) {
  return (is_bf16 ? norm<uint16_t> : norm<float>)(x, ldx, n, C, gamma, beta, eps, y, ldy, mean,
                                                  rstd, stream);
}

hipError_t launch_layer_norm_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx,
                                      int64_t n, int32_t C, const float* gamma, const float* mean,
                                      const float* rstd, int is_bf16, int accumulate, void* dx,
                                      int64_t lddx, float* dgamma, float* dbeta, void* ws,
                                      hipStream_t stream) {
  const bool want_cols = dgamma != nullptr || dbeta != nullptr;
  float* col = want_cols ? static_cast<float*>(ws) : nullptr;
  int blocks = 0;
  if (n > 0 && (want_cols || dx != nullptr)) {
    blocks = is_bf16 ? backward_blocks<uint16_t>(n, C) : backward_blocks<float>(n, C);
    const hipError_t e = (is_bf16 ? norm_backward<uint16_t> : norm_backward<float>)(
        dy, lddy, x, ldx, n, C, gamma, mean, rstd, dx, lddx, col, stream);
    if (e != hipSuccess) return e;
  }
  if (!want_cols || (n == 0 && accumulate)) return hipSuccess;
  column_sum_kernel<<<(2 * C + 63) / 64, 1024, 0, stream>>>(col, blocks, C, accumulate, dgamma,
                                                           dbeta);
  return hipGetLastError();
}

}  // namespace shc
