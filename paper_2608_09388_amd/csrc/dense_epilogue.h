// Activations of the dense layers, their slopes, and the store of a product's values.
#pragma once

#include <type_traits>

#include "dense.h"

namespace shc {
namespace dense {

__device__ __forceinline__ float exp_(float x) {  // e^x as 2^(x log2 e)
  return __builtin_amdgcn_exp2f(x * 1.44269504088896340736f);
}

// Phi(z), the normal distribution, and e^(-z^2 / 2), by Hastings' rational
// approximation (Abramowitz and Stegun 7.1.26): erfc(x) = (a1 t + ... + a5 t^5)
// e^(-x^2) with t = 1 / (1 + p x) for x = |z| / sqrt 2 >= 0, within 1.5e-7.
__device__ __forceinline__ float normal_cdf(float z, float* bell) {
  const float x = fabsf(z) * 0.70710678118654752440f;
  const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, x, 1.f));
  const float e = exp_(-x * x);
  const float p =
      t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f),
                       -0.284496736f), 0.254829592f);
  *bell = e;
  const float tail = 0.5f * p * e;
  return z < 0.f ? tail : 1.f - tail;
}

__device__ __forceinline__ float act_of(int act, float z) {
  if (act == kActRelu) return z < 0.f ? 0.f : z;  // a NaN stays one
  if (act == kActGelu) {
    float bell;
    return z * normal_cdf(z, &bell);
  }
  if (act == kActSilu) return z / (1.f + exp_(-z));
  return z;
}

__device__ __forceinline__ float slope_of(int act, float z) {
  if (act == kActRelu) return z <= 0.f ? 0.f : 1.f;  // of a NaN 1, so that dout's is kept
  if (act == kActGelu) {
    float bell;
    const float cdf = normal_cdf(z, &bell);
    return fmaf(z * bell, 0.39894228040143267794f, cdf);
  }
  if (act == kActSilu) {
    const float s = 1.f / (1.f + exp_(-z));
    return s * fmaf(z, 1.f - s, 1.f);
  }
  return 1.f;
}

// 8 values of a row of N, from column 8 v on (v < ceil(N / 8)).
template <bool BF16>
__device__ __forceinline__ void load8(const void* base, int64_t row, int64_t ld, int v, int N,
                                      float* f) {
  using namespace rowops;
  if constexpr (BF16) {
    Row<uint16_t>::widen(load_vec<uint16_t>(static_cast<const uint16_t*>(base) + row * ld, v, N),
                         f);
  } else {
    load_channels<8>(static_cast<const float*>(base) + row * ld, v, N, f);
  }
}
template <bool BF16>
__device__ __forceinline__ void put8(void* base, int64_t row, int64_t ld, int v, int N,
                                     const float* f) {
  using namespace rowops;
  if constexpr (BF16)
    store_vec<uint16_t>(static_cast<uint16_t*>(base) + row * ld, v, N, Row<uint16_t>::narrow(f));
  else
    store_channels<8>(static_cast<float*>(base) + row * ld, v, N, f);
}

// What a store of 8 values of a row needs from memory, loaded ahead of it.
template <bool BF16>
struct Fetched {
  typedef typename std::conditional<BF16, i32x4, float[8]>::type Raw;
  Raw res;
  int64_t to;
};
template <bool BF16>
__device__ __forceinline__ Fetched<BF16> fetch8(const Store& s, int64_t row, int v, int N) {
  Fetched<BF16> g;
  g.to = s.to != nullptr ? (int64_t)s.to[row] : row;
  if (s.res != nullptr) {
    if constexpr (BF16)
      g.res = rowops::load_vec<uint16_t>(
          static_cast<const uint16_t*>(s.res) + g.to * s.ld_res, v, N);
    else
      rowops::load_channels<8>(static_cast<const float*>(s.res) + g.to * s.ld_res, v, N, g.res);
  }
  return g;
}
__device__ __forceinline__ float scale_of(const Store& s) {
  return s.scale != nullptr ? *s.scale : 1.f;
}
__device__ __forceinline__ void bias8(const Store& s, int v, int N, float (&b)[8]) {
  if (s.bias != nullptr) rowops::load_channels<8>(s.bias, v, N, b);
}

template <bool BF16>
__device__ __forceinline__ void store8(const Store& s, int64_t row, int v, int N,
                                       const float (&values)[8], float scale,
                                       const float (&bias)[8], const Fetched<BF16>& g) {
  float f[8], x[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = values[e];
  if (s.add32 != nullptr) {
    rowops::load_channels<8>(s.add32 + row * N, v, N, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] += x[e];
  }
  if (s.out32 != nullptr) {
    rowops::store_channels<8>(s.out32 + row * N, v, N, f);
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] *= scale;
  if (s.bias != nullptr) {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] += bias[e];
  }
  if (s.pre != nullptr) put8<BF16>(s.pre, row, s.ld_pre, v, N, f);
  if (s.act != kActNone) {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = act_of(s.act, f[e]);
  }
  if (s.res != nullptr) {
    if constexpr (BF16) {
      rowops::Row<uint16_t>::widen(g.res, x);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = g.res[e];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] += x[e];
  }
  put8<BF16>(s.out, g.to, s.ld_out, v, N, f);
}

}  // namespace dense
}  // namespace shc
