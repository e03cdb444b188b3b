// Device helpers of the row operators (embed.hip, layer_norm.hip, distill.hip):
// rows of C elements read and written as 16-byte vectors at any alignment of
// the element, and reductions over the G lanes that share a row.
#pragma once

#include "shc_internal.h"

namespace shc {
namespace rowops {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
// A 16-byte vector at an address aligned to the element only: rows of a stride
// or width that is no multiple of 16 bytes start anywhere.  One load or store
// instruction all the same (global memory takes unaligned vectors).
typedef int i32x4_a2 __attribute__((ext_vector_type(4), aligned(2)));
typedef int int_a2 __attribute__((aligned(2)));  // a pair of bf16
typedef int i32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));
typedef float f32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));

template <typename T>
struct Row;
template <>
struct Row<float> {
  static constexpr int N = 4;  // elements of a vector
  typedef i32x4_a4 mem;
  static __device__ __forceinline__ void widen(const i32x4& v, float* f) {
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = __int_as_float(v[e]);
  }
  static __device__ __forceinline__ i32x4 narrow(const float* f) {
    return i32x4{__float_as_int(f[0]), __float_as_int(f[1]), __float_as_int(f[2]),
                 __float_as_int(f[3])};
  }
  static __device__ __forceinline__ float get(const float* p) { return *p; }
  static __device__ __forceinline__ void put(float* p, float f) { *p = f; }
};
template <>
struct Row<uint16_t> {  // bf16
  static constexpr int N = 8;
  typedef i32x4_a2 mem;
  static __device__ __forceinline__ void widen(const i32x4& v, float* f) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {  // exact: the bits move up
      f[2 * e] = __int_as_float(v[e] << 16);
      f[2 * e + 1] = __int_as_float(v[e] & (int)0xFFFF0000);
    }
  }
  static __device__ __forceinline__ i32x4 narrow(const float* f) {
    i32x4 out;
#pragma unroll
    for (int e = 0; e < 4; ++e) {  // hardware conversion, nearest even
      const bf16x2 h = __builtin_convertvector(f32x2{f[2 * e], f[2 * e + 1]}, bf16x2);
      out[e] = __builtin_bit_cast(int, h);
    }
    return out;
  }
  static __device__ __forceinline__ float get(const uint16_t* p) {
    return bf16_bits_to_f32(*p);
  }
  static __device__ __forceinline__ void put(uint16_t* p, float f) {
    *p = (uint16_t)f32_to_bf16_bits(f);
  }
};

// Vector v (elements [v * N, v * N + N)) of a row of C elements; elements past
// the row's end are `fill` and not read.
template <typename T>
__device__ __forceinline__ i32x4 load_vec(const T* row, int v, int C, uint32_t fill = 0) {
  constexpr int N = Row<T>::N;
  const T* p = row + (int64_t)v * N;
  const int left = C - v * N;
  if (left >= N) return *reinterpret_cast<const typename Row<T>::mem*>(p);
  i32x4 out;
  if constexpr (N == 4) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      out[e] = e < left ? reinterpret_cast<const int*>(p)[e] : (int)fill;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      out[e] = (int)(fill | (fill << 16));
      if (2 * e + 1 < left)
        out[e] = *reinterpret_cast<const int_a2*>(p + 2 * e);
      else if (2 * e < left)
        out[e] = (int)(p[2 * e] | (fill << 16));
    }
  }
  return out;
}

// NT: a non-temporal store, for rows that nothing reads soon.
template <typename T, bool NT = false>
__device__ __forceinline__ void store_vec(T* row, int v, int C, const i32x4& x) {
  constexpr int N = Row<T>::N;
  typedef typename Row<T>::mem mem;
  T* p = row + (int64_t)v * N;
  const int left = C - v * N;
  if (left >= N) {
    if constexpr (NT)
      __builtin_nontemporal_store((mem)x, reinterpret_cast<mem*>(p));
    else
      *reinterpret_cast<mem*>(p) = x;
    return;
  }
  if constexpr (N == 4) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < left) reinterpret_cast<int*>(p)[e] = x[e];
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (2 * e + 1 < left)
        *reinterpret_cast<int_a2*>(p + 2 * e) = x[e];
      else if (2 * e < left)
        p[2 * e] = (uint16_t)(x[e] & 0xFFFF);
    }
  }
}

// N fp32 values of a per-channel array of C from channel v * N on; 0 past its end.
template <int N>
__device__ __forceinline__ void load_channels(const float* a, int v, int C, float* f) {
  const int left = C - v * N;
  if (left >= N) {
#pragma unroll
    for (int q = 0; q < N / 4; ++q) {
      const f32x4_a4 x = *reinterpret_cast<const f32x4_a4*>(a + (int64_t)v * N + 4 * q);
#pragma unroll
      for (int e = 0; e < 4; ++e) f[4 * q + e] = x[e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) f[e] = e < left ? a[(int64_t)v * N + e] : 0.f;
  }
}
template <int N, bool NT = false>
__device__ __forceinline__ void store_channels(float* a, int v, int C, const float* f) {
  const int left = C - v * N;
  if (left >= N) {
#pragma unroll
    for (int q = 0; q < N / 4; ++q) {
      f32x4_a4* to = reinterpret_cast<f32x4_a4*>(a + (int64_t)v * N + 4 * q);
      const f32x4_a4 x = {f[4 * q], f[4 * q + 1], f[4 * q + 2], f[4 * q + 3]};
      if constexpr (NT)
        __builtin_nontemporal_store(x, to);
      else
        *to = x;
    }
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e < left) a[(int64_t)v * N + e] = f[e];
  }
}

// Reductions over aligned groups of G lanes, 8 <= G <= 64: quads and the two
// mirrors within 16 lanes by DPP, rows 16 apart and halves 32 apart by the
// permlane swaps.  All VALU; every lane ends with the result.
template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xF, 0xF, false));
}
template <int G, typename Op>
__device__ __forceinline__ float lanes_reduce(float x, Op op) {
  static_assert(G == 8 || G == 16 || G == 32 || G == 64, "lanes that share a row");
  x = op(x, dpp<0xB1>(x));    // quad_perm [1, 0, 3, 2]
  x = op(x, dpp<0x4E>(x));    // quad_perm [2, 3, 0, 1]
  x = op(x, dpp<0x141>(x));   // row_half_mirror
  if constexpr (G >= 16) x = op(x, dpp<0x140>(x));  // row_mirror
  if constexpr (G >= 32) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                    false);
    x = op(__uint_as_float(a[0]), __uint_as_float(a[1]));
  }
  if constexpr (G >= 64) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                    false);
    x = op(__uint_as_float(a[0]), __uint_as_float(a[1]));
  }
  return x;
}
// Sum over the lanes of a wavefront that have the same place in their groups of G.
template <int G>
__device__ __forceinline__ float groups_sum(float x) {
  if constexpr (G <= 8) x += dpp<0x128>(x);  // row_ror 8
  if constexpr (G <= 16) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                    false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  }
  if constexpr (G <= 32) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                    false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  }
  return x;
}
struct AddOp {
  __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};
struct MaxOp {  // a NaN loses to a number
  __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};

// The same over the G threads that share a row, G a wavefront's part or a
// whole workgroup of G threads (then through `part`, G / 64 floats of LDS that
// no other use touches; two barriers).
template <int G, typename Op>
__device__ __forceinline__ float group_reduce(float x, Op op, float* part) {
  if constexpr (G <= 64) {
    return lanes_reduce<G>(x, op);
  } else {
    x = lanes_reduce<64>(x, op);
    __syncthreads();  // the last reduction's reads of `part` are over
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    x = part[0];
#pragma unroll
    for (int w = 1; w < G / 64; ++w) x = op(x, part[w]);
    return x;
  }
}

// Makes a group's earlier global stores precede its later ones to the same
// address: a barrier of the workgroup, or of the wavefront where it holds the
// whole group (its memory instructions issue in order).
template <int G>
__device__ __forceinline__ void group_fence() {
  if constexpr (G <= 64) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  } else {
    __syncthreads();
  }
}

}  // namespace rowops
}  // namespace shc
