// Distillation of a row of logits z [V] from a teacher's k top logits
// (id_j, t_j), at temperature T:
//
//   p = softmax(t / T) over the row's entries,  q = softmax(z / T) over V
//   loss = T^2 sum_j p_j (log p_j - log q_{id_j})
//   dz_v = w T (q_v - sum of p_j with id_j = v)
//
// Exponentials and logarithms are in base 2: with c = log2(e) / T, m = max z
// and S = sum 2^((z - m) c), q = 2^((z - m) c - log2 S).  The difference is
// taken before the factor, so masks of the type's lowest value stay finite.
// A logit of -inf has q = 0, also in a row that has no other; a row without
// entries has loss 0 and gradient 0 whatever its logits are (they are read: the
// loads do not wait for the entries).
//
// Bound by HBM: V elements read, and V written by the gradient.
// - Rows of up to 4096 vectors are read once, into the registers of the G threads
//   that share them: maximum, sum, loss and gradient from there.  So are, by the step,
//   many fp32 rows of 7,169 to 16,384 vectors (run_rows).
// - A workgroup of 1024 threads reads a longer row twice, the second time from
//   the caches (256 rows in flight fit the Infinity Cache).
// - Long rows of which there are few are cut into parts: a first launch leaves
//   every part's maximum and sum in the workspace, the second joins them in order
//   and computes the loss or its part of the gradient.
// The backward takes q from the saved log-sum-exp, or sums the row again where 32 bits of
// it do not keep the sum (keeps_sum).
// The gradient writes w T q first; the k entries are corrected behind a fence,
// entries of the same id all with the id's whole p, added in their order.
//
// Measured, bf16: step, 4,096 rows of 131,072 with 64 entries: 453 us, 4.7 TB/s;
// gradient, 268,160 rows of 128 with 8: 34.6 us, 4.5 TB/s; loss, 16 rows of 131,072:
// 7.6 us, two launches.
#include <algorithm>

#include "row_ops.h"

namespace shc {
namespace {

using namespace rowops;

constexpr float kLog2E = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_hw(float x) { return __builtin_amdgcn_logf(x); }

template <typename T>
__device__ __forceinline__ uint32_t minus_inf_bits() {
  return sizeof(T) == 2 ? 0xFF80u : 0xFF800000u;
}
// a vector of a row of V logits; -inf past its end
template <typename T>
__device__ __forceinline__ i32x4 load_logits(const T* z, int v, int V) {
  if ((int64_t)v * Row<T>::N < V) return load_vec(z, v, V, minus_inf_bits<T>());
  const int b = sizeof(T) == 2 ? (int)0xFF80FF80u : (int)0xFF800000u;
  return i32x4{b, b, b, b};
}

// Maximum and sum of a row: q_v = 2^((z_v - m) c - l).  m is not -inf, so that a
// logit of -inf has q = 0, and q = NaN in a row with a NaN.
struct RowSoftmax {
  float m, l;
};
__device__ __forceinline__ float finite_max(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ float prob(float z, const RowSoftmax& r, float c) {
  return exp2_hw((z - r.m) * c - r.l);
}

// The teacher's entries of a row, in LDS: id (-1 where there is none), its own p,
// the p of all the row's entries with that id, and the logit there.  Behind them,
// for the gradient of rows of more than kPairs entries, a bit for each of the
// `range` ids that it covers (modulo kMapBits): ids that are all different, the
// usual case, are told by one pass over the entries, and only a row where a bit
// was met twice compares every two entries.  30,000 rows of 1,000 bf16, step: 72 us
// with 256 entries, 176 when all rows compare them; with up to 16 the two are
// within 0.5 us of each other.
constexpr int kPairs = 16;
constexpr int kMapBits = 131072;
__host__ __device__ constexpr int entry_slots(int k) { return (k + 3) & ~3; }
__host__ __device__ constexpr int map_words(int k, int range) {
  return k <= kPairs ? 0 : ((range < kMapBits ? range : kMapBits) + 127) / 128 * 4;
}
__host__ __device__ constexpr int entry_words(int k, int range) {
  return 4 * entry_slots(k) + map_words(k, range);
}
struct Entries {
  int* id;
  float *p, *all, *z;
  uint32_t* map;
  __device__ __forceinline__ Entries(int* lds, int k)
      : id(lds), p(reinterpret_cast<float*>(lds) + entry_slots(k)), all(p + entry_slots(k)),
        z(all + entry_slots(k)),
        map(reinterpret_cast<uint32_t*>(lds) + 4 * entry_slots(k)) {}
};

// Fills them, by L lanes of one wavefront; whether the row has any.  `all` is that
// of the ids in [lo, lo + range).  All of it,
// the logits' gather and the comparison of the ids too, is done before the
// row's maximum is needed, beside the loads of the row.
template <typename T, int L, bool GRAD>
__device__ __forceinline__ bool teach(const T* __restrict__ z, const int32_t* __restrict__ ids,
                                      const float* __restrict__ top, int k, int V, float c,
                                      int lane, const Entries& en, int lo, int range) {
  constexpr int U = 4;  // entries of a lane in flight
  float tm = -INFINITY, any = 0.f;
  for (int e0 = lane; e0 < k; e0 += U * L) {
    int id[U];
    float t[U], at[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int e = e0 + u * L;
      id[u] = e < k ? ids[e] : -1;
      t[u] = e < k ? top[e] : 0.f;
      if (id[u] >= V || t[u] == -INFINITY) id[u] = -1;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) at[u] = id[u] >= 0 ? Row<T>::get(z + id[u]) : 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int e = e0 + u * L;
      if (e >= k) break;
      en.id[e] = max(id[u], -1);
      en.p[e] = t[u];
      en.z[e] = at[u];
      if (id[u] >= 0) {
        tm = fmaxf(tm, t[u]);
        any = 1.f;
      }
    }
  }
  tm = finite_max(lanes_reduce<L>(tm, MaxOp{}));
  if (lanes_reduce<L>(any, MaxOp{}) == 0.f) return false;
  const int words = GRAD ? map_words(k, range) : 0;
  for (int i = 4 * lane; i < words; i += 4 * L)
    *reinterpret_cast<i32x4*>(en.map + i) = i32x4{};
  float s = 0.f;
  for (int e = lane; e < k; e += L) {
    const float x = en.id[e] >= 0 ? exp2_hw((en.p[e] - tm) * c) : 0.f;
    en.p[e] = x;
    s += x;
  }
  s = lanes_reduce<L>(s, AddOp{});
  if (GRAD) group_fence<64>();
  bool twice = false;
  for (int e = lane; e < k; e += L) {
    const float p = en.p[e] / s;
    en.p[e] = p;
    if (GRAD && words > 0) {
      const unsigned at = (unsigned)(en.id[e] - lo);
      en.all[e] = p;
      if (at < (unsigned)range) {
        const uint32_t bit = 1u << (at & 31);
        twice |= atomicOr(en.map + ((at & (kMapBits - 1)) >> 5), bit) & bit;
      }
    }
  }
  if constexpr (GRAD) {
    if (words > 0 && lanes_reduce<L>(twice ? 1.f : 0.f, MaxOp{}) == 0.f) return true;
    const int slots = entry_slots(k);
    if (lane < slots - k) {  // the last four are whole: no id of the row's
      en.id[k + lane] = -2;
      en.p[k + lane] = 0.f;
    }
    group_fence<64>();
    for (int e = lane; e < k; e += L) {
      const int id = en.id[e];
      if ((unsigned)(id - lo) >= (unsigned)range) continue;
      float p = 0.f;
#pragma unroll 4
      for (int o = 0; o < slots; o += 4) {
        const i32x4 ids4 = *reinterpret_cast<const i32x4*>(en.id + o);
        const f32x4 p4 = *reinterpret_cast<const f32x4*>(en.p + o);
#pragma unroll
        for (int q = 0; q < 4; ++q) p += ids4[q] == id ? p4[q] : 0.f;
      }
      en.all[e] = p;
    }
  }
  return true;
}

// sum_j p_j (log p_j - log q_j) over the row's entries, in natural units: an
// entry on a logit of the type's lowest value stays finite.  By the lanes that
// filled them.
template <int L>
__device__ __forceinline__ float loss_terms(int k, float temp, const RowSoftmax& r, int lane,
                                            const Entries& en) {
  float a = 0.f;
  for (int e = lane; e < k; e += L) {
    const float p = en.p[e];
    if (en.id[e] < 0 || p == 0.f) continue;
    const float zi = en.z[e];
    // (l is -inf in a row of nothing but -inf, NaN in one with a NaN)
    const bool none = zi == -INFINITY && r.l == r.l;
    const float lq = none ? -INFINITY : (zi - r.m) / temp - kLn2 * r.l;
    // (the hardware's logarithm takes a subnormal p as 0)
    a += p * (kLn2 * log2_hw(fmaxf(p, 0x1p-126f)) - lq);
  }
  return lanes_reduce<L>(a, AddOp{});
}

// The entries with ids in [lo, hi) of the gradient, behind the row's q, by the
// lanes that filled them.
template <typename T, int L>
__device__ __forceinline__ void fix_entries(T* dz, int k, float c, float wt, const RowSoftmax& r,
                                            int lane, int lo, int hi, const Entries& en) {
  for (int e = lane; e < k; e += L) {
    const int id = en.id[e];
    if (id >= lo && id < hi) Row<T>::put(dz + id, wt * (prob(en.z[e], r, c) - en.all[e]));
  }
}

// Largest logit among vectors of a row.  bf16 pairs are compared as 16-bit
// integers, two to an instruction and without widening: among patterns with a
// positive one the signed maximum is the largest value, among negative ones the
// unsigned minimum is.
template <typename T>
struct VecMax;
template <>
struct VecMax<float> {
  float m = -INFINITY;
  __device__ __forceinline__ void take(const i32x4& v) {
#pragma unroll
    for (int e = 0; e < 4; ++e) m = fmaxf(m, __int_as_float(v[e]));
  }
  __device__ __forceinline__ float value() const { return m; }
};
template <>
struct VecMax<uint16_t> {
  typedef short s16x2 __attribute__((ext_vector_type(2)));
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  s16x2 hi = {(short)0xFF80, (short)0xFF80};                    // -inf
  u16x2 lo = {(unsigned short)0xFF80, (unsigned short)0xFF80};  // -inf
  __device__ __forceinline__ void take(const i32x4& v) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int pair = v[e];  // a bit cast of the element itself reads element 0
      hi = __builtin_elementwise_max(hi, __builtin_bit_cast(s16x2, pair));
      lo = __builtin_elementwise_min(lo, __builtin_bit_cast(u16x2, pair));
    }
  }
  __device__ __forceinline__ float value() const {
    const short h = hi[0] > hi[1] ? hi[0] : hi[1];
    const unsigned short l = lo[0] < lo[1] ? lo[0] : lo[1];
    return bf16_bits_to_f32(h >= 0 ? (uint16_t)h : l);
  }
};

// A row's exponents as one operation: x = z c - mc, mc = m c rounded.  Any
// constant in its place gives the same q, so its rounding costs nothing as long
// as 2^x stays in range: the rounding of mc below 2^20 moves x by less than 1/8.
// Larger ones (logits of 10^5 and more) take (z - m) c.
constexpr float kFar = 1048576.f;
struct Exponent {
  float c, mc, m;
  bool near;
  __device__ __forceinline__ Exponent(float m_, float c_) : c(c_), mc(m_ * c_), m(m_) {
    near = fabsf(mc) < kFar;
  }
  // log2 of sum 2^((z - m) c) from the sum of 2^x
  __device__ __forceinline__ float log_sum(float s) const {
    return near ? log2_hw(s) - fmaf(m, c, -mc) : log2_hw(s);
  }
};
template <typename T, bool NEAR>
__device__ __forceinline__ float exp_sum(const i32x4& v, const Exponent& x, float s) {
  constexpr int N = Row<T>::N;
  float f[N];
  Row<T>::widen(v, f);
#pragma unroll
  for (int e = 0; e < N; ++e)
    s += exp2_hw(NEAR ? fmaf(f[e], x.c, -x.mc) : (f[e] - x.m) * x.c);
  return s;
}
template <typename T, bool NEAR>
__device__ __forceinline__ i32x4 exp_scaled(const i32x4& v, const Exponent& x, float by) {
  constexpr int N = Row<T>::N;
  float f[N];
  Row<T>::widen(v, f);
#pragma unroll
  for (int e = 0; e < N; ++e)
    f[e] = by * exp2_hw(NEAR ? fmaf(f[e], x.c, -x.mc) : (f[e] - x.m) * x.c);
  return Row<T>::narrow(f);
}

// A thread's running maximum and sum over vectors that it does not keep: the sum
// is of 2^(z c - mc) with mc the maximum's z c, or -kFar where that is lower (no
// logit yet, or masks of the lowest value: next to a row's maximum above it they
// add nothing, and a row whose maximum is that far from 0 is summed again).
template <typename T>
struct RunningSum {
  float m = -INFINITY, mc = -kFar, s = 0.f;
  template <int U>
  __device__ __forceinline__ void take(const i32x4 (&v)[U], float c) {
    VecMax<T> vm;
#pragma unroll
    for (int u = 0; u < U; ++u) vm.take(v[u]);
    m = fmaxf(m, vm.value());
    over(fmaxf(m * c, mc));
    Exponent x(0.f, c);
    x.mc = mc;
#pragma unroll
    for (int u = 0; u < U; ++u) s = exp_sum<T, true>(v[u], x, s);
  }
  __device__ __forceinline__ void over(float to) {  // mc = to >= mc
    s *= exp2_hw(mc - to);
    mc = to;
  }
};

// Maximum and sum of 2^((z - m) c) over vectors [v0, v1) of a row, by the G threads that
// share it, U vectors a thread in flight; part: as of group_reduce.
template <typename T, int G, int U>
__device__ __forceinline__ float max_and_sum(const T* __restrict__ z, int V, int v0, int v1,
                                             int lane, float c, float* part, float* sum) {
  const int nvec = (V + Row<T>::N - 1) / Row<T>::N;
  RunningSum<T> run;
  for (int v = v0 + lane; v < v1; v += G * U) {
    i32x4 in[U];
#pragma unroll
    for (int u = 0; u < U; ++u) in[u] = load_logits(z, v + G * u < v1 ? v + G * u : nvec, V);
    run.take(in, c);
  }
  const float m = group_reduce<G>(run.m, MaxOp{}, part);
  const Exponent x(finite_max(m), c);
  float s = 0.f;
  if (x.near) {
    run.over(x.mc);
    s = run.s;
  } else {
    for (int v = v0 + lane; v < v1; v += G) s = exp_sum<T, false>(load_logits(z, v, V), x, s);
  }
  s = group_reduce<G>(s, AddOp{}, part);
  *sum = x.near ? s * exp2_hw(-fmaf(x.m, c, -x.mc)) : s;
  return m;
}

// Whether the backward takes a row's q from its lse, which is m / T + ln S in fp32: the
// rounding of the sum, of its two terms and of its product with T move every q by up to
// 4 |lse| 2^-24, which is 2^-16 at 64, as much as the row's sum may be off, and 2^-12 at
// 1,024, an eighth of bf16's own rounding.  Farther from 0 lse says less and less of S (of
// a row of masks of the lowest value nothing), and the row's maximum and sum are taken again.
template <typename T>
__device__ __forceinline__ bool keeps_sum(float lse) {
  return !(fabsf(lse) > (sizeof(T) == 2 ? 1024.f : 64.f));
}

// What the threads that share a row tell each other; one barrier a value.
template <int G>
struct GroupShare {
  float m[G / 64], s[G / 64];
  int live;
};
template <>
struct GroupShare<8> {};
template <>
struct GroupShare<16> {};
template <>
struct GroupShare<32> {};
template <>
struct GroupShare<64> {};

enum class Pass { kForward, kBackward, kStep };

// A row of logits by the G threads of a wavefront's part, a wavefront or the
// workgroup.  NV > 0: the row is held in registers, NV vectors a thread, and read
// once.  NV = 0: it is read twice, the second time from the caches, where the
// stores of the gradient pass by them (non-temporal).
template <typename T, int G, int NV, Pass PASS>
__global__ __launch_bounds__(G > 256 ? G : 256) void distill_row_kernel(
    const T* __restrict__ z, int64_t ldz, int64_t n, int V, const int32_t* __restrict__ ids,
    const float* __restrict__ top, int k, float temp, const float* __restrict__ weight,
    float* __restrict__ loss, float* __restrict__ lse, T* __restrict__ dz, int64_t lddz) {
  constexpr int N = Row<T>::N, BLOCK = G > 256 ? G : 256, R = BLOCK / G;
  constexpr int L = G < 64 ? G : 64;  // the lanes that take the teacher's entries
  constexpr int U = 4;                // vectors in flight of a row read twice
  extern __shared__ __align__(16) int smem[];       // the groups' entries
  __shared__ GroupShare<G> sh;
  const int lane = threadIdx.x % G, group = threadIdx.x / G;
  const Entries en(
      smem + group * (PASS == Pass::kForward ? entry_words(k, 0) : entry_words(k, V)), k);
  const int64_t row = (int64_t)blockIdx.x * R + group;
  if (row >= n) return;  // whole groups
  const float c = kLog2E / temp;
  const T* zr = z + row * ldz;
  T* dr = PASS == Pass::kForward ? nullptr : dz + row * lddz;
  const int nvec = (V + N - 1) / N;

  i32x4 raw[NV > 0 ? NV : 1];
#pragma unroll
  for (int q = 0; q < NV; ++q) raw[q] = load_logits(zr, q * G + lane, V);
  const float w = PASS != Pass::kForward && weight != nullptr ? weight[row] : 1.f;
  const float saved = PASS == Pass::kBackward ? lse[row] : 0.f;
  bool live = false;
  if (lane < L)
    live = teach<T, L, PASS != Pass::kForward>(zr, ids + row * k, top + row * k, k, V, c, lane,
                                               en, 0, V);

  // maximum; a row read twice has its sum over the running maximum too
  float m = -INFINITY, s = 0.f;
  RunningSum<T> run;
  if constexpr (PASS != Pass::kBackward) {
    if constexpr (NV > 0) {
      VecMax<T> vm;
#pragma unroll
      for (int q = 0; q < NV; ++q) vm.take(raw[q]);
      m = vm.value();
    } else {
      for (int v = lane; v < nvec; v += G * U) {
        i32x4 in[U];
#pragma unroll
        for (int u = 0; u < U; ++u) in[u] = load_logits(zr, v + G * u, V);
        run.take(in, c);
      }
      m = run.m;
    }
  }
  float all = lanes_reduce<L>(m, MaxOp{});
  if constexpr (G > 64) {
    if ((threadIdx.x & 63) == 0) sh.m[threadIdx.x >> 6] = all;
    if (threadIdx.x == 0) sh.live = live;
    __syncthreads();
    live = sh.live;
    all = sh.m[0];
#pragma unroll
    for (int i = 1; i < G / 64; ++i) all = fmaxf(all, sh.m[i]);
  }
  if (!live) {
    if (lane == 0) {
      if (PASS != Pass::kBackward) loss[row] = 0.f;
      if (PASS == Pass::kForward && lse != nullptr) lse[row] = 0.f;
    }
    if constexpr (PASS != Pass::kForward)
      for (int v = lane; v < nvec; v += G) store_vec(dr, v, V, i32x4{});
    return;  // the whole group
  }

  // sum
  RowSoftmax r;
  if constexpr (PASS == Pass::kBackward) {
    if (keeps_sum<T>(saved)) {  // z/T - lse: the saved lse takes the place of the maximum
      r.m = saved * temp;
      r.l = 0.f;
      s = 1.f;
    } else {
      float* part = nullptr;
      if constexpr (G > 64) part = sh.s;
      r.m = finite_max(max_and_sum<T, G, 1>(zr, V, 0, nvec, lane, c, part, &s));
      r.l = log2_hw(s);
    }
  } else {
    r.m = finite_max(all);
  }
  const Exponent x(r.m, c);
  if constexpr (PASS != Pass::kBackward) {
    if (!x.near) {
      for (int v = lane; v < nvec; v += G) s = exp_sum<T, false>(load_logits(zr, v, V), x, s);
    } else if constexpr (NV > 0) {
#pragma unroll
      for (int q = 0; q < NV; ++q) s = exp_sum<T, true>(raw[q], x, s);
    } else {
      run.over(x.mc);
      s = run.s;
    }
    s = lanes_reduce<L>(s, AddOp{});
    if constexpr (G > 64) {
      if ((threadIdx.x & 63) == 0) sh.s[threadIdx.x >> 6] = s;
      __syncthreads();
      s = sh.s[0];
#pragma unroll
      for (int i = 1; i < G / 64; ++i) s += sh.s[i];
    }
    r.l = x.log_sum(s);
    if (lane < L) {
      const float a = loss_terms<L>(k, temp, r, lane, en);
      if (lane == 0) {
        loss[row] = temp * (temp * a);
        if (PASS == Pass::kForward && lse != nullptr) lse[row] = r.m / temp + kLn2 * r.l;
      }
    }
  } else if (x.near) {
    s *= exp2_hw(fmaf(r.m, c, -x.mc));
  }

  if constexpr (PASS != Pass::kForward) {
    const float wt = w * temp;
    if (s == 0.f) r.l = 0.f;  // no logit but -inf: every q is 0
    const float by = s == 0.f ? 0.f : wt / s;
    if (!x.near) {
      for (int v = lane; v < nvec; v += G)
        store_vec(dr, v, V, exp_scaled<T, false>(load_logits(zr, v, V), x, by));
    } else if constexpr (NV > 0) {
#pragma unroll
      for (int q = 0; q < NV; ++q) {
        const int v = q * G + lane;
        if (v < nvec) store_vec(dr, v, V, exp_scaled<T, true>(raw[q], x, by));
      }
    } else {
      for (int v = lane; v < nvec; v += G * U) {
        i32x4 in[U];
#pragma unroll
        for (int u = 0; u < U; ++u) in[u] = load_logits(zr, v + G * u, V);
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (v + G * u < nvec)
            store_vec<T, true>(dr, v + G * u, V, exp_scaled<T, true>(in[u], x, by));
      }
    }
    group_fence<G>();
    if (lane < L) fix_entries<T, L>(dr, k, c, wt, r, lane, 0, V, en);
  }
}

// Maximum and sum of part blockIdx.y (per vectors) of row blockIdx.x.
template <typename T>
__global__ __launch_bounds__(256) void distill_part_kernel(const T* __restrict__ z, int64_t ldz,
                                                           int V, int per, float temp,
                                                           f32x2* __restrict__ parts) {
  __shared__ float part[4];
  const int nvec = (V + Row<T>::N - 1) / Row<T>::N;
  const int v0 = blockIdx.y * per, v1 = min(v0 + per, nvec);
  float s;
  const float m = max_and_sum<T, 256, 4>(z + (int64_t)blockIdx.x * ldz, V, v0, v1, threadIdx.x,
                                         kLog2E / temp, part, &s);
  if (threadIdx.x == 0) parts[(int64_t)blockIdx.x * gridDim.y + blockIdx.y] = f32x2{m, s};
}

// A row's parts joined, by the lanes of a wavefront (every wavefront of the
// workgroup alike); *sum = sum 2^((z - m) c).
__device__ __forceinline__ RowSoftmax join_parts(const f32x2* __restrict__ parts, int count,
                                                 float c, float* sum) {
  const int lane = threadIdx.x & 63;
  const f32x2 first = lane < count ? parts[lane] : f32x2{-INFINITY, 0.f};
  float m = first[0];
  for (int i = lane + 64; i < count; i += 64) m = fmaxf(m, parts[i][0]);
  RowSoftmax r;
  r.m = finite_max(lanes_reduce<64>(m, MaxOp{}));
  // a part of nothing but -inf has the sum 0, and no maximum; one of NaN has none
  // either, but a sum of NaN, which stays
  auto part = [&](const f32x2& p) {
    return p[1] == 0.f ? 0.f : p[1] * exp2_hw((p[0] - r.m) * c);
  };
  float s = part(first);
  for (int i = lane + 64; i < count; i += 64) s += part(parts[i]);
  *sum = lanes_reduce<64>(s, AddOp{});
  r.l = log2_hw(*sum);
  return r;
}

// Loss (and lse) of rows from their parts, a wavefront each.
template <typename T>
__global__ __launch_bounds__(64) void distill_join_kernel(
    const T* __restrict__ z, int64_t ldz, int V, const f32x2* __restrict__ parts, int count,
    const int32_t* __restrict__ ids, const float* __restrict__ top, int k, float temp,
    float* __restrict__ loss, float* __restrict__ lse) {
  extern __shared__ __align__(16) int smem[];
  const Entries en(smem, k);
  const int64_t row = blockIdx.x;
  const int lane = threadIdx.x;
  const float c = kLog2E / temp;
  const bool live =
      teach<T, 64, false>(z + row * ldz, ids + row * k, top + row * k, k, V, c, lane, en, 0, 0);
  if (!live) {
    if (lane == 0) {
      loss[row] = 0.f;
      if (lse != nullptr) lse[row] = 0.f;
    }
    return;
  }
  float s;
  const RowSoftmax r = join_parts(parts + row * count, count, c, &s);
  const float a = loss_terms<64>(k, temp, r, lane, en);
  if (lane == 0) {
    loss[row] = temp * (temp * a);
    if (lse != nullptr) lse[row] = r.m / temp + kLn2 * r.l;
  }
}

// Gradient of part blockIdx.y (per vectors) of row blockIdx.x, from lse (backward)
// or from the row's parts (step: the first part also writes the loss).  A row whose lse
// does not keep its sum is taken whole by the first part's workgroup (1,024 rows of 131,072
// bf16, all of them such: 164 us, 690 where every part sums the row; 64 rows 63, 40; no
// such row: 106).  64 registers at most: 65, without the bound, cost 2%.
template <typename T>
__global__ __launch_bounds__(256, 8) void distill_grad_kernel(
    const T* __restrict__ z, int64_t ldz, int V, int per, const f32x2* __restrict__ parts,
    int count, const float* __restrict__ lse, const int32_t* __restrict__ ids,
    const float* __restrict__ top, int k, float temp, const float* __restrict__ weight,
    float* __restrict__ loss, T* __restrict__ dz, int64_t lddz) {
  constexpr int N = Row<T>::N, U = 4;
  extern __shared__ __align__(16) int smem[];
  __shared__ int live_sh;
  __shared__ float part[4];
  const int lane = threadIdx.x;
  const Entries en(smem, k);
  const int64_t row = blockIdx.x;
  const float c = kLog2E / temp;
  const T* zr = z + row * ldz;
  T* dr = dz + row * lddz;
  const int nvec = (V + N - 1) / N;
  RowSoftmax r;
  float s = 1.f;
  bool whole = false;
  if (lse == nullptr) {
    r = join_parts(parts + row * count, count, c, &s);
  } else if (keeps_sum<T>(lse[row])) {
    r.m = lse[row] * temp;  // z/T - lse: in the place of the maximum
    r.l = 0.f;
  } else {
    if (blockIdx.y > 0) return;
    whole = true;
    r.m = finite_max(max_and_sum<T, 256, U>(zr, V, 0, nvec, lane, c, part, &s));
    r.l = log2_hw(s);
  }
  for (int v0 = blockIdx.y * per;;) {
    const int v1 = min(v0 + per, nvec);
    if (lane < 64) {
      const bool live = teach<T, 64, true>(zr, ids + row * k, top + row * k, k, V, c, lane, en,
                                           v0 * N, (v1 - v0) * N);
      if (loss != nullptr && blockIdx.y == 0) {
        const float a = live ? loss_terms<64>(k, temp, r, lane, en) : 0.f;
        if (lane == 0) loss[row] = temp * (temp * a);
      }
      if (lane == 0) live_sh = live;
    }
    __syncthreads();
    if (!live_sh) {
      for (int v = v0 + lane; v < (whole ? nvec : v1); v += 256) store_vec(dr, v, V, i32x4{});
      return;
    }
    const float wt = (weight != nullptr ? weight[row] : 1.f) * temp;
    if (s == 0.f) r.l = 0.f;  // no logit but -inf: every q is 0
    const Exponent x(r.m, c);
    const float sum = x.near ? s * exp2_hw(fmaf(r.m, c, -x.mc)) : s;
    const float by = s == 0.f ? 0.f : wt / sum;
    if (x.near) {
      for (int v = v0 + lane; v < v1; v += 256 * U) {
        i32x4 in[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
          in[u] = load_logits(zr, v + 256 * u < v1 ? v + 256 * u : nvec, V);
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (v + 256 * u < v1)
            store_vec(dr, v + 256 * u, V, exp_scaled<T, true>(in[u], x, by));
      }
    } else {
      for (int v = v0 + lane; v < v1; v += 256)
        store_vec(dr, v, V, exp_scaled<T, false>(load_logits(zr, v, V), x, by));
    }
    __syncthreads();
    if (lane < 64) fix_entries<T, 64>(dr, k, c, wt, r, lane, v0 * N, min(v1 * N, V), en);
    v0 = v1;
    if (!whole || v0 == nvec) return;
    __syncthreads();  // live_sh and the entries are free again
  }
}

int vectors_of(int32_t V, int is_bf16) { return is_bf16 ? (V + 7) / 8 : (V + 3) / 4; }

// Entries a row up to which 32 (16) rows share a workgroup.  Above 32 a row of 8
// lanes waits for its entries (121,924 rows of 128 bf16, 64 entries, step: 60 us,
// with 16 lanes 50; of 24 entries 28, 33); above 128 those of 16 rows would fill
// more than half of the 64 KB of LDS that a launch has without asking.
constexpr int kTop32 = 32, kTop16 = 128;

constexpr int kRowVectors = 4096;  // the longest row that is always held in registers

// Parts of a row: 1 where a workgroup has a row to itself.  Rows in registers
// always do: one launch, where two wait for the host (16 rows of 16,384 bf16,
// loss: 4.7 us, in parts 6.5).  Longer rows are cut up where they are few: 64
// rows of 131,072 bf16, step: 16.2 us in parts, 19.4 whole; 100 rows: 20.8, 19.8.
int row_parts(int64_t n, int nvec) {
  if (nvec <= kRowVectors || n * 192 >= nvec) return 1;
  const int64_t want = (1024 + n - 1) / n;
  const int64_t most = (nvec + 511) / 512;
  return (int)std::min<int64_t>(want, most);
}

template <typename T, Pass PASS>
hipError_t run_rows(const DistillArgs& a, hipStream_t stream) {
  const int nvec = vectors_of(a.V, sizeof(T) == 2);
  auto go = [&](auto g, auto v) {
    constexpr int G = decltype(g)::value, NV = decltype(v)::value;
    constexpr int BLOCK = G > 256 ? G : 256, R = BLOCK / G;
    const size_t lds = (size_t)R * entry_words(a.k, PASS == Pass::kForward ? 0 : a.V) * 4;
    distill_row_kernel<T, G, NV, PASS><<<(unsigned)((a.n + R - 1) / R), BLOCK, lds, stream>>>(
        static_cast<const T*>(a.z), a.ldz, a.n, a.V, a.ids, a.top, a.k, a.temp, a.weight, a.loss,
        a.lse, static_cast<T*>(a.dz), a.lddz);
    return hipGetLastError();
  };
#define SHC_ROW(limit, g, v) \
  if (nvec <= limit) return go(std::integral_constant<int, g>{}, std::integral_constant<int, v>{})
  // few lanes a row, so that the entries' share of the lanes and the row's steps
  // are spread over more rows: 524,288 rows of 128 bf16, 8 entries, step: 71 us
  // with 8 lanes a row, 94 with 16; of 512 (134,217 rows): 74 with 16, 108 with 64
  if (a.k <= kTop32) SHC_ROW(16, 8, 2);
  if (a.k <= kTop16) SHC_ROW(32, 16, 2);
  if (a.k <= kTop16) SHC_ROW(64, 16, 4);
  SHC_ROW(128, 32, 4);
  SHC_ROW(256, 64, 4);
  SHC_ROW(512, 64, 8);
  SHC_ROW(1024, 256, 4);
  SHC_ROW(2048, 256, 8);
  SHC_ROW(kRowVectors, 512, 8);
  // longer fp32 rows too for the step, whose second pass has as many bytes to store as
  // to read, from 112 MB of them on, when not all of it stays in the caches (1,500 rows
  // of 45,000: 113 us, read twice 126; 1,000 of 65,536: 115, 123; 600 of 50,021: 57.9,
  // 62.3; 600 of 32,768: 40.3, 39.1).  Not up to 7,168 vectors, where it takes more rows
  // to pay (of 24,000 2,000 rows take 84.5, 89.7, but 1,300, also above 112 MB, 62.4,
  // 60.6).  With 16 vectors a thread 14 registers spill: 60 bytes of scratch a thread, and
  // still faster (1,000 of 53,252: 95, 103; 500 of 65,536: 61, 66).  bf16 rows, with twice
  // the arithmetic a byte, gain nothing (2,000 of 65,536: 124, 119).
  if constexpr (sizeof(T) == 4 && PASS == Pass::kStep) {
    if (nvec > 7168 && a.n * nvec >= 7000000) {
      SHC_ROW(8192, 1024, 8);
      SHC_ROW(10240, 1024, 10);
      SHC_ROW(13312, 1024, 13);
      SHC_ROW(16384, 1024, 16);
    }
  }
#undef SHC_ROW
  if constexpr (PASS == Pass::kBackward)
    return hipErrorInvalidValue;  // run_backward takes longer rows in parts
  else
    return go(std::integral_constant<int, 1024>{}, std::integral_constant<int, 0>{});
}

template <typename T>
hipError_t run_grad(const DistillArgs& a, int count, int per, hipStream_t stream) {
  const int nvec = vectors_of(a.V, sizeof(T) == 2);
  const dim3 grid((unsigned)a.n, (nvec + per - 1) / per);
  distill_grad_kernel<T><<<grid, 256, (size_t)entry_words(a.k, per * Row<T>::N) * 4, stream>>>(
      static_cast<const T*>(a.z), a.ldz, a.V, per, static_cast<const f32x2*>(a.parts), count,
      a.lse, a.ids, a.top, a.k, a.temp, a.weight, a.loss, static_cast<T*>(a.dz), a.lddz);
  return hipGetLastError();
}

template <typename T>
hipError_t run_parts(const DistillArgs& a, int count, int* per, hipStream_t stream) {
  const int nvec = vectors_of(a.V, sizeof(T) == 2);
  *per = (nvec + count - 1) / count;
  const dim3 grid((unsigned)a.n, count);
  distill_part_kernel<T><<<grid, 256, 0, stream>>>(static_cast<const T*>(a.z), a.ldz, a.V, *per,
                                                   a.temp, static_cast<f32x2*>(a.parts));
  return hipGetLastError();
}

template <typename T>
hipError_t run_forward(const DistillArgs& a, hipStream_t stream) {
  const int count = row_parts(a.n, vectors_of(a.V, sizeof(T) == 2));
  if (count == 1) return run_rows<T, Pass::kForward>(a, stream);
  int per;
  const hipError_t e = run_parts<T>(a, count, &per, stream);
  if (e != hipSuccess) return e;
  distill_join_kernel<T><<<(unsigned)a.n, 64, (size_t)entry_words(a.k, 0) * 4, stream>>>(
      static_cast<const T*>(a.z), a.ldz, a.V, static_cast<const f32x2*>(a.parts), count, a.ids,
      a.top, a.k, a.temp, a.loss, a.lse);
  return hipGetLastError();
}

template <typename T>
hipError_t run_step(const DistillArgs& a, hipStream_t stream) {
  const int count = row_parts(a.n, vectors_of(a.V, sizeof(T) == 2));
  if (count == 1) return run_rows<T, Pass::kStep>(a, stream);
  int per;
  const hipError_t e = run_parts<T>(a, count, &per, stream);
  return e != hipSuccess ? e : run_grad<T>(a, count, per, stream);
}

template <typename T>
hipError_t run_backward(const DistillArgs& a, hipStream_t stream) {
  // elementwise but for the entries, which every part of a row works out: rows in
  // registers where there are enough of them (31,424 of bf16, 8 entries: 3,000 rows
  // 75.8 us, in parts 78.9, of 200 entries 91, 97; 800 rows 26.4, 23.3), and longer
  // parts where there are many entries (1,500 rows of 120,000, 256 entries: 175, in
  // parts of 1024 vectors 210; of 64 entries 147, 146)
  const int nvec = vectors_of(a.V, sizeof(T) == 2);
  if (nvec <= 1024 || (nvec <= kRowVectors && a.n >= 1536))
    return run_rows<T, Pass::kBackward>(a, stream);
  const int per = a.k > 128 ? 2048 : 1024;
  return run_grad<T>(a, 0, per, stream);
}

}  // namespace

size_t distill_workspace_bytes(int64_t n, int32_t V) {
  // any count of rows up to n that is cut up, in either dtype: at most 1023 parts
  // beside one a row
  const int nvec = std::max(vectors_of(V, 0), vectors_of(V, 1));
  if (nvec <= kRowVectors) return 0;
  return (size_t)(1024 + std::min<int64_t>(n, nvec / 192)) * sizeof(f32x2);
}

hipError_t launch_distill(const DistillArgs& a, DistillPass pass, int is_bf16,
                          hipStream_t stream) {
  // a launch holds fewer than 2^32 threads: 2^20 rows of at most 1024, or of
  // 256 for each of a row's parts
  constexpr int64_t kMost = (int64_t)1 << 20;
  for (int64_t r0 = 0; r0 < a.n; r0 += kMost) {
    DistillArgs c = a;
    const int64_t e = is_bf16 ? 2 : 4;
    c.n = std::min(kMost, a.n - r0);
    c.z = static_cast<const char*>(a.z) + r0 * a.ldz * e;
    c.ids = a.ids + r0 * a.k;
    c.top = a.top + r0 * a.k;
    if (a.weight != nullptr) c.weight = a.weight + r0;
    if (a.loss != nullptr) c.loss = a.loss + r0;
    if (a.lse != nullptr) c.lse = a.lse + r0;
    if (a.dz != nullptr) c.dz = static_cast<char*>(a.dz) + r0 * a.lddz * e;
    hipError_t err;
    switch (pass) {
      case DistillPass::kForward:
        err = is_bf16 ? run_forward<uint16_t>(c, stream) : run_forward<float>(c, stream);
        break;
      case DistillPass::kBackward:
        err = is_bf16 ? run_backward<uint16_t>(c, stream) : run_backward<float>(c, stream);
        break;
      default: err = is_bf16 ? run_step<uint16_t>(c, stream) : run_step<float>(c, stream);
    }
    if (err != hipSuccess) return err;
  }
  return hipSuccess;
}

}  // namespace shc
