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
// entries has loss 0 and gradient 0 and its logits are not read.
//
// Bound by HBM: V elements read, and V written by the gradient.
// - Rows that fit a workgroup's registers (up to 16 vectors a thread) are read
//   once, by G lanes: maximum, sum, loss and, in the step, the gradient from the
//   registers.
// - Longer rows, and long rows of which there are few, are cut into parts: a
//   first launch leaves every part's maximum and sum in the workspace, the
//   second joins them in order and computes the loss or its part of the
//   gradient.
// The gradient writes w T q first; the k entries are corrected behind a fence
// by the lanes that share the row, entries of the same id all with the id's
// whole p, added in their order.
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

// Maximum and sum of a row: q_v = 2^((z_v - m) c - l).
struct RowSoftmax {
  float m, l;
};
__device__ __forceinline__ float finite_max(float m) { return m == -INFINITY ? 0.f : m; }
// What a sum over a maximum m becomes over `base` >= m; 0 where there was no
// logit yet (m = -inf: the sum is 0, and base may be far below 0).
__device__ __forceinline__ float rescale(float m, float base, float c) {
  return m == -INFINITY ? 0.f : exp2_hw((m - base) * c);
}
__device__ __forceinline__ float prob(float z, const RowSoftmax& r, float c) {
  return z == -INFINITY ? 0.f : exp2_hw((z - r.m) * c - r.l);
}

// The teacher's entries of a row, by the G lanes that share it: ids (-1 where
// there is none) and p to LDS.  Returns whether the row has any.
struct Teacher {
  float tm, l;  // log2 p_j = (t_j - tm) c - l
  bool live;
};
template <int G>
__device__ __forceinline__ Teacher teach(const int32_t* __restrict__ ids,
                                         const float* __restrict__ top, int k, int V, float c,
                                         int lane, float* red, int* sid, float* sp) {
  float tm = -INFINITY, any = 0.f;
  for (int e = lane; e < k; e += G) {
    const int id = ids[e];
    const float t = top[e];
    const bool ok = id >= 0 && id < V && t != -INFINITY;
    sid[e] = ok ? id : -1;
    sp[e] = t;
    if (ok) {
      tm = fmaxf(tm, t);
      any = 1.f;
    }
  }
  Teacher out;
  out.tm = finite_max(group_reduce<G>(tm, MaxOp{}, red));
  out.live = group_reduce<G>(any, MaxOp{}, red) != 0.f;
  float s = 0.f;
  for (int e = lane; e < k; e += G)
    if (sid[e] >= 0) s += exp2_hw((sp[e] - out.tm) * c);
  s = group_reduce<G>(s, AddOp{}, red);
  out.l = log2_hw(s);
  for (int e = lane; e < k; e += G)
    sp[e] = sid[e] >= 0 ? exp2_hw((sp[e] - out.tm) * c) / s : 0.f;
  group_fence<G>();
  return out;
}

// sum_j p_j (log p_j - log q_j) over the row's entries (z, top: the row's), in
// natural units: an entry on a logit of the type's lowest value stays finite.
template <typename T, int G>
__device__ __forceinline__ float loss_terms(const T* __restrict__ z,
                                            const float* __restrict__ top, int k, float temp,
                                            const Teacher& t, const RowSoftmax& r, int lane,
                                            float* red, const int* sid, const float* sp) {
  float a = 0.f;
  for (int e = lane; e < k; e += G) {
    if (sid[e] < 0) continue;
    const float zi = Row<T>::get(z + sid[e]), p = sp[e];
    const float lq = zi == -INFINITY ? -INFINITY : (zi - r.m) / temp - kLn2 * r.l;
    const float lp = (top[e] - t.tm) / temp - kLn2 * t.l;
    if (!(p == 0.f)) a += p * (lp - lq);
  }
  return group_reduce<G>(a, AddOp{}, red);
}

// The entries with ids in [lo, hi) of the gradient, behind the row's q.
template <typename T, int G>
__device__ __forceinline__ void fix_entries(const T* __restrict__ z, T* dz, int k, float c,
                                            float wt, const RowSoftmax& r, int lane, int lo,
                                            int hi, const int* sid, const float* sp) {
  for (int e = lane; e < k; e += G) {
    const int id = sid[e];
    if (id < lo || id >= hi) continue;
    float p = 0.f;
    for (int o = 0; o < k; ++o) p += sid[o] == id ? sp[o] : 0.f;
    Row<T>::put(dz + id, wt * (prob(Row<T>::get(z + id), r, c) - p));
  }
}

// Rows in registers: G lanes hold NV vectors each.
template <typename T, int G, int NV, bool STEP>
__global__ __launch_bounds__(G > 256 ? G : 256) void distill_row_kernel(
    const T* __restrict__ z, int64_t ldz, int64_t n, int V, const int32_t* __restrict__ ids,
    const float* __restrict__ top, int k, float temp, const float* __restrict__ weight,
    float* __restrict__ loss, float* __restrict__ lse, T* __restrict__ dz, int64_t lddz) {
  constexpr int N = Row<T>::N, BLOCK = G > 256 ? G : 256, R = BLOCK / G;
  extern __shared__ int smem[];  // per group: k ids, k probabilities
  __shared__ float part[G > 64 ? BLOCK / 64 : 1];
  const int lane = threadIdx.x % G, group = threadIdx.x / G;
  int* sid = smem + (int64_t)group * 2 * k;
  float* sp = reinterpret_cast<float*>(sid + k);
  const int64_t row = (int64_t)blockIdx.x * R + group;
  if (row >= n) return;  // whole groups
  const float c = kLog2E / temp;
  const T* zr = z + row * ldz;
  const int nvec = (V + N - 1) / N;

  i32x4 raw[NV];
#pragma unroll
  for (int q = 0; q < NV; ++q) raw[q] = load_logits(zr, q * G + lane, V);
  const Teacher t = teach<G>(ids + row * k, top + row * k, k, V, c, lane, part, sid, sp);
  if (!t.live) {
    if (lane == 0) {
      loss[row] = 0.f;
      if (!STEP && lse != nullptr) lse[row] = 0.f;
    }
    if constexpr (STEP) {
#pragma unroll
      for (int q = 0; q < NV; ++q)
        if (q * G + lane < nvec) store_vec(dz + row * lddz, q * G + lane, V, i32x4{});
    }
    return;  // the whole group
  }
  float m = -INFINITY;
#pragma unroll
  for (int q = 0; q < NV; ++q) {
    float f[N];
    Row<T>::widen(raw[q], f);
#pragma unroll
    for (int e = 0; e < N; ++e) m = fmaxf(m, f[e]);
  }
  RowSoftmax r;
  r.m = finite_max(group_reduce<G>(m, MaxOp{}, part));
  float s = 0.f;
#pragma unroll
  for (int q = 0; q < NV; ++q) {
    float f[N];
    Row<T>::widen(raw[q], f);
#pragma unroll
    for (int e = 0; e < N; ++e) s += exp2_hw((f[e] - r.m) * c);
  }
  s = group_reduce<G>(s, AddOp{}, part);
  r.l = log2_hw(s);
  const float a = loss_terms<T, G>(zr, top + row * k, k, temp, t, r, lane, part, sid, sp);
  if (lane == 0) {
    loss[row] = temp * temp * a;
    if (!STEP && lse != nullptr) lse[row] = r.m / temp + kLn2 * r.l;
  }
  if constexpr (STEP) {
    const float wt = (weight != nullptr ? weight[row] : 1.f) * temp;
    if (r.l == -INFINITY) r.l = 0.f;  // no logit but -inf: every q is 0
#pragma unroll
    for (int q = 0; q < NV; ++q) {
      const int v = q * G + lane;
      if (v < nvec) {
        float f[N];
        Row<T>::widen(raw[q], f);
#pragma unroll
        for (int e = 0; e < N; ++e) f[e] = wt * exp2_hw((f[e] - r.m) * c - r.l);
        store_vec(dz + row * lddz, v, V, Row<T>::narrow(f));
      }
    }
    group_fence<G>();
    fix_entries<T, G>(zr, dz + row * lddz, k, c, wt, r, lane, 0, V, sid, sp);
  }
}

// Maximum and sum of part blockIdx.y (per vectors) of row blockIdx.x.
template <typename T>
__global__ __launch_bounds__(256) void distill_part_kernel(const T* __restrict__ z, int64_t ldz,
                                                           int V, int per, float temp,
                                                           f32x2* __restrict__ parts) {
  constexpr int N = Row<T>::N, U = 4;
  __shared__ float part[4];
  const T* zr = z + (int64_t)blockIdx.x * ldz;
  const float c = kLog2E / temp;
  const int nvec = (V + N - 1) / N;
  const int v0 = blockIdx.y * per, v1 = min(v0 + per, nvec);
  float m = -INFINITY, s = 0.f;
  for (int v = v0 + threadIdx.x; v < v1; v += 256 * U) {
    i32x4 raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) raw[u] = load_logits(zr, v + 256 * u < v1 ? v + 256 * u : nvec, V);
    float top = m;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float f[N];
      Row<T>::widen(raw[u], f);
#pragma unroll
      for (int e = 0; e < N; ++e) top = fmaxf(top, f[e]);
    }
    const float base = finite_max(top);
    s *= rescale(m, base, c);
    m = top;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float f[N];
      Row<T>::widen(raw[u], f);
#pragma unroll
      for (int e = 0; e < N; ++e) s += exp2_hw((f[e] - base) * c);
    }
  }
  const float all = group_reduce<256>(m, MaxOp{}, part);
  s *= rescale(m, all, c);
  s = group_reduce<256>(s, AddOp{}, part);
  if (threadIdx.x == 0) parts[(int64_t)blockIdx.x * gridDim.y + blockIdx.y] = f32x2{all, s};
}

// A row's parts joined, by the lanes of a wavefront (every wavefront of the
// workgroup alike).
__device__ __forceinline__ RowSoftmax join_parts(const f32x2* __restrict__ parts, int count,
                                                 float c) {
  const int lane = threadIdx.x & 63;
  float m = -INFINITY;
  for (int i = lane; i < count; i += 64) m = fmaxf(m, parts[i][0]);
  RowSoftmax r;
  r.m = finite_max(lanes_reduce<64>(m, MaxOp{}));
  float s = 0.f;
  for (int i = lane; i < count; i += 64)
    s += parts[i][1] * rescale(parts[i][0], r.m, c);
  r.l = log2_hw(lanes_reduce<64>(s, AddOp{}));
  return r;
}

// Loss (and lse) of rows from their parts, a wavefront each.
template <typename T>
__global__ __launch_bounds__(64) void distill_join_kernel(
    const T* __restrict__ z, int64_t ldz, int V, const f32x2* __restrict__ parts, int count,
    const int32_t* __restrict__ ids, const float* __restrict__ top, int k, float temp,
    float* __restrict__ loss, float* __restrict__ lse) {
  extern __shared__ int smem[];
  int* sid = smem;
  float* sp = reinterpret_cast<float*>(sid + k);
  const int64_t row = blockIdx.x;
  const int lane = threadIdx.x;
  const float c = kLog2E / temp;
  const Teacher t = teach<64>(ids + row * k, top + row * k, k, V, c, lane, nullptr, sid, sp);
  if (!t.live) {
    if (lane == 0) {
      loss[row] = 0.f;
      if (lse != nullptr) lse[row] = 0.f;
    }
    return;
  }
  const RowSoftmax r = join_parts(parts + row * count, count, c);
  const float a = loss_terms<T, 64>(z + row * ldz, top + row * k, k, temp, t, r, lane, nullptr, sid,
                                    sp);
  if (lane == 0) {
    loss[row] = temp * temp * a;
    if (lse != nullptr) lse[row] = r.m / temp + kLn2 * r.l;
  }
}

// Gradient of part blockIdx.y (per vectors) of the rows, G lanes a row, from
// lse (backward) or from the row's parts (step: the first part also writes the
// loss).
template <typename T, int G>
__global__ __launch_bounds__(256) void distill_grad_kernel(
    const T* __restrict__ z, int64_t ldz, int64_t n, int V, int per,
    const f32x2* __restrict__ parts, int count, const float* __restrict__ lse,
    const int32_t* __restrict__ ids, const float* __restrict__ top, int k, float temp,
    const float* __restrict__ weight, float* __restrict__ loss, T* __restrict__ dz,
    int64_t lddz) {
  constexpr int N = Row<T>::N, R = 256 / G;
  extern __shared__ int smem[];
  __shared__ float part[4];
  const int lane = threadIdx.x % G, group = threadIdx.x / G;
  int* sid = smem + (int64_t)group * 2 * k;
  float* sp = reinterpret_cast<float*>(sid + k);
  const int64_t row = (int64_t)blockIdx.x * R + group;
  if (row >= n) return;  // whole groups
  const float c = kLog2E / temp;
  const T* zr = z + row * ldz;
  T* dr = dz + row * lddz;
  const int nvec = (V + N - 1) / N;
  const int v0 = blockIdx.y * per, v1 = min(v0 + per, nvec);
  const Teacher t = teach<G>(ids + row * k, top + row * k, k, V, c, lane, part, sid, sp);
  if (!t.live) {
    if (loss != nullptr && lane == 0 && blockIdx.y == 0) loss[row] = 0.f;
    for (int v = v0 + lane; v < v1; v += G) store_vec(dr, v, V, i32x4{});
    return;
  }
  RowSoftmax r;
  if (lse != nullptr) {
    // z/T - lse: the saved lse takes the place of the maximum
    r.m = lse[row] * temp;
    r.l = 0.f;
    if (r.m == -INFINITY) r.m = 0.f;
  } else {
    r = join_parts(parts + row * count, count, c);
    if (loss != nullptr && blockIdx.y == 0) {
      const float a = loss_terms<T, G>(zr, top + row * k, k, temp, t, r, lane, part, sid, sp);
      if (lane == 0) loss[row] = temp * temp * a;
    }
    if (r.l == -INFINITY) r.l = 0.f;
  }
  const float wt = (weight != nullptr ? weight[row] : 1.f) * temp;
  for (int v = v0 + lane; v < v1; v += G) {
    float f[N];
    Row<T>::widen(load_logits(zr, v, V), f);
#pragma unroll
    for (int e = 0; e < N; ++e) f[e] = wt * exp2_hw((f[e] - r.m) * c - r.l);
    store_vec(dr, v, V, Row<T>::narrow(f));
  }
  group_fence<G>();
  fix_entries<T, G>(zr, dr, k, c, wt, r, lane, v0 * N, min(v1 * N, V), sid, sp);
}

int vectors_of(int32_t V, int is_bf16) { return is_bf16 ? (V + 7) / 8 : (V + 3) / 4; }

constexpr int kRowVectors = 1024 * 16;  // vectors of the longest row held in registers

// Parts of a row: 1 where rows are held in registers.
int row_parts(int64_t n, int nvec) {
  if (nvec <= kRowVectors && (n >= 256 || nvec <= 1024)) return 1;
  const int64_t want = std::max<int64_t>(1, (1024 + n - 1) / n);
  const int64_t most = (nvec + 511) / 512;
  return (int)std::max<int64_t>(2, std::min<int64_t>(want, most));
}

template <typename T, bool STEP>
hipError_t run_rows(const DistillArgs& a, hipStream_t stream) {
  const int nvec = vectors_of(a.V, sizeof(T) == 2);
  auto go = [&](auto g, auto v) {
    constexpr int G = decltype(g)::value, NV = decltype(v)::value;
    constexpr int BLOCK = G > 256 ? G : 256, R = BLOCK / G;
    distill_row_kernel<T, G, NV, STEP>
        <<<(unsigned)((a.n + R - 1) / R), BLOCK, (size_t)R * 2 * a.k * 4, stream>>>(
            static_cast<const T*>(a.z), a.ldz, a.n, a.V, a.ids, a.top, a.k, a.temp, a.weight,
            a.loss, a.lse, static_cast<T*>(a.dz), a.lddz);
    return hipGetLastError();
  };
#define SHC_ROW(limit, g, v) \
  if (nvec <= limit) return go(std::integral_constant<int, g>{}, std::integral_constant<int, v>{})
  SHC_ROW(16, 16, 1);
  SHC_ROW(32, 32, 1);
  SHC_ROW(64, 64, 1);
  SHC_ROW(128, 64, 2);
  SHC_ROW(256, 64, 4);
  SHC_ROW(512, 256, 2);
  SHC_ROW(1024, 256, 4);
  SHC_ROW(2048, 256, 8);
  SHC_ROW(4096, 512, 8);
  SHC_ROW(8192, 1024, 8);
  SHC_ROW(kRowVectors, 1024, 16);
#undef SHC_ROW
  return hipErrorInvalidValue;
}

template <typename T>
hipError_t run_grad(const DistillArgs& a, int count, int per, hipStream_t stream) {
  const int nvec = vectors_of(a.V, sizeof(T) == 2);
  const int nparts = (nvec + per - 1) / per;
  auto go = [&](auto g) {
    constexpr int G = decltype(g)::value;
    constexpr int R = 256 / G;
    const dim3 grid((unsigned)((a.n + R - 1) / R), nparts);
    distill_grad_kernel<T, G><<<grid, 256, (size_t)R * 2 * a.k * 4, stream>>>(
        static_cast<const T*>(a.z), a.ldz, a.n, a.V, per,
        static_cast<const f32x2*>(a.parts), count, a.lse, a.ids, a.top, a.k, a.temp, a.weight,
        a.loss, static_cast<T*>(a.dz), a.lddz);
    return hipGetLastError();
  };
  if (nvec <= 16) return go(std::integral_constant<int, 16>{});
  if (nvec <= 256) return go(std::integral_constant<int, 64>{});
  return go(std::integral_constant<int, 256>{});
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
  if (count == 1) return run_rows<T, false>(a, stream);
  int per;
  const hipError_t e = run_parts<T>(a, count, &per, stream);
  if (e != hipSuccess) return e;
  distill_join_kernel<T><<<(unsigned)a.n, 64, (size_t)2 * a.k * 4, stream>>>(
      static_cast<const T*>(a.z), a.ldz, a.V, static_cast<const f32x2*>(a.parts), count, a.ids,
      a.top, a.k, a.temp, a.loss, a.lse);
  return hipGetLastError();
}

template <typename T>
hipError_t run_step(const DistillArgs& a, hipStream_t stream) {
  const int count = row_parts(a.n, vectors_of(a.V, sizeof(T) == 2));
  if (count == 1) return run_rows<T, true>(a, stream);
  int per;
  const hipError_t e = run_parts<T>(a, count, &per, stream);
  return e != hipSuccess ? e : run_grad<T>(a, count, per, stream);
}

template <typename T>
hipError_t run_backward(const DistillArgs& a, hipStream_t stream) {
  // rows cut up only where there are too few to fill the chip
  const int nvec = vectors_of(a.V, sizeof(T) == 2);
  const int64_t want = std::max<int64_t>(1, (2048 + a.n - 1) / a.n);
  const int64_t most = std::max(1, nvec / 256);
  const int count = (int)std::min<int64_t>(want, most);
  return run_grad<T>(a, 0, (nvec + count - 1) / count, stream);
}

}  // namespace

size_t distill_workspace_bytes(int64_t n, int32_t V) {
  // parts of any count of rows up to n, in either dtype: at most 1024 + n, and
  // at least two a row
  const int nvec = std::max(vectors_of(V, 0), vectors_of(V, 1));
  if (nvec <= 1024) return 0;
  return (size_t)(std::max<int64_t>(1024 + n, 2 * n)) * sizeof(f32x2);
}

hipError_t launch_distill(const DistillArgs& a, DistillPass pass, int is_bf16,
                          hipStream_t stream) {
  // a launch holds fewer than 2^32 threads: 2^21 rows of at most 1024
  constexpr int64_t kMost = (int64_t)1 << 21;
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
