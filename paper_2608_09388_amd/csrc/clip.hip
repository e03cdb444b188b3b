// Norm of all gradients together, and their clipping to it:
//
//   norm = sqrt(sum over every tensor and element of g^2)
//   factor = 1 where norm <= max_norm, else max_norm / norm;  out = factor g
//
// Both are bound by HBM: the first pass reads every element, the second reads and writes
// it.  The tensors are cut into chunks of the same number of elements, a workgroup to a
// chunk; a launch's arguments hold the addresses of up to kBatch tensors, so there is no
// table to build or keep.  Squares are summed in fp64: a value's square passes fp32 at
// 2e19, and a long sum keeps its digits.  Every chunk writes its sum, one workgroup adds
// them in a fixed order.  The second pass takes the chunks from the last to the first, of
// which some are still in the caches: 4 GiB of bf16 2,347 us so, 2,370 us from the first.
//
// 4 GiB of fp32 are read for their norm in 713 us (6.0 TB/s), 1.27e9 elements of bf16 (2.55
// GB) normed and clipped in 1,337 us (5.7 TB/s of the 7.65 GB that the two passes move).
#include <algorithm>

#include "row_ops.h"

namespace shc {
namespace {

using namespace rowops;

constexpr int kBatch = 128;

struct Batch {
  const void* data[kBatch];
  void* out[kBatch];
  int32_t first[kBatch + 1];  // a tensor's first chunk of the launch
  int64_t numel[kBatch];
  uint64_t bf16[kBatch / 64];
  int32_t n;
  int32_t chunk;  // elements
};
static_assert(sizeof(Batch) <= 3900, "kernel arguments stay below 4 KB");

// The tensor of a chunk, by halving (tensors without elements have no chunk).
__device__ __forceinline__ int tensor_of(const Batch& b, int chunk) {
  int lo = 0, hi = b.n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (b.first[mid] <= chunk)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

template <typename T>
__device__ __forceinline__ double chunk_squares(const T* p, int n) {
  constexpr int N = Row<T>::N;
  double s[2] = {0.0, 0.0};
  const int nv = (n + N - 1) / N;
#pragma unroll 4
  for (int v = threadIdx.x; v < nv; v += 256) {
    float f[N];
    Row<T>::widen(load_vec<T>(p, v, n), f);
#pragma unroll
    for (int e = 0; e < N; ++e) s[e & 1] = fma((double)f[e], (double)f[e], s[e & 1]);
  }
  return s[0] + s[1];
}

__device__ __forceinline__ double wave_sum(double s) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) s += __shfl_xor(s, d, 64);
  return s;
}

__global__ __launch_bounds__(256) void squares_kernel(Batch b, double* sums) {
  __shared__ double part[4];
  const int t = tensor_of(b, blockIdx.x);
  const int64_t at = (int64_t)(blockIdx.x - b.first[t]) * b.chunk;
  const int64_t left = b.numel[t] - at;
  const int n = left < b.chunk ? (int)left : b.chunk;
  double s;
  if (b.bf16[t >> 6] >> (t & 63) & 1)
    s = chunk_squares(static_cast<const uint16_t*>(b.data[t]) + at, n);
  else
    s = chunk_squares(static_cast<const float*>(b.data[t]) + at, n);
  s = wave_sum(s);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) sums[blockIdx.x] = (part[0] + part[1]) + (part[2] + part[3]);
}

__global__ __launch_bounds__(1024) void norm_kernel(const double* sums, int64_t n, float* norm) {
  __shared__ double part[16];
  double s = 0.0;
#pragma unroll 4
  for (int64_t i = threadIdx.x; i < n; i += 1024) s += sums[i];
  s = wave_sum(s);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x != 0) return;
  for (int w = 1; w < 16; ++w) s += part[w];
  *norm = (float)sqrt(s);
}

template <typename T>
__device__ __forceinline__ void chunk_scale(const T* p, T* q, int n, float factor) {
  constexpr int N = Row<T>::N;
  const int nv = (n + N - 1) / N;
#pragma unroll 4
  for (int v = threadIdx.x; v < nv; v += 256) {
    float f[N];
    Row<T>::widen(load_vec<T>(p, v, n), f);
#pragma unroll
    for (int e = 0; e < N; ++e) f[e] *= factor;
    store_vec<T>(q, v, n, Row<T>::narrow(f));
  }
}

__global__ __launch_bounds__(256) void scale_kernel(Batch b, const float* norm, float most) {
  const float x = *norm;
  const float factor = x <= most ? 1.f : most / x;  // a NaN makes NaN of all
  const int chunk = (int)(gridDim.x - 1 - blockIdx.x);
  const int t = tensor_of(b, chunk);
  if (factor == 1.f && b.data[t] == b.out[t]) return;
  const int64_t at = (int64_t)(chunk - b.first[t]) * b.chunk;
  const int64_t left = b.numel[t] - at;
  const int n = left < b.chunk ? (int)left : b.chunk;
  if (b.bf16[t >> 6] >> (t & 63) & 1)
    chunk_scale(static_cast<const uint16_t*>(b.data[t]) + at,
                static_cast<uint16_t*>(b.out[t]) + at, n, factor);
  else
    chunk_scale(static_cast<const float*>(b.data[t]) + at, static_cast<float*>(b.out[t]) + at, n,
                factor);
}

// Elements of a chunk: `most`, fewer where that leaves CUs idle.  The pass that reads
// alone gains by long chunks, the one that writes too by short ones: 4 GiB of fp32 read,
// us at 4,096, 8,192, 16,384, 32,768: 805, 755, 727, 713; 4 GiB of bf16 read and written
// 1,528, 1,542, 1,622, 1,633.
constexpr int kNormChunk = 32768, kScaleChunk = 8192;
int chunk_of(const ClipTensor* t, int64_t count, int most) {
  int64_t total = 0;
  for (int64_t i = 0; i < count; ++i) total += t[i].numel;
  return (int)std::min<int64_t>(most, std::max<int64_t>(2048, total / 1024 / 2048 * 2048));
}
int64_t chunks_of(const ClipTensor& t, int chunk) { return (t.numel + chunk - 1) / chunk; }

// Calls f(batch, chunks, chunks before it) for every launch; tensors of more chunks
// than a launch takes are given in parts.
template <typename F>
hipError_t batches(const ClipTensor* t, int64_t count, int chunk, F&& f) {
  constexpr int64_t kMost = (int64_t)1 << 22;  // chunks of a launch
  Batch b;
  b.chunk = chunk;
  int64_t before = 0;
  b.n = 0, b.first[0] = 0;
  std::fill(b.bf16, b.bf16 + kBatch / 64, 0);
  const auto flush = [&] {
    const int64_t chunks = b.first[b.n];
    hipError_t e = hipSuccess;
    if (chunks > 0) e = f(b, chunks, before);
    before += chunks;
    b.n = 0;
    std::fill(b.bf16, b.bf16 + kBatch / 64, 0);
    return e;
  };
  for (int64_t i = 0; i < count; ++i) {
    int64_t at = 0;
    while (at < t[i].numel) {
      const int64_t room = kMost - (b.n == 0 ? 0 : b.first[b.n]);
      if (b.n == kBatch || room == 0) {
        const hipError_t e = flush();
        if (e != hipSuccess) return e;
        continue;
      }
      const int64_t take = std::min(t[i].numel - at, room * chunk);
      const int64_t size = t[i].bf16 ? 2 : 4;
      b.data[b.n] = static_cast<const char*>(t[i].data) + at * size;
      b.out[b.n] = t[i].out == nullptr ? nullptr : static_cast<char*>(t[i].out) + at * size;
      b.numel[b.n] = take;
      if (t[i].bf16) b.bf16[b.n >> 6] |= 1ull << (b.n & 63);
      b.first[b.n + 1] = b.first[b.n] + (int32_t)((take + chunk - 1) / chunk);
      ++b.n;
      at += take;
    }
  }
  return flush();
}

}  // namespace

size_t grad_norm_workspace_bytes(const ClipTensor* t, int64_t count) {
  const int chunk = chunk_of(t, count, kNormChunk);
  int64_t chunks = 0;
  for (int64_t i = 0; i < count; ++i) chunks += chunks_of(t[i], chunk);
  return (size_t)std::max<int64_t>(chunks, 1) * sizeof(double);
}

hipError_t launch_grad_norm(const ClipTensor* t, int64_t count, float* norm, void* ws,
                            hipStream_t stream) {
  double* sums = static_cast<double*>(ws);
  int64_t all = 0;
  const int chunk = chunk_of(t, count, kNormChunk);
  const hipError_t e =
      batches(t, count, chunk, [&](const Batch& b, int64_t chunks, int64_t before) {
        squares_kernel<<<(int)chunks, 256, 0, stream>>>(b, sums + before);
        all = before + chunks;
        return hipGetLastError();
      });
  if (e != hipSuccess) return e;
  norm_kernel<<<1, 1024, 0, stream>>>(sums, all, norm);
  return hipGetLastError();
}

hipError_t launch_clip_grads(const ClipTensor* t, int64_t count, const float* norm,
                             float max_norm, hipStream_t stream) {
  const int chunk = chunk_of(t, count, kScaleChunk);
  return batches(t, count, chunk, [&](const Batch& b, int64_t chunks, int64_t) {
    scale_kernel<<<(int)chunks, 256, 0, stream>>>(b, norm, max_norm);
    return hipGetLastError();
  });
}

}  // namespace shc
