// Embedding rows with scaling, and their gradient by sorted ids.
//
//   y[i] = scale * E[id_i] (+ add[i]);   an id outside [0, R) has no row
//   dE[r] = scale * sum over i with id_i = r (and r != pad) of dY[i]
//
// Forward: a gather bound by HBM.  G lanes share a row and walk its 16-byte
// vectors, 256 / G rows a workgroup.
//
// Gradient: three launches.
// 1. embed_sort_kernel orders the positions by id, stably, in one launch and
//    without communication: workgroup p of P owns the ids that are p modulo P
//    (frequent ids, often neighbours, then fall to different workgroups), reads
//    all ids once to count its own per id and to count the ids of the workgroups
//    before it (its first place in the order), and again to place the positions:
//    a chunk of ids at a time goes to a queue in LDS, in order, and the
//    workgroup's 16 wavefronts, each owning a sixteenth of the ids, hand out the
//    places.  It also clears the table rows of its ids that have no position.
// 2. embed_sum_kernel cuts the ordered positions into jobs of equal length,
//    whatever the ids' frequencies; a group of lanes per job and column range
//    adds the rows of each id in order.  An id that lies inside one job is
//    final; the part of an id that continues in or from another job goes to the
//    workspace.
// 3. embed_join_kernel adds those parts, in order, at the job where the id
//    begins.
// Every sum has an order that follows the ids and sizes alone: results repeat
// bit for bit.
#include <algorithm>
#include <mutex>

#include "row_ops.h"

namespace shc {
namespace {

using namespace rowops;

template <typename T, typename ID, int G>
__global__ __launch_bounds__(256) void embed_kernel(const T* __restrict__ E, int64_t R,
                                                    int64_t ldE, const ID* __restrict__ ids,
                                                    int64_t id_stride, int64_t n, int C,
                                                    float scale, const T* __restrict__ add,
                                                    int64_t ldadd, T* __restrict__ out,
                                                    int64_t ldout) {
  constexpr int N = Row<T>::N;
  const int lane = threadIdx.x % G;
  const int64_t row = (int64_t)blockIdx.x * (256 / G) + threadIdx.x / G;
  if (row >= n) return;
  const int64_t id = (int64_t)ids[row * id_stride];
  const bool there = id >= 0 && id < R;
  const T* e = E + (there ? id : 0) * ldE;
  const int nvec = (C + N - 1) / N;
  for (int v = lane; v < nvec; v += G) {
    float f[N], a[N];
    Row<T>::widen(there ? load_vec(e, v, C) : i32x4{}, f);
    if (add != nullptr) {
      Row<T>::widen(load_vec(add + row * ldadd, v, C), a);
#pragma unroll
      for (int k = 0; k < N; ++k) f[k] = there ? fmaf(f[k], scale, a[k]) : a[k];
    } else {
#pragma unroll
      for (int k = 0; k < N; ++k) f[k] *= scale;
    }
    store_vec(out + row * ldout, v, C, Row<T>::narrow(f));
  }
}

constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kSortPer = 8;                          // ids a thread takes from a chunk
constexpr int kSortChunk = kSortThreads * kSortPer;  // ids of a chunk

// Ids of the sort's workgroup p of P = 1 << logP: id & (P - 1) == p, at most
// keys = ceil(R / P) of them, local number id >> logP.
// LDS: count[keys], then the queue (local number, position) of a chunk.
template <typename ID>
__global__ __launch_bounds__(kSortThreads) void embed_sort_kernel(
    const ID* __restrict__ ids, int64_t id_stride, int n, int R, int pad, int logP, int keys,
    int C, int clear, float* __restrict__ dE, int64_t ldE, int32_t* __restrict__ order,
    int32_t* __restrict__ key_of, int32_t* __restrict__ total) {
  extern __shared__ int smem[];
  volatile int* count = smem;
  int* queue_key = smem + keys;
  int* queue_pos = queue_key + kSortChunk;
  __shared__ int wave_sum[kSortWaves];
  __shared__ int base_sh, queued;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int P = 1 << logP, p = blockIdx.x;

  for (int k = tid; k < keys; k += kSortThreads) smem[k] = 0;
  __syncthreads();
  // counts of this workgroup's ids, and of the ids of the workgroups before it
  int below = 0;
  for (int i = tid; i < n; i += kSortThreads) {
    const int64_t id = (int64_t)ids[(int64_t)i * id_stride];
    if (id >= 0 && id < R && id != pad) {
      const int b = (int)id & (P - 1);
      below += b < p;
      if (b == p) atomicAdd(&smem[(int)id >> logP], 1);
    }
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) below += __shfl_xor(below, d, 64);
  if (lane == 0) wave_sum[wave] = below;
  __syncthreads();
  if (tid == 0) {
    int s = 0;
    for (int w = 0; w < kSortWaves; ++w) s += wave_sum[w];
    base_sh = s;
  }
  __syncthreads();

  // rows of ids without a position
  if (clear) {
    for (int k = wave; k < keys; k += kSortWaves) {
      const int r = (k << logP) + p;
      if (r < R && count[k] == 0)
        for (int v = lane; 4 * v < C; v += 64) {
          const float z[4] = {0.f, 0.f, 0.f, 0.f};
          store_channels<4>(dE + (int64_t)r * ldE, v, C, z);
        }
    }
  }
  __syncthreads();

  // counts -> first places: consecutive keys per thread, their sums scanned
  const int per = (keys + kSortThreads - 1) / kSortThreads;
  int mine = 0;
  for (int k = tid * per; k < min(keys, (tid + 1) * per); ++k) mine += count[k];
  int inc = mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int u = __shfl_up(inc, d, 64);
    if (lane >= d) inc += u;
  }
  if (lane == 63) wave_sum[wave] = inc;
  __syncthreads();
  int at = base_sh + inc - mine;
  for (int w = 0; w < wave; ++w) at += wave_sum[w];
  for (int k = tid * per; k < min(keys, (tid + 1) * per); ++k) {
    const int c = count[k];
    count[k] = at;
    at += c;
  }
  // the last workgroup's last place is the number of ids that count
  if (p == P - 1 && tid == kSortThreads - 1) *total = at;
  __syncthreads();

  for (int64_t c0 = 0; c0 < n; c0 += kSortChunk) {
    // this chunk's ids of the workgroup, in order: wavefront w has the w-th
    // part of the chunk
    int key[kSortPer];
    uint64_t has[kSortPer];
    int found = 0;
    const int64_t w0 = c0 + (int64_t)wave * 64 * kSortPer;
#pragma unroll
    for (int u = 0; u < kSortPer; ++u) {
      const int64_t i = w0 + u * 64 + lane;
      key[u] = -1;
      if (i < n) {
        const int64_t id = (int64_t)ids[i * id_stride];
        if (id >= 0 && id < R && id != pad && ((int)id & (P - 1)) == p) key[u] = (int)id >> logP;
      }
      has[u] = __ballot(key[u] >= 0);
      found += __popcll(has[u]);
    }
    if (lane == 0) wave_sum[wave] = found;
    __syncthreads();
    int q = 0;
    for (int w = 0; w < wave; ++w) q += wave_sum[w];
    if (wave == kSortWaves - 1 && lane == 0) queued = q + found;
#pragma unroll
    for (int u = 0; u < kSortPer; ++u) {
      if (key[u] >= 0) {
        const int s = q + __popcll(has[u] & ((1ull << lane) - 1));
        queue_key[s] = key[u];
        queue_pos[s] = (int)(w0 + u * 64 + lane);
      }
      q += __popcll(has[u]);
    }
    __syncthreads();
    // places: every wavefront walks the queue for the local numbers it owns
    const int nq = queued;
    for (int q0 = 0; q0 < nq; q0 += 64) {
      const bool in = q0 + lane < nq;
      const int k = in ? queue_key[q0 + lane] : 0;
      uint64_t todo = __ballot(in && (k & (kSortWaves - 1)) == wave);
      while (todo != 0) {
        const int first = __ffsll((unsigned long long)todo) - 1;
        const int kk = __shfl(k, first, 64);
        const uint64_t same = __ballot(in && k == kk);
        const int place = count[kk];
        if (lane == first) count[kk] = place + __popcll(same);
        if (in && k == kk) {
          const int s = place + __popcll(same & ((1ull << lane) - 1));
          order[s] = queue_pos[q0 + lane];
          key_of[s] = (kk << logP) + p;
        }
        todo &= ~same;
      }
    }
    __syncthreads();
  }
}

// Job j (J positions of the order) and columns [tile * G * N, + G * N): G lanes.
// part [jobs][2][C]: what an id that began in an earlier job gets from this one
// (slot 0), what an id that goes on in the next job gets from this one, where it
// began here (slot 1).
template <typename T, int G>
__global__ __launch_bounds__(256) void embed_sum_kernel(
    const T* __restrict__ dY, int64_t lddy, const int32_t* __restrict__ order,
    const int32_t* __restrict__ key_of, const int32_t* __restrict__ total, int J, int jobs, int C,
    float scale, int accumulate, float* __restrict__ dE, int64_t ldE, float* __restrict__ part) {
  constexpr int N = Row<T>::N, U = 8;
  const int j = blockIdx.x * (256 / G) + threadIdx.x / G;
  const int v = blockIdx.y * G + threadIdx.x % G;
  const int m = *total;
  if (j >= jobs) return;
  const int lo = j * J, hi = min(lo + J, m);
  if (lo >= hi || v * N >= C) return;
  const int before = lo > 0 ? key_of[lo - 1] : -1;
  const int after = hi < m ? key_of[hi] : -1;

  float acc[N];
#pragma unroll
  for (int e = 0; e < N; ++e) acc[e] = 0.f;
  bool from_before = key_of[lo] == before;
  auto put = [&](int key, bool goes_on) {
    if (from_before) {
      store_channels<N>(part + ((int64_t)j * 2) * C, v, C, acc);
    } else if (goes_on) {
      store_channels<N>(part + ((int64_t)j * 2 + 1) * C, v, C, acc);
    } else {
      float* to = dE + (int64_t)key * ldE;
      float f[N];
      if (accumulate) load_channels<N>(to, v, C, f);
#pragma unroll
      for (int e = 0; e < N; ++e) f[e] = accumulate ? fmaf(acc[e], scale, f[e]) : acc[e] * scale;
      store_channels<N>(to, v, C, f);
    }
    from_before = false;
#pragma unroll
    for (int e = 0; e < N; ++e) acc[e] = 0.f;
  };
  int key = key_of[lo];
  for (int t0 = lo; t0 < hi; t0 += U) {
    int pos[U], keys[U];
    i32x4 raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = min(t0 + u, hi - 1);
      pos[u] = order[t];
      keys[u] = key_of[t];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) raw[u] = load_vec(dY + (int64_t)pos[u] * lddy, v, C);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (t0 + u < hi) {
        if (keys[u] != key) {
          put(key, false);
          key = keys[u];
        }
        float f[N];
        Row<T>::widen(raw[u], f);
#pragma unroll
        for (int e = 0; e < N; ++e) acc[e] += f[e];
      }
    }
  }
  put(key, key == after);
}

// The parts of the id that begins in job j and goes on in the next: slot 1 of
// job j, then slot 0 of the jobs after it up to the last with that id.  The
// workgroup's four quarters take every fourth of those, added in order.
__global__ __launch_bounds__(256) void embed_join_kernel(
    const int32_t* __restrict__ key_of, const int32_t* __restrict__ total, int J, int jobs, int C,
    float scale, int accumulate, const float* __restrict__ part, float* __restrict__ dE,
    int64_t ldE) {
  __shared__ float sum[4][64][4];
  const int m = *total;
  const int lane = threadIdx.x & 63, quarter = threadIdx.x >> 6;
  const int v = blockIdx.y * 64 + lane;
  for (int j = blockIdx.x; j < jobs; j += gridDim.x) {
  const int lo = j * J, hi = lo + J;
  if (hi >= m) return;  // the last job: nothing goes on
  const int key = key_of[hi];
  if (key_of[hi - 1] != key) continue;                                  // nothing goes on
  if (key_of[lo] == key && lo > 0 && key_of[lo - 1] == key) continue;  // it began earlier
  // the last job that has the id: it holds every position up to its last
  int last = j + 1;
  for (int b = (m - 1) / J; last < b;) {
    const int mid = (last + b + 1) / 2;
    if (key_of[mid * J] == key)
      last = mid;
    else
      b = mid - 1;
  }
  float acc[4] = {0.f, 0.f, 0.f, 0.f}, f[4];
  if (v * 4 < C) {
    if (quarter == 0) load_channels<4>(part + ((int64_t)j * 2 + 1) * C, v, C, acc);
    for (int q = j + 1 + quarter; q <= last; q += 4) {
      load_channels<4>(part + ((int64_t)q * 2) * C, v, C, f);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] += f[e];
    }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) sum[quarter][lane][e] = acc[e];
  __syncthreads();
  if (quarter == 0 && v * 4 < C) {
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] += (sum[1][lane][e] + sum[2][lane][e]) + sum[3][lane][e];
    float* to = dE + (int64_t)key * ldE;
    if (accumulate) load_channels<4>(to, v, C, f);
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = accumulate ? fmaf(acc[e], scale, f[e]) : acc[e] * scale;
    store_channels<4>(to, v, C, f);
  }
  __syncthreads();
  }
}

struct EmbedPlan {
  int logP, keys, J, jobs;
  size_t lds, off_key, off_total, off_part, total;
};

size_t up256(size_t b) { return (b + 255) & ~(size_t)255; }

void embed_plan(int64_t n, int64_t R, int32_t C, EmbedPlan* p) {
  p->logP = 0;
  while (p->logP < 8 && (1 << p->logP) < R) ++p->logP;
  p->keys = (int)((R + (1 << p->logP) - 1) >> p->logP);
  p->lds = ((size_t)p->keys + 2 * kSortChunk) * sizeof(int);
  p->J = 32;
  p->jobs = (int)((n + p->J - 1) / p->J);
  p->off_key = up256((size_t)n * 4);
  p->off_total = p->off_key + up256((size_t)n * 4);
  p->off_part = p->off_total + 256;
  p->total = p->off_part + (size_t)p->jobs * 2 * (size_t)C * 4;
}

template <typename T, typename ID>
hipError_t embed_rows(const void* E, int64_t R, int64_t ldE, const void* ids, int64_t id_stride,
                      int64_t n, int32_t C, float scale, const void* add, int64_t ldadd, void* out,
                      int64_t ldout, hipStream_t stream) {
  const int nvec = (C + Row<T>::N - 1) / Row<T>::N;
  auto go = [&](auto g) {
    constexpr int G = decltype(g)::value;
    const int64_t blocks = (n + 256 / G - 1) / (256 / G);
    embed_kernel<T, ID, G><<<(unsigned)blocks, 256, 0, stream>>>(
        static_cast<const T*>(E), R, ldE, static_cast<const ID*>(ids), id_stride, n, C, scale,
        static_cast<const T*>(add), ldadd, static_cast<T*>(out), ldout);
    return hipGetLastError();
  };
  if (nvec <= 16) return go(std::integral_constant<int, 16>{});
  if (nvec <= 64) return go(std::integral_constant<int, 64>{});
  return go(std::integral_constant<int, 256>{});
}

template <typename ID>
hipError_t embed_sort(const void* ids, int64_t id_stride, int64_t n, int64_t R, int pad,
                      const EmbedPlan& p, int32_t C, int clear, float* dE, int64_t ldE,
                      int32_t* order, int32_t* key_of, int32_t* total, hipStream_t stream) {
  // allow the large dynamic LDS allocation; once per instantiation
  static std::once_flag once;
  static hipError_t attr_err = hipSuccess;
  std::call_once(once, [&] {
    attr_err = hipFuncSetAttribute(
        reinterpret_cast<const void*>(embed_sort_kernel<ID>),
        hipFuncAttributeMaxDynamicSharedMemorySize,
        (int)(((kMaxEmbedRows >> 8) + 2 * kSortChunk) * sizeof(int)));
  });
  if (attr_err != hipSuccess) return attr_err;
  embed_sort_kernel<ID><<<1 << p.logP, kSortThreads, p.lds, stream>>>(
      static_cast<const ID*>(ids), id_stride, (int)n, (int)R, pad, p.logP, p.keys, C, clear, dE,
      ldE, order, key_of, total);
  return hipGetLastError();
}

template <typename T>
hipError_t embed_sum(const void* dY, int64_t lddy, const int32_t* order, const int32_t* key_of,
                     const int32_t* total, const EmbedPlan& p, int32_t C, float scale,
                     int accumulate, float* dE, int64_t ldE, float* part, hipStream_t stream) {
  const int nvec = (C + Row<T>::N - 1) / Row<T>::N;
  auto go = [&](auto g) {
    constexpr int G = decltype(g)::value;
    const dim3 grid((p.jobs + 256 / G - 1) / (256 / G), (nvec + G - 1) / G);
    embed_sum_kernel<T, G><<<grid, 256, 0, stream>>>(static_cast<const T*>(dY), lddy, order,
                                                     key_of, total, p.J, p.jobs, C, scale,
                                                     accumulate, dE, ldE, part);
    return hipGetLastError();
  };
  if (nvec <= 16) return go(std::integral_constant<int, 16>{});
  return go(std::integral_constant<int, 64>{});
}

}  // namespace

hipError_t launch_embed_rows(const void* E, int64_t R, int64_t ldE, const void* ids, int id64,
                             int64_t id_stride, int64_t n, int32_t C, float scale, const void* add,
                             int64_t ldadd, int is_bf16, void* out, int64_t ldout,
                             hipStream_t stream) {
  auto f = is_bf16 ? (id64 ? embed_rows<uint16_t, int64_t> : embed_rows<uint16_t, int32_t>)
                   : (id64 ? embed_rows<float, int64_t> : embed_rows<float, int32_t>);
  // a launch holds fewer than 2^32 threads: 2^22 rows of at most 256
  constexpr int64_t kMost = (int64_t)1 << 22;
  const int64_t e = is_bf16 ? 2 : 4;
  for (int64_t r0 = 0; r0 < n; r0 += kMost) {
    const void* a = add == nullptr ? nullptr : static_cast<const char*>(add) + r0 * ldadd * e;
    const hipError_t err =
        f(E, R, ldE, static_cast<const char*>(ids) + r0 * id_stride * (id64 ? 8 : 4), id_stride,
          std::min(kMost, n - r0), C, scale, a, ldadd, static_cast<char*>(out) + r0 * ldout * e,
          ldout, stream);
    if (err != hipSuccess) return err;
  }
  return hipSuccess;
}

size_t embed_rows_backward_workspace_bytes(int64_t n, int64_t R, int32_t C) {
  EmbedPlan p;
  embed_plan(n, R, C, &p);
  return p.total;
}

hipError_t launch_embed_rows_backward(const void* dY, int64_t lddy, const void* ids, int id64,
                                      int64_t id_stride, int64_t n, int64_t R, int32_t C,
                                      float scale, int64_t pad, int is_bf16, int accumulate,
                                      float* dE, int64_t ldE, void* ws, hipStream_t stream) {
  if (n == 0 && accumulate) return hipSuccess;
  EmbedPlan p;
  embed_plan(n, R, C, &p);
  char* b = static_cast<char*>(ws);
  int32_t* order = reinterpret_cast<int32_t*>(b);
  int32_t* key_of = reinterpret_cast<int32_t*>(b + p.off_key);
  int32_t* total = reinterpret_cast<int32_t*>(b + p.off_total);
  float* part = reinterpret_cast<float*>(b + p.off_part);
  const int pad32 = pad >= 0 && pad < R ? (int)pad : -1;
  hipError_t e = (id64 ? embed_sort<int64_t> : embed_sort<int32_t>)(
      ids, id_stride, n, R, pad32, p, C, !accumulate, dE, ldE, order, key_of, total, stream);
  if (e != hipSuccess || n == 0) return e;
  e = (is_bf16 ? embed_sum<uint16_t> : embed_sum<float>)(dY, lddy, order, key_of, total, p, C,
                                                          scale, accumulate, dE, ldE, part, stream);
  if (e != hipSuccess) return e;
  const dim3 grid(std::min(p.jobs, 1 << 14), (C + 255) / 256);
  embed_join_kernel<<<grid, 256, 0, stream>>>(key_of, total, p.J, p.jobs, C, scale, accumulate,
                                              part, dE, ldE);
  return hipGetLastError();
}

}  // namespace shc
