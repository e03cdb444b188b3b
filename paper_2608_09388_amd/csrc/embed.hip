// Embedding rows with scaling, and their gradient by sorted ids.
//
//   y[i] = scale * E[id_i] (+ add[i]);   an id outside [0, R) has no row
//   dE[r] = scale * sum over i with id_i = r (and r != pad) of dY[i]
//
// Forward: a gather bound by HBM.  G lanes share a row and walk its 16-byte
// vectors, 256 / G rows a workgroup (67,040 rows of 128 fp32 with an addend, table of
// 10,475: 15.3 us, 4.9 TB/s).
//
// Gradient of few positions (few_rows): one launch, embed_few_kernel; every position
// looks through the list for its id.  Of more: the positions are ordered by id, then
// added.
// 1. embed_split_kernel (past kDirectRows positions) cuts the list of ids into
//    chunks and orders each chunk's positions by bucket, id modulo 1024 (frequent
//    ids, often neighbours, then fall to different buckets): every wavefront
//    ranks 64 ids at a time by ten ballots over the bucket's bits.
// 2. embed_order_kernel, a workgroup a bucket, takes its segments of all chunks in
//    order (of few positions: the ids themselves), counts its ids and hands out
//    the places: wavefronts take a queue in LDS in shares and rank 64 positions at a
//    time by ballots over the ids' bits.  Its first place in the order is the number
//    of positions in buckets before it, which the chunks' offsets give without
//    communication.
// 3. embed_sum_kernel cuts the order into jobs of J positions, whatever the ids'
//    frequencies; lanes that share a job and a column range add each id's rows in
//    order.  A job takes the ids that begin in it, to their end; ids of many
//    positions are cut at the jobs' borders instead, their parts left in
//    the workspace.  Other workgroups of the launch clear the table rows of ids
//    without a position meanwhile.
// 4. embed_join_kernel adds the parts, in order.
// Every sum has an order that follows the ids and sizes alone: results repeat
// bit for bit.
//
// Measured: 16,384 rows of 4,096 bf16 into a table of 32,768, ids as frequent as
// words: 145 us, 4.6 TB/s over all (5, 8, 129 and 5 us: the sums and the clearing are
// bound by HBM, the rest by latency); 268,160 rows of 128 into 10,475: 34 us (5, 11,
// 17 and 3).  One id of very many positions is the worst: its bucket is one workgroup's
// (65,536 rows of 1,024, one id: 315 us).
#include <algorithm>
#include <mutex>

#include "row_ops.h"

namespace shc {
namespace {

using namespace rowops;
// G lanes share a row, with U vectors a lane in flight: of U rows where a row has at
// most G vectors (SHORT), of one row otherwise.
template <typename T, typename ID, int G, int U, bool SHORT>
__global__ __launch_bounds__(256) void embed_kernel(const T* __restrict__ E, int64_t R,
                                                    int64_t ldE, const ID* __restrict__ ids,
                                                    int64_t id_stride, int64_t n, int C,
                                                    float scale, const T* __restrict__ add,
                                                    int64_t ldadd, T* __restrict__ out,
                                                    int64_t ldout) {
  constexpr int N = Row<T>::N, ROWS = SHORT ? U : 1;
  const int lane = threadIdx.x % G;
  const int64_t row0 = ((int64_t)blockIdx.x * (256 / G) + threadIdx.x / G) * ROWS;
  if (row0 >= n) return;
  const int nvec = (C + N - 1) / N;
  int64_t id[ROWS];
#pragma unroll
  for (int u = 0; u < ROWS; ++u) id[u] = row0 + u < n ? (int64_t)ids[(row0 + u) * id_stride] : -1;
  for (int v0 = lane; v0 < nvec; v0 += SHORT ? G : G * U) {
    i32x4 e[U], a[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = SHORT ? u : 0, v = SHORT ? v0 : v0 + u * G;
      e[u] = a[u] = i32x4{};
      if (v < nvec && row0 + r < n) {
        if (add != nullptr) a[u] = load_vec(add + (row0 + r) * ldadd, v, C);
        if (id[r] >= 0 && id[r] < R) e[u] = load_vec(E + id[r] * ldE, v, C);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = SHORT ? u : 0, v = SHORT ? v0 : v0 + u * G;
      if (v < nvec && row0 + r < n) {
        const bool there = id[r] >= 0 && id[r] < R;
        float f[N], g[N];
        Row<T>::widen(e[u], f);
        Row<T>::widen(a[u], g);
#pragma unroll
        for (int k = 0; k < N; ++k)
          f[k] = add == nullptr ? f[k] * scale : there ? fmaf(f[k], scale, g[k]) : g[k];
        store_vec(out + (row0 + r) * ldout, v, C, Row<T>::narrow(f));
      }
    }
  }
}

constexpr int kRound = 1024;                           // segments of a round
constexpr int kQueuePer = 4;                           // positions a thread in LDS at a time
constexpr int kLogBuckets = 10, kBuckets = 1 << kLogBuckets;
constexpr uint32_t kCut = 0x80000000u;  // in key_of: an id whose run is cut at jobs' borders

typedef int i32x2 __attribute__((ext_vector_type(2)));

template <typename ID>
__device__ __forceinline__ int valid_id(const ID* ids, int64_t id_stride, int64_t i, int R,
                                        int pad) {
  const int64_t id = (int64_t)ids[i * id_stride];
  return id >= 0 && id < R && id != pad ? (int)id : -1;
}

__device__ __forceinline__ uint64_t lanes_below(int lane) { return (1ull << lane) - 1; }

// Inclusive sums over the lanes of a wavefront: shifts within 16 lanes, then the
// last lanes of 16 and of 32 handed on, all by DPP.
template <int CTRL, int ROWS>
__device__ __forceinline__ int shifted(int x) {
  return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xF, false);
}
__device__ __forceinline__ int wave_scan(int x) {
  x += shifted<0x111, 0xF>(x);  // row_shr 1, 2, 4, 8
  x += shifted<0x112, 0xF>(x);
  x += shifted<0x114, 0xF>(x);
  x += shifted<0x118, 0xF>(x);
  x += shifted<0x142, 0xA>(x);  // row_bcast 15, into rows 1 and 3
  x += shifted<0x143, 0xC>(x);  // row_bcast 31, into rows 2 and 3
  return x;
}

// Exclusive sums over the threads of W wavefronts; *total their sum.  wave_sum [W]
// is free on entry and on return.
template <int W>
__device__ __forceinline__ int block_scan(int mine, int* wave_sum, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int inc = wave_scan(mine);
  if (lane == 63) wave_sum[wave] = inc;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    const int s = wave_sum[w];
    before += w < wave ? s : 0;
    all += s;
  }
  __syncthreads();
  *total = all;
  return before + inc - mine;
}

// Chunk c's (id, position) by bucket, in order, to split[c * NT * PER + ...];
// where each bucket begins to offs[c][kBuckets + 1].
template <typename ID, int NT, int PER>
__global__ __launch_bounds__(NT) void embed_split_kernel(
    const ID* __restrict__ ids, int64_t id_stride, int64_t n, int R, int pad,
    i32x2* __restrict__ split, int32_t* __restrict__ offs) {
  constexpr int W = NT / 64, BPT = kBuckets / NT;  // wavefronts; buckets a thread
  constexpr int64_t CHUNK = NT * PER;
  extern __shared__ __align__(16) int hist[];  // [W][kBuckets]
  __shared__ int wave_sum[W];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t w0 = blockIdx.x * CHUNK + (int64_t)wave * 64 * PER;
  int id[PER], rank[PER];
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int64_t i = w0 + u * 64 + lane;
    id[u] = i < n ? valid_id(ids, id_stride, i, R, pad) : -1;
  }
  volatile int* mine = hist + wave * kBuckets;
  for (int b = lane; b < kBuckets / 4; b += 64)
    reinterpret_cast<i32x4*>(hist + wave * kBuckets)[b] = i32x4{};
  group_fence<64>();
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int b = id[u] & (kBuckets - 1);
    uint64_t same = __ballot(id[u] >= 0);
#pragma unroll
    for (int k = 0; k < kLogBuckets; ++k) {
      const uint64_t bit = __ballot((b >> k) & 1);
      same &= ((b >> k) & 1) ? bit : ~bit;
    }
    if (id[u] >= 0) {
      const int before = __popcll(same & lanes_below(lane));
      const int start = mine[b];
      rank[u] = start + before;
      if (before == 0) mine[b] = start + __popcll(same);
    }
    group_fence<64>();
  }
  __syncthreads();
  // bucket starts: a thread's BPT buckets, over the wavefronts
  int h[W][BPT], sum[BPT], all = 0;
#pragma unroll
  for (int e = 0; e < BPT; ++e) {
    sum[e] = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      h[w][e] = hist[w * kBuckets + tid * BPT + e];
      sum[e] += h[w][e];
    }
    all += sum[e];
  }
  int total;
  int at = block_scan<W>(all, wave_sum, &total);
  int32_t* o = offs + (int64_t)blockIdx.x * (kBuckets + 1);
  if (tid == 0) o[kBuckets] = total;
#pragma unroll
  for (int e = 0; e < BPT; ++e) {
    o[tid * BPT + e] = at;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      hist[w * kBuckets + tid * BPT + e] = at;
      at += h[w][e];
    }
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < PER; ++u)
    if (id[u] >= 0)
      split[blockIdx.x * CHUNK + mine[id[u] & (kBuckets - 1)] + rank[u]] =
          i32x2{id[u], (int)(w0 + u * 64 + lane)};
}

// Bucket p's positions by id.  Ids of the bucket: at most keys = ceil(R / kBuckets),
// below 2^key_bits, local number id >> kLogBuckets.  order, key_of, run_end [n]:
// position, id (with kCut where its positions are more than `most`) and the end of
// the id's run, at its places; present [kBuckets][words]: a bit for every id with a
// position; *total the number of positions with an id that counts.
// LDS: place[keys], end[keys], at[NT / 64][keys], the queue (local number,
// position), a round of segments.
template <typename ID, int NT, bool DIRECT>
__global__ __launch_bounds__(NT) void embed_order_kernel(
    const ID* __restrict__ ids, int64_t id_stride, int64_t n, int R, int pad, int keys,
    int key_bits, int most, const i32x2* __restrict__ split, const int32_t* __restrict__ offs,
    int chunks, int chunk, int32_t* __restrict__ order, uint32_t* __restrict__ key_of,
    int32_t* __restrict__ run_end, uint32_t* __restrict__ present, int words,
    int32_t* __restrict__ total) {
  extern __shared__ int smem[];
  constexpr int W = NT / 64, PER = kQueuePer, QUEUE = NT * PER, SEGS = kRound / NT;
  int* place = smem;
  int* end = place + keys;
  int* at = end + keys;  // a wavefront's places, then its next ones
  int* queue_key = at + W * keys;
  int* queue_pos = queue_key + QUEUE;
  int* seg_at = queue_pos + QUEUE;  // [kRound]: a segment's first entry
  int* seg_src = seg_at + kRound;    // and where it lies in its chunk
  __shared__ int wave_sum[W];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int p = blockIdx.x;

  // calls f(entries in the queue) for the bucket's entries, in order, a queue at
  // a time; below: the thread's positions in the buckets before
  int below = 0;
  auto each_queue = [&](auto&& f) {
    if constexpr (DIRECT) {
      for (int64_t c0 = 0; c0 < n; c0 += QUEUE) {
        int key[PER];
        uint64_t has[PER];
        int found = 0;
        const int64_t w0 = c0 + (int64_t)wave * 64 * PER;
#pragma unroll
        for (int u = 0; u < PER; ++u) {
          const int64_t i = w0 + u * 64 + lane;
          const int id = i < n ? valid_id(ids, id_stride, i, R, pad) : -1;
          const int b = id & (kBuckets - 1);
          below += id >= 0 && b < p;
          key[u] = id >= 0 && b == p ? id >> kLogBuckets : -1;
        }
#pragma unroll
        for (int u = 0; u < PER; ++u) {
          has[u] = __ballot(key[u] >= 0);
          found += __popcll(has[u]);
        }
        if (lane == 0) wave_sum[wave] = found;
        __syncthreads();
        int q = 0, entries = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) {
          q += w < wave ? wave_sum[w] : 0;
          entries += wave_sum[w];
        }
#pragma unroll
        for (int u = 0; u < PER; ++u) {
          if (key[u] >= 0) {
            const int s = q + __popcll(has[u] & lanes_below(lane));
            queue_key[s] = key[u];
            queue_pos[s] = (int)(w0 + u * 64 + lane);
          }
          q += __popcll(has[u]);
        }
        __syncthreads();
        f(entries);
        __syncthreads();
      }
    } else {
      for (int c0 = 0; c0 < chunks; c0 += kRound) {
        int from[SEGS], len[SEGS], sum = 0;
#pragma unroll
        for (int u = 0; u < SEGS; ++u) {
          const int c = c0 + tid * SEGS + u;
          from[u] = len[u] = 0;
          if (c < chunks) {
            const int32_t* o = offs + (int64_t)c * (kBuckets + 1) + p;
            from[u] = o[0];
            len[u] = o[1] - o[0];
          }
          below += from[u];
          sum += len[u];
        }
        int entries;
        int first = block_scan<W>(sum, wave_sum, &entries);
#pragma unroll
        for (int u = 0; u < SEGS; ++u) {
          seg_at[tid * SEGS + u] = first;
          seg_src[tid * SEGS + u] = from[u];
          first += len[u];
        }
        __syncthreads();
        for (int q0 = 0; q0 < entries; q0 += QUEUE) {
          const int take = min(QUEUE, entries - q0);
          // a thread's entries together: the last segment that begins at or before
          // each, by bisection, then their loads
          int s[PER] = {};
#pragma unroll
          for (int d = kRound / 2; d > 0; d >>= 1)
#pragma unroll
            for (int u = 0; u < PER; ++u)
              if (seg_at[s[u] + d] <= q0 + tid + u * NT) s[u] += d;
          i32x2 e[PER];
#pragma unroll
          for (int u = 0; u < PER; ++u) {
            const int i = tid + u * NT;
            if (i < take)
              e[u] = split[(int64_t)(c0 + s[u]) * chunk + seg_src[s[u]] + (q0 + i - seg_at[s[u]])];
          }
#pragma unroll
          for (int u = 0; u < PER; ++u) {
            const int i = tid + u * NT;
            if (i < take) {
              queue_key[i] = e[u][0] >> kLogBuckets;
              queue_pos[i] = e[u][1];
            }
          }
          __syncthreads();
          f(take);
          __syncthreads();
        }
      }
    }
  };
  // a wavefront's share of a queue: consecutive blocks of 64
  auto share = [&](int entries, int* lo, int* hi) {
    const int blocks = (entries + 63) / 64, each = (blocks + W - 1) / W;
    *lo = min(entries, wave * each * 64);
    *hi = min(entries, (wave + 1) * each * 64);
  };
  auto count_queue = [&](int entries) {
    int lo, hi;
    share(entries, &lo, &hi);
    // lanes with the first one's id count as one: of a frequent id that is most, and
    // additions to one address go one after the other
    for (int i = lo + lane; i < hi; i += 64) {
      const int k = queue_key[i], first = __builtin_amdgcn_readfirstlane(k);
      const uint64_t same = __ballot(k == first);
      if (k != first)
        atomicAdd(&at[wave * keys + k], 1);
      else if ((same & lanes_below(lane)) == 0)
        atomicAdd(&at[wave * keys + k], __popcll(same));
    }
  };

  for (int k = tid; k < (2 + W) * keys; k += NT) smem[k] = 0;
  __syncthreads();
  // counts, and the first place: positions of the buckets before
  int held = 0, queues = 0;
  each_queue([&](int entries) {
    count_queue(entries);
    held += entries;
    ++queues;
  });
  int base;
  block_scan<W>(below, wave_sum, &base);
  for (int k = tid; k < keys; k += NT)
#pragma unroll
    for (int w = 0; w < W; ++w) place[k] += at[w * keys + k];
  __syncthreads();

  // ids present, 64 a wavefront at a time
  for (int k0 = wave * 64; k0 < words * 32; k0 += NT) {
    const uint64_t bits = __ballot(k0 + lane < keys && place[min(k0 + lane, keys - 1)] != 0);
    if (lane < 2 && k0 / 32 + lane < words)
      present[(int64_t)p * words + k0 / 32 + lane] = (uint32_t)(bits >> (32 * lane));
  }
  if (p == kBuckets - 1 && tid == 0) *total = base + held;
  if (held == 0) return;  // the whole workgroup

  // counts -> first places (with the cut bit where the id is long) and ends:
  // consecutive ids per thread, their sums scanned
  const int per = (keys + NT - 1) / NT;
  const int k0 = min(keys, tid * per), k1 = min(keys, k0 + per);
  __syncthreads();
  int mine = 0, all;
  for (int k = k0; k < k1; ++k) mine += place[k];
  int next = base + block_scan<W>(mine, wave_sum, &all);
  for (int k = k0; k < k1; ++k) {
    const int c = place[k];
    place[k] = next | (c > most ? (int)kCut : 0);
    next += c;
    end[k] = next;
  }
  __syncthreads();

  // places: a wavefront's blocks of 64 entries of the queue in order, every entry
  // ranked among the block's of its id by ballots over the id's bits
  auto hand_out = [&](int entries) {
    // the wavefronts' counts -> their first places; place: the next queue's
    for (int k = tid; k < keys; k += NT) {
      int to = place[k];
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const int c = at[w * keys + k];
        at[w * keys + k] = to;
        to += c;
      }
      place[k] = to;
    }
    __syncthreads();
    int lo, hi;
    share(entries, &lo, &hi);
    volatile int* mine_at = at + wave * keys;
    for (int q0 = lo; q0 < hi; q0 += 64) {
      const bool in = q0 + lane < hi;
      const int k = in ? queue_key[q0 + lane] : 0;
      uint64_t same = __ballot(in);
      for (int b = 0; b < key_bits; ++b) {
        const uint64_t bit = __ballot((k >> b) & 1);
        same &= ((k >> b) & 1) ? bit : ~bit;
      }
      if (in) {
        const int to = mine_at[k];
        const int before = __popcll(same & lanes_below(lane));
        if (before == 0) mine_at[k] = to + __popcll(same);
        const int s = (to & (int)~kCut) + before;
        order[s] = queue_pos[q0 + lane];
        key_of[s] = (uint32_t)((k << kLogBuckets) + p) | ((uint32_t)to & kCut);
        run_end[s] = end[k];
      }
      group_fence<64>();
    }
  };
  if (queues == 1) {
    hand_out(held);  // the queue and its counts are there
  } else {
    each_queue([&](int entries) {
      for (int k = tid; k < W * keys; k += NT) at[k] = 0;
      __syncthreads();
      count_queue(entries);
      __syncthreads();
      hand_out(entries);
    });
  }
}

// 4 zeros of a row, `past` the caches or not.
__device__ __forceinline__ void clear_vec(float* row, int v, int C, int past) {
  const float z[4] = {0.f, 0.f, 0.f, 0.f};
  if (past)
    store_channels<4, true>(row, v, C, z);
  else
    store_channels<4>(row, v, C, z);
}

// Few positions in one launch.  A workgroup of [0, sums) takes a position and a range
// of 64 vectors, and wavefront w the positions [64 M w, 64 M (w + 1)) of the same id,
// found by ballots; where the position is the id's first, each adds its rows in
// order, and their sums are added in order.  The others clear the table rows of ids
// without a position, `rows` at a time.  Into a table of 5,000: 64 rows of 1,024 bf16
// 6.4 us, by the launches below 13.8; 512 rows 7.9, 18.0 (one id throughout: 13.9,
// 17.4).
constexpr int kFewThreads = 512;
template <typename T, typename ID, int M>
__global__ __launch_bounds__(kFewThreads) void embed_few_kernel(
    const T* __restrict__ dY, int64_t lddy, const ID* __restrict__ ids, int64_t id_stride, int n,
    int R, int pad, int sums, int rows, int past, int C, float scale, int accumulate,
    float* __restrict__ dE, int64_t ldE) {
  constexpr int N = Row<T>::N, U = 8, W = kFewThreads / 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int mine[M];
#pragma unroll
  for (int m = 0; m < M; ++m) {
    const int i = (wave * M + m) * 64 + lane;
    mine[m] = i < n ? valid_id(ids, id_stride, i, R, pad) : -1;
  }
  if ((int)blockIdx.x >= sums) {
    __shared__ uint32_t there[2 * W];  // a bit a row
    const int nv = (C + 3) / 4;
    int wide = 64;
    while (wide > 1 && wide / 2 >= nv) wide /= 2;
    const int step = (gridDim.x - sums) * rows;
    for (int r0 = (blockIdx.x - sums) * rows; r0 < R; r0 += step) {
      if (threadIdx.x < 2 * W) there[threadIdx.x] = 0;
      __syncthreads();
#pragma unroll
      for (int m = 0; m < M; ++m) {
        const int at = mine[m] - r0;
        if (mine[m] >= 0 && at >= 0 && at < rows) atomicOr(&there[at >> 5], 1u << (at & 31));
      }
      __syncthreads();
      const int end = min(rows, R - r0);
      for (int i = threadIdx.x / wide; i < end; i += kFewThreads / wide)
        if (!((there[i >> 5] >> (i & 31)) & 1))
          for (int v = lane % wide; v < nv; v += wide)
            clear_vec(dE + (int64_t)(r0 + i) * ldE, v, C, past);
      __syncthreads();
    }
    return;
  }
  __shared__ int some[W];
  __shared__ f32x4 sum[W > 1 ? W - 1 : 1][N / 4][64];
  const int tiles = ((C + N - 1) / N + 63) / 64;
  const int i = blockIdx.x / tiles, v = blockIdx.x % tiles * 64 + lane;
  const int key = valid_id(ids, id_stride, i, R, pad);
  uint64_t same[M];
  int begin = n;  // the wavefront's first position of that id
#pragma unroll
  for (int m = M - 1; m >= 0; --m) {
    same[m] = __ballot(mine[m] >= 0 && mine[m] == key);
    if (same[m] != 0)
      begin = (wave * M + m) * 64 + __ffsll((unsigned long long)same[m]) - 1;
  }
  if (lane == 0) some[wave] = begin;
  __syncthreads();
  int first = n;
#pragma unroll
  for (int w = W - 1; w >= 0; --w)
    if (some[w] < n) first = some[w];
  if (first != i) return;  // the whole workgroup
  float acc[N];
#pragma unroll
  for (int e = 0; e < N; ++e) acc[e] = 0.f;
#pragma unroll
  for (int m = 0; m < M; ++m) {
    while (same[m] != 0) {
      i32x4 raw[U];
      int count = 0;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        raw[u] = i32x4{};
        if (same[m] != 0) {
          const int64_t at = (wave * M + m) * 64 + __ffsll((unsigned long long)same[m]) - 1;
          same[m] &= same[m] - 1;
          if (v * N < C) raw[u] = load_vec(dY + at * lddy, v, C);
          ++count;
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float f[N];
        Row<T>::widen(raw[u], f);
#pragma unroll
        for (int e = 0; e < N; ++e) acc[e] = u < count ? acc[e] + f[e] : acc[e];
      }
    }
  }
  if (wave > 0) {
#pragma unroll
    for (int e = 0; e < N; e += 4)
      sum[wave - 1][e / 4][lane] = f32x4{acc[e], acc[e + 1], acc[e + 2], acc[e + 3]};
  }
  __syncthreads();
  if (wave > 0 || v * N >= C) return;
#pragma unroll
  for (int w = 1; w < W; ++w)
    if (some[w] < n) {
#pragma unroll
      for (int e = 0; e < N; ++e) acc[e] += sum[w - 1][e / 4][lane][e % 4];
    }
  float* to = dE + (int64_t)key * ldE;
  float f[N];
  if (accumulate) load_channels<N>(to, v, C, f);
#pragma unroll
  for (int e = 0; e < N; ++e) f[e] = accumulate ? fmaf(acc[e], scale, f[e]) : acc[e] * scale;
  store_channels<N>(to, v, C, f);
}

// Workgroups [0, sums): jobs of J positions, G lanes each, by column ranges of
// G vectors.  part [jobs][2][C]: of a cut id that began in an earlier job, what
// this job adds (slot 0); of one that goes on in the next job, what this one, in
// which it began, adds (slot 1).  A job takes fewer than 3 J positions: its own,
// and the rest of an id that begins in it (of 2 J at most where it is not cut).
// The others clear the table rows of the ids without a position.
template <typename T, int G, int J>
__global__ __launch_bounds__(256) void embed_sum_kernel(
    const T* __restrict__ dY, int64_t lddy, int64_t n, const int32_t* __restrict__ order,
    const uint32_t* __restrict__ key_of, const int32_t* __restrict__ run_end,
    const uint32_t* __restrict__ present, int words, const int32_t* __restrict__ total, int jobs,
    int sums, int clear, int past, int R, int C, float scale, int accumulate,
    float* __restrict__ dE, int64_t ldE, float* __restrict__ part,
    int32_t* __restrict__ begins) {
  constexpr int N = Row<T>::N, U = 8, TAKE = 3 * J;
  __shared__ __align__(16) int pos_sh[256 / G][TAKE];
  __shared__ __align__(16) uint32_t key_sh[256 / G][TAKE];
  if ((int)blockIdx.x >= sums) {
    // a wavefront clears `clear` rows at a time (up to 64), its lanes looking up
    // one each; rows shorter than 64 vectors several together
    const int lane = threadIdx.x & 63;
    const int nv = (C + 3) / 4;
    int wide = 64;
    while (wide > 1 && wide / 2 >= nv) wide /= 2;
    const int step = (gridDim.x - sums) * 4 * clear;
    for (int r0 = ((blockIdx.x - sums) * 4 + (threadIdx.x >> 6)) * clear; r0 < R; r0 += step) {
      const int r = r0 + lane, k = r >> kLogBuckets;
      bool none = false;
      if (lane < clear && r < R)
        none = !((present[(int64_t)(r & (kBuckets - 1)) * words + (k >> 5)] >> (k & 31)) & 1);
      const uint64_t rows = __ballot(none);
      for (int i = lane / wide; i < clear; i += 64 / wide)
        if ((rows >> i) & 1)
          for (int v = lane % wide; v < nv; v += wide)
            clear_vec(dE + (int64_t)(r0 + i) * ldE, v, C, past);
    }
    return;
  }
  const int tiles = ((C + N - 1) / N + G - 1) / G;
  const int group = threadIdx.x / G, lane = threadIdx.x % G;
  int j = (blockIdx.x / tiles) * (256 / G) + group;
  if constexpr (G == 64) j = __builtin_amdgcn_readfirstlane(j);
  const int v = (blockIdx.x % tiles) * G + lane;
  if (j >= jobs) return;
  // everything the job may need at once: places past the total hold anything
  int lo = j * J;
  const int64_t next = min((int64_t)lo + J, n);
  const int m = *total;
  uint32_t key = key_of[lo];
  const uint32_t before = lo > 0 ? key_of[lo - 1] : ~0u;
  const int first_end = run_end[lo];
  uint32_t last = key_of[next - 1];
  int last_end = run_end[next - 1];
  const uint32_t after = next < n ? key_of[next] : ~0u;
  int* pos = pos_sh[group];
  uint32_t* keys = key_sh[group];
#pragma unroll
  for (int i = 0; i < (TAKE + G - 1) / G; ++i) {
    const int t = i * G + lane;
    if (t < TAKE && lo + t < n) {
      pos[t] = order[lo + t];
      keys[t] = key_of[lo + t];
    }
  }
  if (v == 0) begins[j] = 0;  // the last job of a cut id that begins here; none yet
  group_fence<64>();
  if (lo >= m) return;
  int hi = (int)next;
  if (hi > m) {
    hi = m;
    last = key_of[m - 1];
    last_end = run_end[m - 1];
  }
  const int lo0 = lo;
  bool from_before = before == key;
  if (from_before && !(key & kCut)) {  // an earlier job takes it to its end
    lo = first_end;
    if (lo >= hi) return;
    key = keys[lo - lo0];
    from_before = false;
  }
  const bool goes_on = (last & kCut) && hi < m && after == last;
  if (!(last & kCut)) hi = last_end;
  if (v * N >= C) return;

  float acc[N];
#pragma unroll
  for (int e = 0; e < N; ++e) acc[e] = 0.f;
  auto put = [&](bool to_next) {
    if (from_before || to_next) {
      store_channels<N>(part + ((int64_t)j * 2 + (from_before ? 0 : 1)) * C, v, C, acc);
    } else {
      float* to = dE + (int64_t)(key & ~kCut) * ldE;
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
  for (int t0 = lo - lo0; t0 < hi - lo0; t0 += U) {
    i32x4 raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = min(t0 + u, hi - lo0 - 1);
      raw[u] = load_vec(dY + (int64_t)pos[t] * lddy, v, C);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (t0 + u < hi - lo0) {
        if (keys[t0 + u] != key) {
          put(false);
          key = keys[t0 + u];
        }
        float f[N];
        Row<T>::widen(raw[u], f);
#pragma unroll
        for (int e = 0; e < N; ++e) acc[e] += f[e];
      }
    }
  }
  if (goes_on && !from_before && v == 0) begins[j] = (last_end - 1) / J;
  put(goes_on);
}

// The parts of the cut ids that begin in jobs [blockIdx.x * range, + range): slot 1 of
// the job, then slot 0 of the jobs after it up to the last with that id.  L lanes hold
// four columns each.  Ids of up to kShortParts parts are taken by a group of L lanes
// each, in order; of longer ones the workgroup's groups take the parts in turn, each
// adding its own in order, and the groups are added in order.  16,384 rows of 4,096:
// 4.7 us; 400,000 rows of 64 on 10,475 ids, all of which are cut in two or three: 43
// us in all, 111 where a whole workgroup took each.
constexpr int kJoinThreads = 512, kJoinRange = 64, kShortParts = 8;
template <int L>
__global__ __launch_bounds__(kJoinThreads) void embed_join_kernel(
    const uint32_t* __restrict__ key_of, const int32_t* __restrict__ begins, int J, int jobs,
    int range, int C, float scale, int accumulate, const float* __restrict__ part,
    float* __restrict__ dE, int64_t ldE) {
  constexpr int SHARES = kJoinThreads / L, U = 8;
  __shared__ f32x4 sum[SHARES][L];
  __shared__ int from_job[2][kJoinRange], to_job[2][kJoinRange];
  // every wavefront looks through the jobs, a lane each
  const int wlane = threadIdx.x & 63, j0 = blockIdx.x * range;
  const int last = wlane < range && j0 + wlane < jobs ? begins[j0 + wlane] : 0;
  const bool is_long = last - (j0 + wlane) > kShortParts;
  const uint64_t some[2] = {__ballot(last != 0 && !is_long), __ballot(last != 0 && is_long)};
  if ((some[0] | some[1]) == 0) return;  // the whole workgroup
  if (threadIdx.x < 64 && last != 0) {
    const int at = __popcll((is_long ? some[1] : some[0]) & lanes_below(wlane));
    from_job[is_long][at] = j0 + wlane;
    to_job[is_long][at] = last;
  }
  __syncthreads();
  const int lane = threadIdx.x % L, share = threadIdx.x / L;
  const int v = blockIdx.y * L + lane;
  const int64_t step = (int64_t)2 * C;
  const float* from = part + (int64_t)v * 4;
  float acc[4], f[4];
  // acc += slot 0 of jobs q, q + by, ... up to the last
  auto add = [&](int q, int to, int by) {
    if (v * 4 + 4 <= C) {  // U parts in flight
      for (; q + (U - 1) * by <= to; q += U * by) {
        f32x4_a4 x[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
          x[u] = *reinterpret_cast<const f32x4_a4*>(from + (q + u * by) * step);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[e] += x[u][e];
      }
    }
#pragma unroll 4
    for (; q <= to; q += by) {
      load_channels<4>(part + q * step, v, C, f);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] += f[e];
    }
  };
  auto put = [&](int j) {
    float* to = dE + (int64_t)(key_of[(int64_t)(j + 1) * J] & ~kCut) * ldE;
    if (accumulate) load_channels<4>(to, v, C, f);
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = accumulate ? fmaf(acc[e], scale, f[e]) : acc[e] * scale;
    store_channels<4>(to, v, C, f);
  };
  if (v * 4 < C) {
    for (int i = share; i < __popcll(some[0]); i += SHARES) {
      const int j = from_job[0][i];
      load_channels<4>(part + j * step + C, v, C, acc);
      add(j + 1, to_job[0][i], 1);
      put(j);
    }
  }
  for (int i = 0; i < __popcll(some[1]); ++i) {
    const int j = from_job[1][i];
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] = 0.f;
    if (v * 4 < C) {
      if (share == 0) load_channels<4>(part + j * step + C, v, C, acc);
      add(j + 1 + share, to_job[1][i], SHARES);
    }
    sum[share][lane] = f32x4{acc[0], acc[1], acc[2], acc[3]};
    __syncthreads();
    if (share == 0 && v * 4 < C) {
#pragma unroll 8
      for (int q = 1; q < SHARES; ++q)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] += sum[q][lane][e];
      put(j);
    }
    __syncthreads();
  }
}

// Positions up to which every bucket reads the ids itself: one launch less (1,024
// rows of 5,000 bf16: 34.8 us, 40.0 with the split; 2,048: 42.9, 45.6).
constexpr int64_t kDirectRows = 2048;
// Positions from which a chunk is 4096 of them, split by 1024 threads, not 1024 by 512:
// fewer, longer segments (1,340,800 rows of 64 bf16 took 20 us less; 268,160 29.4 us,
// 32.3 with long chunks).
constexpr int64_t kWideRows = 524288;

// Positions from which a bucket is ordered by 512 threads, a queue of 2,048 at a time:
// frequent ids' buckets are the last to end (268,160 rows of 64 bf16, ids as frequent
// as words: 75 us, 105 by 256 threads; evenly, 32.1, 33.2; 16,384: 30.6, 30.0 and 22.4,
// 22.1).  Up to kWideKeys ids a bucket: the counts of each wavefront fit LDS.
constexpr int64_t kWideOrder = 32768;
constexpr int kWideThreads = 512, kWideKeys = 1024;
constexpr size_t order_lds(int threads, int keys) {
  return ((2 + threads / 64) * (size_t)keys + 2 * kQueuePer * threads + 2 * kRound) * sizeof(int);
}

// Workspace: what the launches leave each other.
struct EmbedPlan {
  int keys, key_bits, words, chunk, chunks, J, jobs, order_threads;
  size_t off_key, off_end, off_present, off_total, off_begins, off_split, off_offs, off_part, total;
};

// Positions of a job; an id of more than 2 J is cut.  Short jobs where there are
// few wavefronts (16,384 rows of 64 bf16: 31 us with 8, 33 with 16, 43 with 32),
// long ones where the parts' traffic counts (of 4,096: 160, 153, 150).
constexpr int64_t kJobs16 = 32768, kJobs32 = 131072;  // wavefronts of one position each, about
[[nodiscard]] int job_rows(int64_t n, int32_t C) {
  const int64_t w = n * C >> 9;
  return w >= kJobs32 ? 32 : w >= kJobs16 ? 16 : 8;
}
[[nodiscard]] int job_count(int64_t n, int32_t C) {
  const int J = job_rows(n, C);
  return (int)((n + J - 1) / J);
}
[[nodiscard]] int chunk_rows(int64_t n) { return n < kWideRows ? 1024 : 4096; }
[[nodiscard]] int chunk_count(int64_t n) {
  return n > kDirectRows ? (int)((n + chunk_rows(n) - 1) / chunk_rows(n)) : 0;
}

size_t up256(size_t b) { return (b + 255) & ~(size_t)255; }

// The workspace of n positions serves any smaller number too: every part of it has
// the size that the number up to n with the most jobs, or chunks, needs.
void embed_plan(int64_t n, int64_t R, int32_t C, EmbedPlan* p) {
  p->keys = (int)((R + kBuckets - 1) >> kLogBuckets);
  p->key_bits = 0;
  while ((1 << p->key_bits) < p->keys) ++p->key_bits;
  p->words = (p->keys + 31) / 32;
  p->order_threads = n >= kWideOrder && p->keys <= kWideKeys ? kWideThreads : 256;
  p->chunk = chunk_rows(n);
  p->chunks = chunk_count(n);
  p->J = job_rows(n, C);
  p->jobs = job_count(n, C);
  // the largest counts below the changes of rule
  const int64_t most_chunks = std::max(p->chunks, chunk_count(std::min(n, kWideRows - 1)));
  int64_t most_jobs = p->jobs;
  for (const int64_t w : {kJobs16, kJobs32})
    most_jobs = std::max<int64_t>(most_jobs, job_count(std::min(n, ((w << 9) - 1) / C), C));
  size_t at = 0;
  auto place = [&](size_t bytes) {
    const size_t here = at;
    at += up256(bytes);
    return here;
  };
  place((size_t)n * 4);  // order
  p->off_key = place((size_t)n * 4);
  p->off_end = place((size_t)n * 4);
  p->off_present = place((size_t)kBuckets * p->words * 4);
  p->off_total = place(4);
  p->off_begins = place((size_t)most_jobs * 4);
  p->off_split = place((size_t)p->chunks * p->chunk * 8);
  p->off_offs = place((size_t)most_chunks * (kBuckets + 1) * 4);
  p->off_part = place((size_t)most_jobs * 2 * (size_t)C * 4);
  p->total = at;
}

template <typename T, typename ID>
hipError_t embed_rows(const void* E, int64_t R, int64_t ldE, const void* ids, int64_t id_stride,
                      int64_t n, int32_t C, float scale, const void* add, int64_t ldadd, void* out,
                      int64_t ldout, hipStream_t stream) {
  const int nvec = (C + Row<T>::N - 1) / Row<T>::N;
  auto go = [&](auto g, auto u, auto is_short) {
    constexpr int G = decltype(g)::value, U = decltype(u)::value;
    constexpr bool SHORT = decltype(is_short)::value;
    constexpr int ROWS = 256 / G * (SHORT ? U : 1);
    embed_kernel<T, ID, G, U, SHORT><<<(unsigned)((n + ROWS - 1) / ROWS), 256, 0, stream>>>(
        static_cast<const T*>(E), R, ldE, static_cast<const ID*>(ids), id_stride, n, C, scale,
        static_cast<const T*>(add), ldadd, static_cast<T*>(out), ldout);
    return hipGetLastError();
  };
  // two vectors a lane in flight (67,040 rows of 128 fp32 with an addend: 15.5 us;
  // one 16.0, four 20.1)
  using std::integral_constant;
  integral_constant<int, 2> two;
  if (nvec <= 8) return go(integral_constant<int, 8>{}, two, std::true_type{});
  if (nvec <= 16) return go(integral_constant<int, 16>{}, two, std::true_type{});
  if (nvec <= 32) return go(integral_constant<int, 32>{}, two, std::true_type{});
  if (nvec <= 64) return go(integral_constant<int, 64>{}, two, std::true_type{});
  if (nvec <= 128) return go(integral_constant<int, 64>{}, two, std::false_type{});
  return go(integral_constant<int, 256>{}, two, std::false_type{});
}

struct EmbedWork {
  EmbedPlan p;
  int32_t *order, *run_end, *total, *begins, *offs;
  uint32_t *key_of, *present;
  i32x2* split;
  float* part;
};

template <typename ID>
hipError_t embed_order(const void* ids, int64_t id_stride, int64_t n, int64_t R, int pad,
                       const EmbedWork& w, hipStream_t stream) {
  // allow the large dynamic LDS allocation; once per instantiation
  static std::once_flag once;
  static hipError_t attr_err = hipSuccess;
  constexpr int kMostKeys = kMaxEmbedRows >> kLogBuckets;
  std::call_once(once, [&] {
    auto allow = [&](const void* kernel, size_t bytes) {
      if (attr_err == hipSuccess)
        attr_err = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize,
                                       (int)bytes);
    };
    allow(reinterpret_cast<const void*>(embed_split_kernel<ID, 1024, 4>),
          16 * kBuckets * sizeof(int));
    allow(reinterpret_cast<const void*>(embed_order_kernel<ID, 256, true>),
          order_lds(256, kMostKeys));
    allow(reinterpret_cast<const void*>(embed_order_kernel<ID, 256, false>),
          order_lds(256, kMostKeys));
    allow(reinterpret_cast<const void*>(embed_order_kernel<ID, kWideThreads, false>),
          order_lds(kWideThreads, kWideKeys));
  });
  if (attr_err != hipSuccess) return attr_err;
  const ID* in = static_cast<const ID*>(ids);
  if (w.p.chunks > 0) {
    // two ids a thread of 512: 268,160 ids 5.3 us, four of 256 6.1
    if (w.p.chunk == 1024)
      embed_split_kernel<ID, 512, 2><<<w.p.chunks, 512, 8 * kBuckets * sizeof(int), stream>>>(
          in, id_stride, n, (int)R, pad, w.split, w.offs);
    else
      embed_split_kernel<ID, 1024, 4><<<w.p.chunks, 1024, 16 * kBuckets * sizeof(int), stream>>>(
          in, id_stride, n, (int)R, pad, w.split, w.offs);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  auto order = [&](auto kernel) {
    kernel<<<kBuckets, w.p.order_threads, order_lds(w.p.order_threads, w.p.keys), stream>>>(
        in, id_stride, n, (int)R, pad, w.p.keys, w.p.key_bits, 2 * w.p.J, w.split, w.offs,
        w.p.chunks, w.p.chunk, w.order, w.key_of, w.run_end, w.present, w.p.words, w.total);
    return hipGetLastError();
  };
  if (w.p.chunks == 0) return order(embed_order_kernel<ID, 256, true>);
  return w.p.order_threads == 256 ? order(embed_order_kernel<ID, 256, false>)
                                  : order(embed_order_kernel<ID, kWideThreads, false>);
}

// Rows that a wavefront clears at a time, about 16 KB of them.
int clear_rows(int32_t C) { return std::max(1, std::min(64, 4096 / C)); }
// Whether the cleared rows go past the caches: where the table does not fit the
// Infinity Cache, so that dY may stay there (4,096 rows, table of 32,768 x 4,096:
// 113 us, 133 through the caches; of 64 rows: 107, 103).
int clear_past(int64_t R, int32_t C) { return R * C >= (int64_t)1 << 26; }

// Whether one launch does it: a position's workgroups, one for each range of columns,
// look through the whole list, so that the work grows with the positions' square
// (5,000 ids, bf16: 1,024 rows of 2,000 take 17.1 us, by the launches below 20.2; 2,048
// rows of 500 10.6, 24.2, of 2,000 30.2, 25.3; 1,186 of 2,345 27.9, 24.6).  One id
// throughout is the worst of it: 2,048 rows of 64 take 40 us, 26.
constexpr int kFewMost = 4 * kFewThreads;
bool few_rows(int64_t n, int32_t C, int is_bf16) {
  const int per = is_bf16 ? 512 : 256;
  return n <= kFewThreads || (n <= kFewMost && n * ((C + per - 1) / per) <= 5120);
}

template <typename T, typename ID>
hipError_t embed_few(const void* dY, int64_t lddy, const void* ids, int64_t id_stride, int64_t n,
                     int64_t R, int pad, int32_t C, float scale, int accumulate, float* dE,
                     int64_t ldE, hipStream_t stream) {
  const int tiles = ((C + Row<T>::N - 1) / Row<T>::N + 63) / 64;
  const int sums = (int)n * tiles, rows = kFewThreads / 64 * clear_rows(C);
  const int clears = accumulate ? 0 : (int)std::min<int64_t>((R + rows - 1) / rows, 16384);
  if (sums + clears == 0) return hipSuccess;
  auto go = [&](auto m) {
    embed_few_kernel<T, ID, decltype(m)::value><<<sums + clears, kFewThreads, 0, stream>>>(
        static_cast<const T*>(dY), lddy, static_cast<const ID*>(ids), id_stride, (int)n, (int)R,
        pad, sums, rows, clear_past(R, C), C, scale, accumulate, dE, ldE);
    return hipGetLastError();
  };
  if (n <= kFewThreads) return go(std::integral_constant<int, 1>{});
  if (n <= 2 * kFewThreads) return go(std::integral_constant<int, 2>{});
  return go(std::integral_constant<int, 4>{});
}

template <typename T>
hipError_t embed_sum(const void* dY, int64_t lddy, int64_t n, int64_t R, const EmbedWork& w,
                     int32_t C, float scale, int accumulate, float* dE, int64_t ldE,
                     hipStream_t stream) {
  const int nvec = (C + Row<T>::N - 1) / Row<T>::N;
  auto go = [&](auto g, auto job) {
    constexpr int G = decltype(g)::value, J = decltype(job)::value;
    const int sums = (w.p.jobs + 256 / G - 1) / (256 / G) * ((nvec + G - 1) / G);
    const int clear = clear_rows(C);
    const int clears =
        accumulate ? 0 : (int)std::min<int64_t>((R + 4 * clear - 1) / (4 * clear), 16384);
    const int past = clear_past(R, C);
    if (sums + clears == 0) return hipSuccess;
    embed_sum_kernel<T, G, J><<<sums + clears, 256, 0, stream>>>(
        static_cast<const T*>(dY), lddy, n, w.order, w.key_of, w.run_end, w.present, w.p.words,
        w.total, w.p.jobs, sums, clear, past, (int)R, C, scale, accumulate, dE, ldE, w.part,
        w.begins);
    return hipGetLastError();
  };
  using std::integral_constant;
  auto lanes = [&](auto job) {
    if (nvec <= 8) return go(integral_constant<int, 8>{}, job);
    if (nvec <= 16) return go(integral_constant<int, 16>{}, job);
    if (nvec <= 32) return go(integral_constant<int, 32>{}, job);
    return go(integral_constant<int, 64>{}, job);
  };
  if (w.p.J == 8) return lanes(integral_constant<int, 8>{});
  if (w.p.J == 16) return lanes(integral_constant<int, 16>{});
  return lanes(integral_constant<int, 32>{});
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
  const int pad32 = pad >= 0 && pad < R ? (int)pad : -1;
  if (few_rows(n, C, is_bf16)) {
    auto few = is_bf16 ? (id64 ? embed_few<uint16_t, int64_t> : embed_few<uint16_t, int32_t>)
                       : (id64 ? embed_few<float, int64_t> : embed_few<float, int32_t>);
    return few(dY, lddy, ids, id_stride, n, R, pad32, C, scale, accumulate, dE, ldE, stream);
  }
  EmbedWork w;
  embed_plan(n, R, C, &w.p);
  char* b = static_cast<char*>(ws);
  w.order = reinterpret_cast<int32_t*>(b);
  w.key_of = reinterpret_cast<uint32_t*>(b + w.p.off_key);
  w.run_end = reinterpret_cast<int32_t*>(b + w.p.off_end);
  w.present = reinterpret_cast<uint32_t*>(b + w.p.off_present);
  w.total = reinterpret_cast<int32_t*>(b + w.p.off_total);
  w.begins = reinterpret_cast<int32_t*>(b + w.p.off_begins);
  w.split = reinterpret_cast<i32x2*>(b + w.p.off_split);
  w.offs = reinterpret_cast<int32_t*>(b + w.p.off_offs);
  w.part = reinterpret_cast<float*>(b + w.p.off_part);
  hipError_t e = (id64 ? embed_order<int64_t> : embed_order<int32_t>)(ids, id_stride, n, R, pad32,
                                                                      w, stream);
  if (e != hipSuccess) return e;
  e = (is_bf16 ? embed_sum<uint16_t> : embed_sum<float>)(dY, lddy, n, R, w, C, scale, accumulate,
                                                         dE, ldE, stream);
  if (e != hipSuccess) return e;
  auto join = [&](auto l) {
    constexpr int L = decltype(l)::value;
    const int tiles = (C + 4 * L - 1) / (4 * L);
    // few idle wavefronts, and few long ids one after the other: 2,048 workgroups
    // (1,048,576 rows of 512: 425 us, with 512 of them 439), of 16 to 64 jobs
    const int range = (int)std::clamp<int64_t>((int64_t)w.p.jobs * tiles / 2048, 16, kJoinRange);
    const dim3 grid((unsigned)((w.p.jobs + range - 1) / range), tiles);
    embed_join_kernel<L><<<grid, kJoinThreads, 0, stream>>>(
        w.key_of, w.begins, w.p.J, w.p.jobs, range, C, scale, accumulate, w.part, dE, ldE);
    return hipGetLastError();
  };
  if (C <= 64) return join(std::integral_constant<int, 16>{});
  if (C <= 128) return join(std::integral_constant<int, 32>{});
  return join(std::integral_constant<int, 64>{});
}

}  // namespace shc
