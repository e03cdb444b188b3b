// The matrix product of the dense layers (linear.hip, xent.hip): one workgroup's
// tile of D = A B^T in fp32, from bf16 operands in either order,
//
//   D[m][n] = sum over k of A[m][k] B[n][k],
//
// or from fp32 operands as three bf16 terms each (`split`).  An operand's
// element (r, k) is at r * ld + k ("rows": the sum runs along memory) or at
// k * ld + r ("cols": it runs across rows), so that x W, dz W^T and x^T dz read
// their tensors as they are.
//
// A tile of BM x BN is WM x WN wavefronts of (32 MB) x (32 NB), in 32 x 32 x 16 matrix
// instructions: half as many operand registers are read per product as with 16 x 16
// x 32, and the large products run at the power limit.  The tile's operands pass
// through LDS in steps of 64 along k, in two buffers, brought by loads that write LDS
// directly.  A step is two halves of 32; each half's fragments are read into registers
// while the matrix instructions of the half before run, so that they wait neither for
// LDS nor, with a whole step between a load and its first use, for memory, and there
// is one barrier to a step:
//
//   read half 1 of step t;  multiply half 0 of t;
//   wait for those reads and for step t + 1 in LDS;  barrier;
//   load step t + 2 over step t;  read half 0 of t + 1;  multiply half 1 of t
//
// LDS holds a rows operand as [R][64] and a cols operand as [64][R], in chunks of
// 16 bytes whose place in a row is XORed with bits of the row's number so that the
// lanes of a read fall on different banks.  The load of a chunk to its place is a
// matter of the lane's address: a lane writes 16 bytes at its own place of a
// contiguous kilobyte.  Fragments of a cols operand come from the transposing LDS
// read: 16 lanes give the addresses of 4 x 16 elements and each gets a column.
//
// Few rows of fp32 and small products are not split: both operands are read from memory
// into registers, for the fp32 matrix cores.
//
// Split fp32: x = h + m + l, and of the nine products of terms the six largest, h h in
// one sum and the others, at most 2^-7 of it, in a second.  The three planes of both
// operands pass through LDS together, 32 of k at a time in three buffers, so that a
// fragment is read once for its two or three products.
//
// The products run transposed (D^T = B A^T): a lane holds columns 8 b + 4 (lane / 32)
// + e of row lane % 32 of a 32 x 32 block.  At the end they pass through LDS, 32 rows of
// the wavefront's 64 columns at a time, so that 8 lanes have 64 adjacent columns of a
// row: stores, and loads of a residual, are of whole 128 bytes.
//
// Loads past the ends give zeros: a buffer descriptor covers exactly the rows that
// are there, and chunks past a row's end get an offset outside of it.  Operands
// start at multiples of 16 bytes, with rows of a multiple of 8 elements, a
// multiple of 8 elements apart.  A load's place is a 32-bit offset from the tile's first
// element, and a descriptor covers kReach bytes: how far apart rows may be follows from how
// many a tile has (see `in_reach`).
#pragma once

#include <type_traits>

#include "row_ops.h"

namespace shc {
namespace dense {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr int BK = 64, BKS = 32;  // of k to a step; split
constexpr int64_t kReach = 0x7FFFFFF0;  // bytes from a tile's first element that a load reaches
typedef float f32x16 __attribute__((ext_vector_type(16)));

struct Operand {
  const uint16_t* p;
  int64_t ld;      // elements from row to row of memory (r of rows, k of cols)
  int64_t extent;  // r that may be read (cols: a multiple of 8)
  int64_t k;       // k that may be read (rows: a multiple of 8)
  int64_t plane;   // elements from term to term of an operand of several
  // where a device count of rows is below their number: the chosen rows, packed
  const uint16_t* alt;
  int64_t alt_ld;
  // split operands: the values themselves, memory row r at idx[r] (NULL: r)
  const float* f32;
  int64_t f32_ld;
  const int32_t* idx;
};

// How a tile multiplies: bf16, fp32 in three terms, fp32 from memory.
enum Mode { kPlain, kSplit, kDirect };

template <int MB_, int NB_, int WM_, int WN_>
struct Shape {
  static constexpr int MB = MB_, NB = NB_, WM = WM_, WN = WN_;
  static constexpr int BM = 32 * MB * WM, BN = 32 * NB * WN, NW = WM * WN, THREADS = 64 * NW;
  static constexpr int LDS_A = BM * BK * 2, LDS_B = BN * BK * 2, STAGE = LDS_A + LDS_B;
  // split: three planes of half a step in three buffers
  static constexpr int SPLIT_A = BM * BKS * 2, SPLIT_B = BN * BKS * 2,
                       SPLIT_STAGE = 3 * (SPLIT_A + SPLIT_B), SPLIT_BUFFERS = 3;
  template <Mode MODE>
  static constexpr int lds() {  // direct: for the epilogues alone
    return MODE == kDirect ? NW * 8192 + 2048 : MODE == kSplit ? SPLIT_BUFFERS * SPLIT_STAGE
                                                               : 2 * STAGE;
  }
};

// What the place of a chunk in its row of LDS is XORed with: rows operand, 8 chunks (or 4,
// split) to row r (a read takes 16 rows at a time, two or four of them 256 bytes of
// banks); cols operand, 16 or more chunks to row k (32 lanes have 64 bytes of 4 rows).
template <int K>
__device__ __forceinline__ int rows_key(int r) {
  return K == 64 ? (r >> 1) & 7 : (r >> 2) & 3;
}
__device__ __forceinline__ int cols_key(int k) { return (k & 3) << 2; }

// One operand's side of the tile.
template <int R, bool ROWS, int NW, int K_>
struct Side {
  static constexpr int INSTR = R * K_ * 2 / 1024;  // loads of a kilobyte
  static constexpr int PER_WAVE = (INSTR + NW - 1) / NW;
  const char* base;   // first element of the tile at k = 0
  int64_t bytes;      // from there to the end of what the tile may read
  int64_t step;       // bytes from one k step to the next
  uint32_t off;       // the lane's byte offset of its first load
  int32_t inc;        // bytes from one of a wave's loads to the next
  int kl;             // the lane's first k within a step (cols: row k of its first load)

  // rows r0 on; lane's place in wave w's loads
  __device__ __forceinline__ void init(const Operand& o, int64_t r0, int w, int lane) {
    if constexpr (ROWS) {
      base = reinterpret_cast<const char*>(o.p + r0 * o.ld);
      const int64_t left = o.extent - r0 < R ? o.extent - r0 : R;
      bytes = ((left - 1) * o.ld + o.k) * 2;
      constexpr int C = K_ / 8, RL = 64 / C;  // chunks of a row; rows of a load
      static_assert(RL * NW % 16 == 0, "the key repeats");
      step = K_ * 2;
      const int r = w * RL + lane / C;
      kl = ((lane % C) ^ rows_key<K_>(r)) * 8;
      off = (uint32_t)((r * o.ld + kl) * 2);
      inc = (int32_t)(RL * NW * o.ld * 2);
    } else {
      constexpr int S = R / 8, KR = 64 / S;  // chunks of a row; rows of a load
      base = reinterpret_cast<const char*>(o.p + r0);
      const int64_t left = o.extent - r0;    // a multiple of 8
      bytes = ((o.k - 1) * o.ld + left) * 2;
      step = o.ld * K_ * 2;
      kl = w * KR + lane / S;
      static_assert(R >= 128, "16 chunks to a row");
      const int c = (lane % S) ^ cols_key(kl);
      off = c * 8 < left ? (uint32_t)((kl * o.ld + c * 8) * 2) : 0xFFFFFFF0u;
      inc = (int32_t)(KR * NW * o.ld * 2);
    }
  }
  // loads step kt (K elements in all) of the plane `plane` bytes on into lds
  __device__ __forceinline__ void load(char* lds, int64_t plane, int kt, int64_t K, int w) const {
    const int64_t at = plane + kt * step;
    int64_t left = bytes - kt * step;
    if (left > kReach) left = kReach;
    const auto rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base + at), 0, (int)left,
                                                      0x00020000);
#pragma unroll
    for (int i = 0; i < PER_WAVE; ++i) {
      if (INSTR % NW != 0 && i * NW + w >= INSTR) break;
      uint32_t o = off == 0xFFFFFFF0u ? off : off + i * inc;
      if constexpr (ROWS) {
        if ((int64_t)kt * K_ + kl >= K) o = 0xFFFFFFF0u;
      } else {
        static_assert((64 / (R / 8) * NW) % 4 == 0 || INSTR <= NW, "the key repeats");
      }
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void*)(lds + (i * NW + w) * 1024), 16, o, 0,
                                               0, 0);
    }
  }
};

// The transposing read.  `restrict` gives it the alias information without which the
// compiler waits, at every such read, for all loads into LDS that are under way; here
// the steps' own waits and barriers order them.
__device__ __forceinline__ s16x4 read_transposed(const char* __restrict__ p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
}

// Fragments of 32 rows by 16 k: lane l has row l % 32, k 8 (l / 32) to 8 (l / 32) + 7.
template <int R, bool ROWS, int K_>
struct Frags {
  int at;  // LDS byte offset of the lane in the first fragment; others by XOR

  // r0: the wave's first row, a multiple of 32
  __device__ __forceinline__ void init(int r0, int lane) {
    const int h = lane >> 5;
    if constexpr (ROWS) {
      const int r = r0 + (lane & 31);
      at = r * (K_ * 2) + ((h ^ rows_key<K_>(r)) * 16);
    } else {
      const int i = lane & 15, k = 8 * h + (i >> 2);
      const int c = r0 / 8 + ((lane >> 4) & 1) * 2 + ((i & 3) >> 1);
      at = k * (R * 2) + ((c ^ cols_key(k)) * 16) + (i & 1) * 8;
    }
  }
  // rows 32 f on, k 16 s on
  __device__ __forceinline__ bf16x8 get(const char* lds, int f, int s) const {
    if constexpr (ROWS) {
      return *reinterpret_cast<const bf16x8*>(lds + (at ^ (s * 32)) + f * 32 * (K_ * 2));
    } else {
      // 64 bytes a fragment; f & 3 meets the key's bits (r0 is a multiple of 32 MB or NB)
      const char* p = lds + (at ^ ((f & 3) * 64)) + (f >> 2) * 256 + s * 16 * R * 2;
      union {
        s16x4 v[2];
        bf16x8 all;
      } u;
#pragma unroll
      for (int e = 0; e < 2; ++e)
        u.v[e] = read_transposed(p + e * 4 * R * 2);
      return u.all;
    }
  }
};

// Waits until all but the last VM of the wavefront's loads and all of its LDS accesses
// are done, then for the workgroup.  No access to memory moves across; the compiler
// sees the wait and adds none of its own for what it covers.
template <int VM>
__device__ __forceinline__ void wait_and_sync() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((VM & 15) | (7 << 4) | ((VM >> 4) << 14));
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Element (r, k) of a split operand as it was given; 0 outside of it.
template <bool ROWS>
__device__ __forceinline__ float original(const Operand& o, int64_t r, int64_t k, int64_t R,
                                          int64_t K) {
  if (r >= R || k >= K) return 0.f;
  const int64_t row = ROWS ? r : k, col = ROWS ? k : r;
  return o.f32[(o.idx != nullptr ? (int64_t)o.idx[row] : row) * o.f32_ld + col];
}

// Split fp32 terms are of the value times 2^24, so that every nonzero term is a
// normal bf16 number (the last bit of the smallest fp32 number is 2^-149); sums
// are scaled back.
constexpr float kSplitScale = 0x1p24f, kSplitBack = 0x1p-48f;

template <class S, bool AROWS, bool BROWS, Mode MODE>
struct Tile {
  static constexpr int MB = S::MB, NB = S::NB;
  static constexpr int LDS = S::template lds<MODE>();
  f32x16 acc[MB][NB];

  // The tile at (m0, n0) of the M x N of which both operands hold enough rows,
  // over steps [t0, t1) of 64 along K.  smem: LDS bytes at a multiple of 1024.
  __device__ __forceinline__ void run(const Operand& A, const Operand& B, int64_t M, int64_t N,
                                      int64_t K, int64_t m0, int64_t n0, int t0, int t1,
                                      char* smem) {
    clear(acc);
    add(A, B, M, N, K, m0, n0, t0, t1, smem);
  }
  // adds to what the tile holds (bf16)
  __device__ __forceinline__ void add(const Operand& A, const Operand& B, int64_t M, int64_t N,
                                      int64_t K, int64_t m0, int64_t n0, int t0, int t1,
                                      char* smem) {
    if (t0 >= t1) return;
    if constexpr (MODE == kDirect) {
      run_direct(A, B, M, N, K, m0, n0, t0, t1);
    } else if constexpr (MODE == kSplit) {
      run_split(A, B, m0, n0, t0 * (BK / BKS),
                (int)min((int64_t)t1 * (BK / BKS), (K + BKS - 1) / BKS), smem);
      again(A, B, M, N, K, row_of(m0, 0, 0) - ((threadIdx.x & 63) >> 3),
            col_of(n0) - (threadIdx.x & 7) * 8, t0, t1);
    } else {
      run_plain(A, B, m0, n0, t0, t1, smem);
    }
  }

  static __device__ __forceinline__ void clear(f32x16 (&a)[MB][NB]) {
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) a[i][j][e] = 0.f;
  }

  __device__ __forceinline__ void run_plain(const Operand& A, const Operand& B, int64_t m0,
                                            int64_t n0, int t0, int t1, char* smem) {
    const int lane = threadIdx.x & 63;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Side<S::BM, AROWS, S::NW, BK> sa;
    Side<S::BN, BROWS, S::NW, BK> sb;
    sa.init(A, m0, w, lane);
    sb.init(B, n0, w, lane);
    Frags<S::BM, AROWS, BK> fa;
    Frags<S::BN, BROWS, BK> fb;
    fa.init(w / S::WN * 32 * MB, lane);
    fb.init(w % S::WN * 32 * NB, lane);
    const int64_t ka = A.k, kb = B.k;
    const auto load = [&](int t, int buf) {
      char* to = smem + buf * S::STAGE;
      sa.load(to, 0, t, ka, w);
      sb.load(to + S::LDS_A, 0, t, kb, w);
    };
    bf16x8 a0[MB][2], b0[NB][2], a1[MB][2], b1[NB][2];
    const auto read = [&](bf16x8(&a)[MB][2], bf16x8(&b)[NB][2], int buf, int h) {
      const char* from = smem + buf * S::STAGE;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
#pragma unroll
        for (int j = 0; j < NB; ++j) b[j][s] = fb.get(from + S::LDS_A, j, 2 * h + s);
#pragma unroll
        for (int i = 0; i < MB; ++i) a[i][s] = fa.get(from, i, 2 * h + s);
      }
    };
    const auto multiply = [&](const bf16x8(&a)[MB][2], const bf16x8(&b)[NB][2]) {
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
          for (int j = 0; j < NB; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b[j][s], a[i][s], acc[i][j], 0, 0,
                                                                0);
    };
    load(t0, 0);
    if (t0 + 1 < t1) load(t0 + 1, 1);
    wait_and_sync<0>();
    read(a0, b0, 0, 0);
    int buf = 0;
    for (int t = t0; t < t1; ++t) {
      read(a1, b1, buf, 1);
      multiply(a0, b0);
      __builtin_amdgcn_sched_barrier(0);  // the products are not moved behind the wait
      wait_and_sync<0>();
      if (t + 2 < t1) load(t + 2, buf);
      buf ^= 1;
      if (t + 1 < t1) read(a0, b0, buf, 0);
      multiply(a1, b1);
    }
  }

  // Steps of 32 of k, their fragments read while the step before is multiplied; a load
  // has two steps to arrive.
  __device__ __forceinline__ void run_split(const Operand& A, const Operand& B, int64_t m0,
                                            int64_t n0, int t0, int t1, char* smem) {
    const int lane = threadIdx.x & 63;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Side<S::BM, AROWS, S::NW, BKS> sa;
    Side<S::BN, BROWS, S::NW, BKS> sb;
    sa.init(A, m0, w, lane);
    sb.init(B, n0, w, lane);
    Frags<S::BM, AROWS, BKS> fa;
    Frags<S::BN, BROWS, BKS> fb;
    fa.init(w / S::WN * 32 * MB, lane);
    fb.init(w % S::WN * 32 * NB, lane);
    const int64_t ka = A.k, kb = B.k;
    constexpr int BUFFERS = S::SPLIT_BUFFERS;
    constexpr int LOADS = 3 * (decltype(sa)::PER_WAVE + decltype(sb)::PER_WAVE);
    static_assert(decltype(sa)::INSTR % S::NW == 0 && decltype(sb)::INSTR % S::NW == 0,
                  "every wavefront has as many loads");
    const auto load = [&](int t) {
      char* to = smem + (t - t0) % BUFFERS * S::SPLIT_STAGE;
#pragma unroll
      for (int p = 0; p < 3; ++p) {
        sa.load(to + p * S::SPLIT_A, p * A.plane * 2, t, ka, w);
        sb.load(to + 3 * S::SPLIT_A + p * S::SPLIT_B, p * B.plane * 2, t, kb, w);
      }
    };
    f32x16 low[MB][NB];
    clear(low);
    bf16x8 a0[3][MB][2], b0[3][NB][2], a1[3][MB][2], b1[3][NB][2];
    const auto read = [&](bf16x8(&a)[3][MB][2], bf16x8(&b)[3][NB][2], int t) {
      const char* from = smem + (t - t0) % BUFFERS * S::SPLIT_STAGE;
#pragma unroll
      for (int p = 0; p < 3; ++p)
#pragma unroll
        for (int s = 0; s < 2; ++s) {
#pragma unroll
          for (int j = 0; j < NB; ++j)
            b[p][j][s] = fb.get(from + 3 * S::SPLIT_A + p * S::SPLIT_B, j, s);
#pragma unroll
          for (int i = 0; i < MB; ++i) a[p][i][s] = fa.get(from + p * S::SPLIT_A, i, s);
        }
    };
    const auto multiply = [&](const bf16x8(&a)[3][MB][2], const bf16x8(&b)[3][NB][2]) {
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int p = 0; p < 3; ++p)
#pragma unroll
          for (int q = 0; q < 3 - p; ++q)
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
              for (int j = 0; j < NB; ++j) {
                f32x16& to = p + q == 0 ? acc[i][j] : low[i][j];
                to = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b[q][j][s], a[p][i][s], to, 0, 0, 0);
              }
    };
    // Step t is in registers; t + 1 has arrived when all but the last step's loads have.
    // The steady loop has no condition in it: past a branch the compiler waits for the
    // reads that are under way.
    const auto steady = [&](int t, bf16x8(&a)[3][MB][2], bf16x8(&b)[3][NB][2],
                            bf16x8(&an)[3][MB][2], bf16x8(&bn)[3][NB][2]) {
      wait_and_sync<LOADS*(BUFFERS - 2)>();
      load(t + BUFFERS);
      read(an, bn, t + 1);
      multiply(a, b);
      // one wavefront to a SIMD: loads and reads are issued between the products
      constexpr int READS = 3 * 2 * (MB * (AROWS ? 1 : 2) + NB * (BROWS ? 1 : 2));
      constexpr int PRODUCTS = 6 * 2 * MB * NB;
#pragma unroll
      for (int i = 0; i < READS; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);  // an LDS read
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);    // a product
      }
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x10, 1, 0);  // a load
        if (READS + i < PRODUCTS) __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    };
    const auto last = [&](int t, bf16x8(&a)[3][MB][2], bf16x8(&b)[3][NB][2],
                          bf16x8(&an)[3][MB][2], bf16x8(&bn)[3][NB][2]) {
      wait_and_sync<0>();
      if (t + BUFFERS < t1) load(t + BUFFERS);
      if (t + 1 < t1) read(an, bn, t + 1);
      multiply(a, b);
      __builtin_amdgcn_sched_barrier(0);
    };
    for (int t = t0; t < t0 + BUFFERS && t < t1; ++t) load(t);
    if (t0 + BUFFERS <= t1)
      wait_and_sync<LOADS*(BUFFERS - 1)>();
    else
      wait_and_sync<0>();
    read(a0, b0, t0);
    int t = t0;
    for (; t + 1 + BUFFERS < t1; t += 2) {
      steady(t, a0, b0, a1, b1);
      steady(t + 1, a1, b1, a0, b0);
    }
    for (; t < t1; t += 2) {
      last(t, a0, b0, a1, b1);
      if (t + 1 < t1) last(t + 1, a1, b1, a0, b0);
    }
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j) acc[i][j] += low[i][j];
  }

  // 8 of k at a time, 4 adjacent ones to a lane: lane l has row l % 32 of both operands.
  // A cols operand is read 32 columns of a row of memory at a time.
  __device__ __forceinline__ void run_direct(const Operand& A, const Operand& B, int64_t M,
                                             int64_t N, int64_t K, int64_t m0, int64_t n0, int t0,
                                             int t1) {
    static_assert(MODE != kDirect || (AROWS && MB == 1 && S::WM == 1), "few rows");
    const int r = threadIdx.x & 31, h = (threadIdx.x >> 5) & 1;
    const int64_t k0 = (int64_t)t0 * BK, end = (int64_t)t1 * BK < K ? (int64_t)t1 * BK : K;
    const int64_t n = col_of(n0) - (threadIdx.x & 7) * 8 + r;
    // rows past the last repeat row 0, whose values are not kept
    const int64_t ra = m0 + r < M ? m0 + r : 0;
    const float* a = A.f32 + (A.idx != nullptr ? (int64_t)A.idx[ra] : ra) * A.f32_ld;
    const float* b[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      const int64_t nj = n + 32 * j < N ? n + 32 * j : 0;
      b[j] = BROWS ? B.f32 + nj * B.f32_ld : B.f32 + nj;
    }
    // U times 8 of k, all loads ahead of the products; the lane's first k, and how many
    // of its 4 are there
    const auto steps = [&](int64_t k, int left, auto uc) {
      constexpr int U = decltype(uc)::value;
      rowops::f32x4_a4 x[U], y[U][NB];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t at = k + 8 * u;
        if (left >= 4) {
          x[u] = *reinterpret_cast<const rowops::f32x4_a4*>(a + at);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) x[u][e] = e < left ? a[at + e] : 0.f;
        }
#pragma unroll
        for (int j = 0; j < NB; ++j) {
          if (BROWS && left >= 4) {
            y[u][j] = *reinterpret_cast<const rowops::f32x4_a4*>(b[j] + at);
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              y[u][j][e] = e < left ? b[j][(at + e) * (BROWS ? 1 : B.f32_ld)] : 0.f;
          }
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int j = 0; j < NB; ++j)
            acc[0][j] =
                __builtin_amdgcn_mfma_f32_32x32x2f32(y[u][j][e], x[u][e], acc[0][j], 0, 0, 0);
    };
    int64_t k = k0;
    for (; k + 64 <= end; k += 64) steps(k + 4 * h, 4, std::integral_constant<int, 8>{});
    for (; k < end; k += 8)
      steps(k + 4 * h, (int)min((int64_t)4, end - k - 4 * h), std::integral_constant<int, 1>{});
  }

  // Scales the sums of split products back.  Sums that are not finite (an infinity, a
  // NaN, a value of 2^104 or more, a sum of 2^80) are taken again on the fp32 matrix
  // cores from the values, 32 x 32 at a time, and replaced; the others stay.
  __device__ __forceinline__ void again(const Operand& A, const Operand& B, int64_t M, int64_t N,
                                        int64_t K, int64_t m0, int64_t n0, int t0, int t1) {
    const int r = threadIdx.x & 31, h = (threadIdx.x >> 5) & 1;
    const int64_t end = (int64_t)t1 * BK < K ? (int64_t)t1 * BK : K;
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        bool fine = true;
#pragma unroll
        for (int e = 0; e < 16; ++e) fine &= __builtin_isfinite(acc[i][j][e]);
        if (__any(!fine)) {
          f32x16 sum;
#pragma unroll
          for (int e = 0; e < 16; ++e) sum[e] = 0.f;
#pragma unroll 1
          for (int64_t k = (int64_t)t0 * BK; k < end; k += 2)
            sum = __builtin_amdgcn_mfma_f32_32x32x2f32(
                original<BROWS>(B, n0 + j * 32 + r, k + h, N, end),
                original<AROWS>(A, m0 + i * 32 + r, k + h, M, end), sum, 0, 0, 0);
#pragma unroll
          for (int e = 0; e < 16; ++e)
            acc[i][j][e] = __builtin_isfinite(acc[i][j][e]) ? acc[i][j][e] * kSplitBack : sum[e];
        } else {
          acc[i][j] *= kSplitBack;
        }
      }
  }

  // What the lane stores of block i: rows of D and first column of row t of 4.
  static __device__ __forceinline__ int64_t row_of(int64_t m0, int i, int t) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    return m0 + (w / S::WN) * 32 * MB + 32 * i + 8 * t + (lane >> 3);
  }
  static __device__ __forceinline__ int64_t col_of(int64_t n0) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    return n0 + (w % S::WN) * 64 + (lane & 7) * 8;
  }
  // g[t] = fetch(row, column) of block i
  template <typename G, typename Fetch>
  static __device__ __forceinline__ void fetch_block(int64_t m0, int64_t n0, int i, G (&g)[4],
                                                     Fetch&& fetch) {
#pragma unroll
    for (int t = 0; t < 4; ++t) g[t] = fetch(row_of(m0, i, t), col_of(n0));
  }
  // f(row of D, first column, 8 adjacent values, what was fetched for them): lane l has
  // 8 (l % 8) of the wavefront's 64 columns, rows l / 8 and 8 on.  Through 8 KB of smem
  // a wavefront, 16 chunks of 16 bytes to a row, placed by the row's number.  `got` is
  // block 0's; each next block's is fetched before the block at hand is stored, where
  // there are registers for both.
  template <typename G, typename Fetch, typename F>
  __device__ __forceinline__ void each(int64_t m0, int64_t n0, char* smem, G (&got)[4],
                                       Fetch&& fetch, F&& f) const {
    static_assert(NB == 2 && S::NW * 8192 <= LDS, "64 columns to a wavefront");
    const int lane = threadIdx.x & 63;
    char* mine = smem + (threadIdx.x >> 6) * 8192;
    const int r = lane & 31, h = lane >> 5, r8 = lane >> 3, q = lane & 7;
#pragma unroll
    for (int i = 0; i < MB; ++i) {
      constexpr bool kAhead = sizeof(G) <= 24;
      G next[4];
      if (kAhead && i + 1 < MB) fetch_block(m0, n0, i + 1, next, fetch);
      if (!kAhead && i > 0) fetch_block(m0, n0, i, got, fetch);
      rowops::group_fence<64>();  // the reads of the rows before are over
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int b = 0; b < 4; ++b)
          *reinterpret_cast<f32x4*>(mine + r * 256 + (((8 * j + 2 * b + h) ^ (r & 15)) * 16)) =
              f32x4{acc[i][j][4 * b], acc[i][j][4 * b + 1], acc[i][j][4 * b + 2],
                    acc[i][j][4 * b + 3]};
      rowops::group_fence<64>();
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int at = 8 * t + r8;
        float v[8];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const f32x4 x =
              *reinterpret_cast<const f32x4*>(mine + at * 256 + (((2 * q + u) ^ (at & 15)) * 16));
#pragma unroll
          for (int e = 0; e < 4; ++e) v[4 * u + e] = x[e];
        }
        f(row_of(m0, i, t), col_of(n0), v, got[t]);
      }
      if (kAhead && i + 1 < MB) {
#pragma unroll
        for (int t = 0; t < 4; ++t) got[t] = next[t];
      }
    }
  }
  template <typename F>  // with nothing to fetch
  __device__ __forceinline__ void each(int64_t m0, int64_t n0, char* smem, F&& f) const {
    int none[4];
    each(m0, n0, smem, none, [](int64_t, int64_t) { return 0; },
         [&](int64_t row, int64_t col, float (&v)[8], int) { f(row, col, v); });
  }
};

// The tile of workgroup b of tm x tn, false past them (tm counts the live rows' tiles,
// so that these spread evenly): a contiguous range of tiles to an XCD, in
// bands of kBand rows of tiles taken column by column, so that the tiles an XCD
// works on at a time share rows of both operands in its L2.  Loss and gradients of 4,096
// rows of 4,096 over 131,072 classes, us with bands of 1, 4, 8, 16: 11,930, 11,460,
// 11,290, 11,770; 67,040 rows of 128 over 10,475: 1,334, 1,308, 1,300, 1,422.
constexpr int kBand = 8;
__device__ __forceinline__ bool tile_of(int b, int tm, int tn, int* m, int* n) {
  if (b >= tm * tn) return false;
  const int t = xcd_tile(b, tm * tn);
  const int band = t / (kBand * tn), rows = min(tm - band * kBand, kBand);
  const int r = t - band * kBand * tn;
  *m = band * kBand + r % rows;
  *n = r / rows;
  return true;
}

// Rows that a device count leaves of `all` from row0 on (count NULL: all).
__device__ __forceinline__ int64_t rows_left(const int32_t* count, int64_t row0, int64_t all) {
  if (count == nullptr) return all;
  const int64_t left = *count - row0;
  return left < 0 ? 0 : left < all ? left : all;
}

}  // namespace dense
}  // namespace shc
