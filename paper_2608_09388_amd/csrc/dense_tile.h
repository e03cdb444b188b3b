// The matrix product of the dense layers (linear.hip, xent.hip): one workgroup's
// tile of D = A B^T in fp32, from bf16 operands in either order,
//
//   D[m][n] = sum over p, k of A_p[m][k] B_p[n][k],
//
// p over the term pairs of split fp32 operands (one pair for bf16).  An operand's
// element (r, k) is at r * ld + k ("rows": the sum runs along memory) or at
// k * ld + r ("cols": it runs across rows), so that x W, dz W^T and x^T dz read
// their tensors as they are.
//
// A tile of BM x BN is WM x WN wavefronts of (16 MI) x (64 NG).  Its operands pass
// through LDS in steps of 64 along k, in two buffers, brought by loads that write
// LDS directly.  A step is two halves of 32; each half's fragments are read into
// registers while the matrix instructions of the half before run, so that they
// wait neither for LDS nor, with a whole step between a load and its first use,
// for memory, and there is one barrier to a step:
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
// The products run transposed (D^T = B A^T), and the rows of B that a fragment
// takes are chosen so that a lane ends with 16 adjacent columns of one row of D:
// row lane % 16, columns 16 (lane / 16) + 4 j + i of the 64, in register i of
// fragment j.
//
// Loads past the ends give zeros: a buffer descriptor covers exactly the rows that
// are there, and chunks past a row's end get an offset outside of it.  Operands
// start at multiples of 16 bytes, with rows of a multiple of 8 elements, a
// multiple of 8 elements and less than 2^22 apart (see `direct`).
#pragma once

#include "row_ops.h"

namespace shc {
namespace dense {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr int BK = 64;

struct Operand {
  const uint16_t* p;
  int64_t ld;      // elements from row to row of memory (r of rows, k of cols)
  int64_t extent;  // r that may be read (cols: a multiple of 8)
  int64_t k;       // k that may be read (rows: a multiple of 8)
  int64_t plane;   // elements from term to term of a split fp32 operand
  // where a device count of rows is below their number: the chosen rows, packed
  const uint16_t* alt;
  int64_t alt_ld;
  // split operands: the values themselves, memory row r at idx[r] (NULL: r)
  const float* f32;
  int64_t f32_ld;
  const int32_t* idx;
};

// Term pairs of split fp32 products, the small ones first: terms of A and B in
// two bits each.  (2, 2), (1, 2) and (2, 1) are below fp32's last place.
constexpr int kPairs = 6;
__device__ __forceinline__ int pair_a(int p) { return (0x012010 >> (4 * (5 - p))) & 0xF; }
__device__ __forceinline__ int pair_b(int p) { return (0x210100 >> (4 * (5 - p))) & 0xF; }

template <int MI_, int NG_, int WM_, int WN_>
struct Shape {
  static constexpr int MI = MI_, NG = NG_, WM = WM_, WN = WN_;
  static constexpr int BM = 16 * MI * WM, BN = 64 * NG * WN, NW = WM * WN, THREADS = 64 * NW;
  static constexpr int LDS_A = BM * BK * 2, LDS_B = BN * BK * 2, STAGE = LDS_A + LDS_B;
  static constexpr int LDS = 2 * STAGE;
};

// The place of chunk c of a row in LDS.  PERM: the fragments take rows
// 16 q + 4 j + i of 64 (operand B), else 16 adjacent rows (operand A).
// rows operand: R rows of 8 chunks, key from the row; cols operand: 64 rows (k)
// of R / 8 chunks, key from k.
template <bool PERM>
__device__ __forceinline__ int rows_key(int r) {
  return PERM ? (r & 3) | ((r >> 2) & 4) : r & 7;
}
template <int R, bool PERM>
__device__ __forceinline__ int cols_key(int k) {
  if constexpr (R == 64) return PERM ? (k >> 1) & 1 : k & 2;
  return PERM ? (k & 1) | ((k & 2) << 2) : (k & 3) << 1;
}

// One operand's side of the tile.
template <int R, bool ROWS, bool PERM, int NW>
struct Side {
  static constexpr int INSTR = R * BK * 2 / 1024;          // loads of a kilobyte
  static constexpr int PER_WAVE = (INSTR + NW - 1) / NW;
  const char* base;   // first element of the tile at k = 0 of the current pair
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
      step = BK * 2;
      const int r = w * 8 + (lane >> 3);
      kl = ((lane & 7) ^ rows_key<PERM>(r)) * 8;
      off = (uint32_t)((r * o.ld + kl) * 2);
      inc = (int32_t)(8 * NW * o.ld * 2);
    } else {
      constexpr int S = R / 8, KR = 64 / S;  // chunks of a row; rows of a load
      base = reinterpret_cast<const char*>(o.p + r0);
      const int64_t left = o.extent - r0;    // a multiple of 8
      bytes = ((o.k - 1) * o.ld + left) * 2;
      step = o.ld * BK * 2;
      kl = w * KR + lane / S;
      const int c = (lane % S) ^ cols_key<R, PERM>(kl);
      off = c * 8 < left ? (uint32_t)((kl * o.ld + c * 8) * 2) : 0xFFFFFFF0u;
      inc = (int32_t)(KR * NW * o.ld * 2);
    }
  }
  // loads k step kt (K elements in all) of the pair at `plane` bytes into lds
  __device__ __forceinline__ void load(char* lds, int64_t plane, int kt, int64_t K, int w) const {
    const int64_t at = plane + kt * step;
    int64_t left = bytes - kt * step;
    if (left > 0x7FFFFFF0) left = 0x7FFFFFF0;
    const auto rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base + at), 0, (int)left,
                                                      0x00020000);
#pragma unroll
    for (int i = 0; i < PER_WAVE; ++i) {
      if (INSTR % NW != 0 && i * NW + w >= INSTR) break;
      uint32_t o = off == 0xFFFFFFF0u ? off : off + i * inc;
      if constexpr (ROWS) {
        // the key of PERM rows changes with the load only through bit 4 of the row
        int k = kl;
        if constexpr (PERM && (8 * NW) % 32 != 0) {
          const int flip = (rows_key<PERM>(i * NW * 8 + w * 8) ^ rows_key<PERM>(w * 8)) * 8;
          o += ((kl ^ flip) - kl) * 2;
          k = kl ^ flip;
        }
        if ((int64_t)kt * BK + k >= K) o = 0xFFFFFFF0u;
      } else {
        static_assert((64 / (R / 8) * NW) % 4 == 0 || INSTR <= NW, "the key repeats");
      }
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void*)(lds + (i * NW + w) * 1024), 16, o, 0,
                                               0, 0);
    }
  }
};

// Fragments of one half step: F of 16 rows by 32 k.
template <int R, bool ROWS, bool PERM, int F>
struct Frags {
  static constexpr int BASES = ROWS ? 2 : PERM ? 2 : (R == 64 ? 2 : 4);
  int at[BASES];  // LDS byte offsets of the lane

  // r0: the wave's first row (a multiple of 64 with PERM)
  __device__ __forceinline__ void init(int r0, int lane) {
    const int i = lane & 15, g = lane >> 4;
    if constexpr (ROWS) {
      const int r = r0 + (PERM ? 16 * (i >> 2) + (i & 3) : i);
#pragma unroll
      for (int h = 0; h < 2; ++h) at[h] = r * 128 + (((4 * h + g) ^ rows_key<PERM>(r)) * 16);
    } else {
      const int k = 8 * g + (i >> 2), q = i & 3, key = cols_key<R, PERM>(k);
#pragma unroll
      for (int b = 0; b < BASES; ++b) {
        // PERM: fragment j = 2 b (+ 1: 8 bytes on); else fragment f = b modulo BASES
        const int c = r0 / 8 + (PERM ? 2 * q + b : 2 * b + (q >> 1));
        at[b] = k * (R * 2) + ((c ^ key) * 16) + (PERM ? 0 : (q & 1) * 8);
      }
    }
  }
  __device__ __forceinline__ bf16x8 get(const char* lds, int f, int h) const {
    if constexpr (ROWS) {
      const int add = PERM ? (f >> 2) * 64 * 128 + (f & 3) * 4 * 128 : f * 16 * 128;
      return *reinterpret_cast<const bf16x8*>(lds + at[h] + add);
    } else {
      const int b = PERM ? (f >> 1) & 1 : f % BASES;
      const int add = (PERM ? (f >> 2) * 128 + (f & 1) * 8 : f / BASES * (BASES * 32)) +
                      h * 32 * R * 2;
      union {
        s16x4 s[2];
        bf16x8 v;
      } u;
#pragma unroll
      for (int e = 0; e < 2; ++e)
        u.s[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (lds_s16x4*)(lds + at[b] + add + e * 4 * R * 2));
      return u.v;
    }
  }
};

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

template <class S, bool AROWS, bool BROWS, int PAIRS>
struct Tile {
  f32x4 acc[S::MI][4 * S::NG];

  // The tile at (m0, n0) of the M x N of which both operands hold enough rows,
  // over steps [t0, t1) of 64 along K.  smem: S::LDS bytes at a multiple of 1024.
  __device__ __forceinline__ void run(const Operand& A, const Operand& B, int64_t M, int64_t N,
                                      int64_t K, int64_t m0, int64_t n0, int t0, int t1,
                                      char* smem) {
    constexpr int MI = S::MI, NJ = 4 * S::NG;
    const int lane = threadIdx.x & 63;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = w / S::WN, wn = w % S::WN;
    Side<S::BM, AROWS, false, S::NW> sa;
    Side<S::BN, BROWS, true, S::NW> sb;
    sa.init(A, m0, w, lane);
    sb.init(B, n0, w, lane);
    Frags<S::BM, AROWS, false, MI> fa;
    Frags<S::BN, BROWS, true, NJ> fb;
    fa.init(wm * 16 * MI, lane);
    fb.init(wn * 64 * S::NG, lane);
    clear();
    if (t0 >= t1) return;

    int lp = 0, lk = t0;  // the next step to load: its pair, and its place along K
    const int64_t ka = A.k, kb = B.k;
    const auto load = [&](int buf) {
      char* to = smem + buf * S::STAGE;
      const int64_t pa = PAIRS == 1 ? 0 : pair_a(lp) * A.plane * 2;
      const int64_t pb = PAIRS == 1 ? 0 : pair_b(lp) * B.plane * 2;
      sa.load(to, pa, lk, ka, w);
      sb.load(to + S::LDS_A, pb, lk, kb, w);
      if (++lk == t1 && PAIRS > 1) lk = t0, ++lp;
    };
    bf16x8 a0[MI], b0[NJ], a1[MI], b1[NJ];
    const auto read = [&](bf16x8(&a)[MI], bf16x8(&b)[NJ], int buf, int h) {
      const char* from = smem + buf * S::STAGE;
#pragma unroll
      for (int j = 0; j < NJ; ++j) b[j] = fb.get(from + S::LDS_A, j, h);
#pragma unroll
      for (int i = 0; i < MI; ++i) a[i] = fa.get(from, i, h);
    };
    const auto multiply = [&](const bf16x8(&a)[MI], const bf16x8(&b)[NJ]) {
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[j], a[i], acc[i][j], 0, 0, 0);
    };
    // Waits and barriers in one asm block each: no access to LDS moves across.
    const int steps = PAIRS * (t1 - t0);
    load(0);
    asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
    if (steps > 1) load(1);
    read(a0, b0, 0, 0);
    int buf = 0;
    for (int t = 0; t < steps; ++t) {
      read(a1, b1, buf, 1);
      multiply(a0, b0);
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
      if (t + 2 < steps) load(buf);
      buf ^= 1;
      if (t + 1 < steps) read(a0, b0, buf, 0);
      multiply(a1, b1);
    }
    if constexpr (PAIRS > 1) again(A, B, M, N, K, m0 + wm * 16 * MI, n0 + wn * 64 * S::NG, t0, t1);
  }

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < S::MI; ++i)
#pragma unroll
      for (int j = 0; j < 4 * S::NG; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // Scales the sums of split products back.  Sums that are not finite (an infinity, a
  // NaN, a value of 2^104 or more, a sum of 2^80) are taken again on the fp32 matrix
  // cores from the values, 16 x 16 at a time, and replaced; the others stay.
  __device__ __forceinline__ void again(const Operand& A, const Operand& B, int64_t M, int64_t N,
                                        int64_t K, int64_t m0, int64_t n0, int t0, int t1) {
    const int i16 = threadIdx.x & 15, g = (threadIdx.x >> 4) & 3;
    const int64_t end = (int64_t)t1 * BK < K ? (int64_t)t1 * BK : K;
#pragma unroll
    for (int i = 0; i < S::MI; ++i)
#pragma unroll
      for (int j = 0; j < 4 * S::NG; ++j) {
        bool fine = true;
#pragma unroll
        for (int e = 0; e < 4; ++e) fine &= __builtin_isfinite(acc[i][j][e]);
        if (__any(!fine)) {
          const int64_t m = m0 + i * 16 + i16;
          const int64_t n = n0 + (j >> 2) * 64 + (i16 >> 2) * 16 + (j & 3) * 4 + (i16 & 3);
          f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
          for (int64_t k = (int64_t)t0 * BK; k < end; k += 4)
            sum = __builtin_amdgcn_mfma_f32_16x16x4f32(original<BROWS>(B, n, k + g, N, end),
                                                       original<AROWS>(A, m, k + g, M, end), sum,
                                                       0, 0, 0);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            acc[i][j][e] = __builtin_isfinite(acc[i][j][e]) ? acc[i][j][e] * kSplitBack : sum[e];
        } else {
          acc[i][j] *= kSplitBack;
        }
      }
  }

  // f(row of D, first column, 16 adjacent values) for what the lane holds.
  template <typename F>
  __device__ __forceinline__ void each(int64_t m0, int64_t n0, F&& f) const {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t row = m0 + (w / S::WN) * 16 * S::MI + (lane & 15);
    const int64_t col = n0 + (w % S::WN) * 64 * S::NG + (lane >> 4) * 16;
#pragma unroll
    for (int i = 0; i < S::MI; ++i)
#pragma unroll
      for (int q = 0; q < S::NG; ++q) {
        float v[16];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) v[4 * j + e] = acc[i][4 * q + j][e];
        f(row + 16 * i, col + 64 * q, v);
      }
  }
};

// The tile of workgroup b of tm x tn: a contiguous range of tiles to an XCD, in
// bands of kBand rows of tiles taken column by column, so that the tiles an XCD
// works on at a time share rows of both operands in its L2.
constexpr int kBand = 4;
__device__ __forceinline__ void tile_of(int b, int tm, int tn, int* m, int* n) {
  const int t = xcd_tile(b, tm * tn);
  const int band = t / (kBand * tn), rows = min(tm - band * kBand, kBand);
  const int r = t - band * kBand * tn;
  *m = band * kBand + r % rows;
  *n = r / rows;
}

// Rows that a device count leaves of `all` from row0 on (count NULL: all).
__device__ __forceinline__ int64_t rows_left(const int32_t* count, int64_t row0, int64_t all) {
  if (count == nullptr) return all;
  const int64_t left = *count - row0;
  return left < 0 ? 0 : left < all ? left : all;
}

}  // namespace dense
}  // namespace shc
