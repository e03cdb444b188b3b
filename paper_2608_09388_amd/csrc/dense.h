// Host interface of the matrix products (dense.hip) behind the dense linear layer
// (linear.hip) and the cross entropy of a linear layer (xent.hip).
#pragma once

#include "dense_tile.h"

namespace shc {
namespace dense {

// Activations: the layer's SHC_ACT_* codes.
constexpr int kActNone = 0, kActRelu = 1, kActGelu = 2, kActSilu = 3;

// What becomes of a product's element v at (row, col), in this order:
//   v += add32[row][col];  out32[row][col] = v, and nothing else, where out32 is set
//   v += bias[col];  pre[row][col] = v;  v = act(v);
//   v += res[to[row]][col];  out[to[row]][col] = v
// res, pre and out are bf16, or fp32 of a split product; res may be out itself.
struct Store {
  const float* add32;
  float* out32;  // both [M][N], N apart
  const float* scale;  // of the sums, on the device, or NULL
  const float* bias;
  int act;
  const void* res;
  int64_t ld_res;
  void* pre;
  int64_t ld_pre;
  void* out;
  int64_t ld_out;
  const int32_t* to;  // NULL: row
};

struct Product {
  Operand A, B;
  bool a_rows, b_rows;  // the order of each operand (see dense_tile.h)
  bool split;           // fp32 as three bf16 terms
  bool direct;          // fp32 as it is (with split; A in rows)
  bool a_low;           // A (bf16) is the sum of two terms, `plane` apart
  int64_t M, N, K;
  // the device count of live rows, from row0 on, bounds M (rows of D) or K; NULL: all
  const int32_t* count;
  int64_t row0;
  bool count_is_k;
  int64_t full;  // the count at which an operand's `alt` is not needed
  Store store;
  float* partials;  // where K is cut into parts: their sums
  size_t partial_bytes;
};

// Bytes of partial sums with which a product of up to M x N x K may be cut along K;
// grows with each of the sizes.
size_t partial_bytes(int64_t M, int64_t N, int64_t K);
hipError_t launch_product(const Product& p, hipStream_t stream);

// Whether the loads of a tile of R rows (or columns) of an operand stay within kReach of its
// first element: of a rows operand all R rows, of a cols operand the BK rows of a step.
inline bool in_reach(const Operand& o, bool rows_order, int64_t R) {
  const int64_t ld = o.alt_ld > o.ld ? o.alt_ld : o.ld;
  return (rows_order ? (R - 1) * ld + BK : (BK - 1) * ld + R) * 2 <= kReach;
}

// Whether rows of C elements, ld apart, can be read as they are (bf16).
inline bool direct(const void* p, int64_t ld, int64_t C) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 8 == 0 && C % 8 == 0 &&
         ld < ((int64_t)1 << 21);
}
// Rows of a packed copy are a multiple of this many elements long, zeros at the end.
inline int64_t packed_width(int64_t C) { return C <= 64 ? (C + 7) / 8 * 8 : (C + 63) / 64 * 64; }
inline size_t align256(size_t b) { return (b + 255) & ~(size_t)255; }
inline size_t packed_bytes(int64_t rows, int64_t C, bool split) {
  return align256((size_t)rows * packed_width(C) * 2 * (split ? 3 : 1));
}

// Packs n rows of C elements into rows of packed_width(C) bf16: copies of bf16, or
// the three terms of fp32, `rows` * packed_width(C) elements from term to term.
// Packed row r is row idx[r] (NULL: r) for r below *count - row0 (NULL: n); with
// `unless_full`, nothing is written where *count is that number.
struct Pack {
  const void* src;
  int64_t ld;
  int64_t n, rows;
  int32_t C;
  int split;
  const int32_t* idx;
  const int32_t* count;
  int64_t row0;
  int64_t unless_full;  // -1: none
  uint16_t* dst;
};
hipError_t launch_pack(const Pack& p, hipStream_t stream);

// out[c] (+)= sum over `rows` partial rows of C, `ld` apart, in ascending order.
hipError_t launch_sum_rows(const float* parts, int64_t rows, int64_t ld, int32_t C, int accumulate,
                           float* out, hipStream_t stream);

// Shape of the workgroups' tiles and parts along K for a product.
enum class TileKind { k256, k128, k64, k32 };  // rows; columns: 256, else 128 (split: not the first)
struct Plan {
  TileKind kind;
  int parts;
};
// few_rows: tiles of fewer than 128 rows too (operand A in rows); logits: the epilogues
// of xent.hip; reach: an operand A in rows that a tile has to reach, or NULL.
Plan plan_product(int64_t M, int64_t N, int64_t K, Mode mode, bool few_rows,
                  size_t partial_bytes, bool logits = false, double* time = nullptr,
                  const Operand* reach = nullptr);
Plan plan_of(const Product& p);

// Rows of fp32 up to which a product reads its operands as they are: the packing of the
// second one would move more than the product.
constexpr int64_t kFewRows = 32;

using Shape256 = Shape<4, 2, 2, 4>;
using Shape128 = Shape<2, 2, 2, 2>;
using Shape64 = Shape<1, 2, 2, 2>;
using Shape32 = Shape<1, 2, 1, 2>;
constexpr int tile_m(TileKind k) {
  return k == TileKind::k256   ? Shape256::BM
         : k == TileKind::k128 ? Shape128::BM
         : k == TileKind::k64  ? Shape64::BM
                               : Shape32::BM;
}
constexpr int tile_n(TileKind k) { return k == TileKind::k256 ? Shape256::BN : Shape128::BN; }

// Tiles of a launch, for fewer than 2^32 threads.  Products of fewer than 2^22 tiles of
// 128 x 128 have fewer with every kind: four of 32 rows and 128 threads in the place of one.
constexpr int64_t kMostTiles = (int64_t)1 << 24;

// Calls f(shape) for the kind.
template <typename F>
hipError_t with_tile(TileKind kind, F&& f) {
  switch (kind) {
    case TileKind::k256: return f(Shape256{});
    case TileKind::k128: return f(Shape128{});
    case TileKind::k64: return f(Shape64{});
    default: return f(Shape32{});
  }
}

}  // namespace dense
}  // namespace shc
