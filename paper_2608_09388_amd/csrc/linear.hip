// The dense linear layer with bias, activation and residual, and its gradients:
//
//   z = x W + b,  out = act(z) + residual
//   dz = dout (.) act'(z),  dx = dz W^T,  dW = x^T dz,  db = sum over rows of dz
//
// on the matrix products of dense.hip: x W reads W [Cin][Cout] across its rows, dz W^T
// along them, x^T dz both operands across.  The backward forms dz once (one pass over
// dout and z, which also sums db) and multiplies it twice.
//
// Tensors that the products cannot read as they are (bf16 rows that do not start at
// multiples of 16 bytes or are not a multiple of 8 long, fp32 rows, which become three
// bf16 terms) are packed into the workspace first.
//
// Forward, 8,192 rows, 16,384 -> 4,096, bf16, 909 us (1.21 PFLOP/s); backward of 4,096 ->
// 8,192 989 us, 95 of them dz and db (4.2 TB/s), the products at 1.23 PFLOP/s.
// 67,040 rows of 128 -> 128 with GELU, residual and z kept: 22 us (3.1 TB/s).
#include <algorithm>

#include "dense.h"
#include "dense_epilogue.h"

namespace shc {

using namespace dense;

namespace {

// dz rows and, per chunk of rows, their column sums.  A group of G lanes to a row's
// vectors of 8; the rows of a chunk go to the 256 / G groups in turn.
struct GradRows {
  const void* dout;
  int64_t ld_dout;
  const void* pre;
  int64_t ld_pre;
  int act;
  int64_t n, chunk;
  int C, G;
  void* dz;  // NULL: not written
  int64_t ld_dz;
  int width;     // columns of dz that are written, those from C on as zeros
  float* sums;   // [chunks][C] or NULL
};

template <bool BF16>
__global__ __launch_bounds__(256) void grad_rows_kernel(GradRows a) {
  __shared__ float part[256 * 8];
  const int lane = threadIdx.x & (a.G - 1), group = threadIdx.x / a.G, groups = 256 / a.G;
  const int v = blockIdx.x * a.G + lane;  // the thread's vector
  const int64_t r0 = (int64_t)blockIdx.y * a.chunk;
  const int64_t r1 = r0 + a.chunk < a.n ? r0 + a.chunk : a.n;
  float sum[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) sum[e] = 0.f;
  if (8 * v < a.width) {
#pragma unroll 2
    for (int64_t r = r0 + group; r < r1; r += groups) {
      float d[8], z[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) d[e] = 0.f;
      if (8 * v < a.C) {
        load8<BF16>(a.dout, r, a.ld_dout, v, a.C, d);
        if (a.act != kActNone) {
          load8<BF16>(a.pre, r, a.ld_pre, v, a.C, z);
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (8 * v + e < a.C) d[e] *= slope_of(a.act, z[e]);
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[e] += d[e];
      if (a.dz != nullptr) put8<BF16>(a.dz, r, a.ld_dz, v, a.width, d);
    }
  }
  if (a.sums == nullptr) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) part[threadIdx.x * 8 + e] = sum[e];
  __syncthreads();
  if (group != 0 || 8 * v >= a.C) return;
  for (int g = 1; g < groups; ++g)
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] += part[(g * a.G + lane) * 8 + e];
  rowops::store_channels<8>(a.sums + (int64_t)blockIdx.y * a.C, v, a.C, sum);
}

// Lanes to a row and chunks of rows: up to 64 lanes, about four workgroups to a CU,
// 16 rows to a chunk at least.  Backward of 8,192 rows, 4,096 -> 8,192, and of 67,040 rows,
// 128 -> 128, us with 256, 1,024, 4,096 workgroups: 1,185, 1,033, 1,035; 82.7, 77.5, 140.9
// (as many partial rows to sum).
struct GradShape {
  int G, cols;
  int64_t chunks, chunk;
};
GradShape grad_shape(int64_t n, int32_t C) {
  GradShape s;
  const int nv = (int)(packed_width(C) / 8);
  s.G = 8;
  while (s.G < 64 && s.G < nv) s.G *= 2;
  s.cols = (nv + s.G - 1) / s.G;
  s.chunks = std::max<int64_t>(1, std::min<int64_t>((n + 15) / 16, std::max(1, 1024 / s.cols)));
  s.chunk = std::max<int64_t>(1, (n + s.chunks - 1) / s.chunks);
  return s;
}

// Where things lie in the workspace; offsets in bytes.
struct Forward {
  size_t x, W, partials, partial_bytes, total;
};
bool fits(int32_t C, bool aligned) { return aligned && C % 8 == 0; }

Forward forward_layout(int64_t n, int32_t Cin, int32_t Cout, bool bf16, bool aligned) {
  Forward w{};
  size_t at = 0;
  const auto take = [&](size_t bytes) {
    const size_t here = at;
    at += align256(bytes);
    return here;
  };
  w.x = take(bf16 && fits(Cin, aligned) ? 0 : packed_bytes(n, Cin, !bf16));
  w.W = take(bf16 && fits(Cout, aligned) ? 0 : packed_bytes(Cin, Cout, !bf16));
  w.partial_bytes = partial_bytes(n, Cout, Cin);
  w.partials = take(w.partial_bytes);
  w.total = at;
  return w;
}

struct Backward {
  size_t x, W, dz, dz32, sums, partials, partial_bytes, total;
};
Backward backward_layout(int64_t n, int32_t Cin, int32_t Cout, bool bf16, bool aligned, int act) {
  Backward w{};
  size_t at = 0;
  const auto take = [&](size_t bytes) {
    const size_t here = at;
    at += align256(bytes);
    return here;
  };
  w.x = take(bf16 && fits(Cin, aligned) ? 0 : packed_bytes(n, Cin, !bf16));
  w.W = take(bf16 && fits(Cout, aligned) ? 0 : packed_bytes(Cin, Cout, !bf16));
  w.dz = take(bf16 && act == kActNone && fits(Cout, aligned) ? 0 : packed_bytes(n, Cout, !bf16));
  w.dz32 = take(bf16 || act == kActNone ? 0 : (size_t)n * Cout * 4);
  w.sums = take((size_t)grad_shape(n, Cout).chunks * Cout * 4);
  w.partial_bytes = std::max(partial_bytes(n, Cin, Cout), partial_bytes(Cin, Cout, n));
  w.partials = take(w.partial_bytes);
  w.total = at;
  return w;
}

char* byte(void* ws, size_t at) { return static_cast<char*>(ws) + at; }

// An operand over rows of C elements that lie as they are (bf16) or are packed.
// `rows_order`: the sum runs along the rows, else across them.
Operand plain(const void* p, int64_t ld, int64_t n, int64_t C, bool rows_order) {
  Operand o{};
  o.p = static_cast<const uint16_t*>(p);
  o.ld = ld;
  o.extent = rows_order ? n : C;
  o.k = rows_order ? C : n;
  return o;
}
// fp32 rows for a product that reads them as they are.
Operand direct_rows(const void* p, int64_t ld) {
  Operand o{};
  o.f32 = static_cast<const float*>(p);
  o.f32_ld = ld;
  return o;
}
// Packs the rows at `to` unless they can be read as they are.
hipError_t operand(const void* p, int64_t ld, int64_t n, int32_t C, bool bf16, bool rows_order,
                   void* to, bool packed, Operand* o, hipStream_t stream) {
  if (bf16 && direct(p, ld, C)) {
    *o = plain(p, ld, n, C, rows_order);
    return hipSuccess;
  }
  const int64_t width = packed_width(C);
  *o = plain(to, width, n, width, rows_order);
  if (!bf16) {
    o->plane = n * width;
    o->f32 = static_cast<const float*>(p);
    o->f32_ld = ld;
  }
  if (packed) return hipSuccess;
  return launch_pack(Pack{p, ld, n, n, C, !bf16, nullptr, nullptr, 0, -1,
                          static_cast<uint16_t*>(to)},
                     stream);
}

// Whether a product of fp32 rows, M x N over K, goes to the fp32 matrix cores as its operands
// are: few rows, for which packing the second operand moves more than the product, and small
// products, where the packing's launches cost more than the slower instructions.  M x K x N,
// us so / in three terms: 58,059 x 35 x 64 22.5 / 34.3, 67,040 x 128 x 128 46.7 / 63.1, 64 x 4,096
// x 4,096 44.7 / 54.7, 256 x 512 x 512 12.2 / 16.5, 5,000 x 300 x 300 19.1 / 24.8; 20,000 x 512 x 64
// 50.7 / 49.1, 1,023 x 1,001 x 2,503 113.5 / 59.9, 84,210 x 1,216 x 166 730 / 514.
bool direct_pays(int64_t M, int64_t K, int64_t N) {
  constexpr int64_t kMost = 1200000000;  // of whole tiles
  return M <= kFewRows || (M + 31) / 32 * 32 * ((N + 127) / 128 * 128) <= kMost / K;
}

#define SHC_LAUNCH(...)                    \
  do {                                     \
    const hipError_t _e = (__VA_ARGS__);   \
    if (_e != hipSuccess) return _e;       \
  } while (0)

}  // namespace

bool linear_aligned(const LinearArgs& a, bool backward) {
  if (!a.bf16) return true;
  return direct(a.x, a.ldx, 8) && direct(a.W, a.ldw, 8) &&
         (!backward || a.act != kActNone || direct(a.dout, a.lddout, 8));
}

size_t linear_workspace_bytes(int64_t n, int32_t Cin, int32_t Cout, bool bf16, bool aligned) {
  return forward_layout(n, Cin, Cout, bf16, aligned).total;
}
size_t linear_backward_workspace_bytes(int64_t n, int32_t Cin, int32_t Cout, bool bf16,
                                       bool aligned, int act) {
  return backward_layout(n, Cin, Cout, bf16, aligned, act).total;
}

hipError_t launch_linear(const LinearArgs& a, hipStream_t stream) {
  const bool aligned = linear_aligned(a, false);
  const Forward w = forward_layout(a.n, a.Cin, a.Cout, a.bf16, aligned);
  Product p{};
  p.direct = !a.bf16 && direct_pays(a.n, a.Cin, a.Cout);
  if (p.direct) {
    p.A = direct_rows(a.x, a.ldx), p.B = direct_rows(a.W, a.ldw);
  } else {
    SHC_LAUNCH(operand(a.x, a.ldx, a.n, a.Cin, a.bf16, true, byte(a.ws, w.x), false, &p.A,
                       stream));
    SHC_LAUNCH(operand(a.W, a.ldw, a.Cin, a.Cout, a.bf16, false, byte(a.ws, w.W), false, &p.B,
                       stream));
  }
  p.a_rows = true, p.b_rows = false, p.split = !a.bf16;
  p.M = a.n, p.N = a.Cout, p.K = a.Cin;
  p.store.bias = a.bias, p.store.act = a.act;
  p.store.res = a.res, p.store.ld_res = a.ldres;
  p.store.pre = a.pre, p.store.ld_pre = a.ldpre;
  p.store.out = a.out, p.store.ld_out = a.ldout;
  p.partials = reinterpret_cast<float*>(byte(a.ws, w.partials));
  p.partial_bytes = w.partial_bytes;
  return launch_product(p, stream);
}

hipError_t launch_linear_backward(const LinearArgs& a, hipStream_t stream) {
  const bool aligned = linear_aligned(a, true);
  const Backward w = backward_layout(a.n, a.Cin, a.Cout, a.bf16, aligned, a.act);
  const bool products = a.dx != nullptr || a.dW != nullptr;
  // dz as the products read it: dout itself, or dz in the workspace
  const void* dz = a.dout;
  int64_t ld = a.lddout;
  const bool as_is = a.act == kActNone && (!a.bf16 || direct(a.dout, a.lddout, a.Cout));
  const bool write = products && !as_is;
  if (a.n > 0 && (write || a.db != nullptr)) {
    const GradShape g = grad_shape(a.n, a.Cout);
    GradRows r{a.dout, a.lddout, a.pre, a.ldpre, a.act, a.n, g.chunk, a.Cout, g.G, nullptr, 0,
               a.Cout, a.db != nullptr ? reinterpret_cast<float*>(byte(a.ws, w.sums)) : nullptr};
    if (write) {
      ld = a.bf16 ? packed_width(a.Cout) : a.Cout;
      r.dz = byte(a.ws, a.bf16 ? w.dz : w.dz32);
      r.ld_dz = ld;
      r.width = (int)ld;
      dz = r.dz;
    }
    const dim3 grid(g.cols, (unsigned)((a.n + g.chunk - 1) / g.chunk));
    if (a.bf16)
      grad_rows_kernel<true><<<grid, 256, 0, stream>>>(r);
    else
      grad_rows_kernel<false><<<grid, 256, 0, stream>>>(r);
    SHC_LAUNCH(hipGetLastError());
    if (a.db != nullptr)
      SHC_LAUNCH(launch_sum_rows(r.sums, grid.y, a.Cout, a.Cout, a.accumulate, a.db, stream));
  } else if (a.db != nullptr && !a.accumulate) {
    SHC_LAUNCH(launch_sum_rows(nullptr, 0, 0, a.Cout, 0, a.db, stream));
  }
  if (!products) return hipSuccess;
  if (a.n == 0 && (a.dW == nullptr || a.accumulate)) return hipSuccess;

  // the packed rows of dz in bf16 are read as they are: their width is dz's
  const int32_t dzC = a.bf16 && write ? (int32_t)ld : a.Cout;
  Operand rows{}, cols{};
  const bool dx_direct = !a.bf16 && direct_pays(a.n, a.Cout, a.Cin);
  if (a.n > 0) {
    void* to = byte(a.ws, w.dz);
    const bool pack = a.dW != nullptr || !dx_direct;
    SHC_LAUNCH(operand(dz, ld, a.n, dzC, a.bf16, true, to, !pack, &rows, stream));
    SHC_LAUNCH(operand(dz, ld, a.n, dzC, a.bf16, false, to, true, &cols, stream));
  }
  Product p{};
  p.split = !a.bf16;
  p.partials = reinterpret_cast<float*>(byte(a.ws, w.partials));
  p.partial_bytes = w.partial_bytes;
  if (a.dx != nullptr && a.n > 0) {
    p.direct = dx_direct;
    if (dx_direct) {
      p.A = direct_rows(dz, ld), p.B = direct_rows(a.W, a.ldw);
    } else {
      p.A = rows;
      SHC_LAUNCH(operand(a.W, a.ldw, a.Cin, a.Cout, a.bf16, true, byte(a.ws, w.W), false, &p.B,
                         stream));
    }
    p.a_rows = p.b_rows = true;
    p.M = a.n, p.N = a.Cin, p.K = a.Cout;
    p.store.out = a.dx, p.store.ld_out = a.lddx;
    SHC_LAUNCH(launch_product(p, stream));
  }
  if (a.dW != nullptr) {
    if (a.n > 0)
      SHC_LAUNCH(operand(a.x, a.ldx, a.n, a.Cin, a.bf16, false, byte(a.ws, w.x), false, &p.A,
                         stream));
    p.B = cols;
    p.direct = false;
    p.a_rows = p.b_rows = false;
    p.M = a.Cin, p.N = a.Cout, p.K = a.n;
    p.store.out = a.dW, p.store.ld_out = a.lddW;
    if (a.accumulate) p.store.res = a.dW, p.store.ld_res = a.lddW;
    SHC_LAUNCH(launch_product(p, stream));
  }
  return hipSuccess;
}

}  // namespace shc
