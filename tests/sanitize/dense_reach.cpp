// The offsets that the loads of the cross entropy's and the linear layer's products form, at the
// tile that is chosen for them, over their sizes: within 32 bits and what a descriptor covers.
// Host code alone, linked to the library; nothing is launched.
#include <stdio.h>

#include "../../paper_2608_09388_amd/csrc/dense.h"

using namespace shc::dense;

static long checked, bad;

// The largest offset that Side<R, rows_order, ...> forms from a tile's first element, in bytes,
// of the K_ of k to a step.
static int64_t last_byte(const Operand& o, bool rows_order, int64_t R, int64_t K_) {
  return rows_order ? ((R - 1) * o.ld + K_) * 2 : ((K_ - 1) * o.ld + R) * 2;
}

static void look(const Product& p, const char* what, long n, long C, long V) {
  const Plan plan = plan_of(p);
  const int64_t K_ = p.split ? BKS : BK;
  const int64_t a = last_byte(p.A, p.a_rows, tile_m(plan.kind), K_);
  const int64_t b = last_byte(p.B, p.b_rows, tile_n(plan.kind), K_);
  ++checked;
  if (a > 0x7FFFFFF0 || b > 0x7FFFFFF0) {
    if (++bad <= 5)
      printf("%s: n %ld C %ld V %ld split %d: tile %d, bytes %lld %lld\n", what, n, C, V, p.split,
             tile_m(plan.kind), (long long)a, (long long)b);
  }
}

static Operand at(int64_t ld) {
  Operand o{};
  o.ld = ld;
  return o;
}

int main() {
  const long ns[] = {1, 16, 33, 64, 65, 127, 128, 200, 256, 300, 1000, 4000, 67040};
  const long Cs[] = {1, 16, 64, 100, 256, 512, 1000, 1024, 2048, 4095, 16384, 65536};
  const long Vs[] = {1, 300, 50021, 131072, 1l << 20, 1l << 21, 4200000, 4210700, 4210800,
                     4500000, 8454600, 8454700, 8500000, (1l << 24) - 1, 1l << 24};
  float partials;
  for (long n : ns)
    for (long C : Cs)
      for (long V : Vs)
        for (int split = 0; split < 2; ++split) {
          const auto tiles = [](long a, long b) { return (a + 127) / 128 * ((b + 127) / 128); };
          if (tiles(n, V) >= 1l << 22 || tiles(V, C) >= 1l << 22) continue;
          const long rows = n < 256 ? n : 256;  // what a piece of so many classes has
          Product p{};
          p.split = split, p.a_low = !split && n <= 64;
          p.partials = &partials;
          p.partial_bytes = (size_t)128 << 20;
          p.A = at(packed_width(V));
          for (long ld : {(long)packed_width(C), (1l << 21) - 8}) {  // packed, or as they lie
            p.B = at(ld);
            p.a_rows = true, p.b_rows = false, p.M = rows, p.N = C, p.K = V;
            look(p, "dx", n, C, V);
            p.a_rows = p.b_rows = false, p.M = V, p.N = C, p.K = rows;
            look(p, "dW", n, C, V);
            Product l{};  // the linear layer's, C -> V
            if (V > 65536) continue;
            l.split = split, l.partials = &partials, l.partial_bytes = (size_t)128 << 20;
            l.A = l.B = at(ld);
            l.a_rows = true, l.b_rows = false, l.M = n, l.N = V, l.K = C;
            look(l, "linear", n, C, V);
            l.b_rows = true, l.N = C, l.K = V;
            look(l, "linear dx", n, C, V);
            l.a_rows = l.b_rows = false, l.M = C, l.N = V, l.K = n;
            look(l, "linear dW", n, C, V);
          }
        }
  // an operand that no tile reaches is refused before anything is launched
  Product p{};
  p.A = at(1l << 26), p.B = at(64);
  p.a_rows = true, p.M = 100, p.N = 64, p.K = 1l << 26;
  if (launch_product(p, nullptr) != hipErrorInvalidValue) ++bad;
  p.A = at(64), p.B = at(1l << 26);
  p.a_rows = p.b_rows = false, p.M = p.N = 64, p.K = 100;
  if (launch_product(p, nullptr) != hipErrorInvalidValue) ++bad;
  printf("checked %ld bad %ld\n", checked, bad);
  return bad != 0;
}
