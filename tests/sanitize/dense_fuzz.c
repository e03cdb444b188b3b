/* The dense operators' host code under a sanitizer, without a GPU: random arguments, most
 * of them wrong in one place.  Valid ones end in a HIP error (no device). */
#include <stdio.h>
#include <stdlib.h>

#include "shc.h"

static uint64_t seed = 88172645463325252ull;
static uint64_t next(void) {
  seed ^= seed << 13;
  seed ^= seed >> 7;
  return seed ^= seed << 17;
}
static int64_t pick(const int64_t* v, int n) { return v[next() % n]; }
#define PICK(...) pick((const int64_t[]){__VA_ARGS__}, sizeof((int64_t[]){__VA_ARGS__}) / 8)

static void* ptr(void) {
  return (void*)(uintptr_t)PICK(0, 0x10000, 0x10002, 0x10004, 0x10001, 0x7fff0000, 0x10000, 0x10000);
}
static int64_t rows(void) {
  return PICK(0, 1, 2, 32, 33, 100, 4096, 70000, -1, (1 << 27) - 1, 1 << 27, INT64_MAX, 300, 1000);
}
static int32_t width(void) {
  return (int32_t)PICK(1, 8, 63, 64, 65, 128, 1000, 4096, 65536, 65537, 0, -5, INT32_MAX, 16);
}
static int64_t stride(int32_t w) {
  return PICK(w, w, w, (int64_t)w + 1, (int64_t)w + 64, 0, -1, INT64_MAX, (int64_t)1 << 40, 1 << 21);
}
static int32_t small(void) { return (int32_t)PICK(0, 0, 1, 1, 2, 3, -1, 7); }

static long calls, bad;
static void check(int rc) {
  ++calls;
  if (rc > 0 || rc < SHC_ERR_HIP || (rc != 0) != (shc_last_error()[0] != 0)) ++bad;
}

int main(void) {
  int devices = 0;
  if (hipGetDeviceCount(&devices) == hipSuccess && devices > 0) {
    fprintf(stderr, "a GPU is present\n");
    return 2;
  }
  const size_t big = (size_t)1 << 62;
  for (int i = 0; i < 60000; ++i) {
    const int64_t n = rows();
    const int32_t a = width(), b = width(), dt = (int32_t)PICK(0, 1, 0, 1, 0, 1, 2);
    const int32_t V = (int32_t)PICK(1, 48, 1000, 50021, 131072, 1 << 24, (1 << 24) + 1, 0, a > 0 ? a : 1);
    const int32_t act = small(), acc = (int32_t)PICK(0, 1, 0, 1, 2), al = small();
    const size_t ws = PICK(0, 16, 1) == 0 ? big : (size_t)PICK(0, 1000, 1 << 20);
    check(shc_linear(ptr(), stride(a), n, a, ptr(), stride(b), b, ptr(), act, ptr(), stride(b), dt,
                     ptr(), stride(b), ptr(), stride(b), ptr(), ws, 0));
    check(shc_linear_backward(ptr(), stride(b), ptr(), stride(a), n, a, ptr(), stride(b), b, ptr(),
                              stride(b), act, dt, acc, ptr(), stride(a), ptr(), stride(b), ptr(),
                              ptr(), ws, 0));
    check(shc_linear_cross_entropy(ptr(), stride(a), n, a, ptr(), stride(a), V, ptr(), ptr(),
                                   small(), PICK(0, 1, 2, -1, INT64_MAX), dt, ptr(), ptr(), ptr(),
                                   ws, 0));
    check(shc_linear_cross_entropy_backward(ptr(), stride(a), n, a, ptr(), stride(a), V, ptr(),
                                            ptr(), small(), 1, ptr(), ptr(), dt, acc, ptr(),
                                            stride(a), ptr(), stride(a), ptr(), ptr(), ws, 0));
    check(shc_linear_cross_entropy_step(ptr(), stride(a), n, a, ptr(), stride(a), V, ptr(), ptr(),
                                        small(), 1, ptr(), dt, acc, ptr(), ptr(), stride(a),
                                        ptr(), stride(a), ptr(), ptr(), ws, 0));
    shc_grad g[300];
    const int64_t count = PICK(0, 1, 2, 5, 127, 128, 129, 300, -1);
    for (int64_t k = 0; k < 300; ++k) {
      const int odd = next() % 97 == 0;
      g[k].data = odd ? ptr() : (void*)(uintptr_t)(0x100000 + k * 0x10000);
      g[k].out = odd ? ptr() : (void*)(uintptr_t)(next() % 2 ? 0x10000000 + k * 0x10000
                                                             : 0x100000 + k * 0x10000);
      g[k].numel = odd ? PICK(0, -1, INT64_MAX, (int64_t)1 << 40, 100000) : (int64_t)(next() % 4096);
      g[k].dtype = odd ? small() : (int32_t)(next() % 2);
    }
    check(shc_grad_norm(g, count, ptr(), ptr(), ws, 0));
    check(shc_clip_grads(g, count, ptr(), (float)PICK(0, 1, -1, 5), 0));
    volatile size_t sizes = shc_linear_workspace(n, a, b, dt, al) +
                            shc_linear_backward_workspace(n, a, b, dt, act, al) +
                            shc_linear_cross_entropy_workspace(n, a, V, dt, small(), al) +
                            shc_grad_norm_workspace(g, count);
    (void)sizes;
  }
  /* calls that pass validation, stopped at their first launch */
#define AT(k) ((void*)(uintptr_t)((uint64_t)(k) << 41))
  long launched = 0;
  for (int i = 0; i < 3000; ++i) {
    const int64_t n = PICK(1, 2, 31, 32, 33, 300, 5000, 67040);
    const int32_t a = (int32_t)PICK(1, 7, 64, 128, 1000, 4096), dt = (int32_t)PICK(0, 1);
    const int32_t b = (int32_t)PICK(1, 9, 64, 512, 5001, 16384);
    const int32_t act = (int32_t)PICK(0, 1, 2, 3), acc = (int32_t)PICK(0, 1);
    const int64_t lda = a + PICK(0, 0, 3, 8), ldb = b + PICK(0, 0, 5, 16);
    int rc[7];
    check(rc[0] = shc_linear(AT(1), lda, n, a, AT(2), ldb, b, AT(3), act, AT(4), ldb, dt, AT(5),
                             ldb, AT(6), ldb, AT(9), big, 0));
    check(rc[1] = shc_linear_backward(AT(1), ldb, AT(2), lda, n, a, AT(3), ldb, b,
                                      act ? AT(4) : 0, ldb, act, dt, acc, AT(5), lda, AT(6), ldb,
                                      AT(7), AT(9), big, 0));
    check(rc[2] = shc_linear_cross_entropy(AT(1), lda, n, a, AT(2), lda, b, AT(3), AT(4), dt, 1,
                                           dt, AT(5), AT(6), AT(9), big, 0));
    check(rc[3] = shc_linear_cross_entropy_backward(AT(1), lda, n, a, AT(2), lda, b, AT(3), AT(4),
                                                    0, 2, AT(5), AT(6), dt, acc, AT(7), lda,
                                                    AT(8), lda, AT(10), AT(9), big, 0));
    check(rc[4] = shc_linear_cross_entropy_step(AT(1), lda, n, a, AT(2), lda, b, AT(3), AT(4), 1,
                                                1, AT(5), dt, acc, AT(6), AT(7), lda, AT(8), lda,
                                                AT(10), AT(9), big, 0));
    shc_grad g[300];
    for (int k = 0; k < 300; ++k)
      g[k] = (shc_grad){AT(k + 1), next() % 2 ? AT(k + 1) : AT(k + 1000), (int64_t)(next() % 100000),
                        (int32_t)(next() % 2)};
    const int64_t count = PICK(1, 127, 128, 129, 300);
    check(rc[5] = shc_grad_norm(g, count, AT(2000), AT(2001), big, 0));
    check(rc[6] = shc_clip_grads(g, count, AT(2000), 1.f, 0));
    for (int k = 0; k < 7; ++k) {
      launched += rc[k] == SHC_ERR_HIP;
      bad += rc[k] != SHC_ERR_HIP;
    }
  }
  printf("calls %ld bad %ld launched %ld\n", calls, bad, launched);
  return bad != 0;
}
