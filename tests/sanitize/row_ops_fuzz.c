/*
 * Host-side fuzz of the row operators' entry points under AddressSanitizer and
 * UndefinedBehaviorSanitizer, as abi_fuzz.c does for the others: arguments drawn
 * from edge values, run only where no GPU is present (a call that passes
 * validation then stops at its first HIP call).
 */
#include <limits.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include "shc.h"

static uint64_t g_state = 0x9E3779B97F4A7C15ULL;
static uint64_t next_u64(void) { /* xorshift64* */
  g_state ^= g_state >> 12;
  g_state ^= g_state << 25;
  g_state ^= g_state >> 27;
  return g_state * 0x2545F4914F6CDD1DULL;
}
#define PICK(a) (a[(next_u64() >> 20) % (sizeof(a) / sizeof(a[0]))])

static void* const kP[] = {NULL, (void*)(uintptr_t)0x10000, (void*)(uintptr_t)0x10000,
                           (void*)(uintptr_t)0x20000, (void*)(uintptr_t)0x10002,
                           (void*)(uintptr_t)0x10001, (void*)(uintptr_t)0x7f0000001000ULL};
static const int64_t kN[] = {-7, -1, 0, 1, 2, 31, 33, 255, 256, 1000, 67040, 1 << 20, 1 << 28,
                             (1 << 28) + 1, INT32_MAX, (int64_t)INT32_MAX + 1, INT64_MAX / 2,
                             INT64_MAX};
static const int64_t kS[] = {INT64_MIN, -1, 0, 1, 2, 64, 128, 4096, 65536, 140001, 1 << 24,
                             (int64_t)1 << 40, ((int64_t)1 << 40) + 1, INT64_MAX};
static const int32_t kC[] = {INT32_MIN, -1, 0, 1, 7, 16, 64, 128, 1000, 4096, 5001, 16384, 16385,
                             65536, 65537, 140001, 1 << 24, (1 << 24) + 1, INT32_MAX};
static const int32_t kK[] = {-1, 0, 1, 8, 64, 256, 257, INT32_MAX};
static const int32_t kCode[] = {-1, 0, 1, 0, 1, 2};
static const float kF[] = {0.0f, 1e-5f, 1.0f, 2.0f, -1.0f, 3e38f, INFINITY, NAN};
static const size_t kB[] = {0, 15, 4096, (size_t)1 << 40, SIZE_MAX};

#define P() PICK(kP)
#define N() PICK(kN)
#define S() PICK(kS)
#define C() PICK(kC)
#define K() PICK(kK)
#define CODE() PICK(kCode)
#define F() PICK(kF)
#define B() PICK(kB)

static long g_calls = 0, g_ok = 0;
static int g_bad = 0;

static void check(int rc, const char* fn) {
  ++g_calls;
  g_ok += rc == 0;
  const char* e = shc_last_error();
  if (rc > 0 || rc < -5 || e == NULL || strnlen(e, 1024) >= 512) {
    fprintf(stderr, "%s returned %d\n", fn, rc);
    g_bad = 1;
  }
}

int main(void) {
  int count = 0;
  if (hipGetDeviceCount(&count) == hipSuccess && count > 0) {
    fprintf(stderr, "a GPU is present\n");
    return 2;
  }
  for (int i = 0; i < 40000 && !g_bad; ++i) {
    check(shc_embed_rows(P(), S(), N(), P(), CODE(), S(), N(), C(), F(), P(), S(), CODE(), P(),
                         S(), NULL), "shc_embed_rows");
    check(shc_embed_rows_backward(P(), S(), P(), CODE(), S(), N(), N(), C(), F(), S(), CODE(),
                                  CODE(), P(), S(), P(), B(), NULL), "shc_embed_rows_backward");
    check(shc_layer_norm(P(), S(), N(), C(), P(), P(), F(), CODE(), P(), S(), P(), P(), NULL),
          "shc_layer_norm");
    check(shc_layer_norm_backward(P(), S(), P(), S(), N(), C(), P(), P(), P(), CODE(), CODE(), P(),
                                  S(), P(), P(), P(), B(), NULL), "shc_layer_norm_backward");
    check(shc_distill_top(P(), S(), N(), C(), P(), P(), K(), F(), CODE(), P(), P(), P(), B(),
                          NULL), "shc_distill_top");
    check(shc_distill_top_backward(P(), S(), N(), C(), P(), P(), K(), F(), P(), P(), CODE(), P(),
                                   S(), NULL), "shc_distill_top_backward");
    check(shc_distill_top_step(P(), S(), N(), C(), P(), P(), K(), F(), P(), CODE(), P(), P(), S(),
                               P(), B(), NULL), "shc_distill_top_step");
    (void)shc_embed_rows_backward_workspace(N(), N(), C());
    (void)shc_layer_norm_backward_workspace(N(), C());
    (void)shc_distill_top_workspace(N(), C());
  }
  /* calls that pass validation, stopped at the launch (no GPU here) */
  void* a = (void*)(uintptr_t)0x10000;
  const size_t big = (size_t)1 << 40;
  for (int i = 0; i < 2000 && !g_bad; ++i) {
    static const int64_t n_ok[] = {1, 3, 255, 256, 5000, 67040, 3000000};
    static const int32_t c_ok[] = {1, 7, 64, 128, 1000, 4096, 9000, 16384};
    const int64_t n = PICK(n_ok);
    const int32_t c = PICK(c_ok), dt = (int32_t)(next_u64() >> 40 & 1);
    check(shc_embed_rows(a, c, 100, a, dt, 1, n, c, 1.0f, NULL, 0, dt, a, c, NULL), "embed");
    check(shc_embed_rows_backward(a, c, a, dt, 1, n, 100, c, 1.0f, -1, dt, 0, a, c, a, big, NULL),
          "embed backward");
    check(shc_layer_norm(a, c, n, c, a, a, 1e-5f, dt, a, c, a, a, NULL), "norm");
    check(shc_layer_norm_backward(a, c, a, c, n, c, a, a, a, dt, 0, a, c, a, a, a, big, NULL),
          "norm backward");
    check(shc_distill_top(a, 16 * c, n, 16 * c, a, a, 8, 1.0f, dt, a, a, a, big, NULL), "distill");
    check(shc_distill_top_backward(a, 16 * c, n, 16 * c, a, a, 8, 1.0f, a, a, dt, a, 16 * c, NULL),
          "distill backward");
    check(shc_distill_top_step(a, 16 * c, n, 16 * c, a, a, 8, 1.0f, a, dt, a, a, 16 * c, a, big,
                               NULL), "distill step");
  }
  printf("calls %ld ok %ld bad %d\n", g_calls, g_ok, g_bad);
  return g_bad;
}
