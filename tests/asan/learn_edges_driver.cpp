// Drives ends of the ranges that the learning entry points accept, on the CPU against the
// stub HIP runtime, under the address and undefined-behaviour sanitizers.
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include "sagips.h"

extern "C" {
long stub_bad_launches();
long stub_live_events();
long stub_live_allocs();
}

namespace {

int g_fail = 0, g_checks = 0;

// Fake device memory, 16 GiB apart.
template <class T = float>
T* dev(uint64_t i) {
  return reinterpret_cast<T*>((uintptr_t)0x100000000000ull + (i << 34));
}

void expect(const char* what, long got, long want, sagips_ctx* c) {
  ++g_checks;
  if (got == want) return;
  ++g_fail;
  printf("FAIL %s: %ld, expected %ld (%s)\n", what, got, want, sagips_last_error(c));
}

sagips_newton_schulz coefficients(int steps, double a, double b, double c) {
  sagips_newton_schulz ns;
  memset(&ns, 0, sizeof(ns));
  ns.steps = steps;
  ns.coef[0] = a;
  ns.coef[1] = b;
  ns.coef[2] = c;
  ns.eps = 1e-7;
  return ns;
}

// The polynomial's largest value lies inside its range, also where c is so small that
// sqrt(9 b^2 - 20 a c) rounds to 3 |b|: 9 s - 9 s^3 reaches 3.46 and then diverges.
void bounds_of_coefficients(sagips_ctx* c) {
  const double tiny[] = {0.0, 1e-30, -1e-30, 1e-12};
  for (double k : tiny) {
    const sagips_newton_schulz one = coefficients(1, 9.0, -9.0, k), two = coefficients(2, 9.0, -9.0, k);
    expect("one step of 9 s - 9 s^3", sagips_orthogonalise(c, &one, SAGIPS_F32, dev(1), 1, 8, 8, dev(2)), SAGIPS_OK, c);
    expect("two steps of 9 s - 9 s^3", sagips_orthogonalise(c, &two, SAGIPS_F32, dev(1), 1, 8, 8, dev(2)), SAGIPS_E_UNSUPPORTED, c);
    const sagips_newton_schulz neg = coefficients(2, -9.0, 9.0, -k);
    expect("its negative", sagips_orthogonalise(c, &neg, SAGIPS_F32, dev(1), 1, 8, 8, dev(2)), SAGIPS_E_UNSUPPORTED, c);
  }
  const sagips_newton_schulz odd[] = {coefficients(5, 0.0, 0.0, 1.0), coefficients(5, 0.0, 1.0, 0.0), coefficients(5, 1.0, 0.0, 0.0),
                                      coefficients(5, 0.0, 1.0, -1.0)};
  for (const sagips_newton_schulz& ns : odd)
    expect("some coefficients zero", sagips_orthogonalise(c, &ns, SAGIPS_F32, dev(1), 1, 8, 8, dev(2)), SAGIPS_OK, c);
}

}  // namespace

int main() {
  sagips_ctx* c = nullptr;
  expect("create", sagips_create(&c, 0, nullptr), SAGIPS_OK, nullptr);
  bounds_of_coefficients(c);
  sagips_destroy(c);
  expect("events left behind", stub_live_events(), 0, nullptr);
  expect("allocations left behind", stub_live_allocs(), 0, nullptr);
  expect("bad launches", stub_bad_launches(), 0, nullptr);
  printf("%d checks, %d failures\n", g_checks, g_fail);
  if (!g_fail) printf("ALL OK\n");
  return g_fail ? 1 : 0;
}
