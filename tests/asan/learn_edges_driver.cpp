// Drives ends of the ranges that the learning entry points accept, on the CPU against the
// stub HIP runtime, under the address and undefined-behaviour sanitizers.
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include <initializer_list>

#include "sagips.h"

extern "C" {
long stub_launches();
long stub_mallocs();
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

// Stacks of every accepted size have a workspace of at most 2 GiB, which is as much as the stub gives,
// or of one matrix.
void large_stacks(sagips_ctx* c) {
  const sagips_newton_schulz ns = coefficients(5, 0.0, 0.0, 0.0);
  const int shapes[][3] = {{65535, 1, 16384}, {65535, 16384, 1}, {65535, 2, 16383}, {65535, 1, 513}, {7000, 513, 513}, {1000, 1024, 2048},
                           {4, 4096, 16384}, {2, 16384, 16384}};
  for (const auto& s : shapes)
    for (int type : {SAGIPS_F32, SAGIPS_BF16}) {
      const bool large = s[1] == 16384 && s[2] == 16384;    // one matrix alone needs more
      expect("orthogonalise a large stack", sagips_orthogonalise(c, &ns, type, dev(1), s[0], s[1], s[2], dev(8)),
             large ? SAGIPS_E_NOMEM : SAGIPS_OK, c);
    }
  sagips_matrix_set set;
  memset(&set, 0, sizeof(set));
  set.n_tensors = 3;
  for (int i = 0; i < 3; ++i) {
    set.param[i] = dev(10 + 3 * i);
    set.grad[i] = dev(11 + 3 * i);
    set.m[i] = dev(12 + 3 * i);
    set.count[i] = 20000;
    set.rows[i] = i == 1 ? 16384 : 1;
    set.cols[i] = i == 1 ? 1 : 16384;
  }
  sagips_muon mu;
  memset(&mu, 0, sizeof(mu));
  mu.lr = 0.02;
  mu.ns = ns;
  expect("step on large stacks", sagips_muon_step(c, &set, &mu), SAGIPS_OK, c);
}

// The launches and allocations of one small policy loss.
struct Cost {
  long launches, mallocs;
};
Cost policy_cost(sagips_ctx* c) {
  sagips_policy p;
  memset(&p, 0, sizeof(p));
  p.theta = dev(1);
  p.theta_old = dev(2);
  p.n_theta = 4;
  p.d = 2;
  p.events_per_theta = 100;
  const long n = stub_launches(), m = stub_mallocs();
  expect("policy", sagips_policy_loss(c, &p, dev(4), dev(5), nullptr, dev(7), nullptr, nullptr, dev(8)), SAGIPS_OK, c);
  return {stub_launches() - n, stub_mallocs() - m};
}

// A call that ends in its last workgroup launches and allocates nothing else, the context's first
// no more than a later one: a first call that is being captured into a graph leaves no preparation
// to the replay.  Contexts beyond those that have counters launch twice; one that ends gives its
// counters on.
void counters_of_contexts() {
  const int n = 70, sets = 64;
  static sagips_ctx* c[n];
  for (int again = 0; again < 2; ++again) {
    int once = 0;
    for (int i = 0; i < n; ++i) {
      expect("create", sagips_create(&c[i], 0, nullptr), SAGIPS_OK, nullptr);
      const Cost first = policy_cost(c[i]), second = policy_cost(c[i]);
      expect("workspace of the first call", first.mallocs, 1, c[i]);
      expect("allocations of the second", second.mallocs, 0, c[i]);
      expect("launches of the second", second.launches, first.launches, c[i]);
      if (first.launches == 1) ++once;
      else expect("launches without counters", first.launches, 2, c[i]);
    }
    expect("contexts with counters", once, sets, nullptr);
    for (int i = 0; i < n; ++i) sagips_destroy(c[i]);
  }
}

}  // namespace

int main() {
  sagips_ctx* c = nullptr;
  expect("create", sagips_create(&c, 0, nullptr), SAGIPS_OK, nullptr);
  bounds_of_coefficients(c);
  large_stacks(c);
  sagips_destroy(c);
  counters_of_contexts();
  expect("events left behind", stub_live_events(), 0, nullptr);
  expect("allocations left behind", stub_live_allocs(), 0, nullptr);
  expect("bad launches", stub_bad_launches(), 0, nullptr);
  printf("%d checks, %d failures\n", g_checks, g_fail);
  if (!g_fail) printf("ALL OK\n");
  return g_fail ? 1 : 0;
}
