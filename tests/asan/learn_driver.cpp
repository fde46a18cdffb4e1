// Drives the learning entry points of libsagips's C ABI (advantages, policy and
// preference loss, orthogonalisation, the step on it) on the CPU against the stub
// HIP runtime, under the address and undefined-behaviour sanitizers: every
// documented error path, and valid calls over the range of sizes, whose launch
// shapes the stub checks.
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include <initializer_list>

#include "sagips.h"

extern "C" {
long stub_launches();
long stub_bad_launches();
long stub_live_events();
long stub_live_allocs();
void stub_set_malloc_limit(size_t n);
}

namespace {

int g_fail = 0, g_checks = 0;

// Fake device memory, 16 GiB apart.
template <class T = float>
T* dev(uint64_t i) {
  return reinterpret_cast<T*>((uintptr_t)0x100000000000ull + (i << 34));
}

void expect(const char* what, sagips_status got, sagips_status want, sagips_ctx* c) {
  ++g_checks;
  const char* msg = sagips_last_error(c);
  if (got != want || !msg || (want != SAGIPS_OK && strlen(msg) == 0)) {
    ++g_fail;
    printf("FAIL %s: status %d, expected %d (%s)\n", what, (int)got, (int)want, msg ? msg : "(null message)");
  }
}

sagips_policy policy(int n, int d, int64_t E) {
  sagips_policy p;
  memset(&p, 0, sizeof(p));
  p.theta = dev(1);
  p.theta_old = dev(2);
  p.theta_ref = dev(3);
  p.n_theta = n;
  p.d = d;
  p.events_per_theta = E;
  p.clip_low = p.clip_high = 0.2;
  p.kl_coef = 0.1;
  return p;
}
sagips_preference preference(int n, int d, int64_t pairs, int64_t T, int64_t T2) {
  sagips_preference p;
  memset(&p, 0, sizeof(p));
  p.theta = dev(1);
  p.theta_ref = dev(2);
  p.n_theta = n;
  p.d = d;
  p.pairs_per_theta = pairs;
  p.len_chosen = T;
  p.len_rejected = T2;
  p.beta = 0.1;
  return p;
}
sagips_matrix_set matrices(int n, int count, int rows, int cols, int type) {
  sagips_matrix_set s;
  memset(&s, 0, sizeof(s));
  s.n_tensors = n;
  s.grad_type = type;
  for (int i = 0; i < n; ++i) {
    s.param[i] = dev(10 + 3 * i);
    s.grad[i] = dev(11 + 3 * i);
    s.m[i] = dev(12 + 3 * i);
    s.count[i] = count;
    s.rows[i] = rows + i;
    s.cols[i] = cols;
  }
  return s;
}

}  // namespace

int main() {
  const sagips_status OK = SAGIPS_OK, INVAL = SAGIPS_E_INVAL, UNSUP = SAGIPS_E_UNSUPPORTED, NOMEM = SAGIPS_E_NOMEM;
  sagips_ctx* c = nullptr;
  expect("create", sagips_create(&c, 0, nullptr), OK, nullptr);

  // ---- advantages
  const auto adv = [&](const float* r, const uint8_t* m, int n, int64_t E, double eps, float* a) {
    return sagips_group_advantage(c, r, m, n, E, 1, eps, a);
  };
  const int64_t lengths[] = {1, 2, 63, 64, 65, 1023, 1024, 1025, 16384, 16385, 1000000};
  for (int64_t E : lengths)
    for (int64_t n : {(int64_t)1, (int64_t)7, (((int64_t)1 << 31) - 1) / E})
      expect("advantage ok", adv(dev(1), E % 2 ? dev<uint8_t>(2) : nullptr, (int)n, E, 1e-6, dev(3)), OK, c);
  expect("advantage in place", adv(dev(1), nullptr, 4, 100, 0.0, dev(1)), OK, c);
  expect("advantage ctx NULL", sagips_group_advantage(nullptr, dev(1), nullptr, 1, 1, 1, 0.0, dev(2)), INVAL, nullptr);
  expect("advantage reward NULL", adv(nullptr, nullptr, 4, 100, 0.0, dev(1)), INVAL, c);
  expect("advantage adv NULL", adv(dev(1), nullptr, 4, 100, 0.0, nullptr), INVAL, c);
  expect("advantage misaligned", adv(dev(1) + 1, nullptr, 4, 100, 0.0, dev(2)), INVAL, c);
  expect("advantage no rows", adv(dev(1), nullptr, 0, 100, 0.0, dev(2)), INVAL, c);
  expect("advantage no events", adv(dev(1), nullptr, 4, 0, 0.0, dev(2)), INVAL, c);
  expect("advantage 2^31 events", adv(dev(1), nullptr, 1 << 16, 1 << 15, 0.0, dev(2)), INVAL, c);
  expect("advantage eps < 0", adv(dev(1), nullptr, 4, 100, -1.0, dev(2)), INVAL, c);
  expect("advantage eps NaN", adv(dev(1), nullptr, 4, 100, NAN, dev(2)), INVAL, c);
  expect("advantage overlap", adv(dev(1), nullptr, 4, 100, 0.0, dev(1) + 16), INVAL, c);
  expect("advantage mask overlap", adv(dev(1), reinterpret_cast<uint8_t*>(dev(2) + 4), 4, 100, 0.0, dev(2)), INVAL, c);

  // ---- policy loss
  const auto pol = [&](const sagips_policy* p) {
    return sagips_policy_loss(c, p, dev(4), dev(5), dev<uint8_t>(6), dev(7), dev(8), dev(9), dev(10));
  };
  for (int d : {2, 3})
    for (int64_t E : lengths)
      for (int64_t n : {(int64_t)1, (int64_t)9, (int64_t)65535}) {
        if (n * E >= ((int64_t)1 << 31)) continue;
        sagips_policy p = policy((int)n, d, E);
        p.average = E % 2;
        if (E % 3 == 0) p.theta_ref = nullptr;
        expect("policy ok", pol(&p), OK, c);
      }
  {
    sagips_policy p = policy(4, 2, 100);
    expect("policy only the loss", sagips_policy_loss(c, &p, dev(4), dev(5), nullptr, dev(7), nullptr, nullptr, nullptr), OK, c);
    expect("policy only the gradient", sagips_policy_loss(c, &p, dev(4), dev(5), nullptr, nullptr, nullptr, nullptr, dev(7)), OK, c);
    expect("policy no output", sagips_policy_loss(c, &p, dev(4), dev(5), nullptr, nullptr, nullptr, nullptr, nullptr), INVAL, c);
    expect("policy ctx NULL", sagips_policy_loss(nullptr, &p, dev(4), dev(5), nullptr, dev(7), nullptr, nullptr, nullptr), INVAL, nullptr);
    expect("policy P NULL", pol(nullptr), INVAL, c);
    expect("policy x NULL", sagips_policy_loss(c, &p, nullptr, dev(5), nullptr, dev(7), nullptr, nullptr, nullptr), INVAL, c);
    expect("policy adv NULL", sagips_policy_loss(c, &p, dev(4), nullptr, nullptr, dev(7), nullptr, nullptr, nullptr), INVAL, c);
    expect("policy x misaligned", sagips_policy_loss(c, &p, dev(4) + 1, dev(5), nullptr, dev(7), nullptr, nullptr, nullptr), INVAL, c);
#define BAD(what, change)              \
  {                                    \
    sagips_policy q = p;               \
    change;                            \
    expect("policy " what, pol(&q), INVAL, c); \
  }
    BAD("theta NULL", q.theta = nullptr)
    BAD("theta_old NULL", q.theta_old = nullptr)
    BAD("theta_ref misaligned", q.theta_ref = reinterpret_cast<float*>((char*)dev(3) + 2))
    BAD("no rows", q.n_theta = 0)
    BAD("65536 rows", q.n_theta = 65536)
    BAD("d 4", q.d = 4)
    BAD("no events", q.events_per_theta = 0)
    BAD("2^31 events", q.events_per_theta = (int64_t)1 << 29)
    BAD("events overflow", q.events_per_theta = INT64_MAX)
    BAD("clip_low 1.1", q.clip_low = 1.1)
    BAD("clip_high NaN", q.clip_high = NAN)
    BAD("kl_coef < 0", q.kl_coef = -0.1)
    BAD("kl_coef inf", q.kl_coef = INFINITY)
    BAD("average 2", q.average = 2)
#undef BAD
  }

  // ---- preference loss
  const auto pref = [&](const sagips_preference* p) {
    return sagips_preference_loss(c, p, dev(4), dev<int32_t>(5), dev(6), nullptr, dev(7), dev(8), dev(9));
  };
  for (int d : {2, 3})
    for (int64_t T : lengths)
      for (int64_t pairs : {(int64_t)1, (int64_t)13, (int64_t)5000})
        for (int n : {1, 17, 65535}) {
          if (T * pairs * n >= ((int64_t)1 << 31)) continue;
          sagips_preference p = preference(n, d, pairs, T, T % 2 ? T : 1);
          expect("preference ok", pref(&p), OK, c);
        }
  {
    sagips_preference p = preference(4, 2, 3, 10, 12);
    expect("preference only the margin", sagips_preference_loss(c, &p, dev(4), nullptr, dev(6), nullptr, nullptr, dev(8), nullptr), OK, c);
    expect("preference no output", sagips_preference_loss(c, &p, dev(4), nullptr, dev(6), nullptr, nullptr, nullptr, nullptr), INVAL, c);
    expect("preference ctx NULL", sagips_preference_loss(nullptr, &p, dev(4), nullptr, dev(6), nullptr, dev(7), nullptr, nullptr), INVAL, nullptr);
    expect("preference P NULL", pref(nullptr), INVAL, c);
    expect("preference chosen NULL", sagips_preference_loss(c, &p, nullptr, nullptr, dev(6), nullptr, dev(7), nullptr, nullptr), INVAL, c);
    expect("preference rejected misaligned", sagips_preference_loss(c, &p, dev(4), nullptr, dev(6) + 2, nullptr, dev(7), nullptr, nullptr), INVAL, c);
    expect("preference lengths misaligned",
           sagips_preference_loss(c, &p, dev(4), reinterpret_cast<int32_t*>((char*)dev(5) + 2), dev(6), nullptr, dev(7), nullptr, nullptr),
           INVAL, c);
#define BAD(what, change)                          \
  {                                                \
    sagips_preference q = p;                       \
    change;                                        \
    expect("preference " what, pref(&q), INVAL, c); \
  }
    BAD("theta_ref NULL", q.theta_ref = nullptr)
    BAD("d 1", q.d = 1)
    BAD("no pairs", q.pairs_per_theta = 0)
    BAD("no events", q.len_chosen = 0)
    BAD("rejected < 0", q.len_rejected = -1)
    BAD("2^31 events", q.len_chosen = (int64_t)1 << 28)
    BAD("beta 0", q.beta = 0.0)
    BAD("beta NaN", q.beta = NAN)
    BAD("label_smoothing 2", q.label_smoothing = 2.0)
#undef BAD
  }

  // ---- orthogonalisation and the step
  sagips_newton_schulz ns;
  memset(&ns, 0, sizeof(ns));
  ns.eps = 1e-7;
  const auto orth = [&](const sagips_newton_schulz* o, int type, int n, int r, int k) {
    return sagips_orthogonalise(c, o, type, dev(1), n, r, k, dev(2));
  };
  for (int type : {SAGIPS_F32, SAGIPS_BF16})
    for (int r : {1, 31, 32, 33, 64, 65, 128, 129, 200, 513, 2048})
      for (int k : {1, 40, 128, 129, 256, 300, 512, 700, 4096})
        for (int n : {1, 3, 300}) {
          if ((int64_t)n * r * k > 20000000) continue;     // the stub's memory
          expect("orthogonalise ok", orth(&ns, type, n, r, k), OK, c);
        }
  expect("orthogonalise 65535", orth(&ns, SAGIPS_F32, 65535, 8, 8), OK, c);
  expect("orthogonalise in place", sagips_orthogonalise(c, &ns, SAGIPS_F32, dev(1), 2, 30, 30, dev(1)), OK, c);
  expect("orthogonalise overlap", sagips_orthogonalise(c, &ns, SAGIPS_F32, dev(1), 2, 30, 30, dev(1) + 64), INVAL, c);
  expect("orthogonalise ctx NULL", sagips_orthogonalise(nullptr, &ns, SAGIPS_F32, dev(1), 2, 30, 30, dev(2)), INVAL, nullptr);
  expect("orthogonalise ns NULL", orth(nullptr, SAGIPS_F32, 1, 8, 8), INVAL, c);
  expect("orthogonalise x NULL", sagips_orthogonalise(c, &ns, SAGIPS_F32, nullptr, 2, 30, 30, dev(1)), INVAL, c);
  expect("orthogonalise misaligned", sagips_orthogonalise(c, &ns, SAGIPS_F32, dev(1) + 1, 2, 30, 30, dev(2)), INVAL, c);
  expect("orthogonalise type 2", orth(&ns, 2, 1, 8, 8), INVAL, c);
  expect("orthogonalise no matrices", orth(&ns, SAGIPS_F32, 0, 8, 8), INVAL, c);
  expect("orthogonalise 65536 matrices", orth(&ns, SAGIPS_F32, 65536, 8, 8), INVAL, c);
  expect("orthogonalise 0 rows", orth(&ns, SAGIPS_F32, 1, 0, 8), INVAL, c);
  expect("orthogonalise 16385 cols", orth(&ns, SAGIPS_F32, 1, 8, 16385), INVAL, c);
  expect("orthogonalise 2^31 elements", orth(&ns, SAGIPS_F32, 8, 16384, 16384), INVAL, c);
  {
    sagips_newton_schulz o = ns;
    o.steps = 17;
    expect("steps 17", orth(&o, SAGIPS_F32, 1, 8, 8), INVAL, c);
    o = ns;
    o.steps = -1;
    expect("steps -1", orth(&o, SAGIPS_F32, 1, 8, 8), INVAL, c);
    o = ns;
    o.eps = 0.0;
    expect("eps 0", orth(&o, SAGIPS_F32, 1, 8, 8), INVAL, c);
    o = ns;
    o.coef[0] = NAN;
    expect("coef NaN", orth(&o, SAGIPS_F32, 1, 8, 8), INVAL, c);
    o = ns;
    o.coef[0] = 3.0;
    expect("coef that diverge", orth(&o, SAGIPS_F32, 1, 8, 8), UNSUP, c);
    o.coef[0] = 1.5;
    o.coef[1] = -0.5;
    expect("cubic coef", orth(&o, SAGIPS_F32, 1, 8, 8), OK, c);
    o.coef[0] = 1.0;
    o.coef[1] = -20.0;
    expect("coef of a large polynomial", orth(&o, SAGIPS_F32, 1, 8, 8), UNSUP, c);
    stub_set_malloc_limit(1 << 20);
    sagips_ctx* c2 = nullptr;
    expect("create", sagips_create(&c2, 0, nullptr), OK, nullptr);
    expect("orthogonalise without memory", sagips_orthogonalise(c2, &ns, SAGIPS_F32, dev(1), 1, 2048, 2048, dev(2)), NOMEM, c2);
    expect("orthogonalise small without workspace", sagips_orthogonalise(c2, &ns, SAGIPS_F32, dev(1), 9, 100, 100, dev(2)), OK, c2);
    stub_set_malloc_limit(0);
    sagips_policy p = policy(4, 2, 10);
    expect("policy without memory",
           sagips_policy_loss(c2, &p, dev(4), dev(5), nullptr, dev(7), nullptr, nullptr, nullptr), NOMEM, c2);
    stub_set_malloc_limit((size_t)1 << 31);
    sagips_destroy(c2);
  }
  sagips_muon mu;
  memset(&mu, 0, sizeof(mu));
  mu.lr = 0.02;
  mu.momentum = 0.95;
  mu.nesterov = 1;
  mu.scale = SAGIPS_SCALE_SHAPE;
  mu.ns = ns;
  for (int type : {SAGIPS_F32, SAGIPS_BF16})
    for (int n : {1, 5, 16}) {
      sagips_matrix_set s = matrices(n, 3, 100, 140, type);    // rows 100 .. 115: of two kinds of launches
      for (int scale : {SAGIPS_SCALE_NONE, SAGIPS_SCALE_SHAPE, SAGIPS_SCALE_RMS}) {
        mu.scale = scale;
        expect("muon ok", sagips_muon_step(c, &s, &mu), OK, c);
      }
    }
  {
    const sagips_matrix_set s = matrices(2, 3, 20, 40, SAGIPS_F32);
    expect("muon ctx NULL", sagips_muon_step(nullptr, &s, &mu), INVAL, nullptr);
    expect("muon set NULL", sagips_muon_step(c, nullptr, &mu), INVAL, c);
    expect("muon options NULL", sagips_muon_step(c, &s, nullptr), INVAL, c);
#define BAD(what, change)                                 \
  {                                                       \
    sagips_matrix_set q = s;                              \
    sagips_muon o = mu;                                   \
    change;                                               \
    expect("muon " what, sagips_muon_step(c, &q, &o), INVAL, c); \
  }
    BAD("no tensors", q.n_tensors = 0)
    BAD("17 tensors", q.n_tensors = 17)
    BAD("grad_type 3", q.grad_type = 3)
    BAD("param NULL", q.param[1] = nullptr)
    BAD("grad NULL", q.grad[0] = nullptr)
    BAD("m misaligned", q.m[1] = dev(60) + 1)
    BAD("rows 0", q.rows[1] = 0)
    BAD("cols < 0", q.cols[0] = -3)
    BAD("count 0", q.count[1] = 0)
    BAD("lr < 0", o.lr = -1.0)
    BAD("lr NaN", o.lr = NAN)
    BAD("momentum 1", o.momentum = 1.0)
    BAD("weight_decay < 0", o.weight_decay = -1.0)
    BAD("scale 3", o.scale = 3)
    BAD("steps 20", o.ns.steps = 20)
    BAD("grad is param", q.grad[0] = q.param[0])
    BAD("shared param", q.param[1] = q.param[0] + 4)
    BAD("shared m", q.m[1] = q.m[0])
    BAD("m is the other's grad", q.m[1] = (float*)q.grad[0])
    BAD("m is the other's param", q.m[0] = q.param[1])
#undef BAD
    sagips_matrix_set many = matrices(2, 40000, 4, 4, SAGIPS_F32);
    expect("muon 80000 matrices", sagips_muon_step(c, &many, &mu), INVAL, c);
  }

  // ---- with timing on, and on another stream
  expect("timing", sagips_set_timing(c, 1), OK, c);
  {
    sagips_policy p = policy(4, 2, 100);
    expect("policy timed", pol(&p), OK, c);
    sagips_matrix_set s = matrices(3, 2, 120, 200, SAGIPS_F32);
    expect("muon timed", sagips_muon_step(c, &s, &mu), OK, c);
    const char* names[32];
    int64_t launches[32];
    double ms[32];
    const int n = sagips_kernel_times(c, names, launches, ms, 32);
    ++g_checks;
    if (n < 4) {
      ++g_fail;
      printf("FAIL kernel_times: %d kernels\n", n);
    }
  }
  sagips_destroy(c);
  if (stub_live_events() || stub_live_allocs()) {
    ++g_fail;
    printf("FAIL left behind: %ld events, %ld allocations\n", stub_live_events(), stub_live_allocs());
  }
  if (stub_bad_launches()) ++g_fail;
  printf("%d checks, %ld launches (%ld bad), %d failures\n", g_checks, stub_launches(), stub_bad_launches(), g_fail);
  if (!g_fail) printf("ALL OK\n");
  return g_fail ? 1 : 0;
}
