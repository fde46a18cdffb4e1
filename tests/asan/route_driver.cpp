// Drives the choices' and the mixture's entry points of libsagips's C ABI on the CPU
// against the stub HIP runtime, under the address and undefined-behaviour
// sanitizers: every documented error path, and valid calls over the range of sizes,
// whose launch shapes the stub checks.
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

// Fake device memory, 1 TiB apart.
template <class T = float>
T* dev(uint64_t i) {
  return reinterpret_cast<T*>((uintptr_t)0x100000000000ull + (i << 40));
}

void expect(const char* what, sagips_status got, sagips_status want, sagips_ctx* c) {
  ++g_checks;
  const char* msg = sagips_last_error(c);
  if (got != want || !msg || (want != SAGIPS_OK && strlen(msg) == 0)) {
    ++g_fail;
    printf("FAIL %s: status %d, expected %d (%s)\n", what, (int)got, (int)want, msg ? msg : "(null message)");
  }
}
#define OK(call) expect(#call, call, SAGIPS_OK, c)
#define BAD(call) expect(#call, call, SAGIPS_E_INVAL, c)

sagips_choices choices(int64_t rows, int n, int top, int type, int64_t stride = 0) {
  sagips_choices C;
  memset(&C, 0, sizeof(C));
  C.logits = dev<char>(1);
  C.rows = rows;
  C.n_choices = n;
  C.stride = stride ? stride : n;
  C.type = type;
  C.top = top;
  C.scale = 1.0;
  return C;
}
sagips_status forward(sagips_ctx* c, const sagips_choices& C) {
  return sagips_choice_logprob(c, &C, dev<int32_t>(2), dev(3), dev(4), C.top ? dev<int32_t>(5) : nullptr, C.top ? dev(6) : nullptr, dev(7));
}
sagips_choice_grads grads(const sagips_choices& C) {
  sagips_choice_grads g;
  memset(&g, 0, sizeof(g));
  g.choice = dev<int32_t>(2);
  g.logp = dev(3);
  g.entropy = dev(4);
  g.top_choice = C.top ? dev<int32_t>(5) : nullptr;
  g.stats = dev(7);
  g.d_logp = dev(8);
  g.d_entropy = dev(9);
  g.d_top = C.top ? dev(10) : nullptr;
  return g;
}

void run_choices(sagips_ctx* c) {
  const int sizes[] = {1, 2, 3, 8, 9, 64, 65, 500, 1000, 5000, 20000, 70000, 140000, 1 << 24, 1 << 29};
  for (int type = 0; type < 2; ++type)
    for (int n : sizes)
      for (int64_t rows : {(int64_t)1, (int64_t)1000, (int64_t)0x7fffffff})
        for (int top : {0, 1, 32}) {
          if (rows * n > ((int64_t)1 << 38)) continue;
          const sagips_choices C = choices(rows, n, top, type, n + 3);
          OK(forward(c, C));
          const sagips_choice_grads g = grads(C);
          OK(sagips_choice_backward(c, &C, &g, dev<char>(11), n));
          OK(sagips_choice_backward(c, &C, &g, dev<char>(1), n + 3));        // in place
        }
  sagips_choices C = choices(10, 20, 2, SAGIPS_F32);
  expect("ctx NULL", sagips_choice_logprob(nullptr, &C, nullptr, nullptr, dev(4), nullptr, nullptr, nullptr), SAGIPS_E_INVAL, nullptr);
  BAD(sagips_choice_logprob(c, nullptr, nullptr, nullptr, dev(4), nullptr, nullptr, nullptr));
  const auto with = [&](auto set) {
    sagips_choices D = C;
    set(D);
    return D;
  };
  sagips_choices bad[] = {with([](auto& D) { D.logits = nullptr; }), with([](auto& D) { D.type = 2; }),
                          with([](auto& D) { D.type = -1; }), with([](auto& D) { D.logits = dev<char>(1) + 2; }),
                          with([](auto& D) { D.rows = 0; }), with([](auto& D) { D.rows = (int64_t)1 << 31; }),
                          with([](auto& D) { D.n_choices = 0; }), with([](auto& D) { D.n_choices = (1 << 29) + 1; D.stride = 1 << 30; }),
                          with([](auto& D) { D.stride = 19; }), with([](auto& D) { D.stride = (int64_t)1 << 31; }),
                          with([](auto& D) { D.top = -1; }), with([](auto& D) { D.top = 33; }), with([](auto& D) { D.scale = 0.0; }),
                          with([](auto& D) { D.scale = -1.0; }), with([](auto& D) { D.scale = NAN; }),
                          with([](auto& D) { D.scale = INFINITY; }), with([](auto& D) { D.scale = 1e300; })};
  for (const sagips_choices& D : bad) {
    BAD(forward(c, D));
    const sagips_choice_grads g = grads(C);
    BAD(sagips_choice_backward(c, &D, &g, dev<char>(11), 20));
  }
  // outputs that belong together, overlaps, alignment
  BAD(sagips_choice_logprob(c, &C, nullptr, dev(3), dev(4), dev<int32_t>(5), dev(6), nullptr));
  BAD(sagips_choice_logprob(c, &C, dev<int32_t>(2), nullptr, dev(4), dev<int32_t>(5), dev(6), nullptr));
  BAD(sagips_choice_logprob(c, &C, nullptr, nullptr, dev(4), nullptr, dev(6), nullptr));
  BAD(sagips_choice_logprob(c, &C, nullptr, nullptr, dev(4), dev<int32_t>(5), nullptr, nullptr));
  BAD(sagips_choice_logprob(c, &C, nullptr, nullptr, dev(4), dev<int32_t>(5), dev(4), nullptr));
  BAD(sagips_choice_logprob(c, &C, nullptr, nullptr, dev(1), dev<int32_t>(5), dev(6), nullptr));
  BAD(sagips_choice_logprob(c, &C, dev<int32_t>(3), dev(3), dev(4), dev<int32_t>(5), dev(6), nullptr));
  BAD(sagips_choice_logprob(c, &C, nullptr, nullptr, reinterpret_cast<float*>(dev<char>(4) + 2), dev<int32_t>(5), dev(6), nullptr));
  C.top = 0;
  BAD(sagips_choice_logprob(c, &C, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr));
  BAD(sagips_choice_logprob(c, &C, nullptr, nullptr, dev(4), dev<int32_t>(5), dev(6), nullptr));
  OK(sagips_choice_logprob(c, &C, nullptr, nullptr, nullptr, nullptr, nullptr, dev(7)));
  C.top = 2;
  const auto back = [&](auto set, void* out, int64_t stride) {
    sagips_choice_grads g = grads(C);
    set(g);
    return sagips_choice_backward(c, &C, &g, out, stride);
  };
  const auto none = [](auto&) {};
  OK(back(none, dev<char>(11), 20));
  BAD(sagips_choice_backward(c, &C, nullptr, dev<char>(11), 20));
  BAD(back(none, nullptr, 20));
  BAD(back(none, dev<char>(11), 19));
  BAD(back(none, dev<char>(11) + 2, 20));
  BAD(back(none, dev<char>(1) + 4, 20));
  BAD(back(none, dev<char>(1), 21));
  BAD(back(none, dev<char>(7), 20));
  BAD(back([](auto& g) { g.stats = nullptr; }, dev<char>(11), 20));
  BAD(back([](auto& g) { g.choice = nullptr; }, dev<char>(11), 20));
  BAD(back([](auto& g) { g.logp = nullptr; }, dev<char>(11), 20));
  BAD(back([](auto& g) { g.entropy = nullptr; }, dev<char>(11), 20));
  BAD(back([](auto& g) { g.top_choice = nullptr; }, dev<char>(11), 20));
  BAD(back([](auto& g) { g.d_logp = g.d_entropy = g.d_top = nullptr; }, dev<char>(11), 20));
  BAD(back([](auto& g) { g.d_logp = reinterpret_cast<const float*>(dev<char>(8) + 1); }, dev<char>(11), 20));
  OK(back([](auto& g) { g.d_logp = g.d_top = nullptr; g.choice = nullptr; g.logp = nullptr; g.top_choice = nullptr; }, dev<char>(11), 20));
}

sagips_routed routed(int64_t rows, int slots, int width, int type) {
  sagips_routed R;
  memset(&R, 0, sizeof(R));
  R.place = dev<int32_t>(1);
  R.rows = rows;
  R.slots = slots;
  R.width = width;
  R.type = type;
  return R;
}

void run_routes(sagips_ctx* c) {
  int32_t *m = dev<int32_t>(1), *off = dev<int32_t>(2), *ord = dev<int32_t>(3), *pl = dev<int32_t>(4);
  for (int64_t rows : {(int64_t)1, (int64_t)63, (int64_t)16384, (int64_t)16385, (int64_t)1000000, (((int64_t)1 << 31) - (1 << 20) - 1) / 32})
    for (int slots : {1, 2, 32})
      for (int M : {1, 2, 65, 1024}) OK(sagips_route(c, m, rows, slots, M, off, ord, pl));
  expect("ctx NULL", sagips_route(nullptr, m, 1, 1, 1, off, ord, pl), SAGIPS_E_INVAL, nullptr);
  BAD(sagips_route(c, nullptr, 1, 1, 1, off, ord, pl));
  BAD(sagips_route(c, m, 1, 1, 1, nullptr, ord, pl));
  BAD(sagips_route(c, m, 1, 1, 1, off, nullptr, pl));
  BAD(sagips_route(c, m, 1, 1, 1, off, ord, nullptr));
  BAD(sagips_route(c, m, 0, 1, 1, off, ord, pl));
  BAD(sagips_route(c, m, -5, 1, 1, off, ord, pl));
  BAD(sagips_route(c, m, 1, 0, 1, off, ord, pl));
  BAD(sagips_route(c, m, 1, 33, 1, off, ord, pl));
  BAD(sagips_route(c, m, (int64_t)1 << 31, 1, 1, off, ord, pl));
  BAD(sagips_route(c, m, (((int64_t)1 << 31) - (1 << 20)) / 32, 32, 1, off, ord, pl));
  BAD(sagips_route(c, m, INT64_MAX, 32, 1, off, ord, pl));
  BAD(sagips_route(c, m, 10, 2, 0, off, ord, pl));
  BAD(sagips_route(c, m, 10, 2, 1025, off, ord, pl));
  BAD(sagips_route(c, m, 10, 2, 3, off, ord, m));
  BAD(sagips_route(c, m, 10, 2, 3, off, ord, ord + 5));
  BAD(sagips_route(c, m, 10, 2, 3, reinterpret_cast<int32_t*>(dev<char>(2) + 2), ord, pl));
  for (int type = 0; type < 2; ++type)
    for (int64_t rows : {(int64_t)1, (int64_t)1000, (((int64_t)1 << 31) - (1 << 20) - 1) / 2})
      for (int width : {1, 6, 8, 333, 2048, 100000}) {
        if (rows * width > (int64_t)1 << 42) continue;                       // beyond what the fake memory holds apart
        const sagips_routed R = routed(rows, 2, width, type);
        OK(sagips_dispatch(c, &R, dev<char>(2), dev<char>(300)));
        OK(sagips_combine(c, &R, dev<char>(300), dev(4), dev<char>(1200)));
        OK(sagips_combine(c, &R, dev<char>(300), nullptr, dev<char>(1200)));
        OK(sagips_combine_backward(c, &R, dev<char>(1200), dev<char>(300), dev(4), dev<char>(2400), dev(6)));
        OK(sagips_combine_backward(c, &R, dev<char>(1200), nullptr, nullptr, dev<char>(2400), nullptr));
        OK(sagips_combine_backward(c, &R, dev<char>(1200), dev<char>(300), dev(4), nullptr, dev(6)));
      }
  sagips_routed R = routed(10, 2, 6, SAGIPS_F32);
  expect("ctx NULL", sagips_dispatch(nullptr, &R, dev(2), dev(3)), SAGIPS_E_INVAL, nullptr);
  BAD(sagips_dispatch(c, nullptr, dev(2), dev(3)));
  BAD(sagips_dispatch(c, &R, nullptr, dev(3)));
  BAD(sagips_dispatch(c, &R, dev(2), nullptr));
  BAD(sagips_dispatch(c, &R, dev(2), dev(2)));
  BAD(sagips_dispatch(c, &R, dev<char>(2) + 2, dev(3)));
  BAD(sagips_combine(c, &R, nullptr, dev(4), dev(5)));
  BAD(sagips_combine(c, &R, dev(3), dev(4), nullptr));
  BAD(sagips_combine(c, &R, dev(3), dev(4), dev(4) + 3));
  BAD(sagips_combine(c, &R, dev(3), reinterpret_cast<float*>(dev<char>(4) + 1), dev(5)));
  BAD(sagips_combine_backward(c, &R, nullptr, dev(3), dev(4), dev(5), dev(6)));
  BAD(sagips_combine_backward(c, &R, dev(2), nullptr, dev(4), dev(5), dev(6)));
  BAD(sagips_combine_backward(c, &R, dev(2), dev(3), dev(4), dev(5), nullptr));
  BAD(sagips_combine_backward(c, &R, dev(2), nullptr, dev(4), nullptr, nullptr));
  BAD(sagips_combine_backward(c, &R, dev(2), dev(3), dev(4), dev(3), dev(6)));
  BAD(sagips_combine_backward(c, &R, dev(2), dev(3), dev(4), dev(5), dev(5)));
  for (int i = 0; i < 6; ++i) {
    sagips_routed B = R;
    if (i == 0) B.place = nullptr;
    if (i == 1) B.type = 7;
    if (i == 2) B.width = 0;
    if (i == 3) B.rows = 0;
    if (i == 4) B.slots = 33;
    if (i == 5) B.place = reinterpret_cast<int32_t*>(dev<char>(1) + 3);
    BAD(sagips_dispatch(c, &B, dev(2), dev(3)));
    BAD(sagips_combine(c, &B, dev(3), dev(4), dev(5)));
    BAD(sagips_combine_backward(c, &B, dev(2), dev(3), dev(4), dev(5), dev(6)));
  }
}

sagips_gen members(int M, int hidden, int in, int out) {
  sagips_gen G;
  memset(&G, 0, sizeof(G));
  G.n_layers = hidden + 2;
  G.n_members = M;
  G.leaky_slope = 0.2f;
  G.width[0] = in;
  for (int l = 1; l <= hidden + 1; ++l) G.width[l] = 128;
  G.width[hidden + 2] = out;
  for (int l = 0; l < G.n_layers; ++l) {
    G.W[l] = dev(20 + l);
    G.b[l] = dev(30 + l);
  }
  return G;
}

void run_members(sagips_ctx* c) {
  float *dW[SAGIPS_MAX_LAYERS], *db[SAGIPS_MAX_LAYERS];
  for (int l = 0; l < SAGIPS_MAX_LAYERS; ++l) {
    dW[l] = dev(40 + l);
    db[l] = dev(50 + l);
  }
  const int32_t* off = dev<int32_t>(2);
  for (int hidden : {1, 2, 3})
    for (int M : {1, 8, 100, 2000})
      for (int64_t n : {(int64_t)1, (int64_t)16, (int64_t)1000, (int64_t)4096, (int64_t)8192, (int64_t)100000, ((int64_t)1 << 29) - 1}) {
        const sagips_gen G = members(M, hidden, 6, 6);
        OK(sagips_gen_forward_routed(c, &G, dev(1), off, n, dev(3)));
        OK(sagips_gen_backward_routed(c, &G, dev(1), off, n, dev(4), dW, db, dev(5)));
        OK(sagips_gen_backward_routed(c, &G, dev(1), off, n, dev(4), dW, db, nullptr));
      }
  sagips_gen G = members(4, 3, 6, 6);
  expect("ctx NULL", sagips_gen_forward_routed(nullptr, &G, dev(1), off, 10, dev(3)), SAGIPS_E_INVAL, nullptr);
  BAD(sagips_gen_forward_routed(c, nullptr, dev(1), off, 10, dev(3)));
  BAD(sagips_gen_forward_routed(c, &G, nullptr, off, 10, dev(3)));
  BAD(sagips_gen_forward_routed(c, &G, dev(1), nullptr, 10, dev(3)));
  BAD(sagips_gen_forward_routed(c, &G, dev(1), off, 0, dev(3)));
  BAD(sagips_gen_forward_routed(c, &G, dev(1), off, (int64_t)1 << 29, dev(3)));
  BAD(sagips_gen_forward_routed(c, &G, dev(1), off, 10, nullptr));
  BAD(sagips_gen_forward_routed(c, &G, dev(1), off, 10, dev(1)));
  BAD(sagips_gen_forward_routed(c, &G, reinterpret_cast<float*>(dev<char>(1) + 2), off, 10, dev(3)));
  BAD(sagips_gen_backward_routed(c, &G, dev(1), off, 10, nullptr, dW, db, nullptr));
  BAD(sagips_gen_backward_routed(c, &G, dev(1), off, 10, dev(4), nullptr, db, nullptr));
  BAD(sagips_gen_backward_routed(c, &G, dev(1), off, 10, dev(4), dW, nullptr, nullptr));
  BAD(sagips_gen_backward_routed(c, &G, dev(1), off, 10, dev(4), dW, db, dev(4)));
  float* hole[SAGIPS_MAX_LAYERS];
  memcpy(hole, dW, sizeof(hole));
  hole[2] = nullptr;
  BAD(sagips_gen_backward_routed(c, &G, dev(1), off, 10, dev(4), hole, db, nullptr));
  for (int i = 0; i < 6; ++i) {
    sagips_gen B = G;
    sagips_status want = SAGIPS_E_INVAL;
    if (i == 0) B.n_members = 0;
    if (i == 1) B.n_members = 65536;
    if (i == 2) B.n_layers = 9;
    if (i == 3) B.W[1] = nullptr;
    if (i == 4) B.b[1] = dev(31) + 1;
    if (i == 5) { B.width[2] = 64; want = SAGIPS_E_UNSUPPORTED; }
    expect("generator", sagips_gen_forward_routed(c, &B, dev(1), off, 10, dev(3)), want, c);
    expect("generator", sagips_gen_backward_routed(c, &B, dev(1), off, 10, dev(4), dW, db, nullptr), want, c);
  }
}

}  // namespace

int main() {
  stub_set_malloc_limit((size_t)1 << 40);
  sagips_ctx* c = nullptr;
  expect("create", sagips_create(&c, 0, nullptr), SAGIPS_OK, nullptr);
  run_choices(c);
  run_routes(c);
  run_members(c);
  // a refused workspace, then a smaller call
  stub_set_malloc_limit(0);
  sagips_ctx* d = nullptr;
  expect("create", sagips_create(&d, 0, nullptr), SAGIPS_OK, nullptr);
  expect("no memory", sagips_route(d, dev<int32_t>(1), 1000000, 2, 64, dev<int32_t>(2), dev<int32_t>(3), dev<int32_t>(4)), SAGIPS_E_NOMEM, d);
  expect("none needed", sagips_route(d, dev<int32_t>(1), 100, 2, 64, dev<int32_t>(2), dev<int32_t>(3), dev<int32_t>(4)), SAGIPS_OK, d);
  stub_set_malloc_limit((size_t)1 << 40);
  // timing on: events are taken and given back
  expect("timing", sagips_set_timing(d, 1), SAGIPS_OK, d);
  run_routes(d);
  const char* names[64];
  int64_t launches[64];
  double ms[64];
  if (sagips_kernel_times(d, names, launches, ms, 64) < 4) {
    ++g_fail;
    printf("FAIL kernel_times\n");
  }
  expect("destroy", sagips_destroy(d), SAGIPS_OK, nullptr);
  expect("destroy", sagips_destroy(c), SAGIPS_OK, nullptr);
  if (stub_bad_launches()) {
    ++g_fail;
    printf("FAIL %ld bad launches\n", stub_bad_launches());
  }
  if (stub_live_events() || stub_live_allocs()) {
    ++g_fail;
    printf("FAIL %ld events, %ld allocations left\n", stub_live_events(), stub_live_allocs());
  }
  printf("%d checks, %ld launches\n", g_checks, stub_launches());
  if (g_fail) return 1;
  printf("ALL OK\n");
  return 0;
}
