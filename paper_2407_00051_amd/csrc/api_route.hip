// C ABI of the choices and of the mixture of members (declared in include/sagips.h, 13. to
// 17.): argument validation, workspace and dispatch to the kernel files.
#include <hip/hip_runtime.h>

#include <math.h>

#include "../../include/sagips.h"
#include "context.hpp"
#include "kernels.hpp"

using namespace sagips;

namespace {

// An array of a call: what is read and what is written must not meet.
struct Span {
  const void* p;
  size_t bytes;
  const char* name;
};
bool meet(const Span& a, const Span& b) {
  const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
  return a.p && b.p && x < y + b.bytes && y < x + a.bytes;
}
// Every output against every input and the outputs before it.
template <size_t I, size_t O>
sagips_status apart(sagips_ctx* c, const Span (&in)[I], const Span (&out)[O]) {
  for (size_t o = 0; o < O; ++o) {
    for (size_t i = 0; i < I; ++i)
      if (meet(out[o], in[i])) return fail(c, SAGIPS_E_INVAL, "%s overlaps %s", out[o].name, in[i].name);
    for (size_t i = 0; i < o; ++i)
      if (meet(out[o], out[i])) return fail(c, SAGIPS_E_INVAL, "%s overlaps %s", out[o].name, out[i].name);
  }
  return SAGIPS_OK;
}
template <size_t N>
sagips_status aligned_to(sagips_ctx* c, size_t bytes, const Span (&a)[N]) {
  for (const Span& s : a)
    if ((uintptr_t)s.p % bytes) return fail(c, SAGIPS_E_INVAL, "%s is not %d-byte aligned", s.name, (int)bytes);
  return SAGIPS_OK;
}

size_t value_bytes(int32_t type) { return type == SAGIPS_BF16 ? 2 : 4; }
bool known_type(int32_t type) { return type == SAGIPS_F32 || type == SAGIPS_BF16; }

sagips_status check_choices(sagips_ctx* c, const sagips_choices* C) {
  if (!c) return fail(nullptr, SAGIPS_E_INVAL, "ctx is NULL");
  if (!C) return fail(c, SAGIPS_E_INVAL, "C is NULL");
  if (!C->logits) return fail(c, SAGIPS_E_INVAL, "logits is NULL");
  if (!known_type(C->type)) return fail(c, SAGIPS_E_INVAL, "unknown type %d", C->type);
  if ((uintptr_t)C->logits % value_bytes(C->type)) return fail(c, SAGIPS_E_INVAL, "logits is not aligned to its values");
  if (C->rows < 1 || C->rows >= ((int64_t)1 << 31)) return fail(c, SAGIPS_E_INVAL, "rows = %lld outside [1, 2^31)", (long long)C->rows);
  if (C->n_choices < 1 || C->n_choices > (1 << 29)) return fail(c, SAGIPS_E_INVAL, "n_choices = %d outside [1, 2^29]", C->n_choices);
  if (C->stride < C->n_choices || C->stride >= ((int64_t)1 << 31))
    return fail(c, SAGIPS_E_INVAL, "stride = %lld outside [n_choices = %d, 2^31)", (long long)C->stride, C->n_choices);
  if (C->top < 0 || C->top > SAGIPS_MAX_TOP) return fail(c, SAGIPS_E_INVAL, "top = %d outside [0, %d]", C->top, SAGIPS_MAX_TOP);
  // 1.4427 scale has to be a finite fp32 number too
  if (!(C->scale >= 0x1p-100 && C->scale <= 0x1p100)) return fail(c, SAGIPS_E_INVAL, "scale outside [2^-100, 2^100]");
  return SAGIPS_OK;
}
Span logits_of(const sagips_choices& C) {
  return {C.logits, ((size_t)(C.rows - 1) * C.stride + C.n_choices) * value_bytes(C.type), "logits"};
}

sagips_status check_items(sagips_ctx* c, int64_t rows, int32_t slots) {
  if (slots < 1 || slots > 32) return fail(c, SAGIPS_E_INVAL, "slots = %d outside [1, 32]", slots);
  if (rows < 1 || rows >= ((int64_t)1 << 31) || rows * slots >= ((int64_t)1 << 31) - (1 << 20))
    return fail(c, SAGIPS_E_INVAL, "rows = %lld: must be >= 1, and rows * slots < 2^31 - 2^20", (long long)rows);
  return SAGIPS_OK;
}
sagips_status check_routed(sagips_ctx* c, const sagips_routed* R) {
  if (!c) return fail(nullptr, SAGIPS_E_INVAL, "ctx is NULL");
  if (!R) return fail(c, SAGIPS_E_INVAL, "R is NULL");
  if (!R->place) return fail(c, SAGIPS_E_INVAL, "place is NULL");
  if (!known_type(R->type)) return fail(c, SAGIPS_E_INVAL, "unknown type %d", R->type);
  if (R->width < 1) return fail(c, SAGIPS_E_INVAL, "width = %d, must be >= 1", R->width);
  return check_items(c, R->rows, R->slots);
}
Span rows_of(const sagips_routed& R, const void* p, const char* name) {
  return {p, (size_t)R.rows * R.width * value_bytes(R.type), name};
}
Span items_of(const sagips_routed& R, const void* p, const char* name) {
  return {p, (size_t)R.rows * R.slots * R.width * value_bytes(R.type), name};
}
Span table_of(const sagips_routed& R, const void* p, const char* name) { return {p, (size_t)R.rows * R.slots * 4, name}; }

sagips_status check_members(sagips_ctx* c, const sagips_gen* G, const float* x, const int32_t* offsets, int64_t n_rows) {
  if (!c) return fail(nullptr, SAGIPS_E_INVAL, "ctx is NULL");
  if (!G) return fail(c, SAGIPS_E_INVAL, "G is NULL");
  if (!x || !offsets) return fail(c, SAGIPS_E_INVAL, "x or offsets is NULL");
  if ((uintptr_t)x % 4 || (uintptr_t)offsets % 4) return fail(c, SAGIPS_E_INVAL, "x or offsets is not 4-byte aligned");
  if (G->n_members < 1 || G->n_members > 65535) return fail(c, SAGIPS_E_INVAL, "n_members = %d outside [1, 65535]", G->n_members);
  if (G->n_layers < 2 || G->n_layers > SAGIPS_MAX_LAYERS)
    return fail(c, SAGIPS_E_INVAL, "n_layers = %d outside [2, %d]", G->n_layers, SAGIPS_MAX_LAYERS);
  for (int l = 0; l <= G->n_layers; ++l)
    if (G->width[l] < 1) return fail(c, SAGIPS_E_INVAL, "width[%d] < 1", l);
  for (int l = 0; l < G->n_layers; ++l) {
    if (!G->W[l] || !G->b[l]) return fail(c, SAGIPS_E_INVAL, "W[%d] or b[%d] is NULL", l, l);
    if (!aligned16(G->W[l]) || !aligned16(G->b[l])) return fail(c, SAGIPS_E_INVAL, "W[%d] or b[%d] is not 16-byte aligned", l, l);
  }
  if (n_rows < 1 || n_rows >= ((int64_t)1 << 29)) return fail(c, SAGIPS_E_INVAL, "n_rows = %lld outside [1, 2^29)", (long long)n_rows);
  const char* why = nullptr;
  if (!gen_supported(*G, &why)) return fail(c, SAGIPS_E_UNSUPPORTED, "%s", why);
  return SAGIPS_OK;
}

// Host allocations (messages, the timer's records) may throw; no exception leaves the C ABI.
template <class F>
sagips_status guarded(F&& f) {
  try {
    return f();
  } catch (...) {
    return SAGIPS_E_NOMEM;
  }
}
sagips_status done(sagips_ctx* c, hipError_t e, const char* what) { return e == hipSuccess ? SAGIPS_OK : hip_fail(c, e, what); }

}  // namespace

extern "C" {

sagips_status sagips_choice_logprob(sagips_ctx* c, const sagips_choices* C, const int32_t* choice, float* logp,
                                    float* entropy, int32_t* top_choice, float* top_logp, float* stats) {
  return guarded([&]() -> sagips_status {
    sagips_status s = check_choices(c, C);
    if (s != SAGIPS_OK) return s;
    if ((choice == nullptr) != (logp == nullptr)) return fail(c, SAGIPS_E_INVAL, "choice and logp must be given together");
    if ((top_choice == nullptr) != (C->top == 0) || (top_logp == nullptr) != (C->top == 0))
      return fail(c, SAGIPS_E_INVAL, "top_choice and top_logp must be given with top > 0, and only then");
    if (!logp && !entropy && !top_choice && !stats) return fail(c, SAGIPS_E_INVAL, "no output is given");
    const size_t n = (size_t)C->rows * 4;
    const Span in[] = {logits_of(*C), {choice, n, "choice"}};
    const Span out[] = {{logp, n, "logp"}, {entropy, n, "entropy"}, {top_choice, n * C->top, "top_choice"},
                        {top_logp, n * C->top, "top_logp"}, {stats, 2 * n, "stats"}};
    const Span mine[] = {in[1]};
    s = aligned_to(c, 4, mine);
    if (s == SAGIPS_OK) s = aligned_to(c, 4, out);
    if (s == SAGIPS_OK) s = apart(c, in, out);
    if (s != SAGIPS_OK) return s;
    DeviceGuard g(c->device);
    s = ensure_ws(c, choice_workspace(*C));
    if (s != SAGIPS_OK) return s;
    return done(c, launch_choice(*C, choice, logp, entropy, top_choice, top_logp, stats, c->ws, c->ticket, c->stream, timer_of(c)),
                "choice_logprob launch");
  });
}

sagips_status sagips_choice_backward(sagips_ctx* c, const sagips_choices* C, const sagips_choice_grads* g, void* dlogits,
                                     int64_t dstride) {
  return guarded([&]() -> sagips_status {
    sagips_status s = check_choices(c, C);
    if (s != SAGIPS_OK) return s;
    if (!g || !dlogits) return fail(c, SAGIPS_E_INVAL, "g or dlogits is NULL");
    if (!g->stats) return fail(c, SAGIPS_E_INVAL, "stats is NULL");
    if (!g->d_logp && !g->d_entropy && !g->d_top) return fail(c, SAGIPS_E_INVAL, "d_logp, d_entropy and d_top are all NULL");
    if (g->d_logp && (!g->choice || !g->logp)) return fail(c, SAGIPS_E_INVAL, "d_logp needs choice and logp");
    if (g->d_entropy && !g->entropy) return fail(c, SAGIPS_E_INVAL, "d_entropy needs entropy");
    if (g->d_top && (!g->top_choice || C->top == 0)) return fail(c, SAGIPS_E_INVAL, "d_top needs top_choice and top > 0");
    const size_t size = value_bytes(C->type), n = (size_t)C->rows * 4;
    if ((uintptr_t)dlogits % size) return fail(c, SAGIPS_E_INVAL, "dlogits is not aligned to its values");
    if (dstride < C->n_choices || dstride >= ((int64_t)1 << 31))
      return fail(c, SAGIPS_E_INVAL, "dstride = %lld outside [n_choices = %d, 2^31)", (long long)dstride, C->n_choices);
    const Span in[] = {{g->choice, n, "choice"}, {g->logp, n, "logp"}, {g->entropy, n, "entropy"},
                       {g->top_choice, n * C->top, "top_choice"}, {g->stats, 2 * n, "stats"}, {g->d_logp, n, "d_logp"},
                       {g->d_entropy, n, "d_entropy"}, {g->d_top, n * C->top, "d_top"}};
    const Span out[] = {{dlogits, ((size_t)(C->rows - 1) * dstride + C->n_choices) * size, "dlogits"}};
    s = aligned_to(c, 4, in);
    if (s == SAGIPS_OK) s = apart(c, in, out);
    if (s != SAGIPS_OK) return s;
    if (meet(out[0], logits_of(*C)) && (dlogits != C->logits || dstride != C->stride))
      return fail(c, SAGIPS_E_INVAL, "dlogits overlaps logits without being them");
    DeviceGuard guard(c->device);
    return done(c, launch_choice_backward(*C, *g, dlogits, dstride, c->stream, timer_of(c)), "choice_backward launch");
  });
}

sagips_status sagips_route(sagips_ctx* c, const int32_t* member, int64_t rows, int32_t slots, int32_t n_members,
                           int32_t* offsets, int32_t* order, int32_t* place) {
  return guarded([&]() -> sagips_status {
    if (!c) return fail(nullptr, SAGIPS_E_INVAL, "ctx is NULL");
    if (!member || !offsets || !order || !place) return fail(c, SAGIPS_E_INVAL, "member, offsets, order or place is NULL");
    sagips_status s = check_items(c, rows, slots);
    if (s != SAGIPS_OK) return s;
    if (n_members < 1 || n_members > 1024) return fail(c, SAGIPS_E_INVAL, "n_members = %d outside [1, 1024]", n_members);
    const int64_t n = rows * slots;
    const Span in[] = {{member, (size_t)n * 4, "member"}};
    const Span out[] = {{offsets, ((size_t)n_members + 1) * 4, "offsets"}, {order, (size_t)n * 4, "order"},
                        {place, (size_t)n * 4, "place"}};
    s = aligned_to(c, 4, in);
    if (s == SAGIPS_OK) s = aligned_to(c, 4, out);
    if (s == SAGIPS_OK) s = apart(c, in, out);
    if (s != SAGIPS_OK) return s;
    DeviceGuard g(c->device);
    s = ensure_ws(c, route_workspace(n, n_members));
    if (s != SAGIPS_OK) return s;
    return done(c, launch_route(member, n, n_members, offsets, order, place, c->ws, c->stream, timer_of(c)), "route launch");
  });
}

sagips_status sagips_dispatch(sagips_ctx* c, const sagips_routed* R, const void* x, void* sorted) {
  return guarded([&]() -> sagips_status {
    sagips_status s = check_routed(c, R);
    if (s != SAGIPS_OK) return s;
    if (!x || !sorted) return fail(c, SAGIPS_E_INVAL, "x or sorted is NULL");
    const Span in[] = {rows_of(*R, x, "x"), table_of(*R, R->place, "place")};
    const Span out[] = {items_of(*R, sorted, "sorted")};
    const Span values[] = {in[0], out[0]}, tables[] = {in[1]};
    s = aligned_to(c, value_bytes(R->type), values);
    if (s == SAGIPS_OK) s = aligned_to(c, 4, tables);
    if (s == SAGIPS_OK) s = apart(c, in, out);
    if (s != SAGIPS_OK) return s;
    DeviceGuard g(c->device);
    return done(c, launch_dispatch(*R, x, sorted, c->stream, timer_of(c)), "dispatch launch");
  });
}

sagips_status sagips_combine(sagips_ctx* c, const sagips_routed* R, const void* y, const float* weight, void* out_) {
  return guarded([&]() -> sagips_status {
    sagips_status s = check_routed(c, R);
    if (s != SAGIPS_OK) return s;
    if (!y || !out_) return fail(c, SAGIPS_E_INVAL, "y or out is NULL");
    const Span in[] = {items_of(*R, y, "y"), table_of(*R, R->place, "place"), table_of(*R, weight, "weight")};
    const Span out[] = {rows_of(*R, out_, "out")};
    const Span values[] = {in[0], out[0]}, tables[] = {in[1], in[2]};
    s = aligned_to(c, value_bytes(R->type), values);
    if (s == SAGIPS_OK) s = aligned_to(c, 4, tables);
    if (s == SAGIPS_OK) s = apart(c, in, out);
    if (s != SAGIPS_OK) return s;
    DeviceGuard g(c->device);
    return done(c, launch_combine(*R, y, weight, out_, c->stream, timer_of(c)), "combine launch");
  });
}

sagips_status sagips_combine_backward(sagips_ctx* c, const sagips_routed* R, const void* dout, const void* y,
                                      const float* weight, void* dy, float* dweight) {
  return guarded([&]() -> sagips_status {
    sagips_status s = check_routed(c, R);
    if (s != SAGIPS_OK) return s;
    if (!dout) return fail(c, SAGIPS_E_INVAL, "dout is NULL");
    if (!dy && !dweight) return fail(c, SAGIPS_E_INVAL, "no output is given");
    if ((y == nullptr) != (dweight == nullptr)) return fail(c, SAGIPS_E_INVAL, "y and dweight must be given together");
    const Span in[] = {rows_of(*R, dout, "dout"), items_of(*R, y, "y"), table_of(*R, R->place, "place"),
                       table_of(*R, weight, "weight")};
    const Span out[] = {items_of(*R, dy, "dy"), table_of(*R, dweight, "dweight")};
    const Span values[] = {in[0], in[1], out[0]}, tables[] = {in[2], in[3], out[1]};
    s = aligned_to(c, value_bytes(R->type), values);
    if (s == SAGIPS_OK) s = aligned_to(c, 4, tables);
    if (s == SAGIPS_OK) s = apart(c, in, out);
    if (s != SAGIPS_OK) return s;
    DeviceGuard g(c->device);
    return done(c, launch_combine_backward(*R, dout, y, weight, dy, dweight, c->stream, timer_of(c)), "combine_backward launch");
  });
}

sagips_status sagips_gen_forward_routed(sagips_ctx* c, const sagips_gen* G, const float* x, const int32_t* offsets,
                                        int64_t n_rows, float* theta) {
  return guarded([&]() -> sagips_status {
    sagips_status s = check_members(c, G, x, offsets, n_rows);
    if (s != SAGIPS_OK) return s;
    if (!theta) return fail(c, SAGIPS_E_INVAL, "theta is NULL");
    const Span in[] = {{x, (size_t)n_rows * G->width[0] * 4, "x"}, {offsets, ((size_t)G->n_members + 1) * 4, "offsets"}};
    const Span out[] = {{theta, (size_t)n_rows * G->width[G->n_layers] * 4, "theta"}};
    s = aligned_to(c, 4, out);
    if (s == SAGIPS_OK) s = apart(c, in, out);
    if (s != SAGIPS_OK) return s;
    DeviceGuard g(c->device);
    return done(c, launch_gen_forward_routed(*G, x, offsets, n_rows, theta, c->n_cu, c->stream, timer_of(c)),
                "gen_forward_routed launch");
  });
}

sagips_status sagips_gen_backward_routed(sagips_ctx* c, const sagips_gen* G, const float* x, const int32_t* offsets,
                                         int64_t n_rows, const float* dL_dtheta, float* const* dW, float* const* db, float* dx) {
  return guarded([&]() -> sagips_status {
    sagips_status s = check_members(c, G, x, offsets, n_rows);
    if (s != SAGIPS_OK) return s;
    if (!dL_dtheta || !dW || !db) return fail(c, SAGIPS_E_INVAL, "dL_dtheta, dW or db is NULL");
    for (int l = 0; l < G->n_layers; ++l) {
      if (!dW[l] || !db[l]) return fail(c, SAGIPS_E_INVAL, "dW[%d] or db[%d] is NULL", l, l);
      if ((uintptr_t)dW[l] % 4 || (uintptr_t)db[l] % 4) return fail(c, SAGIPS_E_INVAL, "dW[%d] or db[%d] is not 4-byte aligned", l, l);
    }
    const Span in[] = {{x, (size_t)n_rows * G->width[0] * 4, "x"}, {offsets, ((size_t)G->n_members + 1) * 4, "offsets"},
                       {dL_dtheta, (size_t)n_rows * G->width[G->n_layers] * 4, "dL_dtheta"}};
    const Span out[] = {{dx, (size_t)n_rows * G->width[0] * 4, "dx"}};
    const Span tables[] = {in[2], out[0]};
    s = aligned_to(c, 4, tables);
    if (s == SAGIPS_OK) s = apart(c, in, out);
    if (s != SAGIPS_OK) return s;
    DeviceGuard g(c->device);
    s = ensure_ws(c, gen_backward_routed_workspace(*G, n_rows, c->n_cu));
    if (s != SAGIPS_OK) return s;
    return done(c, launch_gen_backward_routed(*G, x, offsets, n_rows, dL_dtheta, dW, db, dx, c->ws, c->n_cu, c->stream,
                                              timer_of(c)),
                "gen_backward_routed launch");
  });
}

}  // extern "C"
