// C ABI of the learning operators (declared in include/sagips.h, 9. to 12.):
// argument validation, workspace and dispatch to the kernel files.
#include <hip/hip_runtime.h>

#include <math.h>

#include "../../include/sagips.h"
#include "context.hpp"
#include "kernels.hpp"

using namespace sagips;

namespace {

bool aligned_to(const void* p, size_t bytes) { return (uintptr_t)p % bytes == 0; }
bool aligned4(const void* p) { return aligned_to(p, 4); }

bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return x < y + nb && y < x + na;
}

// n * m where both are at least 1 and the product stays below 2^31; -1 otherwise.
int64_t product31(int64_t n, int64_t m) {
  if (n < 1 || m < 1 || m >= ((int64_t)1 << 31) || n >= ((int64_t)1 << 31) || n * m >= ((int64_t)1 << 31)) return -1;
  return n * m;
}

// A parameter table of n_theta rows of 2d values.
sagips_status check_rows(sagips_ctx* c, const float* theta, const char* name) {
  if (!theta) return fail(c, SAGIPS_E_INVAL, "%s is NULL", name);
  if (!aligned4(theta)) return fail(c, SAGIPS_E_INVAL, "%s is not 4-byte aligned", name);
  return SAGIPS_OK;
}
sagips_status check_sizes(sagips_ctx* c, int32_t n_theta, int32_t d) {
  if (n_theta < 1 || n_theta > 65535) return fail(c, SAGIPS_E_INVAL, "n_theta = %d outside [1, 65535]", n_theta);
  if (d != 2 && d != 3) return fail(c, SAGIPS_E_INVAL, "d = %d, must be 2 or 3", d);
  return SAGIPS_OK;
}
bool finite_at_least(double v, double lo) { return v >= lo && isfinite(v); }

// Sizes of a stack of matrices.
sagips_status check_stack(sagips_ctx* c, int32_t count, int32_t rows, int32_t cols, int i) {
  if (count < 1 || count > 65535 || rows < 1 || rows > 16384 || cols < 1 || cols > 16384 ||
      (int64_t)rows * cols * count >= ((int64_t)1 << 31))
    return fail(c, SAGIPS_E_INVAL,
                "stack %d of %d matrices of %d x %d: need 1 <= count <= 65535, 1 <= rows, cols <= 16384 and fewer than "
                "2^31 elements",
                i, count, rows, cols);
  return SAGIPS_OK;
}

// max |a s + b s^3 + c s^5| over 0 <= s <= most: at the end, or where the derivative
// a + 3 b q + 5 c q^2, q = s^2, is zero.
double largest_value(double a, double b, double c, double most) {
  const auto value = [&](double s) { return fabs(s * (a + s * s * (b + c * s * s))); };
  double v = value(most), q[2];
  int n = 0;
  const double disc = 9.0 * b * b - 20.0 * a * c;
  if (disc >= 0.0) {
    // -(3 b + its square root with b's sign): no digits cancel where c is small
    const double t = -(3.0 * b + copysign(sqrt(disc), b));
    if (t != 0.0) q[n++] = 2.0 * a / t;
    if (c != 0.0) q[n++] = t / (10.0 * c);
  }
  for (int i = 0; i < n; ++i)
    if (q[i] > 0.0 && q[i] < most * most) v = fmax(v, value(sqrt(q[i])));
  return v;
}

// max |a + b q + c q^2| over 0 <= q <= most^2: at an end, or where b + 2 c q is zero.
double largest_growth(double a, double b, double c, double most) {
  const auto value = [&](double q) { return fabs(a + q * (b + c * q)); };
  const double q = c != 0.0 ? -b / (2.0 * c) : 0.0;
  const double v = fmax(value(0.0), value(most * most));
  return q > 0.0 && q < most * most ? fmax(v, value(q)) : v;
}

sagips_status fill_steps(sagips_ctx* c, const sagips_newton_schulz& ns, MatrixJobs* js) {
  if (ns.steps < 0 || ns.steps > 16) return fail(c, SAGIPS_E_INVAL, "steps = %d outside [0, 16]", ns.steps);
  if (!(ns.eps > 0.0) || !isfinite(ns.eps)) return fail(c, SAGIPS_E_INVAL, "eps must be finite and > 0");
  static const double standard[3] = {3.4445, -4.7750, 2.0315};
  const bool given = ns.coef[0] != 0.0 || ns.coef[1] != 0.0 || ns.coef[2] != 0.0;
  for (int k = 0; k < 3; ++k) {
    const double v = given ? ns.coef[k] : standard[k];
    if (!isfinite(v)) return fail(c, SAGIPS_E_INVAL, "coef[%d] is not finite", k);
    js->coef[k] = (float)v;
  }
  js->steps = ns.steps ? ns.steps : 5;
  js->eps = ns.eps;
  // The kernels hold 2^12 X, X X^T and the polynomial of it in fp16 terms, up to 15.9, and
  // 2^10 X X^T X, up to 63.9: no entry exceeds the largest singular value, which for X starts
  // below 1 and is bounded step by step (its cube by 59.4).
  const double a = js->coef[0], b = js->coef[1], k = js->coef[2];
  double most = 1.0, growth = 1.0;
  for (int i = 0; i < js->steps; ++i) {
    const double poly = fabs(b) * most * most + fabs(k) * most * most * most * most;
    if (!(most <= 3.9) || !(poly <= 15.9))
      return fail(c, SAGIPS_E_UNSUPPORTED, "coefficients (%g, %g, %g) let singular values grow beyond 3.9 within %d steps", a,
                  b, k, i + 1);
    growth = fmax(growth, largest_growth(a, b, k, most));
    most = largest_value(a, b, k, most);
  }
  js->grow = (int)ceil(log2(growth));
  if (!(most <= 3.9))
    return fail(c, SAGIPS_E_UNSUPPORTED, "coefficients (%g, %g, %g) let singular values grow beyond 3.9", a, b, k);
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

}  // namespace

extern "C" {

sagips_status sagips_group_advantage(sagips_ctx* c, const float* reward, const uint8_t* mask, int32_t n_rows,
                                     int64_t events_per_row, int normalise, double eps, float* adv) {
  return guarded([&]() -> sagips_status {
    if (!c) return fail(nullptr, SAGIPS_E_INVAL, "ctx is NULL");
    if (!reward || !adv) return fail(c, SAGIPS_E_INVAL, "reward or adv is NULL");
    if (!aligned16(reward) || !aligned16(adv)) return fail(c, SAGIPS_E_INVAL, "reward and adv must be 16-byte aligned");
    const int64_t n = product31(n_rows, events_per_row);
    if (n < 0)
      return fail(c, SAGIPS_E_INVAL, "n_rows = %d, events_per_row = %lld: both must be >= 1 and their product < 2^31",
                  n_rows, (long long)events_per_row);
    if (!finite_at_least(eps, 0.0)) return fail(c, SAGIPS_E_INVAL, "eps must be finite and >= 0");
    if (reward != adv && overlap(reward, n * sizeof(float), adv, n * sizeof(float)))
      return fail(c, SAGIPS_E_INVAL, "adv overlaps reward without being it");
    if (mask && overlap(mask, (size_t)n, adv, n * sizeof(float))) return fail(c, SAGIPS_E_INVAL, "adv overlaps mask");
    DeviceGuard g(c->device);
    sagips_status s = ensure_ws(c, advantage_workspace(n_rows, events_per_row));
    if (s != SAGIPS_OK) return s;
    hipError_t e = launch_advantage(reward, mask, n_rows, events_per_row, normalise != 0, eps, adv, c->ws, c->stream,
                                    timer_of(c));
    return e == hipSuccess ? SAGIPS_OK : hip_fail(c, e, "group_advantage launch");
  });
}

sagips_status sagips_policy_loss(sagips_ctx* c, const sagips_policy* P, const float* x, const float* adv,
                                 const uint8_t* mask, float* loss, float* kl, float* clip_frac, float* dtheta) {
  return guarded([&]() -> sagips_status {
    if (!c) return fail(nullptr, SAGIPS_E_INVAL, "ctx is NULL");
    if (!P) return fail(c, SAGIPS_E_INVAL, "P is NULL");
    sagips_status s = check_sizes(c, P->n_theta, P->d);
    if (s == SAGIPS_OK) s = check_rows(c, P->theta, "theta");
    if (s == SAGIPS_OK) s = check_rows(c, P->theta_old, "theta_old");
    if (s == SAGIPS_OK && P->theta_ref) s = check_rows(c, P->theta_ref, "theta_ref");
    if (s != SAGIPS_OK) return s;
    if (product31(P->n_theta, P->events_per_theta) < 0)
      return fail(c, SAGIPS_E_INVAL, "events_per_theta = %lld: must be >= 1, and n_theta * events_per_theta < 2^31",
                  (long long)P->events_per_theta);
    if (!x || !adv) return fail(c, SAGIPS_E_INVAL, "x or adv is NULL");
    if (!aligned16(x) || !aligned16(adv)) return fail(c, SAGIPS_E_INVAL, "x and adv must be 16-byte aligned");
    if (!(P->clip_low >= 0.0 && P->clip_low <= 1.0) || !finite_at_least(P->clip_high, 0.0) || !finite_at_least(P->kl_coef, 0.0))
      return fail(c, SAGIPS_E_INVAL, "need 0 <= clip_low <= 1, clip_high >= 0, kl_coef >= 0");
    if (P->average != SAGIPS_MEAN_EVENTS && P->average != SAGIPS_MEAN_ROWS)
      return fail(c, SAGIPS_E_INVAL, "unknown average %d", P->average);
    if (!loss && !kl && !clip_frac && !dtheta) return fail(c, SAGIPS_E_INVAL, "no output is given");
    if (!aligned4(loss) || !aligned4(kl) || !aligned4(clip_frac) || !aligned4(dtheta))
      return fail(c, SAGIPS_E_INVAL, "outputs must be 4-byte aligned");
    DeviceGuard g(c->device);
    s = ensure_ws(c, policy_workspace(*P));
    if (s != SAGIPS_OK) return s;
    hipError_t e = launch_policy(*P, x, adv, mask, loss, kl, clip_frac, dtheta, c->ws, c->ticket, c->stream,
                                 timer_of(c));
    return e == hipSuccess ? SAGIPS_OK : hip_fail(c, e, "policy_loss launch");
  });
}

sagips_status sagips_preference_loss(sagips_ctx* c, const sagips_preference* P, const float* chosen,
                                     const int32_t* n_chosen, const float* rejected, const int32_t* n_rejected,
                                     float* loss, float* margin, float* dtheta) {
  return guarded([&]() -> sagips_status {
    if (!c) return fail(nullptr, SAGIPS_E_INVAL, "ctx is NULL");
    if (!P) return fail(c, SAGIPS_E_INVAL, "P is NULL");
    sagips_status s = check_sizes(c, P->n_theta, P->d);
    if (s == SAGIPS_OK) s = check_rows(c, P->theta, "theta");
    if (s == SAGIPS_OK) s = check_rows(c, P->theta_ref, "theta_ref");
    if (s != SAGIPS_OK) return s;
    const int64_t pairs = product31(P->n_theta, P->pairs_per_theta);
    if (pairs < 0 || product31(pairs, P->len_chosen) < 0 || product31(pairs, P->len_rejected) < 0)
      return fail(c, SAGIPS_E_INVAL,
                  "pairs_per_theta = %lld, len_chosen = %lld, len_rejected = %lld: each must be >= 1 and the events of "
                  "all pairs < 2^31",
                  (long long)P->pairs_per_theta, (long long)P->len_chosen, (long long)P->len_rejected);
    if (!chosen || !rejected) return fail(c, SAGIPS_E_INVAL, "chosen or rejected is NULL");
    if (!aligned16(chosen) || !aligned16(rejected))
      return fail(c, SAGIPS_E_INVAL, "chosen and rejected must be 16-byte aligned");
    if (!aligned4(n_chosen) || !aligned4(n_rejected))
      return fail(c, SAGIPS_E_INVAL, "n_chosen and n_rejected must be 4-byte aligned");
    if (!finite_at_least(P->beta, 0.0) || P->beta == 0.0 || !(P->label_smoothing >= 0.0 && P->label_smoothing <= 1.0))
      return fail(c, SAGIPS_E_INVAL, "need beta > 0 and 0 <= label_smoothing <= 1");
    if (!loss && !margin && !dtheta) return fail(c, SAGIPS_E_INVAL, "no output is given");
    if (!aligned4(loss) || !aligned4(margin) || !aligned4(dtheta))
      return fail(c, SAGIPS_E_INVAL, "outputs must be 4-byte aligned");
    DeviceGuard g(c->device);
    s = ensure_ws(c, preference_workspace(*P));
    if (s != SAGIPS_OK) return s;
    hipError_t e = launch_preference(*P, chosen, n_chosen, rejected, n_rejected, loss, margin, dtheta, c->ws, c->ticket,
                                     c->stream, timer_of(c));
    return e == hipSuccess ? SAGIPS_OK : hip_fail(c, e, "preference_loss launch");
  });
}

sagips_status sagips_orthogonalise(sagips_ctx* c, const sagips_newton_schulz* ns, int32_t type, const void* x,
                                   int32_t count, int32_t rows, int32_t cols, void* out) {
  return guarded([&]() -> sagips_status {
    if (!c) return fail(nullptr, SAGIPS_E_INVAL, "ctx is NULL");
    if (!ns || !x || !out) return fail(c, SAGIPS_E_INVAL, "ns, x or out is NULL");
    if (type != SAGIPS_F32 && type != SAGIPS_BF16) return fail(c, SAGIPS_E_INVAL, "unknown type %d", type);
    if (!aligned16(x) || !aligned16(out)) return fail(c, SAGIPS_E_INVAL, "x and out must be 16-byte aligned");
    sagips_status s = check_stack(c, count, rows, cols, 0);
    if (s != SAGIPS_OK) return s;
    MatrixJobs js{};
    s = fill_steps(c, *ns, &js);
    if (s != SAGIPS_OK) return s;
    const size_t bytes = (size_t)count * rows * cols * (type == SAGIPS_BF16 ? 2 : 4);
    if (x != out && overlap(x, bytes, out, bytes)) return fail(c, SAGIPS_E_INVAL, "out overlaps x without being it");
    js.n_jobs = 1;
    js.job[0] = MatrixJob{x, nullptr, out, count, rows, cols, 1.0};
    js.src_bf16 = js.out_bf16 = type == SAGIPS_BF16;
    DeviceGuard g(c->device);
    s = ensure_ws(c, muon_workspace(js));
    if (s != SAGIPS_OK) return s;
    hipError_t e = launch_muon(js, c->ws, c->n_cu, c->stream, timer_of(c));
    return e == hipSuccess ? SAGIPS_OK : hip_fail(c, e, "orthogonalise launch");
  });
}

sagips_status sagips_muon_step(sagips_ctx* c, const sagips_matrix_set* set, const sagips_muon* o) {
  return guarded([&]() -> sagips_status {
    if (!c) return fail(nullptr, SAGIPS_E_INVAL, "ctx is NULL");
    if (!set || !o) return fail(c, SAGIPS_E_INVAL, "set or options is NULL");
    if (set->n_tensors < 1 || set->n_tensors > SAGIPS_MAX_TENSORS)
      return fail(c, SAGIPS_E_INVAL, "n_tensors = %d outside [1, %d]", set->n_tensors, SAGIPS_MAX_TENSORS);
    if (set->grad_type != SAGIPS_F32 && set->grad_type != SAGIPS_BF16)
      return fail(c, SAGIPS_E_INVAL, "unknown grad_type %d", set->grad_type);
    if (!finite_at_least(o->lr, 0.0) || !finite_at_least(o->weight_decay, 0.0) || !(o->momentum >= 0.0 && o->momentum < 1.0))
      return fail(c, SAGIPS_E_INVAL, "need lr, weight_decay >= 0 and 0 <= momentum < 1");
    if (o->scale != SAGIPS_SCALE_NONE && o->scale != SAGIPS_SCALE_SHAPE && o->scale != SAGIPS_SCALE_RMS)
      return fail(c, SAGIPS_E_INVAL, "unknown scale %d", o->scale);
    MatrixJobs js{};
    sagips_status s = fill_steps(c, o->ns, &js);
    if (s != SAGIPS_OK) return s;
    const size_t grad_size = set->grad_type == SAGIPS_BF16 ? 2 : 4;
    int64_t matrices = 0;
    for (int i = 0; i < set->n_tensors; ++i) {
      if (!set->param[i] || !set->grad[i] || !set->m[i]) return fail(c, SAGIPS_E_INVAL, "tensor %d has a NULL array", i);
      s = check_stack(c, set->count[i], set->rows[i], set->cols[i], i);
      if (s != SAGIPS_OK) return s;
      // rows of whole quads are read and written four values at a time, others one
      const size_t at_once = set->cols[i] % 4 == 0 ? 4 : 1;
      if (!aligned_to(set->param[i], 4 * at_once) || !aligned_to(set->m[i], 4 * at_once) ||
          !aligned_to(set->grad[i], grad_size * at_once))
        return fail(c, SAGIPS_E_INVAL, "tensor %d has an array that is not aligned to %d values", i, (int)at_once);
      matrices += set->count[i];
      const int32_t rows = set->rows[i], cols = set->cols[i];
      const double scale = o->scale == SAGIPS_SCALE_NONE ? 1.0
                         : o->scale == SAGIPS_SCALE_RMS ? 0.2 * sqrt((double)(rows > cols ? rows : cols))
                         : rows > cols ? sqrt((double)rows / cols) : 1.0;
      js.job[i] = MatrixJob{set->grad[i], set->m[i], set->param[i], set->count[i], rows, cols, scale};
      // every array that is written against every other
      const size_t n = (size_t)set->count[i] * rows * cols;
      for (int k = 0; k < set->n_tensors; ++k) {
        if (set->count[k] < 1 || set->rows[k] < 1 || set->cols[k] < 1) continue;   // refused when its turn comes
        const size_t nk = (size_t)set->count[k] * set->rows[k] * set->cols[k];
        if (overlap(set->param[i], n * 4, set->grad[k], nk * grad_size) || overlap(set->m[i], n * 4, set->grad[k], nk * grad_size) ||
            overlap(set->param[i], n * 4, set->m[k], nk * 4) ||
            (k < i && (overlap(set->param[i], n * 4, set->param[k], nk * 4) || overlap(set->m[i], n * 4, set->m[k], nk * 4))))
          return fail(c, SAGIPS_E_INVAL, "arrays of tensors %d and %d overlap", i, k);
      }
    }
    if (matrices > 65535) return fail(c, SAGIPS_E_INVAL, "%lld matrices, at most 65535", (long long)matrices);
    js.n_jobs = set->n_tensors;
    js.src_bf16 = set->grad_type == SAGIPS_BF16;
    js.nesterov = o->nesterov != 0;
    js.momentum = (float)o->momentum;
    js.decay = (float)(1.0 - o->lr * o->weight_decay);
    js.lr = o->lr;
    DeviceGuard g(c->device);
    s = ensure_ws(c, muon_workspace(js));
    if (s != SAGIPS_OK) return s;
    hipError_t e = launch_muon(js, c->ws, c->n_cu, c->stream, timer_of(c));
    return e == hipSuccess ? SAGIPS_OK : hip_fail(c, e, "muon_step launch");
  });
}

}  // extern "C"
