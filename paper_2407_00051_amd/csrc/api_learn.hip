// C ABI of the learning operators (declared in include/sagips.h, 9. to 11.):
// argument validation, workspace and dispatch to the kernel files.
#include <hip/hip_runtime.h>

#include <math.h>

#include "../../include/sagips.h"
#include "context.hpp"
#include "kernels.hpp"

using namespace sagips;

namespace {

bool aligned4(const void* p) { return ((uintptr_t)p & 3u) == 0; }

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
    hipError_t e = launch_advantage(reward, mask, n_rows, events_per_row, normalise != 0, (float)eps, adv, c->ws, c->stream,
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
    hipError_t e = launch_policy(*P, x, adv, mask, loss, kl, clip_frac, dtheta, c->ws, c->stream, timer_of(c));
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
    hipError_t e = launch_preference(*P, chosen, n_chosen, rejected, n_rejected, loss, margin, dtheta, c->ws, c->stream,
                                     timer_of(c));
    return e == hipSuccess ? SAGIPS_OK : hip_fail(c, e, "preference_loss launch");
  });
}

}  // extern "C"
