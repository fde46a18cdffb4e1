// The library context behind the C ABI and what its entry points share: error
// messages, the device guard, the workspace and kernel timing.
#pragma once

#include <hip/hip_runtime.h>

#include <stdarg.h>
#include <stdint.h>
#include <stdio.h>

#include <string>
#include <vector>

#include "../../include/sagips.h"
#include "kernels.hpp"

namespace sagips {

inline thread_local std::string g_create_error = "no error";

struct EventTimer final : Timer {
  struct Rec {
    const char* name;
    hipEvent_t a, b;
  };
  hipStream_t stream = nullptr;
  std::vector<hipEvent_t> pool;
  std::vector<Rec> recs;
  const char* open_name = nullptr;
  hipEvent_t open_a = nullptr;

  hipEvent_t take() {
    if (!pool.empty()) {
      hipEvent_t e = pool.back();
      pool.pop_back();
      return e;
    }
    hipEvent_t e = nullptr;
    if (hipEventCreate(&e) != hipSuccess) return nullptr;
    return e;
  }
  void begin(const char* name) override {
    open_name = name;
    open_a = take();
    if (open_a) (void)hipEventRecord(open_a, stream);
  }
  void end() override {
    hipEvent_t b = take();
    if (open_a && b) {
      (void)hipEventRecord(b, stream);
      recs.push_back({open_name, open_a, b});
    }
    open_a = nullptr;
  }
  void release() {
    for (auto& r : recs) {
      pool.push_back(r.a);
      pool.push_back(r.b);
    }
    recs.clear();
  }
  ~EventTimer() override {
    release();
    for (hipEvent_t e : pool) (void)hipEventDestroy(e);
  }
};

}  // namespace sagips

struct sagips_ctx {
  int device = 0;
  hipStream_t stream = nullptr;
  int n_cu = 0;
  void* ws = nullptr;
  size_t ws_cap = 0;
  size_t ws_refused = SIZE_MAX; // bf16: the workspace that the device refused last
  uint32_t* ticket = nullptr;   // the counters of ticket_set, or NULL
  int ticket_set = -1;
  std::string err = "no error";
  bool timing = false;
  int bf16_chunk_rows = 0;      // 0: the library's default
  sagips::EventTimer timer;
};

namespace sagips {

inline sagips_status fail(sagips_ctx* c, sagips_status s, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  if (c) c->err = buf;
  else g_create_error = buf;
  return s;
}

inline sagips_status hip_fail(sagips_ctx* c, hipError_t e, const char* what) {
  return fail(c, SAGIPS_E_HIP, "%s: %s", what, hipGetErrorString(e));
}

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

struct DeviceGuard {
  int prev = -1;
  explicit DeviceGuard(int dev) {
    if (hipGetDevice(&prev) == hipSuccess && prev != dev) (void)hipSetDevice(dev);
    else prev = -1;
  }
  ~DeviceGuard() {
    if (prev >= 0) (void)hipSetDevice(prev);
  }
};

inline Timer* timer_of(sagips_ctx* c) { return c->timing ? &c->timer : nullptr; }

inline sagips_status ensure_ws(sagips_ctx* c, size_t bytes) {
  if (bytes <= c->ws_cap) return SAGIPS_OK;
  if (c->ws) {
    hipError_t e = hipStreamSynchronize(c->stream);
    if (e != hipSuccess) return hip_fail(c, e, "hipStreamSynchronize before workspace growth");
    (void)hipFree(c->ws);
    c->ws = nullptr;
    c->ws_cap = 0;
  }
  size_t want = (bytes + ((size_t)1 << 20) - 1) & ~(((size_t)1 << 20) - 1);
  if (hipMalloc(&c->ws, want) != hipSuccess) {
    (void)hipGetLastError();
    c->ws = nullptr;
    return fail(c, SAGIPS_E_NOMEM, "workspace allocation of %zu bytes failed", want);
  }
  c->ws_cap = want;
  return SAGIPS_OK;
}

}  // namespace sagips
