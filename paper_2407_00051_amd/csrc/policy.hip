// Training the parameter rows without a differentiable pipeline: advantages
// within a row's events, the clipped policy loss and the preference loss, each
// with its gradient with respect to theta.  The policy is the sampler's own
// density: an event x drawn at row (a_j, b_j) has
//   l(x) = sum_j ln a_j + ln b_j + (a_j - 1) ln x_j + (b_j - 1) ln(1 - x_j^a_j),
//   dl/da_j = 1/a_j + ln x_j (1 - (b_j - 1) x_j^a_j / (1 - x_j^a_j)),
//   dl/db_j = 1/b_j + ln(1 - x_j^a_j).
// Two rows' densities are only ever needed as a difference, and it is formed
// term by term,
//   l - l' = ln(a/a') + ln(b/b') + (a - a') ln x + (b - 1)(g - g') + (b - b') g',
// g = ln(1 - x^a), g' = ln(1 - x^a'): its rounding then shrinks with the
// distance between the rows instead of staying at that of l.
#include "device_math.hpp"
#include "kernels.hpp"

namespace sagips {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

// Events are read clamped to the open unit interval: a draw may have rounded to
// 0 or 1.  NaN stays NaN.
__device__ __forceinline__ float clamp_event(float x) {
  return __builtin_elementwise_minimum(__builtin_elementwise_maximum(x, 0x1p-126f), 1.0f - 0x1p-24f);
}

// 1 - x^a, from l2 = log2 x < 0.  With t = a l2, 1 - 2^t = -t P(t): above 2^t = 3/4 by the
// polynomial of degree 4 that interpolates P at the Chebyshev nodes of [log2 3/4, 0]
// (relative error 1.3e-8 with these fp32 coefficients), so that no step cancels.
__device__ __forceinline__ float one_minus_power(float a, float l2, float* w_out) {
  const float t = a * l2, w = fast_exp2(t);
  float p = 0x1.364d2ep-10f;
  p = fmaf(p, t, 0x1.396c7ap-7f);
  p = fmaf(p, t, 0x1.c6a02cp-5f);
  p = fmaf(p, t, 0x1.ebfbaap-3f);
  p = fmaf(p, t, 0x1.62e430p-1f);
  *w_out = w;
  return w < 0.75f ? 1.0f - w : -t * p;
}

// A row that the gradient is taken at, and one that its density is compared with.
template <int D>
struct Row {
  float a[D], b[D], bm1[D];
};
template <int D>
struct Against {
  float a[D], da[D], db[D], c;   // c: sum log2(a/a') + log2(b/b')
};

// ln(a / b) of positive a, b, as +- ln(1 + (larger - smaller) / smaller): the difference is exact
// within a factor of two, and the quotient, unlike one over the larger, does not run into -1.  Where
// it is beyond fp32, the difference of two logarithms of 88 or more in all.
__device__ __forceinline__ float log_quotient(float a, float b) {
  const bool below = a < b;
  const float hi = below ? b : a, lo = below ? a : b, q = (hi - lo) / lo;
  const float l = q < INFINITY ? log1pf(q) : logf(hi) - logf(lo);
  return below ? -l : l;
}

// Reads a row and the kOthers it is compared with.  Every group of `step` lanes (this lane its
// l-th) shares the divisions and logarithms out among its lanes, one item a lane where the group
// has as many, and has them back through `shared` (2D (kOthers + 1) floats of the group): with
// each lane taking all of them, 1,850 operations stood before a loop of 190.  The whole
// workgroup calls it.
template <int D, int kOthers>
__device__ __forceinline__ void load_rows(const float* __restrict__ th, const float* const (&others)[kOthers], int l, int step,
                                          float* shared, Row<D>& r, Against<D> (&o)[kOthers]) {
  for (int k = l; k < 2 * D * (kOthers + 1); k += step) {
    const int w = k / (2 * D), j = k % (2 * D);
    const float at = th[j];
    float den = at;
#pragma unroll
    for (int i = 0; i < kOthers; ++i) den = w == i + 1 ? others[i][j] : den;
    shared[k] = w ? log_quotient(at, den) : 1.0f / at;
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < D; ++j) {
    r.a[j] = th[2 * j];
    r.b[j] = th[2 * j + 1];
    r.bm1[j] = r.b[j] - 1.0f;
  }
#pragma unroll
  for (int i = 0; i < kOthers; ++i) {
    o[i].c = 0.0f;
#pragma unroll
    for (int j = 0; j < D; ++j) {
      o[i].a[j] = others[i][2 * j];
      o[i].da[j] = r.a[j] - o[i].a[j];
      o[i].db[j] = r.b[j] - others[i][2 * j + 1];
      o[i].c += (shared[2 * D * (i + 1) + 2 * j] + shared[2 * D * (i + 1) + 2 * j + 1]) * kLog2e;
    }
  }
}

// What the current row needs of an event.
template <int D>
struct Event {
  float l2[D], lg[D], q[D];   // log2 x, log2(1 - x^a), x^a / (1 - x^a)
};
template <int D>
__device__ __forceinline__ Event<D> at_row(const float (&x)[D], const Row<D>& r) {
  Event<D> e;
#pragma unroll
  for (int j = 0; j < D; ++j) {
    float w;
    e.l2[j] = fast_log2(clamp_event(x[j]));
    const float g = one_minus_power(r.a[j], e.l2[j], &w);
    e.lg[j] = fast_log2(g);
    e.q[j] = w * fast_rcp(g);
  }
  return e;
}
// log2 of the density's ratio, current row over the other.
template <int D>
__device__ __forceinline__ float log2_ratio(const Event<D>& e, const Row<D>& r, const Against<D>& o) {
  float s = o.c;
#pragma unroll
  for (int j = 0; j < D; ++j) {
    float w;
    const float lo = fast_log2(one_minus_power(o.a[j], e.l2[j], &w));
    s = fmaf(o.da[j], e.l2[j], s);
    s = fmaf(r.bm1[j], e.lg[j] - lo, s);
    s = fmaf(o.db[j], lo, s);
  }
  return s;
}
// acc += wt * dl/d(a, b), without the terms 1/a and 1/b, which add_constants gives once to a
// lane's finished sum of weights.
template <int D>
__device__ __forceinline__ void add_grad(const Event<D>& e, const Row<D>& r, float wt, float* acc) {
#pragma unroll
  for (int j = 0; j < D; ++j) {
    const float u = wt * e.l2[j];
    acc[2 * j] = fmaf(u, fmaf(-kLn2 * r.bm1[j], e.q[j], kLn2), acc[2 * j]);
    acc[2 * j + 1] = fmaf(wt * kLn2, e.lg[j], acc[2 * j + 1]);
  }
}
// `inverse`: the row's 1/a and 1/b, as load_rows leaves them.
template <int D>
__device__ __forceinline__ void add_constants(const float* inverse, float weights, float* acc) {
#pragma unroll
  for (int j = 0; j < 2 * D; ++j) acc[j] = fmaf(weights, inverse[j], acc[j]);
}

template <int D>
__device__ __forceinline__ void load_event(const float* __restrict__ x, int64_t i, float (&v)[D]) {
  const float* p = x + i * D;
#pragma unroll
  for (int j = 0; j < D; ++j) v[j] = p[j];
}

// e^r - 1 - r: by its series below 1/2 (next term at most 5e-8 of it), where the subtraction would cancel.
__device__ __forceinline__ float exp_minus_line(float r) {
  float p = 1.0f / 40320.0f;
  p = fmaf(p, r, 1.0f / 5040.0f);
  p = fmaf(p, r, 1.0f / 720.0f);
  p = fmaf(p, r, 1.0f / 120.0f);
  p = fmaf(p, r, 1.0f / 24.0f);
  p = fmaf(p, r, 1.0f / 6.0f);
  p = fmaf(p, r, 0.5f);
  float k = r * r * p;
  if (__any(!(fabsf(r) < 0.5f))) k = fabsf(r) < 0.5f ? k : fast_exp(r) - 1.0f - r;   // rarely any lane
  return k;
}

// Sum over groups of 2^lg neighbouring lanes, in every lane of the group.
template <int N>
__device__ __forceinline__ void group_sum(float (&v)[N], int lg) {
  for (int s = 0; s < lg; ++s)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor(v[i], 1 << s, 64);
}

__device__ __forceinline__ double group_sum_d(double v, int lg) {
  for (int s = 0; s < lg; ++s) v += __shfl_xor(v, 1 << s, 64);
  return v;
}
__device__ __forceinline__ double wave_sum_d(double v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
// Sum over the workgroup, in every thread.
template <int N, int kT>
__device__ __forceinline__ void block_sum_d(double (&v)[N]) {
  __shared__ double part[kT / 64][N];
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = wave_sum_d(v[i]);
  __syncthreads();
  if ((threadIdx.x & 63) == 0)
#pragma unroll
    for (int i = 0; i < N; ++i) part[threadIdx.x >> 6][i] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    double s = 0.0;
    for (int w = 0; w < (int)(blockDim.x >> 6); ++w) s += part[w][i];
    v[i] = s;
  }
}

// ---- advantages --------------------------------------------------------------
// (r - mean) / (std + eps) over a row's valid events.  The mean is a 64-bit sum,
// so that a row of equal rewards gives zeros, whatever eps; deviations are formed in
// 64 bits and rounded once.  Bound by memory where rows are many: 1,000,000 x 16 take 26-31 us
// (128 MB at 4.1 to 4.9 TB/s), 16,384 x 1,000 22, 4,096 x 4,097 28; by the time of one read, two
// sums over lanes and one write where they are few (6-7 us a call).

constexpr int kAdvHeld = 16;   // rewards a lane holds between reading and writing, at most
constexpr int kAdvBlock = 1024;

// Whether fp32 deviations times 1 / (sd + eps) in fp32 give a row's advantages.  Else (also where
// sd + eps is 0) write_wide reads the row again and stays in 64 bits until the end.  With 64 bits
// for every row 4,096 x 4,097 take 33 us instead of 28: more registers, fewer waves.
__device__ __forceinline__ bool fits_fp32(float inv) { return inv >= 1e-30f && inv <= 1e30f; }
__device__ __forceinline__ void write_wide(const float* reward, const uint8_t* mask, int e0, int step, int E, double mean, double sd,
                                           double eps, float* adv) {
  const double inv = sd == 0.0 ? 0.0 : 1.0 / (sd + eps);   // no deviations: 0, not 0 / 0
  for (int e = e0; e < E; e += step) adv[e] = !mask || mask[e] ? (float)(((double)reward[e] - mean) * inv) : 0.0f;
}

// Reads a lane's events e0 + i * step < E of the row at `off`: v, 0 where not valid, and a bit for
// each valid one.  All reads are at places inside the row, so that none waits for a branch
// (16,384 rows of 1,000 events: 160 us with a branch for each).
template <int kHeld>
__device__ __forceinline__ uint32_t load_rewards(const float* reward, const uint8_t* __restrict__ mask, int off, int e0, int step,
                                                 int E, float (&v)[kHeld]) {
  uint32_t valid = 0;
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const int e = e0 + i * step;
    v[i] = reward[off + (e < E ? e : E - 1)];
    valid |= e < E ? 1u << i : 0u;
  }
  if (mask) {
    uint8_t k[kHeld];
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      const int e = e0 + i * step;
      k[i] = mask[off + (e < E ? e : E - 1)];
    }
#pragma unroll
    for (int i = 0; i < kHeld; ++i) valid &= k[i] ? ~0u : ~(1u << i);
  }
#pragma unroll
  for (int i = 0; i < kHeld; ++i) v[i] = (valid >> i) & 1u ? v[i] : 0.0f;
  return valid;
}

// A row in a group of 2^lg lanes (kBlock false; up to 64 x 16 events) or in a
// workgroup (up to 1,024 x 16): read once, held in registers, written once.
template <bool kBlock, int kHeld>
__global__ __launch_bounds__(kBlock ? kAdvBlock : kThreads) void k_advantage(const float* reward, const uint8_t* __restrict__ mask,
                                                                            int n_rows, int E, int lg, double eps, int normalise,
                                                                            float* adv) {
  const int lane = threadIdx.x & 63, step = kBlock ? blockDim.x : 1 << lg;
  const int l = kBlock ? threadIdx.x : lane & (step - 1);
  // The workgroup's first row and this lane's, from the first
  const int64_t row0 = kBlock ? blockIdx.x : (int64_t)blockIdx.x * kWaves << (6 - lg);
  const int ahead = kBlock ? 0 : ((threadIdx.x >> 6) << (6 - lg)) + (lane >> lg), last = (int)min((int64_t)255, n_rows - 1 - row0);
  const bool on = kBlock || ahead <= last;
  const int off = kBlock ? 0 : (on ? ahead : last) * E;
  const float* from = reward + row0 * E;
  float* to = adv + row0 * E;
  float v[kHeld];
  double t[2] = {0.0, 0.0};
  const uint32_t valid = load_rewards<kHeld>(from, mask ? mask + row0 * E : nullptr, off, l, step, E, v);
#pragma unroll
  for (int i = 0; i < kHeld; ++i) t[0] += (double)v[i];
  t[1] = (double)__popc(valid);
  if constexpr (kBlock) block_sum_d<2, kAdvBlock>(t);
  else
    for (int s = 0; s < lg; ++s) {
      t[0] += __shfl_xor(t[0], 1 << s, 64);
      t[1] += __shfl_xor(t[1], 1 << s, 64);
    }
  const double n = t[1], mean = n > 0.0 ? t[0] / n : 0.0;
  double q[1] = {0.0};
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const double dev = (valid >> i) & 1u ? (double)v[i] - mean : 0.0;
    q[0] = fma(dev, dev, q[0]);
    v[i] = (float)dev;
  }
  float inv = 1.0f;
  if (normalise) {
    if constexpr (kBlock) block_sum_d<1, kAdvBlock>(q);
    else
      for (int s = 0; s < lg; ++s) q[0] += __shfl_xor(q[0], 1 << s, 64);
    const double sd = n > 0.0 ? sqrt(q[0] / n) : 0.0;
    inv = 1.0f / ((float)sd + (float)eps);
    if (__builtin_expect(!fits_fp32(inv), 0)) {
      if (on) write_wide(from + off, mask ? mask + row0 * E + off : nullptr, l, step, E, mean, sd, eps, to + off);
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const int e = l + i * step;
    if (on && e < E) to[off + e] = (valid >> i) & 1u ? v[i] * inv : 0.0f;
  }
}

// Long rows, in slices of kAdvSlice events: each slice's count, mean and sum of
// squared deviations, then one pass that joins a row's slices (Chan's update)
// and writes.
constexpr int kAdvSlice = 16384;
__global__ __launch_bounds__(kAdvBlock, 8) void k_adv_slices(const float* __restrict__ reward, const uint8_t* __restrict__ mask,
                                                          int64_t E, int n_slices, double* __restrict__ part) {
  const int64_t row = blockIdx.x / n_slices, s = blockIdx.x % n_slices;
  const int64_t base = row * E + s * kAdvSlice;
  const int n = (int)min((int64_t)kAdvSlice, E - s * kAdvSlice);
  float v[kAdvSlice / kAdvBlock];
  double t[2] = {0.0, 0.0};
  const uint32_t valid = load_rewards<kAdvSlice / kAdvBlock>(reward + base, mask ? mask + base : nullptr, 0, threadIdx.x, kAdvBlock,
                                                                       n, v);
#pragma unroll
  for (int i = 0; i < kAdvSlice / kAdvBlock; ++i) t[0] += (double)v[i];
  t[1] = (double)__popc(valid);
  block_sum_d<2, kAdvBlock>(t);
  const double mean = t[1] > 0.0 ? t[0] / t[1] : 0.0;
  double q[1] = {0.0};
#pragma unroll
  for (int i = 0; i < kAdvSlice / kAdvBlock; ++i)
    if ((valid >> i) & 1u) q[0] += ((double)v[i] - mean) * ((double)v[i] - mean);
  block_sum_d<1, kAdvBlock>(q);
  if (threadIdx.x == 0) {
    part[(int64_t)blockIdx.x * 3] = t[1];
    part[(int64_t)blockIdx.x * 3 + 1] = mean;
    part[(int64_t)blockIdx.x * 3 + 2] = q[0];
  }
}
__global__ __launch_bounds__(kAdvBlock, 8) void k_adv_apply(const float* reward, const uint8_t* __restrict__ mask, int64_t E,
                                                         int n_slices, const double* __restrict__ part, double eps,
                                                         int normalise, float* adv) {
  const int64_t row = blockIdx.x / n_slices, s = blockIdx.x % n_slices, base = row * E + s * kAdvSlice;
  const int n = (int)min((int64_t)kAdvSlice, E - s * kAdvSlice);
  float v[kAdvSlice / kAdvBlock];
  const uint32_t valid = load_rewards<kAdvSlice / kAdvBlock>(reward + base, mask ? mask + base : nullptr, 0, threadIdx.x, kAdvBlock,
                                                                       n, v);
  const double* p = part + row * n_slices * 3;
  double t[2] = {0.0, 0.0};
  for (int i = threadIdx.x; i < n_slices; i += kAdvBlock) {
    t[0] += p[3 * i] * p[3 * i + 1];
    t[1] += p[3 * i];
  }
  block_sum_d<2, kAdvBlock>(t);
  const double mean = t[1] > 0.0 ? t[0] / t[1] : 0.0;
  double q[1] = {0.0};
  for (int i = threadIdx.x; i < n_slices; i += kAdvBlock) {
    const double dm = p[3 * i + 1] - mean;
    q[0] += p[3 * i] > 0.0 ? p[3 * i + 2] + p[3 * i] * dm * dm : 0.0;
  }
  float inv = 1.0f;
  if (normalise) {
    block_sum_d<1, kAdvBlock>(q);
    const double sd = t[1] > 0.0 ? sqrt(q[0] / t[1]) : 0.0;
    inv = 1.0f / ((float)sd + (float)eps);
    if (__builtin_expect(!fits_fp32(inv), 0)) {
      write_wide(reward + base, mask ? mask + base : nullptr, threadIdx.x, kAdvBlock, n, mean, sd, eps, adv + base);
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < kAdvSlice / kAdvBlock; ++i) {
    const int e = threadIdx.x + i * kAdvBlock;
    if (e < n) adv[base + e] = (valid >> i) & 1u ? (float)((double)v[i] - mean) * inv : 0.0f;
  }
}

// ---- policy loss ---------------------------------------------------------------
// A record for the launch's last workgroup (kEnds) or for the next launch.  The former goes
// through to where every XCD sees it, so that nothing has to be written back before the
// workgroup is counted: a release, which writes the XCD's whole L2 back, for every workgroup
// cost 45 us at 1,024 of them.
template <bool kEnds>
__device__ __forceinline__ void put_record(float* p, float v) {
  if constexpr (kEnds) __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  else *p = v;
}
// Whether this workgroup is the last of its launch to come here, all the others' records
// visible to it.  16 counters of the context, then one of those that filled theirs (one for all:
// 2 us more at 256 workgroups); whoever fills a counter puts it back to 0.
// Only which workgroup is last depends on the order, not what it computes.
__device__ __forceinline__ bool last_block(uint32_t* ticket) {
  __shared__ bool last;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // every wave's records have arrived before the workgroup is counted
  __syncthreads();
  if (threadIdx.x == 0) {
    const auto fills = [](uint32_t* p, uint32_t n) {
      const bool is = __hip_atomic_fetch_add(p, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == n - 1;
      if (is) __hip_atomic_store(p, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      return is;
    };
    const uint32_t mine = blockIdx.x % kCounters;
    last = fills(ticket + (1 + mine) * kApart, (gridDim.x - mine + kCounters - 1) / kCounters) &&
           fills(ticket, min(gridDim.x, (uint32_t)kCounters));
  }
  __syncthreads();
  if (!last) return false;
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
  return true;
}

// Joins the units' sums in 64 bits and applies the average.  Every workgroup
// forms the totals that its rows' weights need; the first writes the scalars.  Run by a
// launch of its own, or by the last workgroup of k_policy.
struct PolicyFinish {
  const float4* tot;
  const float* grad;
  int64_t rows, E;
  int S, lg, by_rows, masked;   // 2^lg lanes take a row's records (a wave a row: 1,116 us for 4,096 rows of two, 140 so)
  float *loss, *kl, *clip, *dtheta;
};
constexpr int kAhead = 4;   // records a lane asks for before it adds the first
template <int D, int kEach>   // kEach: values of a gradient of one record a row that a thread asks for at a time
__device__ __forceinline__ void policy_finish(const PolicyFinish& p, int block, int blocks) {
  const int step = 1 << p.lg, l = threadIdx.x & (step - 1), group = threadIdx.x >> p.lg, groups = kThreads >> p.lg;
  const int64_t n_grad = p.rows * 2 * D, stride_g = (int64_t)blocks * kThreads;
  float g[kEach], c[kEach];   // and their rows' counts, before the totals are waited for
  const auto ask = [&](int64_t k) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int64_t at = min(k + i * stride_g, n_grad - 1);
      g[i] = p.grad[at];
      c[i] = p.by_rows && p.masked ? p.tot[at / (2 * D)].w : (float)p.E;
    }
  };
  int64_t k_grad = (int64_t)block * kThreads + threadIdx.x;
  if (p.dtheta && p.S == 1) ask(k_grad);
  double t[5] = {};   // loss, KL, clipped, events (all weighted by 1 / events of the row if by_rows), rows with events
  if (p.masked || block == 0) {
    if (p.by_rows && p.S > 1) {
      for (int64_t k = 0; k < p.rows; k += kAhead * groups) {   // all lanes, for the sums over a group
        float4 v[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) v[i] = p.tot[min(k + i * groups + group, p.rows - 1) * p.S + min(l, p.S - 1)];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          if (k + i * groups >= p.rows) break;
          const int64_t row = k + i * groups + group;
          const bool on = row < p.rows;
          double u[4] = {};
          if (on && l < p.S) {
            u[0] = v[i].x; u[1] = v[i].y; u[2] = v[i].z; u[3] = v[i].w;
            for (int s = l + step; s < p.S; s += step) {
              const float4 w = p.tot[row * p.S + s];
              u[0] += w.x; u[1] += w.y; u[2] += w.z; u[3] += w.w;
            }
          }
#pragma unroll
          for (int c = 0; c < 4; ++c) u[c] = group_sum_d(u[c], p.lg);
          if (l == 0 && u[3] > 0.0) {
            const double w = 1.0 / u[3];
#pragma unroll
            for (int c = 0; c < 4; ++c) t[c] += u[c] * w;
            t[4] += 1.0;
          }
        }
      }
    } else {
      const int64_t n = p.rows * p.S;
      for (int64_t k = threadIdx.x; k < n; k += kAhead * kThreads) {
        float4 v[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) v[i] = p.tot[min(k + i * kThreads, n - 1)];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          if (k + i * kThreads >= n) break;
          const double w = !p.by_rows ? 1.0 : v[i].w > 0.0f ? 1.0 / v[i].w : 0.0;
          t[0] += w * v[i].x; t[1] += w * v[i].y; t[2] += w * v[i].z; t[3] += w * v[i].w;
          t[4] += v[i].w > 0.0f ? 1.0 : 0.0;
        }
      }
    }
    block_sum_d<5, kThreads>(t);
  }
  const double all = p.by_rows ? (p.masked ? t[4] : (double)p.rows) : (p.masked ? t[3] : (double)p.rows * (double)p.E);
  const double inv = all > 0.0 ? 1.0 / all : 0.0;
  if (block == 0 && threadIdx.x == 0) {
    if (p.loss) *p.loss = (float)(t[0] * inv);
    if (p.kl) *p.kl = (float)(t[1] * inv);
    if (p.clip) *p.clip = (float)(t[2] * inv);
  }
  if (!p.dtheta) return;
  if (p.S == 1) {
    for (; k_grad < n_grad; k_grad += kEach * stride_g) {
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        if (k_grad + i * stride_g >= n_grad) break;
        // a row's average in fp32, as its sum was; the average over rows in 64 bits
        const float v = !p.by_rows ? g[i] : c[i] > 0.0f ? g[i] / c[i] : 0.0f;
        p.dtheta[k_grad + i * stride_g] = (float)(v * inv);
      }
      if (k_grad + kEach * stride_g < n_grad) ask(k_grad + kEach * stride_g);
    }
    return;
  }
  for (int64_t k = (int64_t)block * groups; k < p.rows; k += (int64_t)blocks * groups) {
    const int64_t row = k + group;
    double u[2 * D + 1] = {};
    if (row < p.rows)
      for (int s = l; s < p.S; s += step) {
        const int64_t at = row * p.S + s;
        u[2 * D] += p.tot[at].w;
#pragma unroll
        for (int j = 0; j < 2 * D; ++j) u[j] += p.grad[at * 2 * D + j];
      }
#pragma unroll
    for (int j = 0; j < 2 * D + 1; ++j) u[j] = group_sum_d(u[j], p.lg);
    const double w = !p.by_rows ? inv : u[2 * D] > 0.0 ? inv / u[2 * D] : 0.0;
    if (l == 0 && row < p.rows)
#pragma unroll
      for (int j = 0; j < 2 * D; ++j) p.dtheta[row * 2 * D + j] = (float)(u[j] * w);
  }
}
template <int D>
__global__ __launch_bounds__(kThreads) void k_policy_finish(PolicyFinish p) {
  policy_finish<D, 2>(p, blockIdx.x, gridDim.x);
}

// A unit is one slice of one row, run by a group of 2^lg lanes (a wave, or less
// where rows have fewer events).  It leaves its sums over valid events: of the
// loss, the KL term, the clipped events and the events, and of the gradient; where
// a row has whole workgroups of slices, a workgroup's four units leave one record.
// Bound by VALU issue: 64 events of three coordinates against two rows take 26
// transcendental and 188 other operations, 51% of all in pairs (adds, products and
// fmas with a literal do; compares, selects, fmac and fmas of three registers do not), and
// the vector units issue in all of the cycles in which a compute unit works.  1,024 x 16,384
// events with mask and KL term: 113-119 us with the second launch; reading them takes 61 at
// the rate of a large copy.  Where no joining follows in it, the kernel is held to 64
// registers, so that the 8,192 waves are resident together: with 71, seven to a SIMD and an
// eighth after them, 139 us.
struct PolicyArgs {
  const float *theta, *theta_old, *theta_ref, *x, *adv;
  const uint8_t* mask;
  int64_t E, chunk, units;
  int S, lg, per_block;
  float lo, hi, beta;
  float4* tot;   // [records]
  float* grad;   // [records][2d]
  uint32_t* ticket;   // or NULL: a launch of k_policy_finish follows
  PolicyFinish fin;
};

// kEnds: the launch ends in its last workgroup.
template <int D, bool kRef, bool kEnds>
__global__ __launch_bounds__(kThreads, kEnds ? 4 : 8) void k_policy(PolicyArgs p) {
  const int lane = threadIdx.x & 63, step = 1 << p.lg, l = lane & (step - 1);
  const int64_t unit = (((int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6)) << (6 - p.lg)) + (lane >> p.lg);
  const bool on = unit < p.units;
  const int64_t row = on ? unit / p.S : 0, s = on ? unit % p.S : 0;
  constexpr int kOthers = kRef ? 2 : 1, kItems = 2 * D * (kOthers + 1);
  __shared__ float items[kThreads * kItems];
  const float* others[kOthers];
  others[0] = p.theta_old + row * 2 * D;
  if constexpr (kRef) others[1] = p.theta_ref + row * 2 * D;
  Row<D> r;
  Against<D> o[kOthers];
  float* const mine = items + (threadIdx.x >> p.lg) * kItems;
  load_rows<D>(p.theta + row * 2 * D, others, l, step, mine, r, o);
  const int64_t e1 = on ? min(p.E, (s + 1) * p.chunk) : 0;
  float acc[2 * D + 4] = {}, weights = 0.0f;   // the gradient, then loss, KL, clipped, events
  for (int64_t e = s * p.chunk + l; e < e1; e += step) {
    const int64_t i = row * p.E + e;
    if (p.mask && !p.mask[i]) continue;
    float x[D];
    load_event<D>(p.x, i, x);
    const float A = p.adv[i];
    const Event<D> ev = at_row<D>(x, r);
    const float rho = fast_exp2(log2_ratio<D>(ev, r, o[0]));
    // min(rho A, clip(rho) A); of A = 0 also where rho is beyond fp32 (the clip keeps a NaN)
    const float in = __builtin_elementwise_maximum(__builtin_elementwise_minimum(rho, p.hi), p.lo) * A;
    const float out = A == 0.0f ? in : rho * A;
    const bool cut = in < out;
    float loss = cut ? -in : -out;
    float wt = cut ? 0.0f : -out;
    if constexpr (kRef) {
      const float t = -log2_ratio<D>(ev, r, o[kOthers - 1]) * kLn2, k = exp_minus_line(t);
      if (p.beta != 0.0f) {   // of all events: no weight, also on a K beyond fp32
        loss = fmaf(p.beta, k, loss);
        wt = fmaf(-p.beta, t + k, wt);
      }
      acc[2 * D + 1] += k;
    }
    acc[2 * D] += loss;
    acc[2 * D + 2] += cut ? 1.0f : 0.0f;
    acc[2 * D + 3] += 1.0f;
    weights += wt;
    add_grad<D>(ev, r, wt, acc);
  }
  add_constants<D>(mine, weights, acc);
  group_sum(acc, p.lg);
  if (p.per_block) {
    __shared__ float sums[kWaves][2 * D + 4];
    if (lane == 0)
#pragma unroll
      for (int j = 0; j < 2 * D + 4; ++j) sums[threadIdx.x >> 6][j] = acc[j];
    __syncthreads();
    if (threadIdx.x < 2 * D + 4) {
      float v = 0.0f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) v += sums[w][threadIdx.x];
      put_record<kEnds>(threadIdx.x < 2 * D ? p.grad + (int64_t)blockIdx.x * 2 * D + threadIdx.x
                                            : reinterpret_cast<float*>(p.tot + blockIdx.x) + threadIdx.x - 2 * D, v);
    }
  } else if (on && l == 0) {
#pragma unroll
    for (int j = 0; j < 4; ++j) put_record<kEnds>(reinterpret_cast<float*>(p.tot + unit) + j, acc[2 * D + j]);
#pragma unroll
    for (int j = 0; j < 2 * D; ++j) put_record<kEnds>(p.grad + unit * 2 * D + j, acc[j]);
  }
  if constexpr (kEnds)
    if (last_block(p.ticket)) policy_finish<D, 12>(p.fin, 0, 1);
}

// ---- preference loss -----------------------------------------------------------
// Joins the units' sums in 64 bits; as policy_finish.
struct PrefFinish {
  const float* in;            // [rows][S][2d + 1]
  int64_t rows;
  int S, lg;                  // 2^lg lanes take a row's records
  double beta, inv_pairs;
  float *loss, *dtheta;
};
template <int D>
__device__ __forceinline__ void pref_finish(const PrefFinish& p, int block, int blocks) {
  const int step = 1 << p.lg, l = threadIdx.x & (step - 1), group = threadIdx.x >> p.lg, groups = kThreads >> p.lg;
  if (block == 0 && p.loss) {
    double t[1] = {0.0};
    const int64_t n = p.rows * p.S;
    for (int64_t k = threadIdx.x; k < n; k += kAhead * kThreads) {
      float v[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) v[i] = p.in[min(k + i * kThreads, n - 1) * (2 * D + 1) + 2 * D];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) t[0] += k + i * kThreads < n ? v[i] : 0.0f;
    }
    block_sum_d<1, kThreads>(t);
    if (threadIdx.x == 0) *p.loss = (float)(t[0] * p.inv_pairs);
  }
  if (!p.dtheta) return;
  const double w = p.beta * p.inv_pairs;
  if (p.S == 1) {
    const int64_t n = p.rows * 2 * D, stride = (int64_t)blocks * kThreads;
    for (int64_t k = (int64_t)block * kThreads + threadIdx.x; k < n; k += kAhead * 2 * stride) {
      float v[kAhead * 2];
#pragma unroll
      for (int i = 0; i < kAhead * 2; ++i) {
        const int64_t at = min(k + i * stride, n - 1);
        v[i] = p.in[at / (2 * D) * (2 * D + 1) + at % (2 * D)];
      }
#pragma unroll
      for (int i = 0; i < kAhead * 2; ++i)
        if (k + i * stride < n) p.dtheta[k + i * stride] = (float)(v[i] * w);
    }
    return;
  }
  const int64_t stride = (int64_t)blocks * groups;
  for (int64_t k = (int64_t)block * groups; k < p.rows; k += kAhead * stride) {
    float v[kAhead][2 * D];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
#pragma unroll
      for (int j = 0; j < 2 * D; ++j)
        v[i][j] = p.in[(min(k + i * stride + group, p.rows - 1) * p.S + min(l, p.S - 1)) * (2 * D + 1) + j];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (k + i * stride >= p.rows) break;
      const int64_t row = k + i * stride + group;
      double u[2 * D] = {};
      if (row < p.rows && l < p.S) {
#pragma unroll
        for (int j = 0; j < 2 * D; ++j) u[j] = v[i][j];
        for (int s = l + step; s < p.S; s += step)
#pragma unroll
          for (int j = 0; j < 2 * D; ++j) u[j] += p.in[(row * p.S + s) * (2 * D + 1) + j];
      }
#pragma unroll
      for (int j = 0; j < 2 * D; ++j) u[j] = group_sum_d(u[j], p.lg);
      if (l == 0 && row < p.rows)
#pragma unroll
        for (int j = 0; j < 2 * D; ++j) p.dtheta[row * 2 * D + j] = (float)(u[j] * w);
    }
  }
}
template <int D>
__global__ __launch_bounds__(kThreads) void k_pref_finish(PrefFinish p) {
  pref_finish<D>(p, blockIdx.x, gridDim.x);
}

// A pair's sums over its two sets, chosen minus rejected: of the log2 ratios and
// of dl/dtheta; both are linear, so one pass over the events gives the margin
// and, once it is known, the gradient.  VALU issue, as k_policy, with one row to compare
// with, in 76% of the busy cycles since a wave's pairs have unequal lengths; 2.9 M events of two
// coordinates 18-19 us of kernel, 25 with the second launch.
struct PrefArgs {
  const float *theta, *theta_ref;
  const float* x[2];          // chosen, rejected
  const int32_t* len[2];      // or NULL
  int64_t T[2];
  int64_t pairs, chunk, units;   // pairs a row; pairs (or, k_pref_slices, events) a unit
  int S, lg;
  float beta, eps;
  float* margin;              // or NULL
  const float* part;          // k_pref with kJoin: [all pairs][slices][2d + 1]
  int slices;
  float* out;                 // [units][2d + 1] (gradient, loss), or the slices' part
  uint32_t* ticket;           // or NULL: a launch of k_pref_finish follows, or nothing
  PrefFinish fin;
};

template <int D>
__device__ __forceinline__ void add_set(const PrefArgs& p, int which, int64_t pair, int64_t e0, int64_t e1, int l, int step,
                                        const Row<D>& r, const Against<D>& ref, float& weights, float (&v)[2 * D + 1]) {
  int64_t n = p.T[which];
  if (p.len[which]) {
    const int64_t given = p.len[which][pair];
    n = given < 0 ? 0 : given < n ? given : n;
  }
  n = min(n, e1);
  const float sign = which ? -1.0f : 1.0f;
  for (int64_t e = e0 + l; e < n; e += step) {
    float x[D];
    load_event<D>(p.x[which], pair * p.T[which] + e, x);
    const Event<D> ev = at_row<D>(x, r);
    v[2 * D] = fmaf(sign, log2_ratio<D>(ev, r, ref), v[2 * D]);
    weights += sign;
    add_grad<D>(ev, r, sign, v);
  }
}

// A unit: one wave, some pairs of one row, 2^lg lanes a pair.  kJoin: the pairs'
// sums come in slices from k_pref_slices.
template <int D, bool kJoin, bool kEnds>
__global__ __launch_bounds__(kThreads) void k_pref(PrefArgs p) {
  const int lane = threadIdx.x & 63, step = 1 << p.lg, l = lane & (step - 1);
  const int64_t unit = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
  const bool any = unit < p.units;   // of the whole wave
  const int64_t row = any ? unit / p.S : 0, s = any ? unit % p.S : 0;
  __shared__ float items[kWaves][4 * D];
  const float* const others[1] = {p.theta_ref + row * 2 * D};
  Row<D> r;
  Against<D> ref[1];
  load_rows<D>(p.theta + row * 2 * D, others, lane, 64, items[threadIdx.x >> 6], r, ref);
  const int64_t q0 = s * p.chunk, q1 = any ? min(p.pairs, q0 + p.chunk) : 0;
  float acc[2 * D + 1] = {};
  for (int64_t q = q0; q < q1; q += 64 >> p.lg) {
    const int64_t mine = q + (lane >> p.lg), pair = row * p.pairs + mine;
    const bool on = mine < q1;
    float v[2 * D + 1] = {};
    if (on) {
      if constexpr (kJoin) {
        for (int i = l; i < p.slices; i += step)
#pragma unroll
          for (int j = 0; j < 2 * D + 1; ++j) v[j] += p.part[(pair * p.slices + i) * (2 * D + 1) + j];
      } else {
        float weights = 0.0f;
        add_set<D>(p, 0, pair, 0, p.T[0], l, step, r, ref[0], weights, v);
        add_set<D>(p, 1, pair, 0, p.T[1], l, step, r, ref[0], weights, v);
        add_constants<D>(items[threadIdx.x >> 6], weights, v);
      }
    }
    group_sum(v, p.lg);
    if (on && l == 0) {
      const float h = p.beta * (v[2 * D] * kLn2);
      if (p.margin) p.margin[pair] = h;
      // softplus(-h) and softplus(h) = softplus(-h) + h; the sigmoid of |h| from the same exponential
      const float t = fast_exp(-fabsf(h)), sp = fmaxf(-h, 0.0f) + log1p_k(t);
      const float sig = (h >= 0.0f ? 1.0f : t) * fast_rcp(1.0f + t);       // sigmoid(h)
      const float one_m = (h >= 0.0f ? t : 1.0f) * fast_rcp(1.0f + t);     // 1 - sigmoid(h)
      acc[2 * D] += (1.0f - p.eps) * sp + p.eps * (sp + h);
      const float g = p.eps * sig - (1.0f - p.eps) * one_m;
#pragma unroll
      for (int j = 0; j < 2 * D; ++j) acc[j] = fmaf(g, v[j], acc[j]);
    }
  }
  group_sum(acc, 6);
  if (any && lane == 0)
#pragma unroll
    for (int j = 0; j < 2 * D + 1; ++j) put_record<kEnds>(p.out + unit * (2 * D + 1) + j, acc[j]);
  if constexpr (kEnds)
    if (last_block(p.ticket)) pref_finish<D>(p.fin, 0, 1);
}

// Long sets: a unit is a wave on one slice of one pair's sets.
template <int D>
__global__ __launch_bounds__(kThreads) void k_pref_slices(PrefArgs p) {
  const int lane = threadIdx.x & 63;
  const int64_t unit = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
  const bool any = unit < p.units;
  const int64_t pair = any ? unit / p.slices : 0, s = any ? unit % p.slices : 0, row = pair / p.pairs;
  __shared__ float items[kWaves][4 * D];
  const float* const others[1] = {p.theta_ref + row * 2 * D};
  Row<D> r;
  Against<D> ref[1];
  load_rows<D>(p.theta + row * 2 * D, others, lane, 64, items[threadIdx.x >> 6], r, ref);
  if (!any) return;
  float v[2 * D + 1] = {}, weights = 0.0f;
  add_set<D>(p, 0, pair, s * p.chunk, (s + 1) * p.chunk, lane, 64, r, ref[0], weights, v);
  add_set<D>(p, 1, pair, s * p.chunk, (s + 1) * p.chunk, lane, 64, r, ref[0], weights, v);
  add_constants<D>(items[threadIdx.x >> 6], weights, v);
  group_sum(v, 6);
  if (lane == 0)
#pragma unroll
    for (int j = 0; j < 2 * D + 1; ++j) p.out[unit * (2 * D + 1) + j] = v[j];
}

// ---- plans ---------------------------------------------------------------------
// Whether a launch ends in its last workgroup instead of in a second launch: where one
// workgroup can join what the others left in the time of that launch (up to 256 of them: 1,024
// rows of 100 events 13.7 us a call against 15.7, 1,024 x 100 single-event pairs 11.7 against
// 14.5; beyond, 600 rows of 600 events 27 against 14, 64 x 64 pairs of 100 events 40 against 13).
// Near the bound either may win: 300 rows of 600 events (225 workgroups, three slices a row) take 19
// against 15, 1,300 and 1,600 rows of 90 (325 and 400 workgroups) 17-18 in one launch, 15-19 in two.
// A gradient of more than 8,192 values is too much for one workgroup however few there are: 8,000
// rows of 2 events 35 us against 17, 30,000 92 against 32.
bool ends_in_last(int64_t blocks, int64_t rows, int d) {
  return blocks <= 256 && rows * 2 * d <= 8192;
}
// Waves that share an array of rows.  Policy loss of 1,024 x 16,384 events 116 us; with 4,096 waves
// 133, with 16,384 116.  64 x 65,536: 38, 39 and 41.  The preference loss is alike with each.
constexpr int64_t kTargetUnits = 8192;

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }
// Lanes (as a power of two) for n items: at most a wave.
int lanes_log(int64_t n) {
  int lg = 0;
  while (lg < 6 && ((int64_t)1 << lg) < n) ++lg;
  return lg;
}

struct PolicyPlan {
  int lg, S, per_block, records;   // records: of a row
  int64_t chunk, units;
  size_t grad_off, bytes;
};
PolicyPlan policy_plan(int64_t rows, int64_t E, int d) {
  PolicyPlan p;
  p.lg = lanes_log(E);
  // slices of at least four events a lane
  const int64_t most = ceil_div(E, 256), want = kTargetUnits / rows;
  p.S = (int)(want < 1 ? 1 : want > most ? most : want);
  p.per_block = p.S >= kWaves;
  if (p.per_block) p.S = p.S / kWaves * kWaves;
  p.chunk = ceil_div(E, p.S);       // the last slices may be short or empty
  p.units = rows * p.S;
  p.records = p.per_block ? p.S / kWaves : p.S;
  p.grad_off = align256((size_t)rows * p.records * sizeof(float4));
  p.bytes = p.grad_off + (size_t)rows * p.records * 2 * d * sizeof(float);
  return p;
}

struct PrefPlan {
  int lg, S, slices;          // slices > 0: long sets, joined after
  int64_t chunk, units, slice_chunk;
  size_t part_off, bytes;
};
// Sets beyond this many events are cut into slices.  Where pairs are few that is late: one pair of
// 4,096 events, a wave's, takes 39 us and one of 4,097 15 (cut from 1,024 or 256 on, 14-16 either),
// 64 x 64 pairs of 4,096 110 (97); 64 x 64 ragged pairs of up to 700 take 24 however it is.
constexpr int64_t kLongSet = 4096;
PrefPlan pref_plan(int64_t rows, int64_t pairs, int64_t T, int d) {
  PrefPlan p;
  p.slices = 0;
  p.slice_chunk = T;
  if (T > kLongSet && rows * pairs < kTargetUnits) {
    const int64_t most = ceil_div(T, 256), want = ceil_div(kTargetUnits, rows * pairs);
    p.slices = (int)(want > most ? most : want);
    p.slice_chunk = ceil_div(T, p.slices);
    p.slices = (int)ceil_div(T, p.slice_chunk);
  }
  p.lg = lanes_log(p.slices ? p.slices : T);
  // a wave takes its lanes' pairs at least twice where a pair is an event a lane: fewer records
  const int64_t most = ceil_div(pairs, (64 >> p.lg) * (T <= 64 ? 2 : 1)), want = kTargetUnits / rows;
  p.S = (int)(want < 1 ? 1 : want > most ? most : want);
  p.chunk = ceil_div(pairs, p.S);
  p.S = (int)ceil_div(pairs, p.chunk);
  p.units = rows * p.S;
  p.part_off = align256((size_t)p.units * (2 * d + 1) * sizeof(float));
  p.bytes = p.part_off + (size_t)rows * pairs * p.slices * (2 * d + 1) * sizeof(float);
  return p;
}

unsigned wave_blocks(int64_t waves) { return (unsigned)ceil_div(waves, kWaves); }

template <int D>
hipError_t policy_d(const sagips_policy& P, const PolicyPlan& pl, const float* x, const float* adv, const uint8_t* mask,
                    float* loss, float* kl, float* clip, float* dtheta, char* ws, uint32_t* ticket, hipStream_t st,
                    Timer* tm) {
  PolicyArgs a{P.theta, P.theta_old, P.theta_ref, x, adv, mask, P.events_per_theta, pl.chunk, pl.units, pl.S, pl.lg,
               pl.per_block, (float)(1.0 - P.clip_low), (float)(1.0 + P.clip_high), (float)P.kl_coef,
               reinterpret_cast<float4*>(ws), reinterpret_cast<float*>(ws + pl.grad_off), nullptr, {}};
  a.fin = PolicyFinish{a.tot, a.grad, P.n_theta, P.events_per_theta, pl.records, lanes_log(pl.records),
                       P.average == SAGIPS_MEAN_ROWS, mask != nullptr, loss, kl, clip, dtheta};
  const dim3 grid(wave_blocks(ceil_div(pl.units, 64 >> pl.lg)));
  if (ends_in_last(grid.x, P.n_theta, D)) a.ticket = ticket;
  if (tm) tm->begin("policy");
  const auto kernel = P.theta_ref ? (a.ticket ? k_policy<D, true, true> : k_policy<D, true, false>)
                                  : (a.ticket ? k_policy<D, false, true> : k_policy<D, false, false>);
  hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, st, a);
  if (tm) tm->end();
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.ticket) return e;
  // at most 128 workgroups, since each forms the totals: 65,535 rows of 16 events, averaged over rows,
  // 73 us with the first launch; with up to 1,024 99, with up to 32 84
  const int64_t blocks = pl.records == 1 ? ceil_div((int64_t)P.n_theta * 2 * D, kThreads) : ceil_div(P.n_theta, kThreads >> a.fin.lg);
  if (tm) tm->begin("policy_finish");
  hipLaunchKernelGGL((k_policy_finish<D>), dim3((unsigned)(blocks > 128 ? 128 : blocks)), dim3(kThreads), 0, st, a.fin);
  if (tm) tm->end();
  return hipGetLastError();
}

template <int D>
hipError_t pref_d(const sagips_preference& P, const PrefPlan& pl, const float* chosen, const int32_t* n_chosen,
                  const float* rejected, const int32_t* n_rejected, float* loss, float* margin, float* dtheta, char* ws,
                  uint32_t* ticket, hipStream_t st, Timer* tm) {
  const int64_t all = (int64_t)P.n_theta * P.pairs_per_theta;
  PrefArgs a{};
  a.theta = P.theta;
  a.theta_ref = P.theta_ref;
  a.x[0] = chosen;
  a.x[1] = rejected;
  a.len[0] = n_chosen;
  a.len[1] = n_rejected;
  a.T[0] = P.len_chosen;
  a.T[1] = P.len_rejected;
  a.pairs = P.pairs_per_theta;
  a.beta = (float)P.beta;
  a.eps = (float)P.label_smoothing;
  a.margin = margin;
  a.slices = pl.slices;
  float* sums = reinterpret_cast<float*>(ws);
  float* part = reinterpret_cast<float*>(ws + pl.part_off);
  if (pl.slices) {
    a.chunk = pl.slice_chunk;
    a.units = all * pl.slices;
    a.out = part;
    if (tm) tm->begin("preference_slices");
    hipLaunchKernelGGL((k_pref_slices<D>), dim3(wave_blocks(a.units)), dim3(kThreads), 0, st, a);
    if (tm) tm->end();
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  a.chunk = pl.chunk;
  a.units = pl.units;
  a.S = pl.S;
  a.lg = pl.lg;
  a.part = part;
  a.out = sums;
  a.fin = PrefFinish{sums, P.n_theta, pl.S, lanes_log(pl.S), P.beta, 1.0 / (double)all, loss, dtheta};
  const unsigned blocks = wave_blocks(pl.units);
  const bool finish = loss || dtheta;
  if (finish && ends_in_last(blocks, P.n_theta, D)) a.ticket = ticket;
  if (tm) tm->begin("preference");
  const auto kernel = pl.slices ? (a.ticket ? k_pref<D, true, true> : k_pref<D, true, false>)
                                : (a.ticket ? k_pref<D, false, true> : k_pref<D, false, false>);
  hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kThreads), 0, st, a);
  if (tm) tm->end();
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !finish || a.ticket) return e;
  // only the first workgroup forms a total: any bound will do (128 and 1,024 are within 3% of 4,096)
  const int64_t n = pl.S == 1 ? ceil_div((int64_t)P.n_theta * 2 * D, kThreads) : ceil_div(P.n_theta, kThreads >> a.fin.lg);
  if (tm) tm->begin("preference_finish");
  hipLaunchKernelGGL((k_pref_finish<D>), dim3((unsigned)(n > 4096 ? 4096 : n)), dim3(kThreads), 0, st, a.fin);
  if (tm) tm->end();
  return hipGetLastError();
}

}  // namespace

size_t advantage_workspace(int64_t n_rows, int64_t E) {
  return E <= kAdvSlice ? 0 : (size_t)n_rows * ceil_div(E, kAdvSlice) * 3 * sizeof(double);
}

hipError_t launch_advantage(const float* reward, const uint8_t* mask, int64_t n_rows, int64_t E, bool normalise, double eps,
                            float* adv, void* ws, hipStream_t st, Timer* tm) {
  if (tm) tm->begin("advantage");
  if (E <= 64 * kAdvHeld) {
    // a lane for every event up to 64, for the least time of one row; with more events than lanes
    // on the device, four a lane and fewer sums over lanes
    const bool many = n_rows * E > 256 * 2048;
    const int held = E > 256 ? kAdvHeld : E > 64 || many ? 4 : 1;
    const int lg = lanes_log(many ? ceil_div(E, held) : E);
    const int64_t waves = ceil_div(n_rows, 64 >> lg);
    const auto kernel = held == 1 ? k_advantage<false, 1> : held == 4 ? k_advantage<false, 4> : k_advantage<false, kAdvHeld>;
    hipLaunchKernelGGL(kernel, dim3(wave_blocks(waves)), dim3(kThreads), 0, st, reward, mask, (int)n_rows, (int)E, lg, eps,
                       (int)normalise, adv);
  } else if (E <= kAdvBlock * kAdvHeld) {
    const int threads = (int)(ceil_div(E, 64 * kAdvHeld) * 64);
    hipLaunchKernelGGL((k_advantage<true, kAdvHeld>), dim3((unsigned)n_rows), dim3(threads), 0, st, reward, mask, (int)n_rows, (int)E,
                       6, eps, (int)normalise, adv);
  } else {
    const int slices = (int)ceil_div(E, kAdvSlice);
    const dim3 grid((unsigned)(n_rows * slices));
    double* part = static_cast<double*>(ws);
    hipLaunchKernelGGL(k_adv_slices, grid, dim3(kAdvBlock), 0, st, reward, mask, E, slices, part);
    if (tm) {
      tm->end();
      tm->begin("advantage_apply");
    }
    hipLaunchKernelGGL(k_adv_apply, grid, dim3(kAdvBlock), 0, st, reward, mask, E, slices, part, eps, (int)normalise, adv);
  }
  if (tm) tm->end();
  return hipGetLastError();
}

size_t policy_workspace(const sagips_policy& P) { return policy_plan(P.n_theta, P.events_per_theta, P.d).bytes; }

hipError_t launch_policy(const sagips_policy& P, const float* x, const float* adv, const uint8_t* mask, float* loss,
                         float* kl, float* clip_frac, float* dtheta, void* ws, uint32_t* ticket, hipStream_t st,
                         Timer* tm) {
  const PolicyPlan pl = policy_plan(P.n_theta, P.events_per_theta, P.d);
  char* w = static_cast<char*>(ws);
  return P.d == 2 ? policy_d<2>(P, pl, x, adv, mask, loss, kl, clip_frac, dtheta, w, ticket, st, tm)
                  : policy_d<3>(P, pl, x, adv, mask, loss, kl, clip_frac, dtheta, w, ticket, st, tm);
}

static PrefPlan plan_of(const sagips_preference& P) {
  return pref_plan(P.n_theta, P.pairs_per_theta, P.len_chosen > P.len_rejected ? P.len_chosen : P.len_rejected, P.d);
}

size_t preference_workspace(const sagips_preference& P) { return plan_of(P).bytes; }

hipError_t launch_preference(const sagips_preference& P, const float* chosen, const int32_t* n_chosen,
                             const float* rejected, const int32_t* n_rejected, float* loss, float* margin, float* dtheta,
                             void* ws, uint32_t* ticket, hipStream_t st, Timer* tm) {
  const PrefPlan pl = plan_of(P);
  char* w = static_cast<char*>(ws);
  return P.d == 2 ? pref_d<2>(P, pl, chosen, n_chosen, rejected, n_rejected, loss, margin, dtheta, w, ticket, st, tm)
                  : pref_d<3>(P, pl, chosen, n_chosen, rejected, n_rejected, loss, margin, dtheta, w, ticket, st, tm);
}

}  // namespace sagips
