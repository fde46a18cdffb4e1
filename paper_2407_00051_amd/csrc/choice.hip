// Choices from logits: log probabilities of given choices, entropy and the most
// likely alternatives of a row, and their gradient.  With z = scale x over a row,
// m = max z, s = sum exp(z - m):
//   ln p_v = z_v - m - ln s,   H = ln s - (1/s) sum exp(z - m) (z - m),
//   dL/dz_v = sum_i g_i ([v = c_i] - p_v) - g_H p_v (ln p_v + H).
//
// Forward: one pass over the logits, which stay in registers; a row is taken by
// 2^k lanes, a wave, 256 or 1,024 threads, whatever holds it, or few long rows in parts.  Every thread keeps
// the maximum of its own values and sums relative to that; the waves' sums are
// joined once.  The alternatives of a short row are taken one a round; of others the K-th largest of 64 groups' maxima is a lower
// bound for the K-th largest value, and hardly more than K values reach it (64 ln 2 =
// 44 on average at K = 32, 9 at K = 8); they are collected in LDS and ranked by counting.
// Longer rows are read a second time for the collecting.
#include "device_math.hpp"
#include "kernels.hpp"
#include "split_bf16.hpp"

#include <float.h>

#include <type_traits>

namespace sagips {
namespace {

constexpr float kLowest = -INFINITY;
constexpr uint32_t kMaskedKey = 0x007fffffu;   // order_key(-infinity)

struct ChoiceArgs {
  const void* x;
  int64_t rows, stride;
  int n, top;
  float scale2;                    // scale log2 e
  float twice;                     // 2 scale
  const int32_t* choice;
  float *logp, *entropy;
  int32_t* top_choice;
  float *top_logp, *stats;
  // Rows cut into parts of `per` units: a record of each, and a counter a row that finds the part
  // which ends last (NULL: k_choice_join follows).
  int parts, per;
  char* records;
  uint32_t* ticket;
};

// Values of a 16-byte unit.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint32_t word(u32x4 r, int k) { return k < 2 ? (k == 0 ? r.x : r.y) : (k == 2 ? r.z : r.w); }
template <class T>
struct Unit;
template <>
struct Unit<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ float get(u32x4 r, int j) { return __uint_as_float(word(r, j)); }
};
template <>
struct Unit<u16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ float get(u32x4 r, int j) {
    const uint32_t w = word(r, j >> 1);
    return j & 1 ? bf16_hi(w) : bf16_lo(w);
  }
};
__device__ __forceinline__ uint32_t bits_of(float v) { return __float_as_uint(v); }
__device__ __forceinline__ uint32_t bits_of(u16 v) { return v; }
template <class T>
constexpr uint32_t kFill = sizeof(T) == 4 ? 0xff800000u : 0xff80u;   // -infinity

// A row in 16-byte units of memory, the first of which may begin before the row.
// Value j of unit q is the row's q N + j - lead; values outside the row read as
// -infinity, and nothing outside it is read.
template <class T>
struct RowView {
  static constexpr int N = Unit<T>::N;
  const char* base;
  int lead, n;
  __device__ __forceinline__ RowView(const void* x, int64_t off, int n_) : n(n_) {
    // (by pointer arithmetic: from an integer the reads would be flat ones)
    const char* at = (const char*)((const T*)x + off);
    const int over = (int)((uintptr_t)at & 15);
    base = at - over;
    lead = over / (int)sizeof(T);
  }
  __device__ __forceinline__ int units() const { return (int)(((int64_t)n + lead + N - 1) / N); }
  __device__ __forceinline__ int first(int q) const { return q * N - lead; }
  __device__ __forceinline__ u32x4 load_whole(int q) const { return *reinterpret_cast<const u32x4*>(base + (uint32_t)q * 16u); }
  __device__ __forceinline__ u32x4 load(int q) const {
    const int i0 = first(q);
    const char* at = base + (uint32_t)q * 16u;
    if (i0 >= 0 && i0 <= n - N) return load_whole(q);
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (sizeof(T) == 4) {
        w[k] = i0 + k >= 0 && i0 + k < n ? bits_of(((const T*)at)[k]) : kFill<T>;
      } else {
        const int i = i0 + 2 * k;
        const uint32_t lo = i >= 0 && i < n ? bits_of(((const T*)at)[2 * k]) : kFill<T>;
        const uint32_t hi = i + 1 >= 0 && i + 1 < n ? bits_of(((const T*)at)[2 * k + 1]) : kFill<T>;
        w[k] = lo | hi << 16;
      }
    }
    return u32x4{w[0], w[1], w[2], w[3]};
  }
};

// Order of candidates: the larger value first, of equal ones the lower index (as 64
// bits, larger first).  +0 and -0 are equal.
__device__ __forceinline__ uint32_t order_key(float v) {
  const uint32_t u = __float_as_uint(v + 0.0f);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float order_value(uint32_t k) {
  return __uint_as_float(k ^ (k & 0x80000000u ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ uint64_t candidate(float v, int i) { return (uint64_t)order_key(v) << 32 | (0xffffffffu - (uint32_t)i); }
__device__ __forceinline__ int candidate_index(uint64_t c) { return (int)(0xffffffffu - (uint32_t)c); }

template <int kCtrl>
__device__ __forceinline__ uint32_t dpp_u(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kCtrl, 0xf, 0xf, true);
}
// Over groups of L lanes (a power of two), in every lane of the group.
template <int L, class V, class F>
__device__ __forceinline__ V group_reduce(V v, F f) {
  const auto as = [](uint32_t u) { return __builtin_bit_cast(V, u); };
  const auto un = [](V x) { return __builtin_bit_cast(uint32_t, x); };
  if constexpr (L >= 2) v = f(v, as(dpp_u<0xB1>(un(v))));
  if constexpr (L >= 4) v = f(v, as(dpp_u<0x1B>(un(v))));
  if constexpr (L >= 8) v = f(v, as(dpp_u<0x141>(un(v))));
  if constexpr (L >= 16) v = f(v, as(dpp_u<0x140>(un(v))));
  if constexpr (L >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(un(v), un(v), false, false);
    v = f(as(r[0]), as(r[1]));
  }
  if constexpr (L >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(un(v), un(v), false, false);
    v = f(as(r[0]), as(r[1]));
  }
  return v;
}
template <int L>
__device__ __forceinline__ float group_max(float v) {   // NaN where one is
  return group_reduce<L>(v, [](float a, float b) { return __builtin_elementwise_maximum(a, b); });
}
// The same bits in every lane: every exchange is between two lanes that add the same two numbers.  With a product
// before it one lane's could become a fused one (then which lane writes an alternative would show in its ln p).
template <int L>
__device__ __forceinline__ float group_sum(float v) {
  return group_reduce<L>(v, [](float a, float b) {
#pragma clang fp contract(off)
    return a + b;
  });
}
template <int L>
__device__ __forceinline__ uint32_t group_max(uint32_t v) {
  return group_reduce<L>(v, [](uint32_t a, uint32_t b) { return max(a, b); });
}
// The first candidate of the group.
template <int L>
__device__ __forceinline__ uint64_t group_first(uint64_t c) {
  const uint32_t hi = group_max<L>((uint32_t)(c >> 32));
  const uint32_t lo = group_max<L>((uint32_t)(c >> 32) == hi ? (uint32_t)c : 0u);
  return (uint64_t)hi << 32 | lo;
}

// Sums of a part of a row: m its largest logit, s = sum 2^d, t = sum 2^d d with d = (x - m) scale2 (the
// difference first: a row's only choice has d = 0 and ln p = 0).  A part without choices has
// m = -infinity, s = t = 0.
struct Sums {
  float m, s, t;
};
// 0 where d is below: no 0 times infinity in 2^d d.  NaN stays.
__device__ __forceinline__ float held_up(float d) { return __builtin_elementwise_maximum(d, -300.0f); }
// To a larger (or the same) m.
__device__ __forceinline__ Sums shifted(const Sums& a, float m, float scale2) {
  const float d = a.s == 0.0f ? 0.0f : held_up((a.m - m) * scale2), f = a.s == 0.0f ? 0.0f : fast_exp2(d);
  return {m, a.s * f, f * fmaf(a.s, d, a.t)};
}
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// The largest of a unit's values and m; NaN where one is.
template <class T>
__device__ __forceinline__ float unit_max(u32x4 r, float m) {
#pragma unroll
  for (int j = 0; j < Unit<T>::N; j += 2) m = larger(larger(Unit<T>::get(r, j), Unit<T>::get(r, j + 1)), m);
  return m;
}
// A unit's sums are formed apart, so that a thread's chain is one addition a unit.
template <class T>
__device__ __forceinline__ void add_unit(u32x4 r, float m, float scale2, float& s, float& t) {
  float us = 0.0f, ut = 0.0f;
#pragma unroll
  for (int j = 0; j < Unit<T>::N; ++j) {
    const float d = held_up((Unit<T>::get(r, j) - m) * scale2), e = fast_exp2(d);
    us += e;
    ut = fmaf(e, d, ut);
  }
  s += us;
  t += ut;
}
// What values are taken relative to: their largest, or 0 where there are none.
__device__ __forceinline__ float finite_or_0(float m) { return m == kLowest ? 0.0f : m; }

// ln p of a row's logits that are not masked: (x - m) scale - ln s, in natural units and from halves (exact ones),
// since with x near the type's lowest value x - m, or its product with log2 e, may pass fp32 where ln p does not.
// What lies below fp32 is its lowest number: -infinity means masked, to a caller and to the gradient.  NaN stays.
struct RowLn {
  float half_m, minus_ln_s, s;
  __device__ __forceinline__ RowLn(const Sums& a, float ls) : half_m(0.5f * a.m), minus_ln_s(-kLn2 * ls), s(a.s) {}
  __device__ __forceinline__ float at(const ChoiceArgs& p, float x) const {
    return larger(fmaf(fmaf(0.5f, x, -half_m), p.twice, minus_ln_s), -FLT_MAX);
  }
};

// What a row's sums give: log2 s, and the results that need nothing else.
template <class T>
__device__ __forceinline__ float write_row(const ChoiceArgs& p, int64_t row, const Sums& a) {
  const float ls = log2f(a.s);
  if (p.stats) {
    p.stats[2 * row] = finite_or_0(a.m);
    p.stats[2 * row + 1] = ls;
  }
  if (p.entropy) p.entropy[row] = a.s == 0.0f ? 0.0f : kLn2 * (ls - a.t / a.s);
  if (p.logp) {
    const int c = p.choice[row];
    float v = 0.0f;
    if (c >= 0 && c < p.n) {
      const uint32_t raw = bits_of(((const T*)p.x)[row * p.stride + c]);
      const float x = __uint_as_float(sizeof(T) == 4 ? raw : raw << 16);
      // a masked choice: -infinity, unless the row is NaN
      v = x == kLowest ? (a.s >= 0.0f ? kLowest : a.s) : RowLn(a, ls).at(p, x);
    }
    p.logp[row] = v;
  }
  return ls;
}
__device__ __forceinline__ void write_top(const ChoiceArgs& p, int64_t row, int k, uint64_t c, const RowLn& r) {
  const int64_t at = row * p.top + k;
  const bool nan = !(r.s >= 0.0f), none = (uint32_t)(c >> 32) <= kMaskedKey;
  p.top_choice[at] = nan || none ? -1 : candidate_index(c);
  p.top_logp[at] = nan ? r.s : none ? kLowest : r.at(p, order_value((uint32_t)(c >> 32)));
}

// Values are taken out of a unit again where they are next needed: kept as floats from one use to the
// next they would need twice the registers, and half the waves would be resident.
__device__ __forceinline__ void forget(u32x4& r) { asm volatile("" : "+v"(r)); }

// ---- short rows: L lanes each, R units a lane -----------------------------------
// Several units a lane, since what is done once a row weighs (65,536 rows of 500 bf16 logits with one alternative: 32 us
// by 64 lanes, 27 by 32 and 23 by 16; of 256 with 8 26, 22 and 21).
template <class T, int L, int R>
__global__ __launch_bounds__(256) void k_choice_short(ChoiceArgs p) {
  constexpr int N = Unit<T>::N;
  const int l = threadIdx.x % L;
  // whole groups leave: no exchange crosses them
  for (int64_t row = (int64_t)blockIdx.x * (256 / L) + threadIdx.x / L; row < p.rows; row += (int64_t)gridDim.x * (256 / L)) {
    const RowView<T> v(p.x, row * p.stride, p.n);
    const int i0 = v.first(l);
    u32x4 r[R];
    float best = kLowest;
#pragma unroll
    for (int i = 0; i < R; ++i) r[i] = v.load(i * L + l);
#pragma unroll
    for (int i = 0; i < R; ++i) best = unit_max<T>(r[i], best);
    Sums a{group_max<L>(best), 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < R; ++i) add_unit<T>(r[i], finite_or_0(a.m), p.scale2, a.s, a.t);
    a.s = group_sum<L>(a.s);
    a.t = group_sum<L>(a.t);
    if (l == 0) write_row<T>(p, row, a);
    if (p.top == 0) continue;
    const RowLn ln(a, log2f(a.s));
    // One alternative a round, which lane k % L keeps; L of them are written together.  A bf16 value's key and its
    // index go in one word (an index is below 128 units' 1,024), fp32 values take a second exchange.
    constexpr bool kWord = sizeof(T) == 2;
    uint32_t key[R * N], kept = 0, kept_lo = 0;        // key 0: masked, outside the row, or taken
    const auto index = [&](int e) __attribute__((always_inline)) { return i0 + e / N * (L * N) + e % N; };
#pragma unroll
    for (int e = 0; e < R * N; ++e) {
      const float x = Unit<T>::get(r[e / N], e % N);
      const uint32_t u = order_key(x);
      key[e] = x == kLowest ? 0u : kWord ? (u & 0xffff0000u) | (0xffffu - (uint32_t)index(e)) : u;
    }
    for (int k = 0; k < p.top; ++k) {
      uint32_t hi = 0;
#pragma unroll
      for (int e = 0; e < R * N; ++e) hi = max(hi, key[e]);
      hi = group_max<L>(hi);
      uint32_t lo = 0;
      if constexpr (!kWord) {
#pragma unroll
        for (int e = 0; e < R * N; ++e) lo = max(lo, key[e] == hi ? 0xffffffffu - (uint32_t)index(e) : 0u);   // of equal ones the lowest
        lo = group_max<L>(lo);
      }
#pragma unroll
      for (int e = 0; e < R * N; ++e) key[e] = (kWord ? key[e] == hi : 0xffffffffu - (uint32_t)index(e) == lo) ? 0u : key[e];
      const int at = k % L;
      if (l == at) kept = hi, kept_lo = lo;
      if (at == L - 1 || k == p.top - 1) {
        if (l <= at) {
          if constexpr (kWord) {                       // the whole key again, whose lower bits are the value's zeros
            kept_lo = 0xffff0000u | kept;
            kept = kept & 0x80000000u ? kept & 0xffff0000u : kept ? kept | 0xffffu : 0u;
          }
          write_top(p, row, k - at + l, (uint64_t)kept << 32 | kept_lo, ln);
        }
      }
    }
  }
}

// ---- a row a workgroup of TH threads, R units a thread and pass -------------------
// The k-th largest key of the wave's 64, by its upper 16 bits, which are a bf16 value's all; the lower
// ones are 0: no larger than the k-th largest.
__device__ __forceinline__ uint32_t wave_kth(uint32_t key, int k) {
  uint32_t at = 0;
#pragma unroll
  for (int b = 31; b >= 16; --b) {
    const uint32_t up = at | 1u << b;
    if (__popcll(__ballot(key >= up)) >= k) at = up;
  }
  return at;
}


// A part's record: its alternatives in order, then its sums.  Stored through to where every XCD sees it.
__device__ __forceinline__ size_t record_bytes(int top) { return (size_t)top * 8 + 16; }
struct Record {
  char* at;
  int top;
  __device__ __forceinline__ Record(const ChoiceArgs& p, int64_t row, int part) : at(p.records + (row * p.parts + part) * record_bytes(p.top)), top(p.top) {}
  __device__ __forceinline__ uint64_t* tops() const { return reinterpret_cast<uint64_t*>(at); }
  __device__ __forceinline__ float* sums() const { return reinterpret_cast<float*>(at + (size_t)top * 8); }
  __device__ __forceinline__ void put_top(int k, uint64_t c) const { __hip_atomic_store(tops() + k, c, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
  __device__ __forceinline__ void put(const Sums& a) const {
    __hip_atomic_store(sums(), a.m, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store(sums() + 1, a.s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store(sums() + 2, a.t, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
};

// Joins the records of a row (at most 64), by one wave: a part a lane.  Every part's list is in order, so that,
// with j = (top - 1) / parts, the ceil(top / (j + 1))-th largest of the lists' entries j is no more than the
// top-th largest of all; those from there on are collected and ranked.
constexpr int kJoinHeld = 256;
template <class T>
__device__ __forceinline__ void join_parts(const ChoiceArgs& p, int64_t row, uint64_t* held, uint32_t* count) {
  const int lane = threadIdx.x & 63;
  const bool on = lane < p.parts;
  const Record r(p, row, on ? lane : 0);
  Sums a{kLowest, 0.0f, 0.0f};
  const int j = p.top ? (p.top - 1) / p.parts : 0;
  uint64_t entry = 0;
  if (on) {
    a = Sums{r.sums()[0], r.sums()[1], r.sums()[2]};
    if (p.top) entry = r.tops()[j];
  }
  a = shifted(a, group_max<64>(a.m), p.scale2);
  a.s = group_sum<64>(a.s);
  a.t = group_sum<64>(a.t);
  if (lane == 0) write_row<T>(p, row, a);
  if (p.top == 0) return;
  const RowLn ln(a, log2f(a.s));
  const uint32_t bound = max(wave_kth((uint32_t)(entry >> 32), (p.top + j) / (j + 1)), kMaskedKey + 1);
  if (lane == 0) *count = 0;
  __builtin_amdgcn_wave_barrier();
  for (int k0 = 0; k0 < p.top; k0 += 8) {
    uint64_t c[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = on && k0 + i < p.top ? r.tops()[k0 + i] : 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if ((uint32_t)(c[i] >> 32) >= bound) {
        const uint32_t at = atomicAdd(count, 1u);
        if (at < (uint32_t)kJoinHeld) held[at] = c[i];
      }
    if (!__any((uint32_t)(c[7] >> 32) >= bound)) break;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  const int n = __builtin_amdgcn_readfirstlane((int)*count);
  if (n <= kJoinHeld) {
    for (int i = lane; i < n; i += 64) {
      const uint64_t c = held[i];
      int rank = 0;
      for (int k = 0; k < n; ++k) rank += held[k] > c;
      if (rank < p.top) write_top(p, row, rank, c, ln);
    }
    for (int k = n + lane; k < p.top; k += 64) write_top(p, row, k, 0, ln);
    return;
  }
  // many equal ones: the next of all, one after the other
  int at = 0;
  uint64_t c = on ? r.tops()[0] : 0;
  for (int k = 0; k < p.top; ++k) {
    const uint64_t first = group_first<64>(c);
    if (lane == k) write_top(p, row, k, first, ln);
    if (on && c == first) c = ++at < p.top ? r.tops()[at] : 0;
  }
}
template <class T>
__global__ __launch_bounds__(64) void k_choice_join(ChoiceArgs p) {
  __shared__ uint64_t held[kJoinHeld];
  __shared__ uint32_t count;
  join_parts<T>(p, blockIdx.x, held, &count);
}

// kParts: a workgroup takes a part of a row.
template <class T, int TH, int R, bool kOnePass, bool kParts>
__global__ __launch_bounds__(TH, R <= 8 && !(kParts && TH == 256) ? 8 : 4) void k_choice_row(ChoiceArgs p) {
  constexpr int N = Unit<T>::N, W = TH / 64, G = TH / 64, kHeld = TH == 64 ? 256 : 1024;
  __shared__ Sums part[W];
  __shared__ float group[64];                        // the largest logit of every G threads
  __shared__ uint64_t cand[kHeld], firsts[W];
  __shared__ uint32_t held;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  constexpr uint32_t none = sizeof(T) == 4 ? kFill<T> : kFill<T> << 16 | kFill<T>;
  const u32x4 fill = {none, none, none, none};
  for (int64_t id = blockIdx.x; id < (kParts ? p.rows * p.parts : p.rows); id += gridDim.x) {
    const int64_t row = kParts ? (uint32_t)id / (uint32_t)p.parts : id;
    const int part_of = kParts ? (int)((uint32_t)id % (uint32_t)p.parts) : 0;
    const RowView<T> v(p.x, row * p.stride, p.n);
    const int begin = kParts ? part_of * p.per : 0, units = kParts ? min(v.units(), begin + p.per) : v.units();
    u32x4 r[R];
    // all whole units' reads first, with no branch between them; then those at the row's ends
    const int whole0 = max(v.lead ? 1 : 0, begin), whole1 = min((v.n + v.lead) / N, units) - 1;
    const auto load = [&](int q0) __attribute__((always_inline)) {
      if (whole1 >= whole0) {
#pragma unroll
        for (int i = 0; i < R; ++i) r[i] = v.load_whole(min(max(q0 + i * TH + tid, whole0), whole1));
      }
      if (whole0 <= q0 && q0 + R * TH - 1 <= whole1) return;
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const int q = q0 + i * TH + tid;
        if (q < whole0 || q > whole1) r[i] = q < units ? v.load(q) : fill;
      }
    };
    float best = kLowest;                            // of the thread
    Sums a{kLowest, 0.0f, 0.0f};
    for (int q0 = begin; q0 < units; q0 += TH * R) {
      load(q0);
#pragma unroll
      for (int i = 0; i < R; ++i) best = unit_max<T>(r[i], best);
      if constexpr (!kOnePass) a = shifted(a, best, p.scale2);
      a.m = best;
      const float m = finite_or_0(best);
#pragma unroll
      for (int i = 0; i < R; ++i) {
        forget(r[i]);
        add_unit<T>(r[i], m, p.scale2, a.s, a.t);
        forget(r[i]);
      }
    }
    if (p.top) {
      const float g = group_max<G>(best);
      if (tid % G == 0) group[tid / G] = g;
      if (tid == 0) held = 0;
    }
    a = shifted(a, group_max<64>(a.m), p.scale2);
    a.s = group_sum<64>(a.s);
    a.t = group_sum<64>(a.t);
    if (lane == 0) part[wave] = a;
    __syncthreads();
    if constexpr (W > 1) {
      a = part[lane % W];
      a = shifted(a, group_max<W>(a.m), p.scale2);
      a.s = group_sum<W>(a.s);
      a.t = group_sum<W>(a.t);
    }
    if (tid == 0) {
      if constexpr (kParts) Record(p, row, part_of).put(a);
      else write_row<T>(p, row, a);
    }
    if (p.top) {
      const RowLn ln(a, log2f(a.s));
      const auto put = [&](int k, uint64_t c) __attribute__((always_inline)) {
        if constexpr (kParts) Record(p, row, part_of).put_top(k, c);
        else write_top(p, row, k, c, ln);
      };
      // at least top values are no less than the top-th of the 64 groups' largest
      const uint32_t key = max(wave_kth(order_key(group[lane]), p.top), kMaskedKey + 1);
      const float bound = order_value(key);
      const auto collect = [&](int q0) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < R; ++i) {
          if (!(unit_max<T>(r[i], kLowest) >= bound)) continue;
          uint32_t on = 0;
#pragma unroll
          for (int j = 0; j < N; ++j) on |= Unit<T>::get(r[i], j) >= bound ? 1u << j : 0u;
          while (on) {                                 // a few units of the row
            const int j = __ffs(on) - 1;
            on &= on - 1;
            const uint32_t at = atomicAdd(&held, 1u);
            if (at < (uint32_t)kHeld) cand[at] = candidate(Unit<T>::get(r[i], j), v.first(q0 + i * TH + tid) + j);
          }
        }
      };
      if (best >= bound) {                             // a thread whose largest is below has none
        if constexpr (kOnePass) collect(begin);
        else
          for (int q0 = begin; q0 < units; q0 += TH * R) {
            load(q0);
            collect(q0);
          }
      }
      __syncthreads();
      const int n = (int)held;
      if (n <= kHeld) {
        for (int i = tid; i < n; i += TH) {
          const uint64_t c = cand[i];
          int rank = 0;
          for (int k = 0; k < n; ++k) rank += cand[k] > c;
          if (rank < p.top) put(rank, c);
        }
        for (int k = n + tid; k < p.top; k += TH) put(k, 0);
      } else {
        // more values at the bound than are held (equal ones, fp32 ones equal in their upper 16 bits): one
        // alternative a pass over the row (4,096 equal rows of 65,536 bf16 logits with 8 of them 735 us, normal ones 108)
        uint64_t last = ~0ull;
        for (int k = 0; k < p.top; ++k) {
          uint64_t c = 0;
          for (int q = begin + tid; q < units; q += TH) {
            const u32x4 u = v.load(q);
#pragma unroll
            for (int j = 0; j < N; ++j) {
              const uint64_t one = candidate(Unit<T>::get(u, j), v.first(q) + j);
              if (one < last && one > c) c = one;
            }
          }
          c = group_first<64>(c);
          __syncthreads();
          if (lane == 0) firsts[wave] = c;
          __syncthreads();
          c = group_first<64>(lane < W ? firsts[lane] : 0);
          if (tid == 0) put(k, c);
          last = c;
        }
      }
    }
    if constexpr (kParts) {
      if (p.ticket) {                                  // one part a workgroup: the last of a row joins it
        __shared__ bool last;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // every wave's records have arrived before the part is counted
        __syncthreads();
        if (tid == 0) {
          uint32_t* counter = p.ticket + (1 + row) * kApart;
          last = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)p.parts - 1;
          if (last) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        __syncthreads();
        if (last && wave == 0) {
          __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
          join_parts<T>(p, row, cand, &held);
        }
      }
    }
    __syncthreads();                                   // the next row's part, group and held
  }
}

// ---- gradient ---------------------------------------------------------------------
struct ChoiceGradArgs {
  const void* x;
  void* dx;
  int64_t rows, stride, dstride;
  int n, top;
  float scale, scale2;
  const int32_t *choice, *top_choice;
  const float *logp, *entropy, *stats, *d_logp, *d_entropy, *d_top;
  int chunks;                      // of a row
};

// Entry i of a row: 0 its choice, 1 .. top its alternatives.  c = -1: takes no part.
__device__ __forceinline__ void grad_entry(const ChoiceGradArgs& p, int64_t row, int i, int& c, float& g) {
  c = -1;
  g = 0.0f;
  if (i == 0) {
    // neither masked nor of a NaN row, which is NaN without it, but for its masked choices
    if (p.d_logp && p.logp[row] > kLowest) c = p.choice[row];
  } else if (p.d_top && i <= p.top) {
    c = p.top_choice[row * p.top + i - 1];
  }
  if (c < 0 || c >= p.n) c = -1;
  else g = i == 0 ? p.d_logp[row] : p.d_top[row * p.top + i - 1];
}

// A unit of N values (one, where the two arrays' rows are not aligned alike) of a row.
struct GradRow {
  float m, ls, a, gh, scale2;      // gh in log2 p's terms
  // p (a - gh ln p)
  __device__ __forceinline__ float at(float x) const {
    const float lp = fmaf(x - m, scale2, -ls);
    return x == kLowest ? 0.0f : fast_exp2(lp) * fmaf(-gh, held_up(lp), a);
  }
};
__device__ __forceinline__ GradRow grad_row(const ChoiceGradArgs& p, int64_t row, float total) {
  GradRow g;
  g.m = p.stats[2 * row];
  g.ls = p.stats[2 * row + 1];
  const float gh = p.d_entropy ? p.d_entropy[row] : 0.0f;
  g.a = -total - (p.d_entropy ? gh * p.entropy[row] : 0.0f);
  g.gh = gh * kLn2;
  g.scale2 = p.scale2;
  return g;
}

// Orders a wave's own accesses of shared memory.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}
template <class T>
__device__ __forceinline__ T rounded(float v) {
  if constexpr (sizeof(T) == 4) return __builtin_bit_cast(T, v);
  else return (T)pk_bf16(v, 0.0f);
}
// L lanes (at most a wave) take a chunk of a row, R units a lane; several rows a wave where they are short.  (Long
// rows by 256 threads and a chunk of 1,024 units each: 65,536 rows of 1,100 fp32 logits with 8 alternatives 290 us,
// 160 by a wave a chunk of 256; 4,096 of 50,001 bf16 ones the same 162.)  The choice and the alternatives are
// added to the value they belong to by the lane that has it, which a table in shared memory tells (each lane
// looking through all of them: 65,536 rows of 256 bf16 logits with 8 alternatives 46 us, 35 so, and 22 by as many
// lanes as they need).  Two units a lane from 8 on, since what is done once a row weighs (500 bf16 logits 44 us
// with one, 39 with two).
// kUnits: 16-byte units, the rows of both arrays being aligned alike; otherwise single values (4,096 rows of 50,257 of
// 50,304 bf16 logits to dense rows 469 us, between dense rows 163; 32,001 of 32,007 fp32 ones 239 and 214).
template <class T, int L, int R, bool kUnits>
__global__ __launch_bounds__(256) void k_choice_grad(ChoiceGradArgs p) {
  constexpr int N = kUnits ? Unit<T>::N : 1, P = 256 / L;
  struct Entry {
    int c;
    float g;
  };
  __shared__ unsigned long long owner[256];          // bit i: the thread has entry i
  __shared__ Entry entry[P][SAGIPS_MAX_TOP + 1];
  const int l = threadIdx.x % L;
  const int64_t all = p.rows * p.chunks;
  for (int64_t id = (int64_t)blockIdx.x * P + threadIdx.x / L; id < all; id += (int64_t)gridDim.x * P) {
    const int64_t row = id / p.chunks;
    const int q0 = (int)(id % p.chunks) * (L * R);
    const RowView<T> v(p.x, row * p.stride, p.n);
    const int lead = kUnits ? v.lead : 0;
    const T* x = (const T*)p.x + row * p.stride;
    T* dx = (T*)p.dx + row * p.dstride;
    float val[R][N];
    u32x4 raw[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int q = q0 + i * L + l;
      if constexpr (kUnits) {
        if (q < v.units()) raw[i] = v.load(q);
      } else {
        raw[i].x = q < p.n ? bits_of(x[q]) : 0u;
      }
    }
    int ec = -1;
    float eg = 0.0f, total = 0.0f;
    owner[threadIdx.x] = 0;
    wave_sync();
    for (int i = l; i <= p.top; i += L) {
      grad_entry(p, row, i, ec, eg);
      total += eg;
      const int q = ec < 0 ? -1 : (ec + lead) / N - q0;
      if (q >= 0 && q < L * R) {
        entry[threadIdx.x / L][i] = Entry{ec, eg};
        atomicOr(&owner[threadIdx.x - l + q % L], 1ull << i);
      }
    }
    total = group_sum<L>(total);
    wave_sync();
    const GradRow g = grad_row(p, row, total);
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        if constexpr (kUnits) val[i][j] = g.at(Unit<T>::get(raw[i], j));
        else if constexpr (sizeof(T) == 4) val[i][j] = g.at(__uint_as_float(raw[i].x));
        else val[i][j] = g.at(__uint_as_float(raw[i].x << 16));
      }
    for (unsigned long long mine = owner[threadIdx.x]; mine; mine &= mine - 1) {
      const Entry e = entry[threadIdx.x / L][__ffsll(mine) - 1];
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const int j0 = e.c - ((q0 + i * L + l) * N - lead);
#pragma unroll
        for (int j = 0; j < N; ++j) val[i][j] += j0 == j ? e.g : 0.0f;
      }
    }
    wave_sync();                                       // the next row's
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int q = q0 + i * L + l;
      const int i0 = q * N - lead;
#pragma unroll
      for (int j = 0; j < N; ++j) val[i][j] *= p.scale;
      if constexpr (kUnits) {
        if (i0 >= 0 && i0 <= p.n - N) {
          u32x4 o;
          if constexpr (sizeof(T) == 4) o = u32x4{__float_as_uint(val[i][0]), __float_as_uint(val[i][1]), __float_as_uint(val[i][2]), __float_as_uint(val[i][3])};
          else o = u32x4{pk_bf16(val[i][0], val[i][1]), pk_bf16(val[i][2], val[i][3]), pk_bf16(val[i][4 % N], val[i][5 % N]), pk_bf16(val[i][6 % N], val[i][7 % N])};
          *reinterpret_cast<u32x4*>(dx + i0) = o;
          continue;
        }
      }
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (i0 + j >= 0 && i0 + j < p.n) dx[i0 + j] = rounded<T>(val[i][j]);
    }
  }
}

template <int n>
using Int = std::integral_constant<int, n>;

// Units a row has at most, wherever it begins.
template <class T>
int64_t most_units(const void* x, int64_t stride, int n) {
  constexpr int N = Unit<T>::N;
  const bool aligned = ((uintptr_t)x & 15) == 0 && stride * sizeof(T) % 16 == 0;
  return ((int64_t)n + (aligned ? N - 1 : 2 * N - 2)) / N;
}

// Rows in parts: where fewer rows than half of the compute units are longer than 32 KiB.  A part has 32 KiB, or
// more where there would be over 64 or over 512 of them in all.  (One row of 131,072 bf16 logits, 20
// alternatives: 16 us by one workgroup, 12 in parts.)
constexpr int kPartUnits = 256 * 8, kPartsMost = 64;
int choice_parts(int64_t rows, int64_t units) {
  if (rows >= 128 || units <= kPartUnits) return 1;
  int64_t n = (units + kPartUnits - 1) / kPartUnits;
  n = n < kPartsMost ? n : kPartsMost;
  return (int)(n < 512 / rows ? n : 512 / rows);
}
int64_t choice_units(const sagips_choices& C) {
  return C.type == SAGIPS_BF16 ? most_units<u16>(C.logits, C.stride, C.n_choices) : most_units<float>(C.logits, C.stride, C.n_choices);
}

template <class T>
hipError_t choice_forward(ChoiceArgs a, int64_t units, hipStream_t st) {
  const auto go_short = [&](auto lanes, auto per) {
    constexpr int L = decltype(lanes)::value, R = decltype(per)::value;
    const int64_t blocks = (a.rows + 256 / L - 1) / (256 / L), most = 1 << 20;
    hipLaunchKernelGGL((k_choice_short<T, L, R>), dim3((unsigned)(blocks < most ? blocks : most)), dim3(256), 0, st, a);
  };
  const auto go_row = [&](auto threads, auto per, auto one) {
    constexpr int TH = decltype(threads)::value, R = decltype(per)::value;
    constexpr bool kOne = decltype(one)::value;
    const int64_t most = 256 * (int64_t)(2048 / TH) * 4;
    hipLaunchKernelGGL((k_choice_row<T, TH, R, kOne, false>), dim3((unsigned)(a.rows < most ? a.rows : most)), dim3(TH), 0, st, a);
  };
  const std::true_type one{};
  // Alternatives up to which rounds cost less than the bound (65,536 rows; us in rounds and by the bound): of 256 fp32
  // logits 6 alternatives 29 and 30, 7 32 and 30, 8 34 and 31; of 500 bf16 ones 10 41 and 43, 11 44 and 44, 12 46 and
  // 44 (of 400 10 39 and 38, 12 43 and 40); of 350 fp32 ones 2 31 and 34, 3 35 and 35; of 1,000 bf16 ones 2 39 and 42,
  // 3 44 and 44, 4 49 and 45.  Rows of up to 32 units have too few groups for a bound of many alternatives (128 fp32 logits:
  // 8 of them 19 and 34, 32 80 and 115).
  const int rounds = units <= 32 ? SAGIPS_MAX_TOP : units <= 64 ? (sizeof(T) == 2 ? 10 : 6) : units <= 128 ? 2 : -1;
  if (a.parts > 1) {
    a.per = (int)((units + a.parts - 1) / a.parts);
    const dim3 grid((unsigned)(a.rows * a.parts));
    if (a.rows > kCounters) a.ticket = nullptr;
    if (a.per <= kPartUnits) hipLaunchKernelGGL((k_choice_row<T, 256, 8, true, true>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_choice_row<T, 1024, 8, false, true>), grid, dim3(1024), 0, st, a);
    if (!a.ticket) {
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
      hipLaunchKernelGGL(k_choice_join<T>, dim3((unsigned)a.rows), dim3(64), 0, st, a);
    }
  } else if (a.top <= rounds) {
    if (units <= 1) go_short(Int<1>{}, Int<1>{});
    else if (units <= 2) go_short(Int<2>{}, Int<1>{});
    else if (units <= 4) go_short(Int<4>{}, Int<1>{});
    else if (units <= 8) go_short(Int<4>{}, Int<2>{});
    else if (units <= 16) go_short(Int<8>{}, Int<2>{});
    else if (units <= 32) go_short(Int<8>{}, Int<4>{});
    else if (units <= 64) go_short(Int<16>{}, Int<4>{});
    else go_short(Int<32>{}, Int<4>{});
  // as many units a thread as are needed, in steps: what lies behind the row is summed too (45,000 bf16 logits with 8
  // units a thread 104 us, with 6 90)
  } else if (units <= 64) go_row(Int<64>{}, Int<1>{}, one);
  else if (units <= 64 * 2) go_row(Int<64>{}, Int<2>{}, one);
  else if (units <= 64 * 4) go_row(Int<64>{}, Int<4>{}, one);
  else if (units <= 64 * 8) go_row(Int<64>{}, Int<8>{}, one);
  else if (units <= 256 * 4) go_row(Int<256>{}, Int<4>{}, one);
  else if (units <= 256 * 6) go_row(Int<256>{}, Int<6>{}, one);
  else if (units <= 256 * 8) go_row(Int<256>{}, Int<8>{}, one);
  else if (units <= 1024 * 4) go_row(Int<1024>{}, Int<4>{}, one);
  else if (units <= 1024 * 6) go_row(Int<1024>{}, Int<6>{}, one);
  else if (units <= 1024 * 8) go_row(Int<1024>{}, Int<8>{}, one);
  else if (units <= 1024 * 16) go_row(Int<1024>{}, Int<16>{}, one);
  else go_row(Int<1024>{}, Int<8>{}, std::false_type{});
  return hipGetLastError();
}

template <class T, bool kUnits>
hipError_t choice_grad(ChoiceGradArgs a, hipStream_t st) {
  const int64_t units = kUnits ? most_units<T>(a.x, a.stride, a.n) : a.n;
  const auto go = [&](auto lanes, auto per) {
    constexpr int L = decltype(lanes)::value, R = decltype(per)::value;
    a.chunks = (int)((units + L * R - 1) / (L * R));
    const int64_t blocks = (a.rows * a.chunks + 256 / L - 1) / (256 / L), most = 1 << 20;
    hipLaunchKernelGGL((k_choice_grad<T, L, R, kUnits>), dim3((unsigned)(blocks < most ? blocks : most)), dim3(256), 0, st, a);
  };
  if (units <= 4) go(Int<4>{}, Int<1>{});
  else if (units <= 8) go(Int<4>{}, Int<2>{});
  else if (units <= 16) go(Int<8>{}, Int<2>{});
  else if (units <= 32) go(Int<16>{}, Int<2>{});
  else if (units <= 64) go(Int<32>{}, Int<2>{});
  else if (units <= 64 * 2) go(Int<32>{}, Int<4>{});
  else if (units <= 64 * 3) go(Int<64>{}, Int<3>{});
  else go(Int<64>{}, Int<4>{});
  return hipGetLastError();
}

}  // namespace

size_t choice_workspace(const sagips_choices& C) {
  const int parts = choice_parts(C.rows, choice_units(C));
  return parts > 1 ? (size_t)C.rows * parts * ((size_t)C.top * 8 + 16) : 0;
}

hipError_t launch_choice(const sagips_choices& C, const int32_t* choice, float* logp, float* entropy, int32_t* top_choice,
                         float* top_logp, float* stats, void* ws, uint32_t* ticket, hipStream_t st, Timer* tm) {
  const int64_t units = choice_units(C);
  const ChoiceArgs a{C.logits, C.rows, C.stride, C.n_choices, C.top, (float)(C.scale * 1.4426950408889634), (float)(2 * C.scale),
                     choice, logp, entropy, top_choice, top_logp, stats, choice_parts(C.rows, units), 0,
                     static_cast<char*>(ws), ticket};
  if (tm) tm->begin("choice_logprob");
  const hipError_t e = C.type == SAGIPS_BF16 ? choice_forward<u16>(a, units, st) : choice_forward<float>(a, units, st);
  if (tm) tm->end();
  return e;
}

hipError_t launch_choice_backward(const sagips_choices& C, const sagips_choice_grads& g, void* dlogits, int64_t dstride,
                                  hipStream_t st, Timer* tm) {
  ChoiceGradArgs a{C.logits, dlogits, C.rows, C.stride, dstride, C.n_choices, g.d_top ? C.top : 0, (float)C.scale, (float)(C.scale * 1.4426950408889634),
                   g.choice, g.top_choice, g.logp, g.entropy, g.stats, g.d_logp, g.d_entropy, g.d_top, 0};
  const int size = C.type == SAGIPS_BF16 ? 2 : 4;
  const bool alike = ((uintptr_t)C.logits - (uintptr_t)dlogits) % 16 == 0 && (C.rows == 1 || (C.stride - dstride) * size % 16 == 0);
  if (tm) tm->begin("choice_backward");
  const hipError_t e = C.type == SAGIPS_BF16 ? (alike ? choice_grad<u16, true>(a, st) : choice_grad<u16, false>(a, st))
                                             : (alike ? choice_grad<float, true>(a, st) : choice_grad<float, false>(a, st));
  if (tm) tm->end();
  return e;
}

}  // namespace sagips
