// Rows sorted by the member that they are given to, and back.
//   route     a stable counting sort of rows * slots items by member: offsets, the
//             item at each sorted position, and each item's position
//   dispatch  sorted[place[r][k]] = x[r]
//   combine   out[r] = sum_k w[r][k] y[place[r][k]], and its gradient
// Positions outside the sorted rows are never followed.
#include "device_math.hpp"
#include "kernels.hpp"
#include "split_bf16.hpp"

#include <type_traits>

namespace sagips {
namespace {

// ---- route ------------------------------------------------------------------------
// A workgroup of 16 waves takes `per` items, wave w the w-th part of them in order.  A
// wave counts its members in LDS, then walks its items again: an item's position is
// the member's first of the wave, plus the lanes before it with the same member (a ballot a
// bit of the member).  Beyond one workgroup the counts come from a launch before.
constexpr int kRouteThreads = 1024, kRouteWaves = 16, kRouteMembers = 1024;

struct RouteArgs {
  const int32_t* member;
  int n, members, per;
  int bits;                        // of members - 1
  int32_t *offsets, *order, *place;
  uint32_t* counts;                // [workgroups][members]
};

// Lanes with the same m as this one (of those that are on).
__device__ __forceinline__ uint64_t same_lanes(uint32_t m, bool on, int bits) {
  uint64_t peers = __ballot(on);
  for (int b = 0; b < bits; ++b) {
    const bool set = m >> b & 1;
    const uint64_t with = __ballot(set);
    peers &= set ? with : ~with;
  }
  return peers;
}

struct WaveItems {
  int lo, hi;                      // of the wave
};
__device__ __forceinline__ WaveItems wave_items(const RouteArgs& p, int block, int wave) {
  const int64_t b0 = (int64_t)block * p.per, b1 = min(b0 + p.per, (int64_t)p.n);
  const int each = (p.per + kRouteWaves * 64 - 1) / (kRouteWaves * 64) * 64;
  const int64_t lo = min(b0 + (int64_t)wave * each, b1), hi = min(lo + each, b1);
  return {(int)lo, (int)hi};
}

// counts[wave][m] of the workgroup's items; all zero before.
__device__ __forceinline__ void count_items(const RouteArgs& p, const WaveItems& w, uint32_t* counts) {
  for (int i = w.lo + (int)(threadIdx.x & 63); i < w.hi; i += 64) {
    const uint32_t m = (uint32_t)p.member[i];
    if (m < (uint32_t)p.members) atomicAdd(counts + m, 1u);
  }
}

__global__ __launch_bounds__(kRouteThreads) void k_route_count(RouteArgs p) {
  __shared__ uint32_t counts[kRouteMembers];
  for (int m = threadIdx.x; m < p.members; m += kRouteThreads) counts[m] = 0;
  __syncthreads();
  count_items(p, wave_items(p, blockIdx.x, threadIdx.x >> 6), counts);
  __syncthreads();
  for (int m = threadIdx.x; m < p.members; m += kRouteThreads) p.counts[(int64_t)blockIdx.x * p.members + m] = counts[m];
}

__global__ __launch_bounds__(kRouteThreads) void k_route_place(RouteArgs p) {
  __shared__ uint32_t next[kRouteWaves * kRouteMembers];   // [wave][members]: the next position
  __shared__ uint32_t sums[kRouteWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const bool alone = gridDim.x == 1;
  for (int i = tid; i < kRouteWaves * p.members; i += kRouteThreads) next[i] = 0;
  __syncthreads();
  const WaveItems w = wave_items(p, blockIdx.x, wave);
  count_items(p, w, next + wave * p.members);
  __syncthreads();
  // thread m: member m's items in the workgroups before, in all, and in this one's waves
  uint32_t before = 0, total = 0;
  if (tid < p.members) {
    if (alone) {
      for (int v = 0; v < kRouteWaves; ++v) total += next[v * p.members + tid];
    } else {
#pragma unroll 8
      for (int b = 0; b < (int)gridDim.x; ++b) {
        const uint32_t c = p.counts[(int64_t)b * p.members + tid];
        total += c;
        before += b < (int)blockIdx.x ? c : 0u;
      }
    }
  }
  uint32_t upto = total;                             // members 0 .. tid: in the wave, then over the waves
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t o = (uint32_t)__shfl_up((int)upto, d, 64);
    if (lane >= d) upto += o;
  }
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  uint32_t all = 0;
#pragma unroll
  for (int v = 0; v < kRouteWaves; ++v) {
    upto += v < wave ? sums[v] : 0u;
    all += sums[v];
  }
  if (tid < p.members) {
    uint32_t at = upto - total;
    if (blockIdx.x == 0) {
      p.offsets[tid] = (int32_t)at;
      if (tid == p.members - 1) p.offsets[p.members] = (int32_t)upto;
    }
    at += before;
    for (int v = 0; v < kRouteWaves; ++v) {
      const uint32_t c = next[v * p.members + tid];
      next[v * p.members + tid] = at;
      at += c;
    }
  }
  __syncthreads();
  uint32_t* mine = next + wave * p.members;
  for (int i0 = w.lo; i0 < w.hi; i0 += 64) {
    const int i = i0 + lane;
    const uint32_t m = i < w.hi ? (uint32_t)p.member[i] : 0xffffffffu;
    const bool on = m < (uint32_t)p.members;
    const uint64_t peers = same_lanes(m, on, p.bits);
    int32_t at = -1;
    if (on) {
      at = (int32_t)(mine[m] + (uint32_t)__popcll(peers & ((1ull << lane) - 1)));
      if (at < p.n) p.order[at] = i;                 // always, unless the members change under the call
    }
    // the wave's own counters: its reads before the write, the write before the next reads
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (on && lane == 63 - __builtin_clzll(peers)) mine[m] = (uint32_t)at + 1;   // the last of them
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (i < w.hi) p.place[i] = at;
  }
  // behind the last position; every workgroup a part
  for (int64_t i = (int64_t)all + (int64_t)blockIdx.x * kRouteThreads + tid; i < p.n; i += (int64_t)gridDim.x * kRouteThreads)
    p.order[i] = -1;
}

// ---- rows -------------------------------------------------------------------------
// A row is taken in pieces of 16 bytes, wherever it begins (rows of odd widths begin on any value, and the memory
// takes such reads and writes whole: for 16,384 x 8 rows of 333 bf16 values dispatch took 38 us in single values
// and takes 20 so, combine 73 and 23, its backward 73 and 42), and the values behind the last whole piece one by
// one.  Both go through one loop: with a loop of their own behind it the single values waited for a second round
// trip (combine 34 us, backward 59).  2^lx lanes of a workgroup take a row, several rows a workgroup where they
// are short.
struct RowsArgs {
  const int32_t* place;
  int64_t rows, items;
  int slots, width, lx;
  const void *x, *y;
  const float* weight;
  void *out, *dy;
  float* dweight;
};

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_by2 __attribute__((aligned(2)));
typedef u32x4 u32x4_by4 __attribute__((aligned(4)));
template <class T>
struct Piece {
  static constexpr int N = 16 / sizeof(T);
  typedef std::conditional_t<sizeof(T) == 4, uint32_t, u16> One;
  typedef std::conditional_t<sizeof(T) == 4, u32x4_by4, u32x4_by2> Loose;
  // A single value stands first, with zeros behind it.
  static __device__ __forceinline__ u32x4 load(const T* at, bool whole) {
    u32x4 r = {0, 0, 0, 0};
    if (whole) r = *reinterpret_cast<const Loose*>(at);
    else r.x = *reinterpret_cast<const One*>(at);
    return r;
  }
  static __device__ __forceinline__ void store(T* at, bool whole, u32x4 v) {
    if (whole) *reinterpret_cast<Loose*>(at) = v;
    else *reinterpret_cast<One*>(at) = (One)v.x;
  }
  static __device__ __forceinline__ float get(u32x4 r, int j) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(r[j]);
    else return j & 1 ? bf16_hi(r[j >> 1]) : bf16_lo(r[j >> 1]);
  }
  static __device__ __forceinline__ u32x4 make(const float (&v)[N]) {
    if constexpr (sizeof(T) == 4) return u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    else return u32x4{pk_bf16(v[0], v[1]), pk_bf16(v[2], v[3]), pk_bf16(v[4 % N], v[5 % N]), pk_bf16(v[6 % N], v[7 % N])};
  }
};

constexpr int kRowThreads = 256;
constexpr int kAtOnce = 8;         // items of a row whose reads are in flight together

// Where value v of the row at a position lies.  The position is opaque, so that the addresses of all items are not
// formed before the loop over a row and kept in registers (kLoop; combine's backward, 65,536 rows of 1,000 fp32
// values: 183 us with them, 169 so).
template <bool kLoop, class T>
__device__ __forceinline__ T* item_at(T* base, int32_t position, int width, int v) {
  if constexpr (kLoop) asm volatile("" : "+v"(position));
  return base + (int64_t)position * width + v;
}

// What a thread does of a row: f(first value, whole) for its pieces, the whole ones first.  kWhole: there are no others
// (combine of 16,384 x 8 rows of 2,048 bf16 values: 146 us with the branches about single values, 140 without).
template <class T, bool kWhole, class F>
__device__ __forceinline__ void over_pieces(const RowsArgs& p, F f) {
  constexpr int N = Piece<T>::N;
  const int full = p.width / N, step = 1 << p.lx, u0 = threadIdx.x & (step - 1);
  if constexpr (kWhole) {
    for (int u = u0; u < full; u += step) f(u * N, std::true_type{});
  } else {
    const int all = full + p.width % N;
    for (int u = u0; u < all; u += step) f(u < full ? u * N : full * N + (u - full), u < full);
  }
}

template <class T, bool kWhole>
__global__ __launch_bounds__(kRowThreads) void k_dispatch(RowsArgs p) {
  typedef Piece<T> P;
  const int per = kRowThreads >> p.lx;
  for (int64_t row = (int64_t)blockIdx.x * per + (threadIdx.x >> p.lx); row < p.rows; row += (int64_t)gridDim.x * per) {
    const int32_t* place = p.place + row * p.slots;
    over_pieces<T, kWhole>(p, [&](int v, auto whole) __attribute__((always_inline)) {
      const u32x4 raw = P::load((const T*)p.x + row * p.width + v, whole);
      for (int k = 0; k < p.slots; ++k) {
        const int64_t at = place[k];
        if (at >= 0 && at < p.items) P::store((T*)p.out + at * p.width + v, whole, raw);
      }
    });
  }
}

template <class T, bool kWhole>
__global__ __launch_bounds__(kRowThreads) void k_combine(RowsArgs p) {
  typedef Piece<T> P;
  const int per = kRowThreads >> p.lx;
  for (int64_t row = (int64_t)blockIdx.x * per + (threadIdx.x >> p.lx); row < p.rows; row += (int64_t)gridDim.x * per) {
    const int32_t* place = p.place + row * p.slots;
    const float* weight = p.weight ? p.weight + row * p.slots : nullptr;
    over_pieces<T, kWhole>(p, [&](int v, auto whole) __attribute__((always_inline)) {
      float s[P::N] = {};
      for (int k0 = 0; k0 < p.slots; k0 += kAtOnce) {
        u32x4 y[kAtOnce];
        float w[kAtOnce];
        bool on[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
          const int32_t at = k0 + i < p.slots ? place[k0 + i] : -1;
          on[i] = at >= 0 && at < p.items;
          if (on[i]) {
            y[i] = P::load(item_at<!kWhole>((const T*)p.y, at, p.width, v), whole);
            w[i] = weight ? weight[k0 + i] : 1.0f;
          }
        }
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i)
          if (on[i])
#pragma unroll
            for (int j = 0; j < P::N; ++j) s[j] = fmaf(w[i], P::get(y[i], j), s[j]);
      }
      P::store((T*)p.out + row * p.width + v, whole, P::make(s));
    });
  }
}

// 2^lx lanes take a row: at most a wave (then <dout, y> needs no exchange between waves), or the workgroup.
template <class T, bool kWhole>
__global__ __launch_bounds__(kRowThreads) void k_combine_grad(RowsArgs p) {
  typedef Piece<T> P;
  __shared__ float part[kRowThreads / 64][kAtOnce];
  const int l = threadIdx.x & ((1 << p.lx) - 1), step = 1 << p.lx, per = kRowThreads >> p.lx;
  for (int64_t row = (int64_t)blockIdx.x * per + (threadIdx.x >> p.lx); row < p.rows; row += (int64_t)gridDim.x * per) {
    const int32_t* place = p.place + row * p.slots;
    for (int k0 = 0; k0 < p.slots; k0 += kAtOnce) {
      float dot[kAtOnce] = {}, w[kAtOnce];
      int32_t at[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        at[i] = k0 + i < p.slots ? place[k0 + i] : -1;
        if (at[i] >= p.items) at[i] = -1;
        w[i] = p.weight && k0 + i < p.slots ? p.weight[row * p.slots + k0 + i] : 1.0f;
      }
      over_pieces<T, kWhole>(p, [&](int v, auto whole) __attribute__((always_inline)) {
        const u32x4 g = P::load((const T*)p.x + row * p.width + v, whole);
        u32x4 y[kAtOnce];
        if (p.dweight) {
#pragma unroll
          for (int i = 0; i < kAtOnce; ++i)
            if (at[i] >= 0) y[i] = P::load(item_at<true>((const T*)p.y, at[i], p.width, v), whole);
        }
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
          if (at[i] < 0) continue;
          if (p.dy) {
            float o[P::N];
#pragma unroll
            for (int j = 0; j < P::N; ++j) o[j] = w[i] * P::get(g, j);
            P::store(item_at<true>((T*)p.dy, at[i], p.width, v), whole, P::make(o));
          }
          if (p.dweight)
#pragma unroll
            for (int j = 0; j < P::N; ++j)           // (zeros behind a single value, in both)
              dot[i] = fmaf(P::get(g, j), P::get(y[i], j), dot[i]);
        }
      });
      if (p.dweight) {
        if (step < kAtOnce) {
#pragma unroll
          for (int i = 0; i < kAtOnce; ++i) {
            for (int d = 1; d < step; d <<= 1) dot[i] += __shfl_xor(dot[i], d, 64);
            if (l == 0 && k0 + i < p.slots) p.dweight[row * p.slots + k0 + i] = dot[i];
          }
        } else {
          // the lanes of a pair halve the items between them, three times, and each adds up one item's
#pragma unroll
          for (int h = kAtOnce / 2, d = 1; h; h >>= 1, d <<= 1) {
            const bool up = l & d;
#pragma unroll
            for (int i = 0; i < h; ++i) dot[i] = (up ? dot[i + h] : dot[i]) + __shfl_xor(up ? dot[i] : dot[i + h], d, 64);
          }
          for (int d = kAtOnce; d < min(step, 64); d <<= 1) dot[0] += __shfl_xor(dot[0], d, 64);
          const int i = (l & 1) << 2 | (l & 2) | (l & 4) >> 2;       // the lane's item
          if (step > 64) {                             // the workgroup's only row
            if ((l & 63) < kAtOnce) part[l >> 6][i] = dot[0];
            __syncthreads();
            if (l < kAtOnce && k0 + l < p.slots)
              p.dweight[row * p.slots + k0 + l] = (part[0][l] + part[1][l]) + (part[2][l] + part[3][l]);
            __syncthreads();
          } else if (l < kAtOnce && k0 + i < p.slots) {
            p.dweight[row * p.slots + k0 + i] = dot[0];
          }
        }
      }
    }
  }
}

// Items a workgroup sorts: one workgroup up to 16,384; at most 256 workgroups.
int route_per(int64_t n) {
  if (n <= 16384) return (int)((n + kRouteThreads - 1) / kRouteThreads * kRouteThreads);
  const int64_t per = (n + 255) / 256;
  return (int)((per < 4096 ? 4096 : per + kRouteThreads - 1) / kRouteThreads * kRouteThreads);
}
int route_blocks(int64_t n) { return (int)((n + route_per(n) - 1) / route_per(n)); }

int pieces_of(const sagips_routed& R) {
  const int n = R.type == SAGIPS_BF16 ? 8 : 4;
  return R.width / n + R.width % n;
}
RowsArgs rows_args(const sagips_routed& R) {
  RowsArgs a{};
  a.place = R.place;
  a.rows = R.rows;
  a.items = R.rows * R.slots;
  a.slots = R.slots;
  a.width = R.width;
  while (a.lx < 8 && (1 << a.lx) < pieces_of(R)) ++a.lx;
  return a;
}
typedef void (*RowsKernel)(RowsArgs);
// kernels[bf16][every piece of a row is whole]
void go_rows(const sagips_routed& R, const RowsArgs& a, const RowsKernel (&kernels)[2][2], hipStream_t st) {
  const bool bf16 = R.type == SAGIPS_BF16;
  const int64_t per = kRowThreads >> a.lx, blocks = (a.rows + per - 1) / per, most = 1 << 20;
  hipLaunchKernelGGL(kernels[bf16][R.width % (bf16 ? 8 : 4) == 0], dim3((unsigned)(blocks < most ? blocks : most)), dim3(kRowThreads), 0, st, a);
}

}  // namespace

size_t route_workspace(int64_t n, int members) {
  const int blocks = route_blocks(n);
  return blocks == 1 ? 0 : sizeof(uint32_t) * (size_t)blocks * members;
}

hipError_t launch_route(const int32_t* member, int64_t n, int members, int32_t* offsets, int32_t* order, int32_t* place,
                        void* ws, hipStream_t st, Timer* tm) {
  RouteArgs a{member, (int)n, members, route_per(n), 0, offsets, order, place, static_cast<uint32_t*>(ws)};
  while ((1 << a.bits) < members) ++a.bits;
  const int blocks = route_blocks(n);
  if (blocks > 1) {
    if (tm) tm->begin("route_count");
    hipLaunchKernelGGL(k_route_count, dim3(blocks), dim3(kRouteThreads), 0, st, a);
    if (tm) tm->end();
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (tm) tm->begin("route_place");
  hipLaunchKernelGGL(k_route_place, dim3(blocks), dim3(kRouteThreads), 0, st, a);
  if (tm) tm->end();
  return hipGetLastError();
}

hipError_t launch_dispatch(const sagips_routed& R, const void* x, void* sorted, hipStream_t st, Timer* tm) {
  RowsArgs a = rows_args(R);
  a.x = x;
  a.out = sorted;
  if (tm) tm->begin("dispatch");
  static const RowsKernel kernels[2][2] = {{k_dispatch<float, false>, k_dispatch<float, true>}, {k_dispatch<u16, false>, k_dispatch<u16, true>}};
  go_rows(R, a, kernels, st);
  if (tm) tm->end();
  return hipGetLastError();
}

hipError_t launch_combine(const sagips_routed& R, const void* y, const float* weight, void* out, hipStream_t st, Timer* tm) {
  RowsArgs a = rows_args(R);
  a.y = y;
  a.weight = weight;
  a.out = out;
  if (tm) tm->begin("combine");
  static const RowsKernel kernels[2][2] = {{k_combine<float, false>, k_combine<float, true>}, {k_combine<u16, false>, k_combine<u16, true>}};
  go_rows(R, a, kernels, st);
  if (tm) tm->end();
  return hipGetLastError();
}

hipError_t launch_combine_backward(const sagips_routed& R, const void* dout, const void* y, const float* weight, void* dy,
                                   float* dweight, hipStream_t st, Timer* tm) {
  RowsArgs a = rows_args(R);
  // A row by a workgroup where rows are few or its pieces of all items many, by a wave otherwise (8 slots of 8,192
  // bf16 values: 300 rows 51 us by a wave each and 21 so; 16,384 rows of 8 slots of 2,048 bf16 values 244 and
  // 208, of 4 slots 119 and 113, 65,536 rows of 1 slot of 1,000 fp32 values 159 and 241).
  const int64_t pieces = (int64_t)pieces_of(R) * (R.slots < kAtOnce ? R.slots : kAtOnce);
  if (a.lx > 6) a.lx = R.rows < 2048 || pieces >= 1024 ? 8 : 6;
  a.x = dout;
  a.y = y;
  a.weight = weight;
  a.dy = dy;
  a.dweight = dweight;
  if (tm) tm->begin("combine_backward");
  static const RowsKernel kernels[2][2] = {{k_combine_grad<float, false>, k_combine_grad<float, true>}, {k_combine_grad<u16, false>, k_combine_grad<u16, true>}};
  go_rows(R, a, kernels, st);
  if (tm) tm->end();
  return hipGetLastError();
}

}  // namespace sagips
