// The orthogonalised update of weight matrices: Newton-Schulz steps
//   X <- a X + b (X X^T) X + c (X X^T)^2 X
// on X = U / (||U||_F + eps), with U oriented so that its rows are the shorter
// side (n rows of L).  The steps drive every singular value of X towards one
// band around 1 and keep its singular vectors.
//
// Every matrix M (X, X X^T, the polynomial of it) is held as two fp16 terms of 2^12 M,
//   2^12 m = hi + lo,  hi = fp16(2^12 m), lo = fp16(2^12 m - hi),
// each rounded to nearest even: |2^12 m - hi| <= 2^-12 |2^12 m|, and the rest is at most
// 2^-24 of it, half a unit in the last place of fp32, while lo is not subnormal (|m|
// above 6e-5; below, at most 2^-37).  Products of fp16 values are exact in fp32, and of
// the four term products lo lo is at most 2^-24 of the whole, no more than the rounding
// of one fp32 product.  Three products on the fp16 matrix cores into one fp32
// accumulator, smallest first, therefore replace an fp32 product at 16/3 of the rate of
// the fp32 matrix instructions.  fp16 ends at 65,504, so entries must stay below 15.9:
// they do because the singular values do (the entry points bound them from the
// coefficients).
#include <limits.h>

#include "kernels.hpp"
#include "split_bf16.hpp"

namespace sagips {
namespace {

constexpr int kThreads = 256;
constexpr int kT = 2;                          // terms
constexpr float kScale = 4096.0f, kInvScale = 1.0f / 4096.0f;

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef MatrixJob Job;

// The matrices of one launch: tensors of one shape.  Matrix z lies in the tensor
// t with first[t] <= z < first[t + 1].
struct Jobs {
  const void* src[SAGIPS_MAX_TENSORS];   // gradients, or the matrices to orthogonalise
  float* m[SAGIPS_MAX_TENSORS];          // momenta, or NULL
  void* out[SAGIPS_MAX_TENSORS];         // parameters, or the orthogonalised matrices
  int first[SAGIPS_MAX_TENSORS + 1];
  int rows, cols;                        // of every matrix
  int src_bf16, out_bf16;
  float momentum, decay, rate;           // m <- momentum m + g;  p <- decay p - rate X
  int nesterov;
  float a, b, c;
  double eps;
};

// Tensor of matrix z: first[] is INT_MAX past the last tensor.
__device__ __forceinline__ int tensor_of(const int (&first)[SAGIPS_MAX_TENSORS + 1], int z) {
  int t = 0;
#pragma unroll
  for (int k = 1; k < SAGIPS_MAX_TENSORS; ++k) t += z >= first[k];
  return t;
}
__device__ __forceinline__ float load_src(const void* p, int64_t i, int bf16) {
  return bf16 ? bf16_lo(static_cast<const u16*>(p)[i]) : static_cast<const float*>(p)[i];
}
__device__ __forceinline__ u16 to_bf16(float v) { return (u16)pk_bf16(v, 0.0f); }

__device__ __forceinline__ double wave_sum_d(double v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// The terms of scale a and scale b, packed in pairs; scale is a power of two.
__device__ __forceinline__ float f16_lo(uint32_t p) { return (float)__builtin_bit_cast(f16x2, p)[0]; }
__device__ __forceinline__ float f16_hi(uint32_t p) { return (float)__builtin_bit_cast(f16x2, p)[1]; }
__device__ __forceinline__ void split2(float a, float b, float scale, uint32_t& hi, uint32_t& lo) {
  const f16x2 h = {(_Float16)(a * scale), (_Float16)(b * scale)};
  const f16x2 l = {(_Float16)fmaf(a, scale, -(float)h[0]), (_Float16)fmaf(b, scale, -(float)h[1])};   // the fma is exact
  hi = __builtin_bit_cast(uint32_t, h);
  lo = __builtin_bit_cast(uint32_t, l);
}
__device__ __forceinline__ f32x16 mfma16(f16x8 a, f16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f16x8 lds_row(const char* p) { return *reinterpret_cast<const f16x8*>(p); }
// A column of four values for each lane, from rows that 16 lanes address together.
__device__ __forceinline__ f16x8 lds_col2(const char* p, const char* q) {
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)q);
  return __builtin_bit_cast(f16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}
// The LDS accesses of the workgroup so far are done; global loads stay in flight.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// ---- norm -------------------------------------------------------------------------
// The momentum update, and each matrix's sum of squares of U in 64 bits (neither
// large nor small gradients leave its range), in chunks of kChunk elements.
constexpr int64_t kChunk = 4096;
__global__ __launch_bounds__(kThreads) void k_ns_norm(Jobs j, int chunks, double* __restrict__ part) {
  const int z = blockIdx.x / chunks, k = blockIdx.x % chunks;
  const int t = tensor_of(j.first, z);
  const int64_t size = (int64_t)j.rows * j.cols, base = (z - j.first[t]) * size;
  const int64_t e1 = min(size, (k + 1) * kChunk);
  double s = 0.0;
#pragma unroll 4
  for (int64_t e = k * kChunk + threadIdx.x; e < e1; e += kThreads) {
    float u = load_src(j.src[t], base + e, j.src_bf16);
    if (j.m[t]) {
      const float m = fmaf(j.momentum, j.m[t][base + e], u);
      j.m[t][base + e] = m;
      u = j.nesterov ? fmaf(j.momentum, m, u) : m;
    }
    s = fma((double)u, (double)u, s);
  }
  __shared__ double w[kThreads / 64];
  s = wave_sum_d(s);
  if ((threadIdx.x & 63) == 0) w[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) part[blockIdx.x] = w[0] + w[1] + w[2] + w[3];
}

// 1 / (||U||_F + eps) from the chunks' sums, in every thread.
__device__ __forceinline__ float inverse_norm(const double* __restrict__ part, int chunks, double eps) {
  __shared__ double w[kThreads / 64];
  double s = 0.0;
  for (int k = threadIdx.x; k < chunks; k += kThreads) s += part[k];
  s = wave_sum_d(s);
  if ((threadIdx.x & 63) == 0) w[threadIdx.x >> 6] = s;
  __syncthreads();
  return (float)(1.0 / (sqrt(w[0] + w[1] + w[2] + w[3]) + eps));
}

// Layout of a matrix of np x width values (both multiples of 64) in the workspace:
// blocks of 64 rows x 32 columns, row-major, each block its hi terms and then its lo
// terms.  A stage of a product (32 along K) is then whole blocks or half blocks,
// contiguous, whichever way K runs; in plain rows the pieces of a stage lie a power
// of two apart and meet in one memory channel (2,048 x 2,048: 182 us a product so,
// against 41 us of matrix instructions).
constexpr int kBlockRows = 64, kBlockCols = 32, kTermSize = kBlockRows * kBlockCols, kBlockSize = kT * kTermSize;
__device__ __forceinline__ int64_t at_value(int i, int j, int width) {   // of the hi term; lo: kTermSize further
  return ((int64_t)(i / kBlockRows) * (width / kBlockCols) + j / kBlockCols) * kBlockSize + (i % kBlockRows) * kBlockCols +
         j % kBlockCols;
}

// X's terms, zero beyond n x L, in tiles of 64 x 64.
__global__ __launch_bounds__(kThreads) void k_ns_split(Jobs j, int chunks, const double* __restrict__ part,
                                                       u16* __restrict__ X, int np, int lp) {
  __shared__ float tile[64][65];
  const int z = blockIdx.z, t = tensor_of(j.first, z), i0 = blockIdx.y * 64, l0 = blockIdx.x * 64;
  const bool flip = j.rows > j.cols;
  const int64_t base = (int64_t)(z - j.first[t]) * j.rows * j.cols;
  const float inv = inverse_norm(part + (int64_t)z * chunks, chunks, j.eps);
  // read along the source's rows
  const int r0 = flip ? l0 : i0, c0 = flip ? i0 : l0;
#pragma unroll 8
  for (int q = threadIdx.x; q < 4096; q += kThreads) {
    const int r = q >> 6, c = q & 63;
    float u = 0.0f;
    if (r0 + r < j.rows && c0 + c < j.cols) {
      const int64_t e = base + (int64_t)(r0 + r) * j.cols + c0 + c;
      u = j.m[t] && !j.nesterov ? 0.0f : load_src(j.src[t], e, j.src_bf16);
      if (j.m[t]) u = j.nesterov ? fmaf(j.momentum, j.m[t][e], u) : j.m[t][e];
    }
    if (flip) tile[c][r] = u * inv;
    else tile[r][c] = u * inv;
  }
  __syncthreads();
  u16* x = X + (int64_t)z * kT * np * lp;
#pragma unroll
  for (int q = threadIdx.x; q < 512; q += kThreads) {   // 8 values of a row
    const int i = q >> 3, l = (q & 7) * 8;
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int h = 0; h < 4; ++h) split2(tile[i][l + 2 * h], tile[i][l + 2 * h + 1], kScale, hi[h], lo[h]);
    u16* at = x + at_value(i0 + i, l0 + l, lp);
    *reinterpret_cast<uint4*>(at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
    *reinterpret_cast<uint4*>(at + kTermSize) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
  }
}

// ---- products -----------------------------------------------------------------------
enum Mode { kGram, kPoly, kApply, kStore };

struct GemmArgs {
  const u16* P;      // [matrices][np x kp]: rows i of the result, K along a row
  const u16* Q;      // kGram, kPoly: rows j of the result, K along a row; otherwise [kp x width]: K down a column
  const u16* X;      // kApply, kStore: X, as Q; kPoly: P
  u16* out;          // [matrices][np x width]
  int np, kp, width; // padded sizes
  int tiles_i, tiles_j, tiles, per_xcd;   // of all matrices together
};

// One TI x TI tile of the result, 4 waves of (TI / 2)^2.  K in stages of 32 through
// two LDS buffers.
template <int TI>
struct Tile {
  static constexpr int KB = 32;
  static constexpr int ROWB = 2 * KB;                  // bytes of an operand row along K
  static constexpr int PT = TI * ROWB;                 // bytes of one term of an operand tile
  static constexpr int BUF = 2 * kT * PT;              // both operands
  static constexpr int LOADS = BUF / 16 / kThreads;    // 16-byte loads a thread
  static constexpr int WB = TI / 64;                   // 32-blocks a wave has in each direction
};

// Tile of a workgroup.  Workgroups go to the 8 XCDs in turn; each XCD gets a
// contiguous run of tiles, and within a matrix the tiles run through groups of four
// tile rows, so that the run's operands (4 x 8 tiles of 128: 6 MB at 2,048) are
// shared in the XCD's L2.
__device__ __forceinline__ bool tile_of(const GemmArgs& g, int& z, int& ti, int& tj) {
  const int id = (blockIdx.x & 7) * g.per_xcd + (blockIdx.x >> 3);
  if (id >= g.tiles) return false;
  const int per = g.tiles_i * g.tiles_j;
  z = id / per;
  const int t = id - z * per, group = t / (4 * g.tiles_j), i0 = group * 4, rows = min(4, g.tiles_i - i0);
  const int r = t - i0 * g.tiles_j;
  ti = i0 + r % rows;
  tj = r / rows;
  return true;
}

template <int kMode, int TI>
__global__ __launch_bounds__(kThreads, 2) void k_ns_gemm(GemmArgs g, Jobs jobs) {
  typedef Tile<TI> T;
  constexpr bool kDown = kMode == kApply || kMode == kStore;   // Q's K runs down its columns
  constexpr int WB = T::WB;
  __shared__ __attribute__((aligned(16))) char lds[2][T::BUF];
  const int lane = threadIdx.x & 63, lr = lane & 31, lh = lane >> 5;
  const int wave = threadIdx.x >> 6, wi = wave & 1, wj = wave >> 1;
  int z, ti, tj;
  if (!tile_of(g, z, ti, tj)) return;
  const int64_t pp = (int64_t)kT * g.np * g.kp, qp = (int64_t)kT * g.kp * g.width, op = (int64_t)kT * g.np * g.width;

  // A thread's 16-byte pieces of a stage.  K along a row: piece (term, row, unit u of
  // 4), kept at unit u ^ (row / 2 % 4), so that 8 lanes (rows) of a read hit distinct
  // banks.  K down a column: piece (block of 32 columns, term, k, unit u of 4), whose
  // half u / 2 is kept at u / 2 ^ (k / 2 % 2), so that the 4 rows of a transposed
  // read do.
  const u16* from[T::LOADS];
  uint32_t to[T::LOADS];
#pragma unroll
  for (int n = 0; n < T::LOADS; ++n) {
    const bool isQ = n >= T::LOADS / 2;
    const int m = isQ ? n - T::LOADS / 2 : n;
    if (!isQ || !kDown) {
      const int rb = m / 2, term = m % 2, row = rb * kBlockRows + (threadIdx.x >> 2), u = threadIdx.x & 3;
      from[n] = (isQ ? g.Q + z * qp : g.P + z * pp) +
                (int64_t)((isQ ? tj : ti) * (TI / kBlockRows) + rb) * (g.kp / kBlockCols) * kBlockSize + term * kTermSize +
                threadIdx.x * 8;
      to[n] = ((isQ ? kT : 0) + term) * T::PT + row * T::ROWB + ((u ^ ((row >> 1) & 3)) << 4);
    } else {
      const int term = threadIdx.x >> 7, r = threadIdx.x & 127, k = r >> 2, u = r & 3;
      from[n] = g.Q + z * qp + (int64_t)(tj * (TI / kBlockCols) + m) * kBlockSize + term * kTermSize + r * 8;
      to[n] = (kT + term) * T::PT + m * (T::KB * 64) + k * 64 + ((((u >> 1) ^ ((k >> 1) & 1)) << 1 | (u & 1)) << 4);
    }
  }
  u32x4 hold0[T::LOADS], hold1[T::LOADS];
  const int stages = g.kp / T::KB;                     // even: kp is a multiple of 64
  // past the end: the last stage again, into a buffer that is not read any more
  const auto fetch = [&](int k, u32x4 (&h)[T::LOADS]) __attribute__((always_inline)) {
    k = min(k, stages - 1);
    const int64_t along = (int64_t)k * kBlockSize;
    const int64_t down = (int64_t)(k >> 1) * (g.width / kBlockCols) * kBlockSize + (k & 1) * (T::KB * kBlockCols);
#pragma unroll
    for (int n = 0; n < T::LOADS; ++n)
      h[n] = *reinterpret_cast<const u32x4*>(from[n] + (kDown && n >= T::LOADS / 2 ? down : along));
  };
  const auto put = [&](char* buf, const u32x4 (&h)[T::LOADS]) __attribute__((always_inline)) {
#pragma unroll
    for (int n = 0; n < T::LOADS; ++n) *reinterpret_cast<u32x4*>(buf + to[n]) = h[n];
  };
  // A K step's operands: of 16 along K a lane half has 8.
  struct Frag {
    f16x8 p[WB][kT], q[WB][kT];
  };
  const auto read = [&](const char* buf, int ks, Frag& f) __attribute__((always_inline)) {
#pragma unroll
    for (int y = 0; y < WB; ++y) {
      const int row = wi * (TI / 2) + y * 32 + lr;
      const uint32_t at = row * T::ROWB + (((2 * ks + lh) ^ ((row >> 1) & 3)) << 4);
#pragma unroll
      for (int t = 0; t < kT; ++t) f.p[y][t] = lds_row(buf + t * T::PT + at);
    }
#pragma unroll
    for (int x = 0; x < WB; ++x) {
      if constexpr (!kDown) {
        const int row = wj * (TI / 2) + x * 32 + lr;
        const uint32_t at = row * T::ROWB + (((2 * ks + lh) ^ ((row >> 1) & 3)) << 4);
#pragma unroll
        for (int t = 0; t < kT; ++t) f.q[x][t] = lds_row(buf + (kT + t) * T::PT + at);
      } else {
        // 16 lanes read 4 rows of 16 values and get a column of 4 each
        const int i = lane & 15, half = (lane >> 4) & 1;
        const int k0 = 16 * ks + 8 * lh + (i >> 2);    // and k0 + 4: the same k / 2 % 2
        const uint32_t at = (wj * (TI / 64) + x) * (T::KB * 64) + k0 * 64 + ((half ^ ((k0 >> 1) & 1)) << 5) + (i & 3) * 8;
#pragma unroll
        for (int t = 0; t < kT; ++t) {
          const char* b = buf + (kT + t) * T::PT + at;
          f.q[x][t] = lds_col2(b, b + 4 * 64);
        }
      }
    }
  };
  f32x16 c[WB][WB] = {};                               // [block of j][block of i], 2^24 times the product
  const auto multiply = [&](const Frag& f) __attribute__((always_inline)) {
#pragma unroll
    for (int s = 0; s < 3; ++s)
#pragma unroll
      for (int x = 0; x < WB; ++x)
#pragma unroll
        for (int y = 0; y < WB; ++y) c[x][y] = mfma16(f.q[x][s == 1], f.p[y][s == 0], c[x][y]);
  };

  // Stage k's second half reads the first operands of stage k + 1, whose pieces went
  // to LDS during the first half; two more stages are on their way in registers.
  fetch(0, hold0);
  fetch(1, hold1);
  put(lds[0], hold0);
  fetch(2, hold0);
  lds_barrier();
  Frag f0, f1;
  read(lds[0], 0, f0);
  for (int k = 0; k < stages; k += 2) {
    read(lds[0], 1, f1);
    put(lds[1], hold1);
    multiply(f0);
    lds_barrier();
    read(lds[1], 0, f0);
    fetch(k + 3, hold1);
    multiply(f1);

    read(lds[1], 1, f1);
    put(lds[0], hold0);
    multiply(f0);
    lds_barrier();
    read(lds[0], 0, f0);
    fetch(k + 4, hold0);
    multiply(f1);
  }

  // A lane has row i, columns j .. j + 3 of each group.
  const int t = kMode == kStore ? tensor_of(jobs.first, z) : 0;
#pragma unroll
  for (int x = 0; x < WB; ++x)
#pragma unroll
    for (int y = 0; y < WB; ++y)
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const int i = ti * TI + wi * (TI / 2) + y * 32 + lr, j = tj * TI + wj * (TI / 2) + x * 32 + 8 * s + 4 * lh;
        // kGram: 2^24 times the result; otherwise 2^12 times
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = c[x][y][4 * s + e];
        if constexpr (kMode != kGram) {
          const u16* old = g.X + z * op + at_value(i, j, g.width);
          const float keep = kMode == kPoly ? jobs.b : jobs.a, mul = (kMode == kPoly ? jobs.c : 1.0f) * kInvScale;
          const uint2 h = *reinterpret_cast<const uint2*>(old), l = *reinterpret_cast<const uint2*>(old + kTermSize);
          const float o[4] = {f16_lo(l.x) + f16_lo(h.x), f16_hi(l.x) + f16_hi(h.x), f16_lo(l.y) + f16_lo(h.y),
                              f16_hi(l.y) + f16_hi(h.y)};
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = fmaf(keep, o[e], mul * v[e]);
        }
        if constexpr (kMode != kStore) {
          constexpr float scale = kMode == kGram ? kInvScale : 1.0f;
          uint2 h, l;
          split2(v[0], v[1], scale, h.x, l.x);
          split2(v[2], v[3], scale, h.y, l.y);
          u16* out = g.out + z * op + at_value(i, j, g.width);
          *reinterpret_cast<uint2*>(out) = h;
          *reinterpret_cast<uint2*>(out + kTermSize) = l;
        } else {
          const bool flip = jobs.rows > jobs.cols;
          const int64_t base = (int64_t)(z - jobs.first[t]) * jobs.rows * jobs.cols;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int r = flip ? j + e : i, cc = flip ? i : j + e;
            if (r >= jobs.rows || cc >= jobs.cols) continue;
            const int64_t at = base + (int64_t)r * jobs.cols + cc;
            const float o = v[e] * kInvScale;
            if (jobs.m[t]) {
              float* w = static_cast<float*>(jobs.out[t]) + at;
              *w = fmaf(-jobs.rate, o, jobs.decay * *w);
            } else if (jobs.out_bf16) {
              static_cast<u16*>(jobs.out[t])[at] = to_bf16(o);
            } else {
              static_cast<float*>(jobs.out[t])[at] = o;
            }
          }
        }
      }
}

// ---- small matrices -------------------------------------------------------------------
// All steps of one matrix in one workgroup, from the momentum update to the
// parameters, X never leaving registers and LDS: n <= NP and L <= 16384 / NP, for NP
// of 32, 64 and 128.  Wave (rw, cw) of NP / 32 x 128 / NP owns rows 32 rw .. + 31 of X
// and every (128 / NP)-th block of 32 columns, JB of them (the fewest of 1, 2 and 4
// that hold L); lane lr (of half lh) holds row 32 rw + lr, columns 8 g + 4 lh + 0..3 of
// each block, as accumulators do.
//   A = X X^T: the wave forms columns 32 rw .. of A, summed over its own columns of X,
//   whose terms it has in registers; waves of one rw add their sums through LDS.  A is
//   symmetric, so a lane's accumulators are pieces of a row of A, and in the K order
//   (4 lh + 0..3, 8 + 4 lh + 0..3) of every 16 they are the operand of the next
//   products as they stand: A never leaves the registers.
//   Y = A X, then X <- a X + b Y + c A Y: the other operand is X, then Y, read down
//   its columns from LDS in the same K order.
// LDS holds X (or Y) as [term][row][unit of 8 columns]: unit 4 J + 2 s + h of a row has
// columns 32 J + 16 s + 4 h + 0..3 and + 8..11, what one lane half has of a K step, and
// is kept at unit ^ swz(row), so that 8 lanes (rows) of a 16-byte access and the 4 rows
// of a transposed read hit distinct banks.
struct SmallJob {
  const void* src;
  float* m;
  void* out;
  int rows, cols;
  float rate;
};
struct SmallJobs {
  SmallJob job[SAGIPS_MAX_TENSORS];
  int first[SAGIPS_MAX_TENSORS + 1];
  int src_bf16, out_bf16, nesterov, steps;
  float momentum, decay, a, b, c;
  double eps;
};

constexpr int kSmallValues = 16384;                    // NP x LP
constexpr int kSmallBuffer = kSmallValues * kT * 2;    // X's terms, and Y's
constexpr int kQuads = kSmallValues / 4 / kThreads;

// U of a small matrix into its fp32 copy, the momentum on the way; returns the
// thread's sum of squares.  Quads (cols a multiple of 4) have every load in flight.
template <bool kBf16, bool kMom>
__device__ __forceinline__ double small_load(const SmallJobs& jobs, const SmallJob& job, int64_t base, float* flat, int pitch) {
  const int cols = job.cols, size = job.rows * cols;
  const float inv_cols = 1.0f / cols;
  const float* const f32 = static_cast<const float*>(job.src) + base;
  const u16* const b16 = static_cast<const u16*>(job.src) + base;
  float* const mom = kMom ? job.m + base : nullptr;
  double sq = 0.0;
  if (cols % 4 == 0) {
    f32x4 u[kQuads], m[kQuads];
#pragma unroll
    for (int k = 0; k < kQuads; ++k) {
      const int e = (k * kThreads + threadIdx.x) * 4;
      if (e >= size) break;
      if constexpr (kBf16) {
        const uint2 q = *reinterpret_cast<const uint2*>(b16 + e);
        u[k] = f32x4{bf16_lo(q.x), bf16_hi(q.x), bf16_lo(q.y), bf16_hi(q.y)};
      } else {
        u[k] = *reinterpret_cast<const f32x4*>(f32 + e);
      }
      if constexpr (kMom) m[k] = *reinterpret_cast<const f32x4*>(mom + e);
    }
#pragma unroll
    for (int k = 0; k < kQuads; ++k) {
      const int e = (k * kThreads + threadIdx.x) * 4;
      if (e >= size) break;
      f32x4 v = u[k];
      if constexpr (kMom) {
        const f32x4 w = jobs.momentum * m[k] + v;
        *reinterpret_cast<f32x4*>(mom + e) = w;
        v = jobs.nesterov ? jobs.momentum * w + v : w;
      }
      const int r = (int)((e + 0.5f) * inv_cols);      // e < 2^14: exact
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        sq = fma((double)v[q], (double)v[q], sq);
        flat[r * (pitch - cols) + e + q] = v[q];
      }
    }
  } else {
#pragma unroll 4
    for (int e = threadIdx.x; e < size; e += kThreads) {
      const int r = (int)((e + 0.5f) * inv_cols);
      float u = kBf16 ? bf16_lo(b16[e]) : f32[e];
      if constexpr (kMom) {
        const float w = fmaf(jobs.momentum, mom[e], u);
        mom[e] = w;
        u = jobs.nesterov ? fmaf(jobs.momentum, w, u) : w;
      }
      sq = fma((double)u, (double)u, sq);
      flat[r * (pitch - cols) + e] = u;
    }
  }
  return sq;
}

// The result from the fp32 copy: parameters moved, or the matrix written.
template <bool kBf16, bool kMom>
__device__ __forceinline__ void small_store(const SmallJobs& jobs, const SmallJob& job, int64_t base, const float* flat, int pitch) {
  const int cols = job.cols, size = job.rows * cols;
  const float inv_cols = 1.0f / cols;
  float* const f32 = static_cast<float*>(job.out) + base;
  u16* const b16 = static_cast<u16*>(job.out) + base;
  if (cols % 4 == 0) {
    f32x4 old[kQuads];
    if constexpr (kMom)
#pragma unroll
      for (int k = 0; k < kQuads; ++k) {
        const int e = (k * kThreads + threadIdx.x) * 4;
        if (e >= size) break;
        old[k] = *reinterpret_cast<const f32x4*>(f32 + e);
      }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kQuads; ++k) {
      const int e = (k * kThreads + threadIdx.x) * 4;
      if (e >= size) break;
      const int r = (int)((e + 0.5f) * inv_cols);
      f32x4 v;
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = flat[r * (pitch - cols) + e + q];
      if constexpr (kMom) *reinterpret_cast<f32x4*>(f32 + e) = jobs.decay * old[k] - job.rate * v;
      else if constexpr (kBf16) *reinterpret_cast<uint2*>(b16 + e) = make_uint2(pk_bf16(v[0], v[1]), pk_bf16(v[2], v[3]));
      else *reinterpret_cast<f32x4*>(f32 + e) = v;
    }
  } else {
    __syncthreads();
#pragma unroll 4
    for (int e = threadIdx.x; e < size; e += kThreads) {
      const int r = (int)((e + 0.5f) * inv_cols);
      const float v = flat[r * (pitch - cols) + e];
      if constexpr (kMom) f32[e] = fmaf(-job.rate, v, jobs.decay * f32[e]);
      else if constexpr (kBf16) b16[e] = to_bf16(v);
      else f32[e] = v;
    }
  }
}

template <int NP, int JB>
__global__ __launch_bounds__(kThreads, 1) void k_ns_small(SmallJobs jobs) {
  constexpr int LP = kSmallValues / NP;
  constexpr int RW = NP / 32, CW = 4 / RW, NI = NP / 32;
  constexpr int RB = 2 * LP, PL = NP * RB;             // bytes of a row of one term, of a term
  constexpr int IK = 4 / NI, JK = 4 / JB;              // accumulators a block, so that four products run side by side
  // X's terms, then Y's; before the first and after the last step the fp32 copy (rows
  // one value longer if even: 66 KB at most); Y's part also takes the waves' sums for A
  __shared__ __attribute__((aligned(16))) char lds[2 * kSmallBuffer];
  __shared__ double sums[kThreads / 64];
  char* const ldsX = lds;
  char* const ldsY = lds + kSmallBuffer;
  float* const flat = reinterpret_cast<float*>(lds);
  const int lane = threadIdx.x & 63, lr = lane & 31, lh = lane >> 5;
  const int wave = threadIdx.x >> 6, rw = wave % RW, cw = wave / RW;
  const int t = tensor_of(jobs.first, blockIdx.x);
  const SmallJob job = jobs.job[t];
  const int rows = job.rows, cols = job.cols;
  const bool flip = rows > cols;
  const int n = flip ? cols : rows, L = flip ? rows : cols;
  const int64_t base = (int64_t)((int)blockIdx.x - jobs.first[t]) * rows * cols;
  const int pitch = cols | 1;

  double sq;
  if (job.m) sq = jobs.src_bf16 ? small_load<true, true>(jobs, job, base, flat, pitch) : small_load<false, true>(jobs, job, base, flat, pitch);
  else sq = jobs.src_bf16 ? small_load<true, false>(jobs, job, base, flat, pitch) : small_load<false, false>(jobs, job, base, flat, pitch);
  sq = wave_sum_d(sq);
  if (lane == 0) sums[wave] = sq;
  __syncthreads();
  const float inv = (float)(1.0 / (sqrt(sums[0] + sums[1] + sums[2] + sums[3]) + jobs.eps));

  float one = 1.0f;                                    // not a constant to the compiler: a multiplication by it lets
  asm("" : "+s"(one));                                 // fp16 operands go straight into an fp32 fma
  // Terms of 16 values, two units of 8.
  struct Terms {
    f16x8 v[2][kT];
  };
  const auto split = [](const f32x16& v, float scale, Terms& o) __attribute__((always_inline)) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      u32x4 h, l;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        uint32_t a, c;
        split2(v[8 * s + 2 * q], v[8 * s + 2 * q + 1], scale, a, c);
        h[q] = a;
        l[q] = c;
      }
      o.v[s][0] = __builtin_bit_cast(f16x8, h);
      o.v[s][1] = __builtin_bit_cast(f16x8, l);
    }
  };
  const auto swz = [](int f) { return (uint32_t)(2 * (f & 3) + ((f >> 2) & 1)); };
  const int i = 32 * rw + lr;
  const uint32_t own = i * RB, own_swz = swz(i);       // rows 32 ib + lr: the same swizzle
  const auto put = [&](char* buf, int b, const Terms& o) __attribute__((always_inline)) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      char* at = buf + own + (((4 * (b * CW + cw) + 2 * s + lh) ^ own_swz) << 4);
      *reinterpret_cast<f16x8*>(at) = o.v[s][0];
      *reinterpret_cast<f16x8*>(at + PL) = o.v[s][1];
    }
  };

  Terms xt[JB];
  {
    const int pi = flip ? 1 : pitch, pj = flip ? pitch : 1;   // X's (i, j) in the fp32 copy: i pi + j pj
#pragma unroll
    for (int b = 0; b < JB; ++b) {
      f32x16 x;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int j = 32 * (b * CW + cw) + 8 * (r >> 2) + 4 * lh + (r & 3);
        x[r] = i < n && j < L ? flat[i * pi + j * pj] * inv : 0.0f;
      }
      split(x, kScale, xt[b]);
    }
    __syncthreads();
#pragma unroll
    for (int b = 0; b < JB; ++b) put(ldsX, b, xt[b]);
  }

  // A times the wave's blocks of what buf holds; done(b, 2^24 times that of block b).
  const int i16 = lane & 15, half = (lane >> 4) & 1;
  const uint32_t row0 = 4 * lh + (i16 >> 2), swz0 = swz(row0);   // rows 32 ib + 16 s (+ 8) + row0: the same swizzle
  const auto times = [&](const char* buf, const Terms (&A)[NI], auto done) __attribute__((always_inline)) {
    constexpr int kSteps = NI * 2;                     // along K
    f16x8 q[2][JB][kT];
    const auto read = [&](int ks, int y) __attribute__((always_inline)) {   // 16 rows 16 ks .. of block y
      const int unit = 4 * (y * CW + cw) + 2 * half + (i16 & 1);
      const char* p = buf + (16 * ks + row0) * RB + ((unit ^ swz0) << 4) + 8 * (i16 >> 1 & 1);
#pragma unroll
      for (int w = 0; w < kT; ++w) q[ks & 1][y][w] = lds_col2(p + w * PL, p + w * PL + 8 * RB);
    };
#pragma unroll
    for (int y = 0; y < JB; ++y) read(0, y);
    f32x16 c[JB][JK] = {};
    // a step's first products each with the reads of a block of the next step behind it, in this order
#pragma unroll
    for (int ks = 0; ks < kSteps; ++ks)
#pragma unroll
      for (int s = 0; s < 3; ++s)
#pragma unroll
        for (int y = 0; y < JB; ++y) {
          f32x16& o = c[y][(3 * ks + s) % JK];
          o = mfma16(q[ks & 1][y][s == 1], A[ks / 2].v[ks % 2][s == 0], o);
          if (s == 0 && ks + 1 < kSteps) read(ks + 1, y);
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
    for (int y = 0; y < JB; ++y) {
#pragma unroll
      for (int k = 1; k < JK; ++k) c[y][0] += c[y][k];
      done(y, c[y][0]);
    }
  };

  f32x16 x[JB];                                        // 2^12 times X
  for (int step = 0; step < jobs.steps; ++step) {
    lds_barrier();                                     // X is there, Y has been read
    Terms A[NI];
    {
      constexpr int kSteps = JB * 2;
      f16x8 q[2][NI][kT];
      const auto read = [&](int ks, int y) __attribute__((always_inline)) {
#pragma unroll
        for (int w = 0; w < kT; ++w)
          q[ks & 1][y][w] =
              lds_row(ldsX + w * PL + (32 * y + lr) * RB + (((4 * (ks / 2 * CW + cw) + 2 * (ks % 2) + lh) ^ own_swz) << 4));
      };
#pragma unroll
      for (int y = 0; y < NI; ++y) read(0, y);
      f32x16 c[NI][IK] = {};
#pragma unroll
      for (int ks = 0; ks < kSteps; ++ks)
#pragma unroll
        for (int s = 0; s < 3; ++s)
#pragma unroll
          for (int y = 0; y < NI; ++y) {
            f32x16& v = c[y][(3 * ks + s) % IK];
            v = mfma16(q[ks & 1][y][s == 1], xt[ks / 2].v[ks % 2][s == 0], v);
            if (s == 0 && ks + 1 < kSteps) read(ks + 1, y);
            __builtin_amdgcn_sched_barrier(0);
          }
#pragma unroll
      for (int y = 0; y < NI; ++y) {
#pragma unroll
        for (int k = 1; k < IK; ++k) c[y][0] += c[y][k];
        if constexpr (CW == 1) {
          split(c[y][0], kInvScale, A[y]);
        } else {
          float* part = reinterpret_cast<float*>(ldsY) + (wave * NI + y) * 16 * 64 + lane;
#pragma unroll
          for (int r = 0; r < 16; ++r) part[r * 64] = c[y][0][r];
        }
      }
    }
    if constexpr (CW > 1) {
      lds_barrier();
#pragma unroll
      for (int ib = 0; ib < NI; ++ib) {
        f32x16 v = {};
#pragma unroll
        for (int w = 0; w < CW; ++w) {                 // the same order in every wave
          const float* part = reinterpret_cast<const float*>(ldsY) + ((w * RW + rw) * NI + ib) * 16 * 64 + lane;
#pragma unroll
          for (int r = 0; r < 16; ++r) v[r] += part[r * 64];
        }
        split(v, kInvScale, A[ib]);
      }
      lds_barrier();
    }
    times(ldsX, A, [&](int b, const f32x16& y) __attribute__((always_inline)) {
#pragma unroll
      for (int r = 0; r < 16; ++r)                     // 2^12 X from its terms: exact
        x[b][r] = fmaf(jobs.b * kInvScale, y[r], jobs.a * fmaf((float)xt[b].v[r / 8][0][r % 8], one, (float)xt[b].v[r / 8][1][r % 8]));
      split(y, kInvScale, xt[b]);
      put(ldsY, b, xt[b]);
    });
    lds_barrier();                                     // Y is there, X has been read
    times(ldsY, A, [&](int b, const f32x16& y) __attribute__((always_inline)) {
      x[b] += (jobs.c * kInvScale) * y;
      split(x[b], one, xt[b]);
      put(ldsX, b, xt[b]);
    });
  }

  // the result through the fp32 copy, so that the parameters are read and written in order
  lds_barrier();
  const int pi = flip ? 1 : pitch, pj = flip ? pitch : 1;
#pragma unroll
  for (int b = 0; b < JB; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int j = 32 * (b * CW + cw) + 8 * (r >> 2) + 4 * lh + (r & 3);
      if (i < n && j < L) flat[i * pi + j * pj] = x[b][r] * kInvScale;
    }
  if (job.m) small_store<false, true>(jobs, job, base, flat, pitch);
  else if (jobs.out_bf16) small_store<true, false>(jobs, job, base, flat, pitch);
  else small_store<false, false>(jobs, job, base, flat, pitch);
}

// The workgroup that holds a matrix, as 3 (log2 NP - 5) + log2 JB; -1: none does.
constexpr int kSmallClasses = 9;
int small_class(int rows, int cols) {
  const int n = rows < cols ? rows : cols, L = rows < cols ? cols : rows;
  for (int p = 0; p < 3; ++p)
    for (int b = 0; b < 3 && n <= 32 << p; ++b)
      if (L <= ((32 << b) * 4 >> p)) return 3 * p + b;   // 32 JB columns a wave, 4 / 2^p waves
  return -1;
}
template <int P, int B>
void small_kernel(const SmallJobs& j, hipStream_t st) {
  hipLaunchKernelGGL((k_ns_small<(32 << P), (1 << B)>), dim3(j.first[SAGIPS_MAX_TENSORS]), dim3(kThreads), 0, st, j);
}

// ---- plan ---------------------------------------------------------------------------
int64_t round_up(int64_t n, int64_t m) { return (n + m - 1) / m * m; }
size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

struct Plan {
  int n, L, np, lp, tile, chunks, mats;
  size_t x0, x1, A, B, bytes;   // offsets; the partial sums come first
};
// Tiles of 128 where they alone occupy the device, of 64 otherwise.
constexpr int kManyTiles = 192;
Plan plan_of(int rows, int cols, int mats) {
  Plan p;
  p.n = rows < cols ? rows : cols;
  p.L = rows < cols ? cols : rows;
  p.mats = mats;
  p.tile = round_up(p.n, 128) / 128 * (round_up(p.n, 128) / 128) * mats >= kManyTiles ? 128 : 64;
  p.np = (int)round_up(p.n, p.tile);
  p.lp = (int)round_up(p.L, p.tile);
  p.chunks = (int)(((int64_t)rows * cols + kChunk - 1) / kChunk);
  const size_t part = align256((size_t)mats * p.chunks * sizeof(double));
  const size_t x = align256((size_t)mats * kT * p.np * p.lp * 2), a = align256((size_t)mats * kT * p.np * p.np * 2);
  p.x0 = part;
  p.x1 = p.x0 + x;
  p.A = p.x1 + x;
  p.B = p.A + a;
  p.bytes = p.B + a;
  return p;
}

template <int kMode, int TI>
void gemm(GemmArgs g, const Jobs& j, int mats, hipStream_t st) {
  g.tiles_i = g.np / TI;
  g.tiles_j = g.width / TI;
  g.tiles = g.tiles_i * g.tiles_j * mats;
  g.per_xcd = (g.tiles + 7) / 8;
  hipLaunchKernelGGL((k_ns_gemm<kMode, TI>), dim3(8 * g.per_xcd), dim3(kThreads), 0, st, g, j);
}

template <int TI>
hipError_t steps_of(const Plan& p, const Jobs& j, int steps, char* ws, hipStream_t st, Timer* tm) {
  double* part = reinterpret_cast<double*>(ws);
  u16 *x0 = reinterpret_cast<u16*>(ws + p.x0), *x1 = reinterpret_cast<u16*>(ws + p.x1);
  u16 *A = reinterpret_cast<u16*>(ws + p.A), *B = reinterpret_cast<u16*>(ws + p.B);
  if (tm) tm->begin("ns_norm");
  hipLaunchKernelGGL(k_ns_norm, dim3((unsigned)p.mats * p.chunks), dim3(kThreads), 0, st, j, p.chunks, part);
  if (tm) tm->end();
  if (tm) tm->begin("ns_split");
  hipLaunchKernelGGL(k_ns_split, dim3(p.lp / 64, p.np / 64, p.mats), dim3(kThreads), 0, st, j, p.chunks, part, x0, p.np,
                     p.lp);
  if (tm) tm->end();
  for (int s = 0; s < steps; ++s) {
    if (tm) tm->begin("ns_gram");
    gemm<kGram, TI>(GemmArgs{x0, x0, nullptr, A, p.np, p.lp, p.np}, j, p.mats, st);
    if (tm) tm->end();
    if (tm) tm->begin("ns_poly");
    gemm<kPoly, TI>(GemmArgs{A, A, A, B, p.np, p.np, p.np}, j, p.mats, st);
    if (tm) tm->end();
    if (tm) tm->begin("ns_apply");
    const GemmArgs g{B, x0, x0, x1, p.np, p.np, p.lp};
    if (s + 1 < steps) gemm<kApply, TI>(g, j, p.mats, st);
    else gemm<kStore, TI>(g, j, p.mats, st);
    if (tm) tm->end();
    u16* t = x0;
    x0 = x1;
    x1 = t;
  }
  return hipGetLastError();
}

}  // namespace

// Tensors of one shape go through their launches together; the shapes one after
// the other, in the same workspace.
template <class F>
static hipError_t for_each_shape(const MatrixJobs& js, F&& f) {
  bool done[SAGIPS_MAX_TENSORS] = {};
  for (int i = 0; i < js.n_jobs; ++i) {
    if (done[i] || small_class(js.job[i].rows, js.job[i].cols) >= 0) continue;
    int list[SAGIPS_MAX_TENSORS], n = 0;
    for (int k = i; k < js.n_jobs; ++k)
      if (!done[k] && js.job[k].rows == js.job[i].rows && js.job[k].cols == js.job[i].cols) {
        done[k] = true;
        list[n++] = k;
      }
    hipError_t e = f(list, n);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

static int total_of(const MatrixJobs& js, const int* list, int n) {
  int64_t mats = 0;
  for (int k = 0; k < n; ++k) mats += js.job[list[k]].count;
  return (int)mats;
}

size_t muon_workspace(const MatrixJobs& js) {
  size_t most = 0;
  (void)for_each_shape(js, [&](const int* list, int n) {
    const Job& a = js.job[list[0]];
    const size_t b = plan_of(a.rows, a.cols, total_of(js, list, n)).bytes;
    most = b > most ? b : most;
    return hipSuccess;
  });
  return most;
}

static hipError_t launch_small(const MatrixJobs& js, int which, hipStream_t st, Timer* tm) {
  SmallJobs j{};
  int n = 0, total = 0;
  for (int k = 0; k < js.n_jobs; ++k) {
    const Job& q = js.job[k];
    if (small_class(q.rows, q.cols) != which) continue;
    j.job[n] = SmallJob{q.src, q.m, q.out, q.rows, q.cols, (float)(js.lr * q.scale)};
    j.first[n++] = total;
    total += q.count;
  }
  if (!n) return hipSuccess;
  for (int k = n; k < SAGIPS_MAX_TENSORS; ++k) j.first[k] = INT_MAX;
  j.first[SAGIPS_MAX_TENSORS] = total;
  j.src_bf16 = js.src_bf16;
  j.out_bf16 = js.out_bf16;
  j.nesterov = js.nesterov;
  j.steps = js.steps;
  j.momentum = js.momentum;
  j.decay = js.decay;
  j.a = js.coef[0];
  j.b = js.coef[1];
  j.c = js.coef[2];
  j.eps = js.eps;
  if (tm) tm->begin("ns_small");
  switch (which) {
    case 0: small_kernel<0, 0>(j, st); break;
    case 1: small_kernel<0, 1>(j, st); break;
    case 2: small_kernel<0, 2>(j, st); break;
    case 3: small_kernel<1, 0>(j, st); break;
    case 4: small_kernel<1, 1>(j, st); break;
    case 5: small_kernel<1, 2>(j, st); break;
    case 6: small_kernel<2, 0>(j, st); break;
    case 7: small_kernel<2, 1>(j, st); break;
    default: small_kernel<2, 2>(j, st); break;
  }
  if (tm) tm->end();
  return hipGetLastError();
}

hipError_t launch_muon(const MatrixJobs& js, void* ws, hipStream_t st, Timer* tm) {
  for (int which = 0; which < kSmallClasses; ++which) {
    const hipError_t e = launch_small(js, which, st, tm);
    if (e != hipSuccess) return e;
  }
  return for_each_shape(js, [&](const int* list, int n) {
    const Job& a = js.job[list[0]];
    Jobs j{};
    int total = 0;
    for (int k = 0; k < n; ++k) {
      const Job& q = js.job[list[k]];
      j.src[k] = q.src;
      j.m[k] = q.m;
      j.out[k] = q.out;
      j.first[k] = total;
      total += q.count;
    }
    for (int k = n; k <= SAGIPS_MAX_TENSORS; ++k) j.first[k] = INT_MAX;
    j.rows = a.rows;
    j.cols = a.cols;
    j.src_bf16 = js.src_bf16;
    j.out_bf16 = js.out_bf16;
    j.momentum = js.momentum;
    j.decay = js.decay;
    j.rate = (float)(js.lr * a.scale);
    j.nesterov = js.nesterov;
    j.a = js.coef[0];
    j.b = js.coef[1];
    j.c = js.coef[2];
    j.eps = js.eps;
    const Plan p = plan_of(a.rows, a.cols, total);
    char* w = static_cast<char*>(ws);
    return p.tile == 128 ? steps_of<128>(p, j, js.steps, w, st, tm) : steps_of<64>(p, j, js.steps, w, st, tm);
  });
}

}  // namespace sagips
