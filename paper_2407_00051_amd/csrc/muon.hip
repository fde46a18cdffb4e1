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
// above 6e-5; below, at most 2^-37: X is held up by a power of two while it is small).
// Products of fp16 values are exact in fp32, and of the four term products lo lo is at
// most 2^-24 of the whole, no more than the rounding of one fp32 product.  Three products on the fp16 matrix cores into one fp32
// accumulator, smallest first, therefore replace an fp32 product at 16/3 of the rate of
// the fp32 matrix instructions.  fp16 ends at 65,504, so entries must stay below 15.9:
// they do because the singular values do (the entry points bound them from the
// coefficients).  A X, which the small matrices' kernel forms, has their cubes, up to
// 59.4, and is held as 2^10 times it.
#include <limits.h>

#include "kernels.hpp"
#include "split_bf16.hpp"

namespace sagips {
namespace {

constexpr int kThreads = 256;
constexpr int kT = 2;                          // terms
constexpr int kScaleBits = 12;
constexpr float kScale = 1 << kScaleBits, kInvScale = 1.0f / kScale;
constexpr float kScaleY = 0.25f;               // of A X, over that of the others

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef MatrixJob Job;

// The matrices of one launch: a part of the tensors of one shape.  Matrix z lies in the tensor
// t with first[t] <= z < first[t + 1] (below 0 where a tensor began in an earlier part).
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
// n elements as they lie in memory, converted after all have been asked for.
template <bool kBf16, int N>
struct Raw {
  uint32_t v[N];
  __device__ __forceinline__ void read(int k, const void* p, int64_t i) {
    v[k] = kBf16 ? static_cast<const u16*>(p)[i] : static_cast<const uint32_t*>(p)[i];
  }
  __device__ __forceinline__ float operator[](int k) const { return kBf16 ? bf16_lo(v[k]) : __uint_as_float(v[k]); }
};
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
// large nor small gradients leave its range), in chunks of kChunk elements, whose reads
// are all in flight (with the launch, 7 us for 2,048 x 2,048 fp32, 8 for three of 512 x 512
// with bf16 gradients and momenta; 12 where each conversion waited for its read).
constexpr int kChunk = 4096;
template <bool kBf16, bool kMom>
__global__ __launch_bounds__(kThreads) void k_ns_norm(Jobs j, int chunks, double* __restrict__ part) {
  const int z = blockIdx.x / chunks, k = blockIdx.x % chunks;
  const int t = tensor_of(j.first, z);
  const int64_t size = (int64_t)j.rows * j.cols, base = (z - j.first[t]) * size;
  const int64_t e0 = (int64_t)k * kChunk + threadIdx.x;
  constexpr int kEach = kChunk / kThreads;
  const void* const src = j.src[t];
  float* const mom = j.m[t];
  Raw<kBf16, kEach> g;
  float m[kEach];
#pragma unroll
  for (int q = 0; q < kEach; ++q) {
    const int64_t e = base + min(e0 + q * kThreads, size - 1);   // inside: no read waits for a branch
    g.read(q, src, e);
    if constexpr (kMom) m[q] = mom[e];
  }
  double s = 0.0;
#pragma unroll
  for (int q = 0; q < kEach; ++q) {
    const int64_t e = e0 + q * kThreads;
    float u = g[q];
    if constexpr (kMom) {
      const float w = fmaf(j.momentum, m[q], u);
      if (e < size) mom[base + e] = w;
      u = j.nesterov ? fmaf(j.momentum, w, u) : w;
    }
    u = e < size ? u : 0.0f;
    s = fma((double)u, (double)u, s);
  }
  __shared__ double w[kThreads / 64];
  s = wave_sum_d(s);
  if ((threadIdx.x & 63) == 0) w[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) part[blockIdx.x] = w[0] + w[1] + w[2] + w[3];
}

// X = U / (||U||_F + eps), as 2^up X = u 2^exp mul, mul in (1, 2]: the inverse itself may lie outside
// fp32's range.  A zero matrix stays zero; an infinity or NaN makes all of it NaN.
// Where ||U|| is far below eps, X is small and fp16 would end inside its terms.  They are held of
// 2^up X, whose norm starts in [1/2, 1); a step takes X up to at most 2^grow times its size, and so
// many bits from up, until none is left and the bounds of the singular values hold as they are.
struct Unit {
  float mul;
  int exp, up;
  __device__ __forceinline__ float operator()(float u) const { return __builtin_ldexpf(u, exp) * mul; }
};
__device__ __forceinline__ Unit unit_of(double norm, double eps) {
  if (norm == 0.0) return {0.0f, 0, 0};
  if (!(norm < INFINITY)) return {NAN, 0, 0};
  int e, below;
  const double m = frexp(norm + eps, &e);
  (void)frexp(norm / (norm + eps), &below);
  const int up = max(0, -below);
  return {(float)(1.0 / m), up - e, up};
}
__device__ __forceinline__ int up_after(int up, int bits) { return max(0, up - bits); }
// The same from the chunks' sums, in every thread.
__device__ __forceinline__ Unit unit_of(const double* __restrict__ part, int chunks, double eps) {
  __shared__ double w[kThreads / 64];
  double s = 0.0;
  for (int k = threadIdx.x; k < chunks; k += kThreads) s += part[k];
  s = wave_sum_d(s);
  if ((threadIdx.x & 63) == 0) w[threadIdx.x >> 6] = s;
  __syncthreads();
  return unit_of(sqrt(w[0] + w[1] + w[2] + w[3]), eps);
}

// Layout of an operand of R rows and K columns (K runs along them) in the workspace:
// fragments of 32 rows x 16 columns in the order in which a wave holds them for a
// 32 x 32 x 16 product, [R / 32][K / 16][term][64 lanes][8 values].  Lane lr + 32 h has
// row lr and columns 4 h + 0..3 and 8 + 4 h + 0..3: any order along K serves as long as
// both operands keep it, and this one is that in which accumulators hold a row.  A
// fragment is one contiguous kilobyte and goes from memory straight into registers.
constexpr int kFrag = 512;                             // values of a fragment's term
__device__ __forceinline__ int64_t frag_at(int rb, int ks, int K) { return ((int64_t)rb * (K / 16) + ks) * (kT * kFrag); }

// X's terms, zero beyond n x L, in tiles of 64 x 64: XR with K along X's rows, XC with
// K down its columns (two copies, since a fragment's 8 values are neighbours along K).
// 13-15 us at 2,048 x 2,048 fp32, 50 MB at 3.5 TB/s.
template <bool kBf16, bool kMom>
__global__ __launch_bounds__(kThreads) void k_ns_split(Jobs j, int chunks, const double* __restrict__ part,
                                                       u16* __restrict__ XR, u16* __restrict__ XC, int* __restrict__ up,
                                                       int np, int lp) {
  __shared__ float tile[64][65];
  const int z = blockIdx.z, t = tensor_of(j.first, z), i0 = blockIdx.y * 64, l0 = blockIdx.x * 64;
  const bool flip = j.rows > j.cols;
  const int64_t base = (int64_t)(z - j.first[t]) * j.rows * j.cols;
  // read along the source's rows, before the norm is waited for
  const int r0 = flip ? l0 : i0, c0 = flip ? i0 : l0;
  const int c = threadIdx.x & 63, col = c0 + c;
  const void* const src = j.src[t];
  const float* const mom = j.m[t];
  Raw<kBf16, 16> g;
  float m[16];
#pragma unroll
  for (int q = 0; q < 16; ++q) {
    const int64_t e = base + (int64_t)min(r0 + 4 * q + (int)(threadIdx.x >> 6), j.rows - 1) * j.cols + min(col, j.cols - 1);
    g.read(q, src, e);
    if constexpr (kMom) m[q] = mom[e];
  }
  const Unit unit = unit_of(part + (int64_t)z * chunks, chunks, j.eps);
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) up[z] = unit.up;
#pragma unroll
  for (int q = 0; q < 16; ++q) {
    const int r = 4 * q + (threadIdx.x >> 6);
    float u = g[q];
    if constexpr (kMom) u = j.nesterov ? fmaf(j.momentum, m[q], u) : m[q];
    u = r0 + r < j.rows && col < j.cols ? unit(u) : 0.0f;
    if (flip) tile[c][r] = u;
    else tile[r][c] = u;
  }
  __syncthreads();
  const int64_t size = (int64_t)kT * np * lp;
  const int lane = threadIdx.x & 63, lr = lane & 31, lh = lane >> 5;
#pragma unroll
  for (int q = threadIdx.x >> 6; q < 16; q += kThreads / 64) {   // 8 fragments of either kind
    const bool down = q >= 8;
    const int rb = (q >> 2) & 1, ks = q & 3;
    if ((down ? l0 : i0) + 32 * rb >= (down ? lp : np) || (down ? i0 : l0) + 16 * ks >= (down ? np : lp)) continue;
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      const int row = 32 * rb + lr, k = 16 * ks + 8 * (h >> 1) + 4 * lh + 2 * (h & 1);
      split2(down ? tile[k][row] : tile[row][k], down ? tile[k + 1][row] : tile[row][k + 1], kScale, hi[h], lo[h]);
    }
    u16* at = (down ? XC : XR) + z * size + lane * 8 +
              (down ? frag_at(l0 / 32 + rb, i0 / 16 + ks, np) : frag_at(i0 / 32 + rb, l0 / 16 + ks, lp));
    *reinterpret_cast<uint4*>(at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
    *reinterpret_cast<uint4*>(at + kFrag) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
  }
}

// ---- products -----------------------------------------------------------------------
// One tile of 32 TB x 32 TB of P Q^T in a workgroup whose four waves each take a quarter
// of K: every wave multiplies the whole tile, from fragments that it alone reads and
// that go from memory straight into registers, kDepth steps of 16 ahead.  The loop has no
// LDS traffic and no barrier (the same tile with operands shared through LDS was bound by
// LDS: 61 us a product at 2,048 x 2,048, of which 21 are matrix instructions).  The
// quarters are added through LDS at the end, each wave keeping a quarter of the tile.
// 2,048 x 2,048: the symmetric products take 32-36 us each, the others 51-57, i.e. 0.83 and
// 0.92 PFLOP/s of fp16 products, with the matrix cores 59% and 61% busy while a unit works;
// the rest is the first fragments' latency and the sums at the end.  Small counts (three of
// 512 x 512: 6-8 us a product) are launches that wait for each other.
enum Mode { kGram, kPoly, kApply, kStore };

struct GemmArgs {
  const u16* P;      // [matrices] operands of np rows: rows i of the result
  const u16* Q;      // [matrices] operands of `width` rows: columns j of the result
  const u16* old;    // kPoly: P;  kApply, kStore: X with K along its rows
  u16* out;          // the result with K along its rows
  u16* outT;         // kApply: the same with K down its columns
  const int* up;     // [matrices] of X at the first step
  int spent, grow;   // bits of it that the steps so far took, that a step takes
  int np, kp, width; // rows, K, columns
  int tiles_i, tiles_j, per_mat, tiles, per_xcd;   // per_mat: tiles of a matrix; tiles: of all
};

// Tile of a workgroup.  Workgroups go to the 8 XCDs in turn; each XCD gets a contiguous
// run of tiles.  Of a symmetric result only tiles ti >= tj are formed; otherwise a
// matrix's tiles run through groups of four tile rows, so that the run's operands are
// shared in the XCD's L2.
template <bool kSym>
__device__ __forceinline__ bool tile_of(const GemmArgs& g, int& z, int& ti, int& tj) {
  const int id = (blockIdx.x & 7) * g.per_xcd + (blockIdx.x >> 3);
  if (id >= g.tiles) return false;
  z = id / g.per_mat;
  const int t = id - z * g.per_mat;
  if constexpr (kSym) {
    ti = (int)((sqrtf(8.0f * t + 1.0f) - 1.0f) * 0.5f);
    while ((ti + 1) * (ti + 2) / 2 <= t) ++ti;
    while (ti * (ti + 1) / 2 > t) --ti;
    tj = t - ti * (ti + 1) / 2;
  } else {
    const int group = t / (4 * g.tiles_j), i0 = group * 4, rows = min(4, g.tiles_i - i0), r = t - i0 * g.tiles_j;
    ti = i0 + r % rows;
    tj = r / rows;
  }
  return true;
}

// 16 values of a row of a 32 x 32 block (as accumulators hold them) as terms: the
// fragments of two K steps.
__device__ __forceinline__ void write_block(u16* at, const f32x16& v, float scale) {
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    u32x4 h, l;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      uint32_t a, b;
      split2(v[8 * s + 2 * q], v[8 * s + 2 * q + 1], scale, a, b);
      h[q] = a;
      l[q] = b;
    }
    *reinterpret_cast<u32x4*>(at + s * kT * kFrag) = h;
    *reinterpret_cast<u32x4*>(at + s * kT * kFrag + kFrag) = l;
  }
}

template <int kMode, int TB>
__global__ __launch_bounds__(kThreads, TB == 2 ? 3 : 1) void k_ns_gemm(GemmArgs g, Jobs jobs) {
  constexpr bool kSym = kMode == kGram || kMode == kPoly;
  constexpr int kDepth = TB == 4 ? 3 : TB == 3 ? 4 : 2;
  constexpr int OB = (TB * TB + 3) / 4;                // blocks a wave keeps: x TB + y in [wave OB, wave OB + OB)
  constexpr int PB = OB == 4 ? 2 : 1;                  // of them added at a time
  constexpr int QB = TB == 2 ? 2 : 4;                  // quads of their values at a time
  __shared__ __attribute__((aligned(16))) f32x4 sums[4][4][PB][QB][64];   // [from][to][block][quad of values][lane]
  const int lane = threadIdx.x & 63, lr = lane & 31, lh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int z, ti, tj;
  if (!tile_of<kSym>(g, z, ti, tj)) return;
  // read here: where it is needed, every tile would wait for it
  const int up = kMode == kGram ? 0 : up_after(g.up[z], g.spent), up_next = up_after(up, g.grow);
  const int64_t pp = (int64_t)kT * g.np * g.kp, qp = (int64_t)kT * g.width * g.kp, op = (int64_t)kT * g.np * g.width;
  // a tile may reach past the last block: those rows repeat it, and their results go nowhere
  const int ni = g.np / 32, nj = g.width / 32;
  int64_t P[TB], Q[TB];                                // offsets of the wave's first fragments
#pragma unroll
  for (int b = 0; b < TB; ++b) {
    P[b] = z * pp + frag_at(min(ti * TB + b, ni - 1), min(wave, g.kp / 16 - 1), g.kp);
    Q[b] = z * qp + frag_at(min(tj * TB + b, nj - 1), min(wave, g.kp / 16 - 1), g.kp);
  }
  const int steps = (g.kp / 16 - wave + 3) / 4;        // of this wave: every fourth, none if there are fewer than four

  const uint32_t lane16 = lane * 16;
  struct Frags {
    f16x8 p[TB][kT], q[TB][kT];
  };
  Frags f[kDepth];
  f32x16 c[TB][TB] = {};                               // [block of j][block of i], 2^24 times the product
  const auto fetch = [&](int k, Frags& o) __attribute__((always_inline)) {
    const int64_t at = (int64_t)max(0, min(k, steps - 1)) * (4 * kT * kFrag);
#pragma unroll
    for (int b = 0; b < TB; ++b)
#pragma unroll
      for (int t = 0; t < kT; ++t) {
        o.p[b][t] = *reinterpret_cast<const f16x8*>(reinterpret_cast<const char*>(g.P + P[b] + at) + (lane16 + t * 2 * kFrag));
        o.q[b][t] = *reinterpret_cast<const f16x8*>(reinterpret_cast<const char*>(g.Q + Q[b] + at) + (lane16 + t * 2 * kFrag));
      }
  };
  const auto multiply = [&](const Frags& o) __attribute__((always_inline)) {
#pragma unroll
    for (int s = 0; s < 3; ++s)
#pragma unroll
      for (int x = 0; x < TB; ++x)
#pragma unroll
        for (int y = 0; y < TB; ++y) c[x][y] = mfma16(o.q[x][s == 1], o.p[y][s == 0], c[x][y]);
  };
#pragma unroll
  for (int d = 0; d < kDepth; ++d) fetch(d, f[d]);
  int k = 0;
  for (; k + kDepth <= steps; k += kDepth)
#pragma unroll
    for (int d = 0; d < kDepth; ++d) {
      multiply(f[d]);
      fetch(k + d + kDepth, f[d]);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
  for (int d = 0; d < kDepth - 1; ++d)
    if (k + d < steps) multiply(f[d]);

  // the four quarters of K, in the waves' order
  f32x16 o[OB];
#pragma unroll
  for (int pass = 0; pass < OB / PB * (4 / QB); ++pass) {
    const int b0 = pass / (4 / QB) * PB, q0 = pass % (4 / QB) * QB;
    if (pass) __syncthreads();
#pragma unroll
    for (int to = 0; to < 4; ++to)
#pragma unroll
      for (int b = 0; b < PB; ++b) {
        const int at = to * OB + b0 + b;
        if (at >= TB * TB) continue;
        const f32x16& v = c[at / TB][at % TB];
#pragma unroll
        for (int q = 0; q < QB; ++q) {
          const int r = 4 * (q0 + q);
          sums[wave][to][b][q][lane] = f32x4{v[r], v[r + 1], v[r + 2], v[r + 3]};
        }
      }
    __syncthreads();
#pragma unroll
    for (int b = 0; b < PB; ++b)
#pragma unroll
      for (int q = 0; q < QB; ++q) {
        f32x4 v = sums[0][wave][b][q][lane];
#pragma unroll
        for (int w = 1; w < 4; ++w) v += sums[w][wave][b][q][lane];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[b0 + b][4 * (q0 + q) + e] = v[e];
      }
  }
  __syncthreads();

  // Each kept block: lane lr + 32 h has row i, columns 8 g + 4 h + 0..3.
  float* const turn = reinterpret_cast<float*>(sums) + wave * (32 * 33);
  const int t = kMode == kStore ? tensor_of(jobs.first, z) : 0;
  const bool flip = jobs.rows > jobs.cols;
#pragma unroll
  for (int b = 0; b < OB; ++b) {
    const int at = wave * OB + b, bi = ti * TB + at % TB, bj = tj * TB + at / TB;   // in blocks of 32
    if (at >= TB * TB || bi >= ni || bj >= nj) continue;
    f32x16 v = o[b];
    // kGram: 2^24 times the result; otherwise 2^12 times.  Operands are held up by powers of two:
    // X X^T by 2 up, its square by 4; the polynomial as it is.
    if constexpr (kMode != kGram) {
      const int to = kMode == kApply ? up_next - up : 0;
      const float keep = kMode == kPoly ? __builtin_ldexpf(jobs.b, -2 * up) : __builtin_ldexpf(jobs.a, to);
      const float mul = kMode == kPoly ? __builtin_ldexpf(jobs.c * kInvScale, -4 * up) : __builtin_ldexpf(kInvScale, to);
      const u16* from = g.old + z * op + frag_at(bi, 2 * bj, g.width) + lane * 8;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const f16x8 h = *reinterpret_cast<const f16x8*>(from + s * kT * kFrag);
        const f16x8 l = *reinterpret_cast<const f16x8*>(from + s * kT * kFrag + kFrag);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[8 * s + e] = fmaf(keep, (float)h[e] + (float)l[e], mul * v[8 * s + e]);
      }
    }
    constexpr float scale = kMode == kGram ? kInvScale : 1.0f;
    if constexpr (kMode != kStore) write_block(g.out + z * op + frag_at(bi, 2 * bj, g.width) + lane * 8, v, scale);
    // the block turned round: lane lr has column lr, rows 8 g + 4 h + 0..3
    const bool turned = kMode == kApply || (kSym && ti != tj) || (kMode == kStore && !flip);
    if (turned) {
#pragma unroll
      for (int r = 0; r < 16; ++r) turn[lr * 33 + 8 * (r >> 2) + 4 * lh + (r & 3)] = v[r];
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int r = 0; r < 16; ++r) v[r] = turn[(8 * (r >> 2) + 4 * lh + (r & 3)) * 33 + lr];
      __builtin_amdgcn_wave_barrier();
      if constexpr (kMode != kStore)
        write_block((kSym ? g.out : g.outT) + z * op + frag_at(bj, 2 * bi, g.np) + lane * 8, v, scale);
    }
    if constexpr (kMode == kStore) {
      // lanes run along the rows of the caller's matrix
      const int64_t base = (int64_t)(z - jobs.first[t]) * jobs.rows * jobs.cols;
      const int r0 = 32 * (flip ? bj : bi), col = 32 * (flip ? bi : bj) + lr;
      const auto row_of = [&](int r) __attribute__((always_inline)) { return r0 + 8 * (r >> 2) + 4 * lh + (r & 3); };
      float old[16];   // all parameters before the first is moved, from places inside the matrix
      if (jobs.m[t])
#pragma unroll
        for (int r = 0; r < 16; ++r)
          old[r] = static_cast<const float*>(jobs.out[t])[base + (int64_t)min(row_of(r), jobs.rows - 1) * jobs.cols +
                                                          min(col, jobs.cols - 1)];
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        if (row_of(r) >= jobs.rows || col >= jobs.cols) continue;
        const int64_t to = base + (int64_t)row_of(r) * jobs.cols + col;
        const float x = __builtin_ldexpf(v[r], -kScaleBits - up);
        if (jobs.m[t]) static_cast<float*>(jobs.out[t])[to] = fmaf(-jobs.rate, x, jobs.decay * old[r]);
        else if (jobs.out_bf16) static_cast<u16*>(jobs.out[t])[to] = to_bf16(x);
        else static_cast<float*>(jobs.out[t])[to] = x;
      }
    }
  }
}

// ---- small matrices -------------------------------------------------------------------
// All steps of one matrix in one workgroup, from the momentum update to the
// parameters, X never leaving registers and LDS: n <= NP and L <= 16384 / NP, for NP
// of 32, 64 and 128.  Wave (rw, cw) of RW x CW = W owns rows 32 rw .. + 31 of X and every
// CW-th block of 32 columns, JB of them (the fewest that hold L); lane lr (of half lh)
// holds row 32 rw + lr, columns 8 g + 4 lh + 0..3 of each block, as accumulators do.
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
// Six of 128 x 128 take 43 us (6.5 a step), 300 of them 97-107 on 256 units; the matrix
// cores are 40% busy: between the products stand barriers and the splitting of X, Y and A
// into terms, with one or two waves on a SIMD to hide them.
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
  int src_bf16, out_bf16, nesterov, steps, grow;
  float momentum, decay, a, b, c;
  double eps;
};

constexpr int kSmallValues = 16384;                    // NP x LP
constexpr int kSmallBuffer = kSmallValues * kT * 2;    // X's terms, and Y's

// U of a small matrix into its fp32 copy, the momentum on the way; returns the
// thread's sum of squares.  Quads (cols a multiple of 4) have every load in flight.
template <int kN, bool kBf16, bool kMom>   // kN threads
__device__ __forceinline__ double small_load(const SmallJobs& jobs, const SmallJob& job, int64_t base, float* flat, int pitch) {
  const int cols = job.cols, size = job.rows * cols;
  const float inv_cols = 1.0f / cols;
  const float* const f32 = static_cast<const float*>(job.src) + base;
  const u16* const b16 = static_cast<const u16*>(job.src) + base;
  float* const mom = kMom ? job.m + base : nullptr;
  double sq = 0.0;
  if (cols % 4 == 0) {
    f32x4 u[(kSmallValues / 4 / kN)], m[(kSmallValues / 4 / kN)];
#pragma unroll
    for (int k = 0; k < (kSmallValues / 4 / kN); ++k) {
      const int e = (k * kN + threadIdx.x) * 4;
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
    for (int k = 0; k < (kSmallValues / 4 / kN); ++k) {
      const int e = (k * kN + threadIdx.x) * 4;
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
    for (int e = threadIdx.x; e < size; e += kN) {
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
template <int kN, bool kBf16, bool kMom>   // kN threads
__device__ __forceinline__ void small_store(const SmallJobs& jobs, const SmallJob& job, int64_t base, const float* flat, int pitch) {
  const int cols = job.cols, size = job.rows * cols;
  const float inv_cols = 1.0f / cols;
  float* const f32 = static_cast<float*>(job.out) + base;
  u16* const b16 = static_cast<u16*>(job.out) + base;
  if (cols % 4 == 0) {
    f32x4 old[(kSmallValues / 4 / kN)];
    if constexpr (kMom)
#pragma unroll
      for (int k = 0; k < (kSmallValues / 4 / kN); ++k) {
        const int e = (k * kN + threadIdx.x) * 4;
        if (e >= size) break;
        old[k] = *reinterpret_cast<const f32x4*>(f32 + e);
      }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < (kSmallValues / 4 / kN); ++k) {
      const int e = (k * kN + threadIdx.x) * 4;
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
    for (int e = threadIdx.x; e < size; e += kN) {
      const int r = (int)((e + 0.5f) * inv_cols);
      const float v = flat[r * (pitch - cols) + e];
      if constexpr (kMom) f32[e] = fmaf(-job.rate, v, jobs.decay * f32[e]);
      else if constexpr (kBf16) b16[e] = to_bf16(v);
      else f32[e] = v;
    }
  }
}

template <int NP, int JB, int W>
__global__ __launch_bounds__(64 * W, 1) void k_ns_small(SmallJobs jobs) {
  constexpr int LP = kSmallValues / NP;
  constexpr int RW = NP / 32, CW = W / RW, NI = NP / 32;
  constexpr int kN = 64 * W;
  constexpr bool kShare = W == 8;                      // A's blocks are shared out, otherwise its sums
  constexpr int IB = kShare ? NI / CW : NI;            // blocks of A that the wave forms
  constexpr int RB = 2 * LP, PL = NP * RB;             // bytes of a row of one term, of a term
  // X's terms, then Y's; before the first and after the last step the fp32 copy (rows
  // one value longer if even: 66 KB at most); Y's part also takes the waves' sums for A
  __shared__ __attribute__((aligned(16))) char lds[2 * kSmallBuffer];
  __shared__ double sums[W];
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
  if (job.m) sq = jobs.src_bf16 ? small_load<kN, true, true>(jobs, job, base, flat, pitch) : small_load<kN, false, true>(jobs, job, base, flat, pitch);
  else sq = jobs.src_bf16 ? small_load<kN, true, false>(jobs, job, base, flat, pitch) : small_load<kN, false, false>(jobs, job, base, flat, pitch);
  sq = wave_sum_d(sq);
  if (lane == 0) sums[wave] = sq;
  __syncthreads();
  double total = 0.0;
#pragma unroll
  for (int w = 0; w < W; ++w) total += sums[w];
  const Unit unit = unit_of(sqrt(total), jobs.eps);

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
        x[r] = i < n && j < L ? unit(flat[i * pi + j * pj]) : 0.0f;
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
    f32x16 c[JB] = {};
    // a step's first products each with the reads of a block of the next step behind it, in this order
#pragma unroll
    for (int ks = 0; ks < kSteps; ++ks)
#pragma unroll
      for (int s = 0; s < 3; ++s)
#pragma unroll
        for (int y = 0; y < JB; ++y) {
          c[y] = mfma16(q[ks & 1][y][s == 1], A[ks / 2].v[ks % 2][s == 0], c[y]);
          if (s == 0 && ks + 1 < kSteps) read(ks + 1, y);
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
    for (int y = 0; y < JB; ++y) done(y, c[y]);
  };

  f32x16 x[JB];                                        // 2^(12 + up) times X
  int up = unit.up;
  for (int step = 0; step < jobs.steps; ++step) {
    // a X, b (X X^T) X and c (X X^T)^2 X from what is held 1, 3 and 5 up, to where the next step has it
    const int to = up_after(up, jobs.grow) - up;
    const float ka = __builtin_ldexpf(jobs.a, to), kb = __builtin_ldexpf(jobs.b * kInvScale, to - 2 * up);
    const float kc = __builtin_ldexpf(jobs.c * (kInvScale / kScaleY), to - 4 * up);
    up += to;
    lds_barrier();                                     // X is there, Y has been read
    Terms A[NI];
    {
      // kShare: all of X's columns, the wave's own first; otherwise its own
      constexpr int kSteps = JB * 2 * (kShare ? CW : 1);
      f16x8 q[2][IB][kT], p[2][kT];
      const auto column = [&](int ks) { return 4 * ((ks / 2) % JB * CW + (cw ^ (ks / 2 / JB))) + 2 * (ks % 2) + lh; };
      const auto read = [&](int ks, int y) __attribute__((always_inline)) {
        const int ib = kShare ? IB * cw + y : y;
#pragma unroll
        for (int w = 0; w < kT; ++w) {
          q[ks & 1][y][w] = lds_row(ldsX + w * PL + (32 * ib + lr) * RB + ((column(ks) ^ own_swz) << 4));
          if (y == 0 && ks >= 2 * JB) p[ks & 1][w] = lds_row(ldsX + w * PL + own + ((column(ks) ^ own_swz) << 4));
        }
      };
#pragma unroll
      for (int y = 0; y < IB; ++y) read(0, y);
      f32x16 c[IB] = {};
#pragma unroll
      for (int ks = 0; ks < kSteps; ++ks)
#pragma unroll
        for (int s = 0; s < 3; ++s)
#pragma unroll
          for (int y = 0; y < IB; ++y) {
            const f16x8& o = ks < 2 * JB ? xt[ks / 2 % JB].v[ks % 2][s == 0] : p[ks & 1][s == 0];
            c[y] = mfma16(q[ks & 1][y][s == 1], o, c[y]);
            if (s == 0 && ks + 1 < kSteps) read(ks + 1, y);
            __builtin_amdgcn_sched_barrier(0);
          }
      if constexpr (kShare) {
        // the blocks of a row go to the other waves of that row through LDS
        char* const give = ldsY + (rw * NI + IB * cw) * 4096 + lane * 16;
#pragma unroll
        for (int y = 0; y < IB; ++y) {
          Terms o;
          split(c[y], kInvScale, o);
#pragma unroll
          for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int w = 0; w < kT; ++w) *reinterpret_cast<f16x8*>(give + y * 4096 + (2 * s + w) * 1024) = o.v[s][w];
        }
        lds_barrier();
        const char* const take = ldsY + rw * NI * 4096 + lane * 16;
#pragma unroll
        for (int ib = 0; ib < NI; ++ib)
#pragma unroll
          for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int w = 0; w < kT; ++w) A[ib].v[s][w] = lds_row(take + ib * 4096 + (2 * s + w) * 1024);
        lds_barrier();
      } else {
#pragma unroll
        for (int y = 0; y < NI; ++y) {
          float* part = reinterpret_cast<float*>(ldsY) + (wave * NI + y) * 16 * 64 + lane;
#pragma unroll
          for (int r = 0; r < 16; ++r) part[r * 64] = c[y][r];
        }
      }
    }
    if constexpr (!kShare) {
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
        x[b][r] = fmaf(kb, y[r], ka * fmaf((float)xt[b].v[r / 8][0][r % 8], one, (float)xt[b].v[r / 8][1][r % 8]));
      split(y, kInvScale * kScaleY, xt[b]);
      put(ldsY, b, xt[b]);
    });
    lds_barrier();                                     // Y is there, X has been read
    times(ldsY, A, [&](int b, const f32x16& y) __attribute__((always_inline)) {
      x[b] += kc * y;
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
      if (i < n && j < L) flat[i * pi + j * pj] = __builtin_ldexpf(x[b][r], -kScaleBits - up);
    }
  if (job.m) small_store<kN, false, true>(jobs, job, base, flat, pitch);
  else if (jobs.out_bf16) small_store<kN, true, false>(jobs, job, base, flat, pitch);
  else small_store<kN, false, false>(jobs, job, base, flat, pitch);
}

// The workgroup that holds a matrix: up to 64 rows, 3 (log2 NP - 5) + log2 JB; beyond, 6 (then L is
// beyond 64 as well); -1: none does.
constexpr int kSmallClasses = 7;
int small_class(int rows, int cols) {
  const int n = rows < cols ? rows : cols, L = rows < cols ? cols : rows;
  for (int p = 0; p < 2; ++p)
    for (int b = 0; b < 3 && n <= 32 << p; ++b)
      if (L <= ((32 << b) * 4 >> p)) return 3 * p + b;   // 32 JB columns a wave, 4 / 2^p waves
  return L <= 128 ? 6 : -1;
}
template <int NP, int JB, int W>
void small_kernel(const SmallJobs& j, hipStream_t st) {
  hipLaunchKernelGGL((k_ns_small<NP, JB, W>), dim3(j.first[SAGIPS_MAX_TENSORS]), dim3(64 * W), 0, st, j);
}

// ---- plan ---------------------------------------------------------------------------
int64_t round_up(int64_t n, int64_t m) { return (n + m - 1) / m * m; }
size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

struct Plan {
  int n, L, np, lp, chunks, mats;
  size_t r0, r1, c0, c1, A, B, up, bytes;   // offsets; the partial sums come first
};
Plan plan_of(int rows, int cols, int mats) {
  Plan p;
  p.n = rows < cols ? rows : cols;
  p.L = rows < cols ? cols : rows;
  p.mats = mats;
  p.np = (int)round_up(p.n, 32);
  p.lp = (int)round_up(p.L, 32);
  p.chunks = (int)(((int64_t)rows * cols + kChunk - 1) / kChunk);
  const size_t part = align256((size_t)mats * p.chunks * sizeof(double));
  const size_t x = align256((size_t)mats * kT * p.np * p.lp * 2), a = align256((size_t)mats * kT * p.np * p.np * 2);
  p.r0 = part;
  p.r1 = p.r0 + x;
  p.c0 = p.r1 + x;
  p.c1 = p.c0 + x;
  p.A = p.c1 + x;
  p.B = p.A + a;
  p.up = p.B + a;
  p.bytes = p.up + align256((size_t)mats * sizeof(int));
  return p;
}

// Matrices that go through their launches together: their workspace stays within kPart bytes,
// which 341 of 512 x 512 or 21 of 2,048 x 2,048 fill, with tens of tiles a compute unit.  All at once,
// 65,535 of 1 x 16,384 (4.3 GB, but padded to 32 rows) would take 550 GB.
constexpr size_t kPart = (size_t)2 << 30;
int per_part(int rows, int cols, int mats) {
  const size_t one = plan_of(rows, cols, 1).bytes;   // with the offsets' padding: no less than a matrix's share
  const size_t most = kPart / one;
  return most < 1 ? 1 : most < (size_t)mats ? (int)most : mats;
}

// Blocks in a tile's side: 2, 3 or 4.  Compute units take tiles in rounds; a round takes
// about fixed + per_k K microseconds (measured from K = 256 to 2,048; a larger side reads
// less per product but has more to add up at the end, and only tiles of 2 run three to a
// unit, which the rounds count as one after the other).  Products at 2,048 x 2,048:
// symmetric 43, 30, 37 us with sides 2, 3, 4, others 61, 61, 50; at K = 512 a side of 2 is
// the fastest at every count (16 of 512 x 512: 13, 20, 16 and 21, 39, 22 us).  A round that fills
// part of the units is faster than that (the 136 symmetric tiles of side 4 at 2,048: 37 us, 50 by the
// model), so that a larger side may be passed over where tiles are few.
int tile_side(bool sym, int np, int width, int K, int mats, int n_cu) {
  static const double fixed[5] = {0, 0, 2.6, 7.6, 13.0}, per_k[5] = {0, 0, 0.0064, 0.0115, 0.018};
  int best = 2;
  double least = 0.0;
  for (int tb = 2; tb <= 4; ++tb) {
    const int64_t i = (np / 32 + tb - 1) / tb, j = (width / 32 + tb - 1) / tb, tiles = (sym ? i * (i + 1) / 2 : i * j) * mats;
    const double t = (fixed[tb] + per_k[tb] * K) * (double)((tiles + n_cu - 1) / n_cu);
    if (tb == 2 || t < least) {
      best = tb;
      least = t;
    }
  }
  return best;
}

template <int kMode, int TB>
void gemm_of(GemmArgs g, const Jobs& j, int mats, hipStream_t st) {
  g.tiles_i = (g.np / 32 + TB - 1) / TB;
  g.tiles_j = (g.width / 32 + TB - 1) / TB;
  g.per_mat = kMode == kGram || kMode == kPoly ? g.tiles_i * (g.tiles_i + 1) / 2 : g.tiles_i * g.tiles_j;
  g.tiles = g.per_mat * mats;
  g.per_xcd = (g.tiles + 7) / 8;
  hipLaunchKernelGGL((k_ns_gemm<kMode, TB>), dim3(8 * g.per_xcd), dim3(kThreads), 0, st, g, j);
}
template <int kMode>
void gemm(const GemmArgs& g, const Jobs& j, int mats, int side, hipStream_t st) {
  if (side == 2) gemm_of<kMode, 2>(g, j, mats, st);
  else if (side == 3) gemm_of<kMode, 3>(g, j, mats, st);
  else gemm_of<kMode, 4>(g, j, mats, st);
}

hipError_t steps_of(const Plan& p, const Jobs& j, int steps, int grow, int n_cu, char* ws, hipStream_t st, Timer* tm) {
  const auto at = [&](size_t offset) { return reinterpret_cast<u16*>(ws + offset); };
  double* part = reinterpret_cast<double*>(ws);
  int* up = reinterpret_cast<int*>(ws + p.up);
  u16 *r0 = at(p.r0), *r1 = at(p.r1), *c0 = at(p.c0), *c1 = at(p.c1), *A = at(p.A), *B = at(p.B);
  if (tm) tm->begin("ns_norm");
  const auto norm = j.m[0] ? (j.src_bf16 ? k_ns_norm<true, true> : k_ns_norm<false, true>)
                           : (j.src_bf16 ? k_ns_norm<true, false> : k_ns_norm<false, false>);
  const auto split = j.m[0] ? (j.src_bf16 ? k_ns_split<true, true> : k_ns_split<false, true>)
                            : (j.src_bf16 ? k_ns_split<true, false> : k_ns_split<false, false>);
  hipLaunchKernelGGL(norm, dim3((unsigned)p.mats * p.chunks), dim3(kThreads), 0, st, j, p.chunks, part);
  if (tm) tm->end();
  if (tm) tm->begin("ns_split");
  hipLaunchKernelGGL(split, dim3((p.lp + 63) / 64, (p.np + 63) / 64, p.mats), dim3(kThreads), 0, st, j, p.chunks, part, r0, c0,
                     up, p.np, p.lp);
  if (tm) tm->end();
  const int gram = tile_side(true, p.np, p.np, p.lp, p.mats, n_cu), poly = tile_side(true, p.np, p.np, p.np, p.mats, n_cu);
  const int apply = tile_side(false, p.np, p.lp, p.np, p.mats, n_cu);
  for (int s = 0; s < steps; ++s) {
    if (tm) tm->begin("ns_gram");
    gemm<kGram>(GemmArgs{r0, r0, nullptr, A, nullptr, up, s * grow, grow, p.np, p.lp, p.np}, j, p.mats, gram, st);
    if (tm) tm->end();
    if (tm) tm->begin("ns_poly");
    gemm<kPoly>(GemmArgs{A, A, A, B, nullptr, up, s * grow, grow, p.np, p.np, p.np}, j, p.mats, poly, st);
    if (tm) tm->end();
    if (tm) tm->begin("ns_apply");
    const GemmArgs g{B, c0, r0, r1, c1, up, s * grow, grow, p.np, p.np, p.lp};
    if (s + 1 < steps) gemm<kApply>(g, j, p.mats, apply, st);
    else gemm<kStore>(g, j, p.mats, apply, st);
    if (tm) tm->end();
    u16 *r = r0, *c = c0;
    r0 = r1;
    r1 = r;
    c0 = c1;
    c1 = c;
  }
  return hipGetLastError();
}

}  // namespace

// Tensors of one shape go through their launches together, or in parts; the shapes and
// parts one after the other, in the same workspace.
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
    const size_t b = plan_of(a.rows, a.cols, per_part(a.rows, a.cols, total_of(js, list, n))).bytes;
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
  j.grow = js.grow;
  j.momentum = js.momentum;
  j.decay = js.decay;
  j.a = js.coef[0];
  j.b = js.coef[1];
  j.c = js.coef[2];
  j.eps = js.eps;
  if (tm) tm->begin("ns_small");
  switch (which) {
    case 0: small_kernel<32, 1, 4>(j, st); break;
    case 1: small_kernel<32, 2, 4>(j, st); break;
    case 2: small_kernel<32, 4, 4>(j, st); break;
    case 3: small_kernel<64, 1, 4>(j, st); break;
    case 4: small_kernel<64, 2, 4>(j, st); break;
    case 5: small_kernel<64, 4, 4>(j, st); break;
    default: small_kernel<128, 2, 8>(j, st); break;
  }
  if (tm) tm->end();
  return hipGetLastError();
}

hipError_t launch_muon(const MatrixJobs& js, void* ws, int n_cu, hipStream_t st, Timer* tm) {
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
    const int each = per_part(a.rows, a.cols, total);
    for (int z = 0; z < total; z += each) {
      Jobs part = j;
      for (int k = 0; k < n; ++k) part.first[k] -= z;
      const Plan p = plan_of(a.rows, a.cols, total - z < each ? total - z : each);
      const hipError_t e = steps_of(p, part, js.steps, js.grow, n_cu, static_cast<char*>(ws), st, tm);
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  });
}

}  // namespace sagips
