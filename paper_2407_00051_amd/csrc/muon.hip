// The orthogonalised update of weight matrices: Newton-Schulz steps
//   X <- a X + b (X X^T) X + c (X X^T)^2 X
// on X = U / (||U||_F + eps), with U oriented so that its rows are the shorter
// side (n rows of L).  The steps drive every singular value of X towards one
// band around 1 and keep its singular vectors.
//
// Products run on the bf16 matrix cores from the operands' bf16 terms with fp32
// accumulation (split_bf16.hpp): three terms (24 bits) where the result is fp32,
// two terms (16 bits, three products) where it is rounded to bf16 anyway.  X,
// A = X X^T and B = b A + c A^2 are kept as their terms, which hold an fp32
// value exactly (two terms: to 2^-17 of it), so no fp32 copy is needed.
#include "kernels.hpp"
#include "split_bf16.hpp"

namespace sagips {
namespace {

constexpr int kThreads = 256;

typedef MatrixJob Job;

// The matrices of one launch: tensors of one shape.  Matrix z lies in the tensor
// t with first[t] <= z < first[t + 1].
struct Jobs {
  const void* src[SAGIPS_MAX_TENSORS];   // gradients, or the matrices to orthogonalise
  float* m[SAGIPS_MAX_TENSORS];          // momenta, or NULL
  void* out[SAGIPS_MAX_TENSORS];         // parameters, or the orthogonalised matrices
  int first[SAGIPS_MAX_TENSORS + 1];
  int n_tensors;
  int rows, cols;                        // of every matrix
  int src_bf16, out_bf16;
  float momentum, decay, rate;           // m <- momentum m + g;  p <- decay p - rate X
  int nesterov;
  float a, b, c;
  double eps;
};

__device__ __forceinline__ int tensor_of(const Jobs& j, int z) {
  int t = 0;
  while (t + 1 < j.n_tensors && z >= j.first[t + 1]) ++t;
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

// The terms of two values, kT of them.
template <int kT>
__device__ __forceinline__ void split2(float a, float b, uint32_t (&t)[kT]) {
  uint32_t s[kTerms];
  split_pair(a, b, s);
#pragma unroll
  for (int k = 0; k < kT; ++k) t[k] = s[k];
}

// ---- norm -------------------------------------------------------------------------
// The momentum update, and each matrix's sum of squares of U in 64 bits (neither
// large nor small gradients leave its range), in chunks of kChunk elements.
constexpr int64_t kChunk = 8192;
__global__ __launch_bounds__(kThreads) void k_ns_norm(Jobs j, int chunks, double* __restrict__ part) {
  const int z = blockIdx.x / chunks, k = blockIdx.x % chunks;
  const int t = tensor_of(j, z);
  const int64_t size = (int64_t)j.rows * j.cols, base = (z - j.first[t]) * size;
  const int64_t e1 = min(size, (k + 1) * kChunk);
  double s = 0.0;
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

// X's terms [term][np][lp], zero beyond n x L, in tiles of 64 x 64.
template <int kT>
__global__ __launch_bounds__(kThreads) void k_ns_split(Jobs j, int chunks, const double* __restrict__ part,
                                                       u16* __restrict__ X, int np, int lp) {
  __shared__ float tile[64][65];
  const int z = blockIdx.z, t = tensor_of(j, z), i0 = blockIdx.y * 64, l0 = blockIdx.x * 64;
  const bool flip = j.rows > j.cols;
  const int64_t base = (int64_t)(z - j.first[t]) * j.rows * j.cols;
  double s = 0.0;
  for (int k = 0; k < chunks; ++k) s += part[(int64_t)z * chunks + k];
  const float inv = (float)(1.0 / (sqrt(s) + j.eps));
  // read along the source's rows
  const int r0 = flip ? l0 : i0, c0 = flip ? i0 : l0;
#pragma unroll 4
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
  const int64_t plane = (int64_t)np * lp;
  u16* x = X + (int64_t)z * kT * plane;
#pragma unroll
  for (int q = threadIdx.x; q < 512; q += kThreads) {   // 8 values of a row
    const int i = q >> 3, l = (q & 7) * 8;
    uint32_t v[4][kT];
#pragma unroll
    for (int h = 0; h < 4; ++h) split2<kT>(tile[i][l + 2 * h], tile[i][l + 2 * h + 1], v[h]);
#pragma unroll
    for (int s2 = 0; s2 < kT; ++s2)
      *reinterpret_cast<uint4*>(x + s2 * plane + (int64_t)(i0 + i) * lp + l0 + l) =
          make_uint4(v[0][s2], v[1][s2], v[2][s2], v[3][s2]);
  }
}

// ---- products -----------------------------------------------------------------------
enum Mode { kGram, kPoly, kApply, kStore };

struct GemmArgs {
  const u16* P;      // [matrices][term][np][kp]: rows i of the result, K along a row
  const u16* Q;      // kGram, kPoly: rows j of the result, K along a row; otherwise [kp][width]: K down a column
  const u16* X;      // kApply, kStore: X, as Q; kPoly: P
  u16* out;          // [matrices][term][np][width]
  int np, kp, width; // padded sizes
  int tiles_i, tiles_j;
};

// One TI x TI tile of the result, 4 waves of (TI / 2)^2.  K in steps of 32 through
// two LDS buffers.
template <int kT, int TI>
struct Tile {
  static constexpr int KB = 32;
  static constexpr int ROWB = 2 * KB;                  // bytes of an operand row along K
  static constexpr int PT = TI * ROWB;                 // bytes of one term of an operand tile
  static constexpr int BUF = 2 * kT * PT;              // both operands
  static constexpr int LOADS = BUF / 16 / kThreads;    // 16-byte loads a thread
  static constexpr int WB = TI / 64;                   // 32-blocks a wave has in each direction
};

// Products over one K step of 16: hi hi into c, the corrections, smallest first, into d.
template <int kT, int WB>
__device__ __forceinline__ void products(const bf16x8 (&q)[WB][kT], const bf16x8 (&p)[WB][kT], f32x16 (&c)[WB][WB],
                                         f32x16 (&d)[WB][WB]) {
  constexpr int n = kT == 3 ? 5 : 2;
  constexpr int tq[5] = {kT == 3 ? 2 : 1, 0, 1, 1, 0}, tp[5] = {0, kT == 3 ? 2 : 1, 1, 0, 1};
#pragma unroll
  for (int x = 0; x < WB; ++x)
#pragma unroll
    for (int y = 0; y < WB; ++y) c[x][y] = mfma32(q[x][0], p[y][0], c[x][y]);
#pragma unroll
  for (int k = 0; k < n; ++k)
#pragma unroll
    for (int x = 0; x < WB; ++x)
#pragma unroll
      for (int y = 0; y < WB; ++y) d[x][y] = mfma32(q[x][tq[k]], p[y][tp[k]], d[x][y]);
}

template <int kMode, int kT, int TI>
__global__ __launch_bounds__(kThreads) void k_ns_gemm(GemmArgs g, Jobs jobs) {
  typedef Tile<kT, TI> T;
  constexpr bool kDown = kMode == kApply || kMode == kStore;   // Q's K runs down its columns
  __shared__ __attribute__((aligned(16))) char lds[2][T::BUF];
  const int lane = threadIdx.x & 63, lr = lane & 31, lh = lane >> 5;
  const int wave = threadIdx.x >> 6, wi = wave & 1, wj = wave >> 1;
  const int z = blockIdx.y;
  const int ti = blockIdx.x / g.tiles_j, tj = blockIdx.x % g.tiles_j;
  const int64_t pp = (int64_t)g.np * g.kp, qp = kDown ? (int64_t)g.kp * g.width : (int64_t)g.width * g.kp;
  const u16* P = g.P + z * kT * pp + (int64_t)ti * TI * g.kp;
  const u16* Q = g.Q + z * kT * qp + (kDown ? (int64_t)tj * TI : (int64_t)tj * TI * g.kp);

  // A thread's 16-byte pieces of a K step.  Along K: piece (term, row, unit u of 4),
  // kept at unit u ^ (row / 2 % 4), so that 8 lanes (rows) of a read hit distinct
  // banks.  Down K: piece (term, k, unit u of TI / 8); the 32-byte granule u / 2 is
  // kept at u / 2 ^ k % 4, so that the 4 rows of a transposed read do.
  const u16* from[T::LOADS];
  int64_t step[T::LOADS];
  uint32_t to[T::LOADS];
#pragma unroll
  for (int n = 0; n < T::LOADS; ++n) {
    const int q = n * kThreads + threadIdx.x;
    constexpr int per = T::PT / 16;                    // pieces of a term of one operand
    const int term = q / per % kT, r = q % per;
    if (q < kT * per || !kDown) {
      const int row = r >> 2, u = r & 3;
      from[n] = (q < kT * per ? P + term * pp : Q + term * qp) + (int64_t)row * g.kp + u * 8;
      step[n] = T::KB;
      to[n] = q / per * T::PT + row * T::ROWB + ((u ^ ((row >> 1) & 3)) << 4);
    } else {
      const int k = r / (TI / 8), u = r % (TI / 8);
      from[n] = Q + term * qp + (int64_t)k * g.width + u * 8;
      step[n] = (int64_t)T::KB * g.width;
      to[n] = q / per * T::PT + k * (2 * TI) + ((((u >> 1) ^ (k & 3)) << 1 | (u & 1)) << 4);
    }
  }
  uint4 hold[T::LOADS];
  const auto fetch = [&] {
#pragma unroll
    for (int n = 0; n < T::LOADS; ++n) {
      hold[n] = *reinterpret_cast<const uint4*>(from[n]);
      from[n] += step[n];
    }
  };
  const auto put = [&](char* buf) {
#pragma unroll
    for (int n = 0; n < T::LOADS; ++n) *reinterpret_cast<uint4*>(buf + to[n]) = hold[n];
  };

  f32x16 c[T::WB][T::WB] = {}, d[T::WB][T::WB] = {};   // [block of j][block of i]
  const int steps = g.kp / T::KB;
  fetch();
  put(lds[0]);
  __syncthreads();
  for (int k = 0; k < steps; ++k) {
    const char* buf = lds[k & 1];
    if (k + 1 < steps) fetch();
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      bf16x8 p[T::WB][kT], q[T::WB][kT];
#pragma unroll
      for (int y = 0; y < T::WB; ++y) {
        const int row = wi * (TI / 2) + y * 32 + lr;
        const uint32_t at = row * T::ROWB + (((2 * ks + lh) ^ ((row >> 1) & 3)) << 4);
#pragma unroll
        for (int t = 0; t < kT; ++t) p[y][t] = *reinterpret_cast<const bf16x8*>(buf + t * T::PT + at);
      }
#pragma unroll
      for (int x = 0; x < T::WB; ++x) {
        if constexpr (!kDown) {
          const int row = wj * (TI / 2) + x * 32 + lr;
          const uint32_t at = row * T::ROWB + (((2 * ks + lh) ^ ((row >> 1) & 3)) << 4);
#pragma unroll
          for (int t = 0; t < kT; ++t) q[x][t] = *reinterpret_cast<const bf16x8*>(buf + (kT + t) * T::PT + at);
        } else {
          // 16 lanes read 4 rows of 16 values and get a column of 4 each
          const int i = lane & 15, half = (lane >> 4) & 1;
          const int G = (wj * (TI / 2) + x * 32) / 16 + half;
#pragma unroll
          for (int t = 0; t < kT; ++t) {
            bf16x4 v[2];
#pragma unroll
            for (int s = 0; s < 2; ++s) {
              const int kk = 16 * ks + 8 * lh + 4 * s + (i >> 2);
              const uint32_t at = kk * (2 * TI) + ((G ^ (kk & 3)) << 5) + (i & 3) * 8;
              v[s] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(buf + (kT + t) * T::PT + at));
            }
            q[x][t] = bf16x8{v[0][0], v[0][1], v[0][2], v[0][3], v[1][0], v[1][1], v[1][2], v[1][3]};
          }
        }
      }
      products<kT, T::WB>(q, p, c, d);
    }
    if (k + 1 < steps) put(lds[(k + 1) & 1]);
    __syncthreads();
  }

  // A lane has row i, columns j .. j + 3 of each group.
  const int64_t op = (int64_t)g.np * g.width;
  const int t = kMode == kStore ? tensor_of(jobs, z) : 0;
#pragma unroll
  for (int x = 0; x < T::WB; ++x)
#pragma unroll
    for (int y = 0; y < T::WB; ++y)
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const int i = ti * TI + wi * (TI / 2) + y * 32 + lr, j = tj * TI + wj * (TI / 2) + x * 32 + 8 * s + 4 * lh;
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = c[x][y][4 * s + e] + d[x][y][4 * s + e];
        if constexpr (kMode != kGram) {
          const u16* old = g.X + z * kT * op + (int64_t)i * g.width + j;
          const float keep = kMode == kPoly ? jobs.b : jobs.a, mul = kMode == kPoly ? jobs.c : 1.0f;
          float o[4] = {};
#pragma unroll
          for (int w = kT - 1; w >= 0; --w) {          // smallest term first
            const uint2 r = *reinterpret_cast<const uint2*>(old + w * op);
            o[0] += bf16_lo(r.x); o[1] += bf16_hi(r.x); o[2] += bf16_lo(r.y); o[3] += bf16_hi(r.y);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = fmaf(keep, o[e], mul * v[e]);
        }
        if constexpr (kMode != kStore) {
          uint32_t a[kT], b[kT];
          split2<kT>(v[0], v[1], a);
          split2<kT>(v[2], v[3], b);
          u16* out = g.out + z * kT * op + (int64_t)i * g.width + j;
#pragma unroll
          for (int w = 0; w < kT; ++w) *reinterpret_cast<uint2*>(out + w * op) = make_uint2(a[w], b[w]);
        } else {
          const bool flip = jobs.rows > jobs.cols;
          const int64_t base = (int64_t)(z - jobs.first[t]) * jobs.rows * jobs.cols;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int r = flip ? j + e : i, cc = flip ? i : j + e;
            if (r >= jobs.rows || cc >= jobs.cols) continue;
            const int64_t at = base + (int64_t)r * jobs.cols + cc;
            if (jobs.m[t]) {
              float* w = static_cast<float*>(jobs.out[t]) + at;
              *w = fmaf(-jobs.rate, v[e], jobs.decay * *w);
            } else if (jobs.out_bf16) {
              static_cast<u16*>(jobs.out[t])[at] = to_bf16(v[e]);
            } else {
              static_cast<float*>(jobs.out[t])[at] = v[e];
            }
          }
        }
      }
}

// ---- plan ---------------------------------------------------------------------------
int64_t round_up(int64_t n, int64_t m) { return (n + m - 1) / m * m; }
size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

struct Plan {
  int n, L, np, lp, tile, chunks, mats, terms;
  size_t x0, x1, A, B, bytes;   // offsets; the partial sums come first
};
Plan plan_of(int rows, int cols, int mats, int terms) {
  Plan p;
  p.n = rows < cols ? rows : cols;
  p.L = rows < cols ? cols : rows;
  p.mats = mats;
  p.terms = terms;
  p.tile = 64;
  p.np = (int)round_up(p.n, p.tile);
  p.lp = (int)round_up(p.L, p.tile);
  p.chunks = (int)(((int64_t)rows * cols + kChunk - 1) / kChunk);
  const size_t part = align256((size_t)mats * p.chunks * sizeof(double));
  const size_t x = align256((size_t)mats * terms * p.np * p.lp * 2), a = align256((size_t)mats * terms * p.np * p.np * 2);
  p.x0 = part;
  p.x1 = p.x0 + x;
  p.A = p.x1 + x;
  p.B = p.A + a;
  p.bytes = p.B + a;
  return p;
}

template <int kMode, int kT, int TI>
void gemm(const GemmArgs& g, const Jobs& j, int mats, hipStream_t st) {
  hipLaunchKernelGGL((k_ns_gemm<kMode, kT, TI>), dim3(g.tiles_i * g.tiles_j, mats), dim3(kThreads), 0, st, g, j);
}

template <int kT, int TI>
hipError_t steps_of(const Plan& p, const Jobs& j, int steps, char* ws, hipStream_t st, Timer* tm) {
  double* part = reinterpret_cast<double*>(ws);
  u16 *x0 = reinterpret_cast<u16*>(ws + p.x0), *x1 = reinterpret_cast<u16*>(ws + p.x1);
  u16 *A = reinterpret_cast<u16*>(ws + p.A), *B = reinterpret_cast<u16*>(ws + p.B);
  if (tm) tm->begin("ns_norm");
  hipLaunchKernelGGL(k_ns_norm, dim3((unsigned)p.mats * p.chunks), dim3(kThreads), 0, st, j, p.chunks, part);
  if (tm) tm->end();
  if (tm) tm->begin("ns_split");
  hipLaunchKernelGGL((k_ns_split<kT>), dim3(p.lp / 64, p.np / 64, p.mats), dim3(kThreads), 0, st, j, p.chunks, part, x0,
                     p.np, p.lp);
  if (tm) tm->end();
  const int ti = p.np / TI, tl = p.lp / TI;
  for (int s = 0; s < steps; ++s) {
    if (tm) tm->begin("ns_gram");
    gemm<kGram, kT, TI>(GemmArgs{x0, x0, nullptr, A, p.np, p.lp, p.np, ti, ti}, j, p.mats, st);
    if (tm) tm->end();
    if (tm) tm->begin("ns_poly");
    gemm<kPoly, kT, TI>(GemmArgs{A, A, A, B, p.np, p.np, p.np, ti, ti}, j, p.mats, st);
    if (tm) tm->end();
    if (tm) tm->begin("ns_apply");
    const GemmArgs g{B, x0, x0, x1, p.np, p.np, p.lp, ti, tl};
    if (s + 1 < steps) gemm<kApply, kT, TI>(g, j, p.mats, st);
    else gemm<kStore, kT, TI>(g, j, p.mats, st);
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
    if (done[i]) continue;
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
    const size_t b = plan_of(a.rows, a.cols, total_of(js, list, n), js.out_bf16 ? 2 : 3).bytes;
    most = b > most ? b : most;
    return hipSuccess;
  });
  return most;
}

hipError_t launch_muon(const MatrixJobs& js, void* ws, hipStream_t st, Timer* tm) {
  return for_each_shape(js, [&](const int* list, int n) {
    const Job& a = js.job[list[0]];
    Jobs j{};
    j.n_tensors = n;
    for (int k = 0; k < n; ++k) {
      const Job& q = js.job[list[k]];
      j.src[k] = q.src;
      j.m[k] = q.m;
      j.out[k] = q.out;
      j.first[k + 1] = j.first[k] + q.count;
    }
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
    const Plan p = plan_of(a.rows, a.cols, j.first[n], js.out_bf16 ? 2 : 3);
    char* w = static_cast<char*>(ws);
    return js.out_bf16 ? steps_of<2, 64>(p, j, js.steps, w, st, tm) : steps_of<3, 64>(p, j, js.steps, w, st, tm);
  });
}

}  // namespace sagips
