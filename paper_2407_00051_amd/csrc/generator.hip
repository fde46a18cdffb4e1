// The GAN generator (noise -> parameters) of Sec. III, for a stack of M
// members of the same shape, and the ensemble response of Sec. VI-A.
//
// Network: IN -> H -> (H -> H) x NH -> OUT, LeakyReLU on the hidden layers,
// theta = 1 + softplus(last layer), so that every shape parameter is above 1.
// The paper's generator (51,206 parameters) is 6 -> 128 x 4 -> 6, i.e.
// H = 128, NH = 3.  Member m's parameters sit at W[l] + m * |W[l]|.
//
// Row tiles: T = 64 rows of the noise batch, or 16 when 64-row tiles of all
// members would leave most CUs idle (a single generator on 1,024 rows).
//
// Forward, 64-row tiles: one workgroup of 4 waves per (tile, member); the H x H
// products run on the bf16 matrix cores from split operands (split_bf16.hpp; see
// GenFwd).  16-row tiles take the forward pass below instead: with few tiles the
// time is one tile's latency, which splitting the weights lengthens (1,024 rows,
// one member: 12.9 us on 64 workgroups, 14.9 us split on 32).
//
// Backward (and the 16-row forward): one workgroup of 8 waves per (tile, member).
// The backward kernel recomputes the tile's forward pass (cheaper than storing it): the
// activations A_1 .. A_{NH+1} live in LDS as [T][H+4] fp32; the H x H products run on the fp32
// matrix cores (v_mfma_f32_16x16x4_f32) as out^T = W * in^T, each wave owning 16
// output features of all T rows.  The first layer (K = IN) and the last (N = OUT)
// are VALU work.  Then the backward pass from dL/dtheta: each backward signal
// overwrites the activation it replaces.  Weight gradients of the tile go to a
// per-tile partial; a second kernel sums the partials over tiles in a fixed
// order, so results are deterministic.
#include "device_math.hpp"
#include "kernels.hpp"
#include "split_bf16.hpp"

#include <string.h>

namespace sagips {
namespace {

constexpr int kGThreads = 512;   // 8 waves
constexpr int kGMaxIO = 8;       // largest IN / OUT

__device__ __forceinline__ f32x4 mfma4(float a, float b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ float g_leaky(float v, float s) { return v > 0.0f ? v : s * v; }
__device__ __forceinline__ float g_leaky_grad(float h, float s) { return h > 0.0f ? 1.0f : s; }
__device__ __forceinline__ float g_softplus(float t) { return fmaxf(t, 0.0f) + log1pf(expf(-fabsf(t))); }
__device__ __forceinline__ float g_sigmoid(float t) { return 1.0f / (1.0f + expf(-t)); }

// Workgroups are numbered L = x + y * gridDim.x and dealt to the 8 XCDs in
// turn (XCD = L mod 8); each XCD has its own L2.  The first 8 * floor(M / 8)
// members are placed so that all tiles of a member run on one XCD (member =
// 8 (j / tiles) + L mod 8, tile = j mod tiles, j = L / 8), so its weights are
// fetched into one L2 only; the remaining members are laid out in order.
__device__ __forceinline__ void gen_block(int tiles, int members, int& m, int& tile) {
  const int L = blockIdx.x + blockIdx.y * gridDim.x;
  const int m8 = members - members % 8;
  if (L < tiles * m8) {
    const int j = L >> 3;
    m = 8 * (j / tiles) + (L & 7);
    tile = j % tiles;
  } else {
    const int r = L - tiles * m8;
    m = m8 + r / tiles;
    tile = r % tiles;
  }
}

struct GenParams {
  const float* W[kMaxGenLayers];   // layer l of member 0; member m at + m * wsz[l]
  const float* b[kMaxGenLayers];
  int64_t wsz[kMaxGenLayers], bsz[kMaxGenLayers];
  int in, out;
  int64_t k;                       // rows of the noise batch
  float slope;
  const float* noise;              // [k][in], shared by every member
  float* theta;                    // forward: [M][k][out]
  const float* dtheta;             // backward: [M][k][out]
  float* part;                     // backward: [M][tiles][P]
  int64_t P;                       // floats per partial (all parameters of one member)
  int64_t poff_w[kMaxGenLayers], poff_b[kMaxGenLayers];
  // Members on rows of their own: noise, theta and dtheta are [k][..], of which member m has rows
  // offsets[m] .. offsets[m + 1] - 1.
  const int32_t* offsets;
  int members;
  float* dx;                       // backward: dL/dnoise [k][in], or NULL
  int* slots;                      // backward: [members][2]
  int64_t PS;                      // floats from one partial to the next
  const u16* split;                // backward, 64-row tiles: split copies of the hidden layers
};

// The rows of a tile: first, the first behind the member's rows, and what is added to a row for
// its place in theta.
struct GenTile {
  int m;
  int64_t row0, end, base;
};

// Member m's rows, whatever the offsets hold, lie within [0, k].
__device__ __forceinline__ void member_rows(const GenParams& p, int m, int64_t& lo, int64_t& hi) {
  lo = min(max((int64_t)p.offsets[m], (int64_t)0), p.k);
  hi = min(max((int64_t)p.offsets[m + 1], lo), p.k);
}

// The members' rows in tiles of T rows, in order; a member a lane, 64 at a time.  Up to 64 members stay in
// the lanes; of more, each search reads the offsets again.  The whole wave calls all of it.
template <int T>
struct RoutedRows {
  int lo, hi;                      // rows of member `lane`
  uint32_t upto;                   // tiles of members 0 .. lane
  int64_t tiles;                   // of all members

  __device__ __forceinline__ void read(const GenParams& p, int m0) {
    const int lane = threadIdx.x & 63, m = m0 + lane;
    int64_t a = 0, b = 0;
    if (m < p.members) member_rows(p, m, a, b);
    lo = (int)a;
    hi = (int)b;
    upto = count();                // 64 of them below 2^32: fewer than 2^29 rows
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t o = (uint32_t)__shfl_up((int)upto, d, 64);
      if (lane >= d) upto += o;
    }
  }
  __device__ __forceinline__ uint32_t count() const { return (uint32_t)((hi - lo + T - 1) / T); }
  __device__ __forceinline__ uint32_t sum() const { return (uint32_t)__builtin_amdgcn_readlane((int)upto, 63); }

  __device__ __forceinline__ explicit RoutedRows(const GenParams& p) {
    tiles = 0;
    for (int m0 = (p.members - 1) / 64 * 64; m0 >= 0; m0 -= 64) {   // the first 64 last: they stay
      read(p, m0);
      tiles += sum();
    }
  }
  // Tile `want` of all; false (only where the offsets do not rise, or want is not below tiles): there is none.
  __device__ __forceinline__ bool find(const GenParams& p, int64_t want, GenTile& t) const {
    RoutedRows r = *this;
    int64_t before = 0;
    for (int m0 = 0;;) {
      const uint64_t past = __ballot(before + r.upto > want);
      if (past) {
        const int src = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)past) - 1);
        t.m = m0 + src;
        const int first = __builtin_amdgcn_readlane(r.lo, src);
        t.end = __builtin_amdgcn_readlane(r.hi, src);
        t.row0 = first + (want - before - (uint32_t)__builtin_amdgcn_readlane((int)(r.upto - r.count()), src)) * T;
        t.base = 0;
        return true;
      }
      before += r.sum();
      m0 += 64;
      if (m0 >= p.members) return false;
      r.read(p, m0);
    }
  }
  // The workgroups of a backward pass, of which number g takes the tiles from g tiles / groups on, share the
  // partials of member m between them: slots[m] = (first, number), those of the workgroups that have tiles of it,
  // tile t being workgroup ((t + 1) groups - 1) / tiles's.  One workgroup writes it.
  __device__ __forceinline__ void write_slots(const GenParams& p, int64_t groups) const {
    if (threadIdx.x >= 64) return;
    RoutedRows r = *this;
    int64_t before = 0;
    for (int m0 = 0;;) {
      const int m = m0 + (int)threadIdx.x;
      if (m < p.members) {
        const uint32_t n = r.count();
        const int64_t t1 = before + r.upto, t0 = t1 - n;
        const int64_t g0 = n ? min(((t0 + 1) * groups - 1) / tiles, groups - 1) : 0;
        p.slots[2 * m] = (int)(g0 + m);
        p.slots[2 * m + 1] = n ? (int)(min((t1 * groups - 1) / tiles, groups - 1) - g0) + 1 : 0;
      }
      before += r.sum();
      m0 += 64;
      if (m0 >= p.members) return;
      r.read(p, m0);
    }
  }
};

// Tile of this workgroup.  Routed: the grid may hold more workgroups than there are tiles, and is a
// multiple of 8; an XCD (workgroup mod 8) takes tiles that follow each other.
template <int T, bool kRouted>
__device__ __forceinline__ bool gen_tile(const GenParams& p, GenTile& t) {
  if constexpr (kRouted) {
    const RoutedRows<T> r(p);
    return r.find(p, (int64_t)(blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3), t);
  } else {
    int tile;
    gen_block(gridDim.x, gridDim.y, t.m, tile);
    t.row0 = (int64_t)tile * T;
    t.end = p.k;
    t.base = (int64_t)t.m * p.k;
    return true;
  }
}

template <int H, int NH, int kGT>
struct Gen {
  static constexpr int LD = H + 4;
  static constexpr int WAVES = kGThreads / 64;
  static constexpr int KB = H / 16;
  static constexpr int CB = kGT / 16;
  static_assert(kGT == 16 || kGT == 64, "row tile");
  static constexpr int PPO = kGThreads / H;     // threads per feature in the VALU loops
  static_assert(H == 16 * WAVES, "one wave per 16 features");

  struct Smem {
    float act[NH + 1][kGT][LD];
    float n[kGT][kGMaxIO];
    float o[kGT][kGMaxIO];     // last-layer pre-activation
    float dout[kGT][kGMaxIO];  // dL/d(pre-activation of the last layer)
  };

  // out^T (16 features of this wave x 64 rows) = W[o][k] in[ev][k]; W row-major [H][H].
  static __device__ __forceinline__ void gemm_fwd(const float* __restrict__ W, const float* in, f32x4 (&acc)[CB],
                                                  int o0, int lr, int lg) {
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) acc[cb] = f32x4{0.f, 0.f, 0.f, 0.f};
    const float* wrow = W + (o0 + lr) * H + 4 * lg;
#pragma unroll 2
    for (int kb = 0; kb < KB; ++kb) {
      const f32x4 a = *reinterpret_cast<const f32x4*>(wrow + 16 * kb);
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) {
        const f32x4 bv = *reinterpret_cast<const f32x4*>(in + (16 * cb + lr) * LD + 16 * kb + 4 * lg);
#pragma unroll
        for (int s = 0; s < 4; ++s) acc[cb] = mfma4(a[s], bv[s], acc[cb]);
      }
    }
  }

  // out^T (16 input features k of this wave x 64 rows) = sum_o W[o][k] dl[ev][o]:
  // the backward-data product, reading W column-wise.
  static __device__ __forceinline__ void gemm_bwd(const float* __restrict__ W, const float* dl, f32x4 (&acc)[CB],
                                                  int k0, int lr, int lg) {
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) acc[cb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 2
    for (int kb = 0; kb < KB; ++kb) {
      const int o = 16 * kb + 4 * lg;
      f32x4 a;
#pragma unroll
      for (int s = 0; s < 4; ++s) a[s] = W[(o + s) * H + k0 + lr];
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) {
        const f32x4 bv = *reinterpret_cast<const f32x4*>(dl + (16 * cb + lr) * LD + o);
#pragma unroll
        for (int s = 0; s < 4; ++s) acc[cb] = mfma4(a[s], bv[s], acc[cb]);
      }
    }
  }

  // Forward pass of member m on rows [row0, row0 + 64) into LDS; rows from end on
  // carry zero noise.  Leaves A_1..A_{NH+1} in act and the last layer's
  // pre-activation in o.
  static __device__ void forward(const GenParams& p, Smem& sm, int m, int64_t row0, int64_t end) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int lr = lane & 15, lg = lane >> 4;
    const float slope = p.slope;
    for (int i = tid; i < kGT * kGMaxIO; i += kGThreads) {
      const int ev = i / kGMaxIO, j = i % kGMaxIO;
      const int64_t r = row0 + ev;
      sm.n[ev][j] = (j < p.in && r < end) ? p.noise[r * p.in + j] : 0.0f;
    }
    __syncthreads();
    {   // first layer: thread (feature o, part) over rows part, part + PPO, ...
      const int o = tid % H, part = tid / H;
      const float* W0 = p.W[0] + m * p.wsz[0];
      float w[kGMaxIO];
#pragma unroll
      for (int j = 0; j < kGMaxIO; ++j) w[j] = j < p.in ? W0[o * p.in + j] : 0.0f;
      const float bias = p.b[0][m * p.bsz[0] + o];
      for (int ev = part; ev < kGT; ev += PPO) {
        float v = bias;
#pragma unroll
        for (int j = 0; j < kGMaxIO; ++j) v = fmaf(w[j], sm.n[ev][j], v);
        sm.act[0][ev][o] = g_leaky(v, slope);
      }
    }
    __syncthreads();
    const int o0 = 16 * wave;
#pragma unroll
    for (int l = 0; l < NH; ++l) {
      f32x4 acc[CB];
      gemm_fwd(p.W[1 + l] + m * p.wsz[1 + l], &sm.act[l][0][0], acc, o0, lr, lg);
      const int o = o0 + 4 * lg;
      const f32x4 bias = *reinterpret_cast<const f32x4*>(p.b[1 + l] + m * p.bsz[1 + l] + o);
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) {
        f32x4 v = acc[cb] + bias;
        v.x = g_leaky(v.x, slope); v.y = g_leaky(v.y, slope);
        v.z = g_leaky(v.z, slope); v.w = g_leaky(v.w, slope);
        *reinterpret_cast<f32x4*>(&sm.act[l + 1][16 * cb + lr][o]) = v;
      }
      __syncthreads();
    }
    if ((tid >> 3) < kGT) {   // last layer: thread (row ev, part) sums features 4 part + 32 c (c < H / 32)
      const int ev = tid >> 3, part = tid & 7;
      const float* Wl = p.W[NH + 1] + m * p.wsz[NH + 1];
      const float* hrow = &sm.act[NH][ev][0];
      for (int j = 0; j < p.out; ++j) {
        float z = 0.f;
#pragma unroll
        for (int c = 0; c < H / 32; ++c) {
          const int f = 4 * part + 32 * c;
          const f32x4 hv = *reinterpret_cast<const f32x4*>(hrow + f);
          const f32x4 wv = *reinterpret_cast<const f32x4*>(Wl + j * H + f);
          z = fmaf(hv.x, wv.x, z); z = fmaf(hv.y, wv.y, z);
          z = fmaf(hv.z, wv.z, z); z = fmaf(hv.w, wv.w, z);
        }
#pragma unroll
        for (int s = 1; s < 8; s <<= 1) z += __shfl_xor(z, s, 64);
        if (part == 0) sm.o[ev][j] = z + p.b[NH + 1][m * p.bsz[NH + 1] + j];
      }
    }
    __syncthreads();
  }

  template <bool kRouted>
  static __device__ void run_forward(const GenParams& p) {
    __shared__ Smem sm;
    GenTile t;
    if (!gen_tile<kGT, kRouted>(p, t)) return;
    forward(p, sm, t.m, t.row0, t.end);
    for (int i = threadIdx.x; i < kGT * p.out; i += kGThreads) {
      const int ev = i / p.out, j = i % p.out;
      const int64_t r = t.row0 + ev;
      if (r < t.end) p.theta[(t.base + r) * p.out + j] = 1.0f + g_softplus(sm.o[ev][j]);
    }
  }

  static __device__ void run_backward(const GenParams& p) {
    __shared__ Smem sm;
    GenTile t;
    int tile;
    gen_block(gridDim.x, gridDim.y, t.m, tile);
    t.row0 = (int64_t)tile * kGT;
    t.end = p.k;
    t.base = (int64_t)t.m * p.k;
    backward_tile<false>(p, sm, t, p.part + ((int64_t)t.m * gridDim.x + tile) * p.P, false);
  }

  // Of the `tiles` tiles in the order of their rows, workgroup g of `groups` (at most one a tile) takes
  // those from g tiles / groups on, and adds up what it has of a member in slot g + m of the
  // partials: g + m rises from each of its (g, m) to the next.
  static __device__ void run_backward_routed(const GenParams& p) {
    __shared__ Smem sm;
    const RoutedRows<kGT> rr(p);
    const int64_t groups = min(rr.tiles, (int64_t)gridDim.x);
    const int64_t g = (int64_t)(blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3);
    if (blockIdx.x == 0) rr.write_slots(p, groups);
    if (g >= groups) return;
    int last = -1;
    for (int64_t i = g * rr.tiles / groups; i < (g + 1) * rr.tiles / groups; ++i) {
      GenTile t;
      if (!rr.find(p, i, t)) return;                 // (there is one)
      __syncthreads();                               // the tile before is read
      backward_tile<true>(p, sm, t, p.part + (g + t.m) * p.PS, t.m == last);
      last = t.m;
    }
  }

  // The gradients of a tile to `part`, or added to what it holds.
  template <bool kRouted>
  static __device__ __forceinline__ void backward_tile(const GenParams& p, Smem& sm, const GenTile& t, float* part, bool more) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int lr = lane & 15, lg = lane >> 4;
    const int m = t.m;
    const float slope = p.slope;
    const auto put = [&](float* at, float v) __attribute__((always_inline)) {
      if constexpr (kRouted) *at = more ? *at + v : v;
      else *at = v;
    };
    forward(p, sm, m, t.row0, t.end);

    // dL/d(last pre-activation) = dL/dtheta * sigmoid(o); zero on rows past the end
    for (int i = tid; i < kGT * kGMaxIO; i += kGThreads) {
      const int ev = i / kGMaxIO, j = i % kGMaxIO;
      const int64_t r = t.row0 + ev;
      float d = 0.f;
      if (j < p.out && r < t.end) d = p.dtheta[(t.base + r) * p.out + j] * g_sigmoid(sm.o[ev][j]);
      sm.dout[ev][j] = d;
    }
    __syncthreads();
    const int L = NH + 1;   // index of the last layer
    const float* WL = p.W[L] + m * p.wsz[L];
    {   // last layer: dW[j][k] = sum_ev dout[ev][j] A_{NH+1}[ev][k]; db[j] = sum_ev dout[ev][j]
      const int k = tid % H, g = tid / H;
      for (int j = g; j < p.out; j += PPO) {
        float s = 0.f;
        for (int ev = 0; ev < kGT; ++ev) s = fmaf(sm.dout[ev][j], sm.act[NH][ev][k], s);
        put(part + p.poff_w[L] + j * H + k, s);
      }
      if (tid < p.out) {
        float s = 0.f;
        for (int ev = 0; ev < kGT; ++ev) s += sm.dout[ev][tid];
        put(part + p.poff_b[L] + tid, s);
      }
    }
    __syncthreads();
    {   // delta_{NH+1} = (dout W_L) * leaky'(A_{NH+1}), in place
      const int k = tid % H, g = tid / H;
      float w[kGMaxIO];
#pragma unroll
      for (int j = 0; j < kGMaxIO; ++j) w[j] = j < p.out ? WL[j * H + k] : 0.0f;
      for (int ev = g; ev < kGT; ev += PPO) {
        float s = 0.f;
#pragma unroll
        for (int j = 0; j < kGMaxIO; ++j) s = fmaf(sm.dout[ev][j], w[j], s);
        float& h = sm.act[NH][ev][k];
        h = s * g_leaky_grad(h, slope);
      }
    }
    __syncthreads();
    const int o0 = 16 * wave;
#pragma unroll
    for (int l = NH - 1; l >= 0; --l) {
      // layer 1 + l maps A_{l+1} (act[l]) -> A_{l+2}; its output signal delta_{l+2} is in act[l+1]
      const float* dl = &sm.act[l + 1][0][0];
      float* A = &sm.act[l][0][0];
      {   // dW[o][k] = sum_ev delta[ev][o] A[ev][k]: rows o0.., 8 column blocks, K = 64 rows
        f32x4 acc[KB];
#pragma unroll
        for (int nb = 0; nb < KB; ++nb) acc[nb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int q = 0; q < kGT / 4; ++q) {
          const int ev = 4 * q + lg;
          const float a = dl[ev * LD + o0 + lr];
#pragma unroll
          for (int nb = 0; nb < KB; ++nb) acc[nb] = mfma4(a, A[ev * LD + 16 * nb + lr], acc[nb]);
        }
        float* dW = part + p.poff_w[1 + l];
#pragma unroll
        for (int nb = 0; nb < KB; ++nb)
#pragma unroll
          for (int r = 0; r < 4; ++r) put(dW + (o0 + 4 * lg + r) * H + 16 * nb + lr, acc[nb][r]);
        if (tid < H) {
          float s = 0.f;
          for (int ev = 0; ev < kGT; ++ev) s += dl[ev * LD + tid];
          put(part + p.poff_b[1 + l] + tid, s);
        }
      }
      __syncthreads();   // delta_{l+1} overwrites A_{l+1}, which every wave just read
      f32x4 acc[CB];
      gemm_bwd(p.W[1 + l] + m * p.wsz[1 + l], dl, acc, o0, lr, lg);
      const int k = o0 + 4 * lg;
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) {
        const int ev = 16 * cb + lr;
        f32x4 h = *reinterpret_cast<const f32x4*>(A + ev * LD + k);
        f32x4 v = acc[cb];
        v.x *= g_leaky_grad(h.x, slope); v.y *= g_leaky_grad(h.y, slope);
        v.z *= g_leaky_grad(h.z, slope); v.w *= g_leaky_grad(h.w, slope);
        *reinterpret_cast<f32x4*>(A + ev * LD + k) = v;
      }
      __syncthreads();
    }
    {   // first layer: dW[o][j] = sum_ev delta_1[ev][o] n[ev][j]; db[o] = sum_ev delta_1[ev][o]
      const int o = tid % H, g = tid / H;
      for (int j = g; j < p.in; j += PPO) {
        float s = 0.f;
        for (int ev = 0; ev < kGT; ++ev) s = fmaf(sm.act[0][ev][o], sm.n[ev][j], s);
        put(part + p.poff_w[0] + o * p.in + j, s);
      }
      if (g == 0) {
        float s = 0.f;
        for (int ev = 0; ev < kGT; ++ev) s += sm.act[0][ev][o];
        put(part + p.poff_b[0] + o, s);
      }
    }
    if constexpr (kRouted) {   // dx[ev][j] = sum_o delta_1[ev][o] W_0[o][j]
      if (p.dx) {
        const float* W0 = p.W[0] + m * p.wsz[0];
        for (int i = tid; i < kGT * p.in; i += kGThreads) {
          const int ev = i / p.in, j = i % p.in;
          float s = 0.f;
#pragma unroll 8
          for (int o = 0; o < H; ++o) s = fmaf(sm.act[0][ev][o], W0[o * p.in + j], s);
          if (t.row0 + ev < t.end) p.dx[(t.row0 + ev) * p.in + j] = s;
        }
      }
    }
  }
};

template <int H, int NH, int T>
__global__ __launch_bounds__(kGThreads, 1) void k_gen_backward(GenParams p) {
  Gen<H, NH, T>::run_backward(p);
}

template <int H, int NH>
__global__ __launch_bounds__(kGThreads, 1) void k_gen_backward_routed16(GenParams p) {
  Gen<H, NH, 16>::run_backward_routed(p);
}

template <int H, int NH, bool kRouted>
__global__ __launch_bounds__(kGThreads, 1) void k_gen_forward16(GenParams p) {
  Gen<H, NH, 16>::template run_forward<kRouted>(p);
}

// Forward pass on the bf16 matrix cores, H = 128.  Wave w owns features [32 w,
// 32 w + 32) of every layer for all 64 rows of the tile.  The activations live
// in LDS split (SplitLds) and are overwritten layer by layer, two barriers a
// layer; 52 KB, so three workgroups share a CU and the vector work of one runs
// beside the products of the others.  A member's weights are split as they are read: 8 values per
// lane and K step, between the products of the step before (44 instructions
// against 12 products of 32 cycles), which saves the pass over all members that
// a split copy would need.  The last hidden layer is formed with M = feature, so
// that a lane holds 16 features of its own rows and the output layer (N = OUT)
// needs only one exchange between the wave's halves and one between the waves.
// Bound by the matrix cores and the vector ALU together.  100 members x 1,024
// rows: 138 us with fp32 matrix instructions, 74 us now.
constexpr int kFwdThreads = 256;

template <int NH>
struct GenFwd : SplitLds<128, 64> {
  static constexpr int H = 128, KS = H / 16, MT = 2, R = 32 * MT, WAVES = 4, PD = 2;
  static_assert(WAVES * 32 == H && WAVES * 64 == kFwdThreads, "one wave per 32 features");

  struct Smem {
    union {
      char act[BUF];
      float op[WAVES][kGMaxIO][64];    // last layer: partials over a wave's features
    };
    union {
      float n[kGMaxIO][64];            // noise, transposed
      float wl[kGMaxIO][H];            // last layer's weights
    };
  };

  // 8 weights of row 32 wf + lr, columns 16 ks + 8 lh .. + 7.
  typedef f32x4 Raw[2];
  static __device__ __forceinline__ void split_raw(const Raw& r, bf16x8 (&w)[kTerms]) {
    uint32_t t[4][kTerms];
#pragma unroll
    for (int q = 0; q < 4; ++q) split_pair(r[q >> 1][2 * (q & 1)], r[q >> 1][2 * (q & 1) + 1], t[q]);
#pragma unroll
    for (int k = 0; k < kTerms; ++k) w[k] = __builtin_bit_cast(bf16x8, make_uint4(t[0][k], t[1][k], t[2][k], t[3][k]));
  }

  // acc[m] = act W^T for the wave's features and rows 32 m .. (kSwap: M = feature,
  // N = row).
  template <bool kSwap>
  static __device__ __forceinline__ void product(const float* __restrict__ W, const char* buf, const Lane& L,
                                                 f32x16 (&acc)[MT]) {
    const float* wrow = W + (32 * L.wf + L.lr) * H + 8 * L.lh;
    f32x16 corr[MT];
    Raw raw[PD + 1];
    bf16x8 w[2][kTerms], a[2][MT][kTerms];
    auto load = [&](int ks) __attribute__((always_inline)) {
#pragma unroll
      for (int q = 0; q < 2; ++q) raw[ks % (PD + 1)][q] = *reinterpret_cast<const f32x4*>(wrow + 16 * ks + 4 * q);
    };
#pragma unroll
    for (int q = 0; q < PD; ++q) load(q);
#pragma unroll
    for (int m = 0; m < MT; ++m) read_tr(buf, L, m, 0, a[0][m]);
    split_raw(raw[0], w[0]);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      __builtin_amdgcn_sched_barrier(0);
      if (ks + PD < KS) load(ks + PD);
      if (ks + 1 < KS) {
#pragma unroll
        for (int m = 0; m < MT; ++m) read_tr(buf, L, m, ks + 1, a[(ks + 1) & 1][m]);
        split_raw(raw[(ks + 1) % (PD + 1)], w[(ks + 1) & 1]);
      }
      if (ks == 0) split_mfma_apart<true, kSwap>(a[0], w[0], acc, corr);
      else split_mfma_apart<false, kSwap>(a[ks & 1], w[ks & 1], acc, corr);
      interleave<2, 8 / MT, 6 * MT>();
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int m = 0; m < MT; ++m) acc[m] += corr[m];
  }

  // A_1 of the wave's features (in <= J).
  template <int J>
  static __device__ __forceinline__ void first_layer(const GenParams& p, Smem& sm, int m, const Lane& L) {
    const int fo = 32 * L.wf + L.lr;
    const float* W0 = p.W[0] + m * p.wsz[0];
    float w[J];
#pragma unroll
    for (int j = 0; j < J; ++j) w[j] = j < p.in ? W0[fo * p.in + j] : 0.0f;
    const float bias = p.b[0][m * p.bsz[0] + fo];
#pragma unroll
    for (int s = 0; s < 2 * MT; ++s) {
      Step d;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        f32x4 v = {bias, bias, bias, bias};
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const f32x4 x = *reinterpret_cast<const f32x4*>(&sm.n[j][16 * s + 8 * u + 4 * L.lh]);
#pragma unroll
          for (int q = 0; q < 4; ++q) v[q] = fmaf(w[j], x[q], v[q]);
        }
        const float h[4] = {g_leaky(v.x, p.slope), g_leaky(v.y, p.slope), g_leaky(v.z, p.slope), g_leaky(v.w, p.slope)};
        split4(h, u, d);
      }
      store_step(sm.act, L, s, d);
    }
  }

  template <bool kRouted>
  static __device__ void run(const GenParams& p) {
    __shared__ __attribute__((aligned(1024))) Smem sm;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Lane L = make_lane(wave, 0);
    GenTile at;
    if (!gen_tile<R, kRouted>(p, at)) return;
    const int m = at.m;
    const int64_t row0 = at.row0;
    const float slope = p.slope;
    for (int i = tid; i < R * kGMaxIO; i += kFwdThreads) {
      const int ev = i % R, j = i / R;
      const int64_t r = row0 + ev;
      sm.n[j][ev] = (j < p.in && r < at.end) ? p.noise[r * p.in + j] : 0.0f;
    }
    __syncthreads();
    if (p.in <= 6) first_layer<6>(p, sm, m, L);
    else first_layer<kGMaxIO>(p, sm, m, L);
    __syncthreads();
    const float* WL = p.W[NH + 1] + m * p.wsz[NH + 1];
    for (int i = tid; i < p.out * H; i += kFwdThreads) sm.wl[i / H][i % H] = WL[i];
    f32x16 acc[MT];
#pragma unroll 1
    for (int l = 0; l < NH - 1; ++l) {
      const float bias = p.b[1 + l][m * p.bsz[1 + l] + 32 * L.wf + L.lr];
      product<false>(p.W[1 + l] + m * p.wsz[1 + l], sm.act, L, acc);
      __syncthreads();                           // every wave is done reading this layer's input
#pragma unroll
      for (int s = 0; s < 2 * MT; ++s) {
        Step d;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          float h[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) h[q] = g_leaky(acc[s >> 1][8 * (s & 1) + 4 * u + q] + bias, slope);
          split4(h, u, d);
        }
        store_step(sm.act, L, s, d);
        __builtin_amdgcn_sched_barrier(0);
      }
      __syncthreads();
    }
    // last hidden layer: lane = row 32 m + lr, register i = feature 32 wf + 8 (i / 4) + 4 lh + i % 4
    product<true>(p.W[NH] + m * p.wsz[NH], sm.act, L, acc);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const f32x4 bias = *reinterpret_cast<const f32x4*>(p.b[NH] + m * p.bsz[NH] + 32 * L.wf + 8 * g + 4 * L.lh);
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[t][4 * g + q] = g_leaky(acc[t][4 * g + q] + bias[q], slope);
    }
    __syncthreads();                             // act is read, wl staged
    for (int j = 0; j < p.out; ++j) {
      float z[MT];
#pragma unroll
      for (int t = 0; t < MT; ++t) z[t] = 0.f;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 wv = *reinterpret_cast<const f32x4*>(&sm.wl[j][32 * L.wf + 8 * g + 4 * L.lh]);
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
          for (int q = 0; q < 4; ++q) z[t] = fmaf(acc[t][4 * g + q], wv[q], z[t]);
      }
      // both halves' features; lanes 0..31 keep rows 0..31
      const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(z[0]), __float_as_uint(z[1]), false, false);
      sm.op[wave][j][L.lane] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    __syncthreads();
    for (int i = tid; i < R * p.out; i += kFwdThreads) {
      const int ev = i / p.out, j = i % p.out;
      const int64_t r = row0 + ev;
      float o = p.b[NH + 1][m * p.bsz[NH + 1] + j];
#pragma unroll
      for (int w = 0; w < WAVES; ++w) o += sm.op[w][j][ev];
      if (r < at.end) p.theta[(at.base + r) * p.out + j] = 1.0f + g_softplus(o);
    }
  }
};

template <int NH, bool kRouted>
__global__ __launch_bounds__(kFwdThreads, 3) void k_gen_forward(GenParams p) {
  GenFwd<NH>::template run<kRouted>(p);
}

// Split copies (split_bf16.hpp) of every member's hidden-to-hidden layers: of member m and layer l the copy
// of W at (2 NH m + l), that of W^T at (2 NH m + NH + l).  blockIdx.y = copy, blockIdx.z = member.
__global__ __launch_bounds__(256) void k_split_members(GenParams p, u16* out, int NH) {
  constexpr int H = 128, KS = H / 16;
  const int t = blockIdx.x * 256 + threadIdx.x, lane = t % 64, ks = t / 64 % KS, nb = t / (64 * KS);
  const int copy = blockIdx.y, l = copy % NH, m = blockIdx.z;
  const float* W = (l == 0 ? p.W[1] : l == 1 ? p.W[2] : p.W[3]) + (int64_t)m * H * H;
  const int n = 32 * nb + (lane & 31), k0 = 16 * ks + 8 * (lane >> 5);
  float v[8];
#pragma unroll
  for (int q = 0; q < 8; ++q) v[q] = copy >= NH ? W[(k0 + q) * H + n] : W[n * H + k0 + q];
  split_piece(v, out + ((size_t)m * 2 * NH + copy) * (split_copy_bytes(H) / 2), nb, ks, KS, lane);
}

// Backward pass of members on rows of their own, on the bf16 matrix cores.  One workgroup of 8 waves takes
// tiles of up to 64 rows of a member, in blocks of 32: wave (wf, we) owns features [32 wf, 32 wf + 32) of
// block we, so that the two waves of a SIMD share its matrix core and one's vector work runs beside the
// other's products; a tile of one block leaves the second wave idle and takes half the time.  The
// activations A_1 .. A_NH live split in three buffers (144 KB); the top signal takes A_1's place, which is
// formed again after it.  Every other signal overwrites the activation it belongs to.  Weights come split
// (k_split_members): splitting them as they are read took as long as the products.  A weight
// gradient has K = the tile's rows; each wave has 32 x 64 of it, in the accumulation registers
// for as long as the workgroup stays with a member.
// What decides its time is the code that a workgroup runs once and the registers: a product, its epilogue and
// the stores are there once, in a loop over the 2 NH products (unrolled, 53 KB of code that most workgroups
// run for one tile only, and 265 spilled registers).
template <int NH>
struct GenBwd : SplitLds<128, 64> {
  static constexpr int H = 128, KS = H / 16, PD = 3;
  static constexpr int NBUF = NH < 3 ? NH + 1 : 3, kTop = NH < 3 ? NH : 0;
  static constexpr uint32_t kCopy = (uint32_t)split_copy_bytes(H), kStep = kTerms * 1024;

  struct Smem {
    char act[NBUF * BUF];
    float n[kGMaxIO][64];          // inputs, transposed
    float dout[kGMaxIO][64];       // dL/d(last pre-activation)
    float w0[kGMaxIO][H];          // the member's first layer, transposed, and its last
    float wo[kGMaxIO][H];
    float bias[NH + 1][H], bo[kGMaxIO];
  };
  // Where a member's gradients lie in its partial.
  static constexpr int kHidden = H * H + H;
  static __device__ __forceinline__ int at_hidden(int in, int l) { return H * in + H + l * kHidden; }
  // The wave and the lane, and the lane's offsets in a buffer.
  struct Me {
    int lane, lr, lh, wf, we, fo;
    uint32_t own[2], tr[2];        // units of the block's two 16-row steps; transposed reads of the block
    uint32_t woff;                 // in a split copy
  };
  // An offset for one phase: kept from phase to phase, what the compiler forms of it beforehand would take
  // more registers than there are.
  static __device__ __forceinline__ uint32_t fresh(uint32_t o) {
    asm volatile("" : "+v"(o));
    return o;
  }
  // Sums over the rows of the lane's feature that a wave keeps of a member.
  struct Sums {
    f32x16 W[NH][2];               // rows 32 wf .., columns 64 we .. of a hidden layer's gradient
    float b[NH + 1], bo;
    float in[kGMaxIO / 2], out[kGMaxIO / 2];   // first and last layer: lane half lh has columns 2 k + lh, over both halves' rows
  };
  typedef bf16x8 Ring[PD + 1][kTerms];   // weight steps: the next product's first three between products

  static __device__ __forceinline__ void load_w(Rsrc R, uint32_t woff, uint32_t at, bf16x8 (&w)[kTerms]) {
#pragma unroll
    for (int t = 0; t < kTerms; ++t) w[t] = split_load(R, woff + t * 1024u, at);
  }
  static __device__ __forceinline__ void read_rows(const char* at0, const char* at1, int o, bf16x8 (&a)[kTerms]) {
#pragma unroll
    for (int t = 0; t < kTerms; ++t) {
      const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(at0 + t * PL + o));
      const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(at1 + t * PL + o));
      a[t] = bf16x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    }
  }

  // act B for the wave's features and block, B the split copy at `copy` (bytes); w holds the copy's first steps,
  // and in the end those of the one at `next`.
  static __device__ __forceinline__ f32x16 product(Rsrc R, uint32_t copy, uint32_t next, Ring& w, const char* buf, const Me& L) {
    f32x16 acc[1] = {}, corr[1] = {};
    bf16x8 a[2][1][kTerms];
    const char *at0 = buf + L.tr[0], *at1 = buf + L.tr[1];
    read_rows(at0, at1, 0, a[0][0]);
    uint32_t more = copy + PD * kStep;
#pragma unroll 1
    for (int half = 0; half < 2; ++half) {
      // the step behind the half: the other half's first, or (unused) the first again
      const int turn = half ? -3 * 16 * RB - 4 * 16 * RB : 16 * RB;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        __builtin_amdgcn_sched_barrier(0);
        load_w(R, L.woff, more, w[(q + PD) % (PD + 1)]);
        more = q == 0 && half ? next : more + kStep;   // step 7 is loaded at step 4
        read_rows(at0, at1, q < 3 ? 16 * RB : turn, a[(q + 1) & 1][0]);
        at0 += q < 3 ? 16 * RB : turn;
        at1 += q < 3 ? 16 * RB : turn;
        __builtin_amdgcn_sched_barrier(0);
        split_mfma_apart<false, false>(a[q & 1], w[q], acc, corr);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    return acc[0] + corr[0];
  }

  // W += signal^T A over `steps` times 16 rows.
  static __device__ __forceinline__ void wgrad(const char* sig, const char* A, const Me& L, int steps, f32x16 (&W)[2]) {
    const char *s0 = sig + L.lr * RB + L.wf * 32 * RB, *a0 = A + L.lr * RB + L.we * 64 * RB;
#pragma unroll 1
    for (int s = 0; s < steps; ++s) {
      bf16x8 a[kTerms], b[2][kTerms];
      const uint32_t o = ((uint32_t)(2 * s + L.lh) ^ swz(L.lr)) << 4;
#pragma unroll
      for (int t = 0; t < kTerms; ++t) {
        a[t] = *reinterpret_cast<const bf16x8*>(s0 + o + t * PL);
#pragma unroll
        for (int k = 0; k < 2; ++k) b[k][t] = *reinterpret_cast<const bf16x8*>(a0 + o + t * PL + k * 32 * RB);
      }
      split_mfma2(b[0], b[1], a, W[0], W[1], W[0], W[1]);
    }
  }

  // 16 values of the lane's feature (rows 32 we + 8 (i / 4) + 4 lh + i % 4), split, into a buffer.
  static __device__ __forceinline__ void store_block(char* buf, const Me& L, const float (&v)[16]) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      Step d;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const float h[4] = {v[8 * s + 4 * u], v[8 * s + 4 * u + 1], v[8 * s + 4 * u + 2], v[8 * s + 4 * u + 3]};
        split4(h, u, d);
      }
      char* at = buf + fresh(L.own[s]);
#pragma unroll
      for (int t = 0; t < kTerms; ++t) *reinterpret_cast<uint4*>(at + t * PL) = make_uint4(d[t][0], d[t][1], d[t][2], d[t][3]);
    }
  }
  // v[i] = c + sum_j w[j][fo] x[j][row]: a layer of few inputs, for the wave's features and rows.
  static __device__ __forceinline__ void from_few(const float (&w)[kGMaxIO][H], const float (&x)[kGMaxIO][64], float c, int n, const Me& L,
                                                  float (&v)[16]) {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = c;
    const float *e0 = &x[0][32 * L.we + 4 * L.lh], *w0 = &w[0][L.fo];
#pragma unroll 2
    for (int j = 0; j < n; ++j) {
      const float wj = w0[j * H];
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 e = *reinterpret_cast<const f32x4*>(e0 + 64 * j + 8 * g);
#pragma unroll
        for (int q = 0; q < 4; ++q) v[4 * g + q] = fmaf(wj, e[q], v[4 * g + q]);
      }
    }
  }
  // LeakyReLU of A_1 or of a hidden layer: the signs as bits, and the values.
  static __device__ __forceinline__ uint32_t signs(const float (&v)[16]) {
    uint32_t k = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) k |= v[i] > 0.0f ? 1u << i : 0u;
    return k;
  }
  static __device__ __forceinline__ void leak(float (&v)[16], uint32_t positive, float slope) {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] *= positive >> i & 1 ? 1.0f : slope;
  }
  static __device__ __forceinline__ uint32_t first_layer(Smem& sm, int in, float slope, const Me& L) {
    float v[16];
    from_few(sm.w0, sm.n, sm.bias[0][L.fo], in, L, v);
    const uint32_t k = signs(v);
    leak(v, k, slope);
    store_block(sm.act, L, v);
    return k;
  }
  // op[wf][j][row] = sum over the wave's features of v[i] w[j][fo], two columns j at a time.
  typedef float Op[kGMaxIO][64];
  static __device__ __forceinline__ void over_features(Op* op, const Me& L, const float (&v)[16], const float (&w)[kGMaxIO][H], int n) {
    const int i = L.lr & 15, row = 32 * L.we + 8 * (i >> 2) + 4 * L.lh + (i & 3);
    const float* w0 = &w[0][L.fo];
#pragma unroll 1
    for (int j = 0; j < n; j += 2) {
      const float wa = w0[j * H], wb = w0[(j + 1) * H];   // rows behind the last are 0
      float z[32];
#pragma unroll
      for (int k = 0; k < 16; ++k) z[k] = v[k] * wa, z[16 + k] = v[k] * wb;
      op[L.wf][j + (L.lr >> 4)][row] = half_scatter_sum(z, L.lr);
    }
  }
  // The sums over a lane's rows of v[i] x[j][row], added over the halves: column 2 k + lh to s[k].
  static __device__ __forceinline__ void over_rows(const Me& L, const float (&v)[16], const float (&x)[kGMaxIO][64], int n,
                                                   float (&s)[kGMaxIO / 2]) {
    const float* e0 = &x[0][32 * L.we + 4 * L.lh];
#pragma unroll
    for (int k = 0; k < kGMaxIO / 2; ++k) {
      if (2 * k >= n) break;
      float t[2] = {};
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const f32x4 e = *reinterpret_cast<const f32x4*>(e0 + 64 * (2 * k + h) + 8 * g);
#pragma unroll
          for (int q = 0; q < 4; ++q) t[h] = fmaf(v[4 * g + q], e[q], t[h]);
        }
      const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(t[0]), __float_as_uint(t[1]), false, false);
      s[k] += __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
  }
  static __device__ __forceinline__ float total_of(const float (&v)[16]) {
    float t = 0.0f;
#pragma unroll
    for (int g = 0; g < 4; ++g) t += (v[4 * g] + v[4 * g + 1]) + (v[4 * g + 2] + v[4 * g + 3]);
    return t;
  }

  // A thread's input and dL/dtheta of a tile: row ev, column col of both.
  struct Inputs {
    float x, d;
  };
  static __device__ __forceinline__ Inputs inputs(const GenParams& p, const GenTile& t, int rows) {
    const int ev = min((int)(threadIdx.x & 63), rows - 1), col = threadIdx.x >> 6;
    return {p.noise[(t.row0 + ev) * p.in + min(col, p.in - 1)], p.dtheta[(t.row0 + ev) * p.out + min(col, p.out - 1)]};
  }

  // A tile: `rows` (1 to 64) rows of a member from row0 on.
  static __device__ __forceinline__ void tile(const GenParams& p, Smem& sm, const Me& L, int64_t row0, int rows, Inputs given, Rsrc R,
                                              Ring& w, Sums& S) {
    const int steps = rows > 32 ? 4 : 2;
    const bool on = rows > 32 * L.we;                // the wave has a block
    const float slope = p.slope;
    const auto buf = [&](int i) __attribute__((always_inline)) { return sm.act + i * BUF; };
    const int ev = threadIdx.x & 63, col = threadIdx.x >> 6;   // a thread's row and column of the inputs and outputs
    sm.n[col][ev] = ev < rows && col < p.in ? given.x : 0.0f;
    sm.dout[col][ev] = ev < rows && col < p.out ? given.d : 0.0f;
    __syncthreads();
    uint64_t mask = 0;                               // bit 16 l + i: value i of A_{l+1} positive
    float v[16];
    if (on) mask = first_layer(sm, p.in, slope, L);
    __syncthreads();
    // The products: layer 1 + l maps A_{l+1} (buffer l) -> A_{l+2}, forward in turn, then the signals back.
#pragma unroll 1
    for (int st = 0; st < 2 * NH; ++st) {
      const bool fwd = st < NH;
      const int l = fwd ? st : 2 * NH - 1 - st;
      const char* from = buf(fwd ? l : l == NH - 1 ? kTop : l + 1);
      if (st == NH) {
        // output layer: v = A_{NH+1}; its sums lie where the top signal will
        Op* op = reinterpret_cast<Op*>(buf(kTop));
        if (on) over_features(op, L, v, sm.wo, p.out);
        __syncthreads();
        if (col < p.out && ev < rows) {   // dL/d(last pre-activation) = dL/dtheta * sigmoid(o); zero on rows past the end
          const float o = sm.bo[col] + ((op[0][col][ev] + op[1][col][ev]) + (op[2][col][ev] + op[3][col][ev]));
          const float d = sm.dout[col][ev] * g_sigmoid(o);
          sm.dout[col][ev] = d;
          S.bo += d;
        }
        __syncthreads();
        if (on) {
          over_rows(L, v, sm.dout, p.out, S.out);
          from_few(sm.wo, sm.dout, 0.0f, p.out, L, v);
          leak(v, (uint32_t)(mask >> 16 * NH), slope);
          S.b[NH] += total_of(v);
          store_block(buf(kTop), L, v);
        }
        __syncthreads();
      }
      if (!fwd) {                                    // (a choice: an index would put the sums into memory)
        if (l == 0) wgrad(from, buf(0), L, steps, S.W[0]);
        else if (l == 1) wgrad(from, buf(1), L, steps, S.W[NH > 1 ? 1 : 0]);
        else wgrad(from, buf(2), L, steps, S.W[NH > 2 ? 2 : 0]);
      }
      if (on) {
        // copies 0 .. NH - 1 forward, NH .. 2 NH - 1 the transposed ones, from the last back; then the next tile's first
        const int copy = fwd ? st : NH + l, next = st < NH - 1 ? st + 1 : st == NH - 1 ? 2 * NH - 1 : l > 0 ? copy - 1 : 0;
        const f32x16 acc = product(R, copy * kCopy, next * kCopy, w, from, L);
        const float bias = fwd ? sm.bias[1 + l][L.fo] : 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = acc[i] + bias;
        if (fwd) mask |= (uint64_t)signs(v) << 16 * (l + 1);
        leak(v, (uint32_t)(mask >> 16 * (fwd ? l + 1 : l)), slope);
        if (!fwd) {
          const float t = total_of(v);
#pragma unroll
          for (int k = 0; k < NH; ++k) S.b[k] += k == l ? t : 0.0f;
        }
      }
      if (st == 2 * NH - 1) break;                   // v = delta_1
      if (!fwd) __syncthreads();                     // every wave is done with buffer l and the signal
      if (on && st != NH - 1) store_block(buf(fwd ? l + 1 : l), L, v);
      if (kTop == 0 && st == NH && on) (void)first_layer(sm, p.in, slope, L);
      __syncthreads();
    }
    // ---- first layer
    if (on) over_rows(L, v, sm.n, p.in, S.in);
    if (p.dx) {
      Op* od = reinterpret_cast<Op*>(buf(NBUF - 1));   // of three buffers the last products read the others
      if (NH == 1) __syncthreads();
      if (on) over_features(od, L, v, sm.w0, p.in);
      __syncthreads();
      if (ev < rows && col < p.in) p.dx[(row0 + ev) * p.in + col] = (od[0][col][ev] + od[1][col][ev]) + (od[2][col][ev] + od[3][col][ev]);
    }
  }

  // What the workgroup has of a member, to its partial.  The two blocks' sums of a feature meet in LDS.
  static __device__ __forceinline__ void flush(const GenParams& p, Smem& sm, const Me& L, float* part, const Sums& S) {
    const int in = p.in, out = p.out;
    float* at = part + at_hidden(in, 0) + (32 * L.wf + 4 * L.lh) * H + 64 * L.we + L.lr;
#pragma unroll
    for (int l = 0; l < NH; ++l, at += kHidden - 32 * H)
#pragma unroll
      for (int g = 0; g < 4; ++g, at += 8 * H)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int k = 0; k < 2; ++k) at[i * H + 32 * k] = S.W[l][k][4 * g + i];
    constexpr int K = kGMaxIO / 2;
    float (*stage)[2][H] = reinterpret_cast<float (*)[2][H]>(sm.act);   // [value][lane half][feature]
    __syncthreads();                                 // act is read
    if (L.we == 1) {
#pragma unroll
      for (int k = 0; k < K; ++k) stage[k][L.lh][L.fo] = S.in[k], stage[K + k][L.lh][L.fo] = S.out[k];
#pragma unroll
      for (int l = 0; l <= NH; ++l) stage[2 * K + l][L.lh][L.fo] = S.b[l];
    }
    __syncthreads();
    if (L.we == 0) {
      float* last = part + at_hidden(in, NH);        // [out][H], then out biases
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int j = 2 * k + L.lh;
        if (j < in) part[L.fo * in + j] = S.in[k] + stage[k][L.lh][L.fo];
        if (j < out) last[j * H + L.fo] = S.out[k] + stage[K + k][L.lh][L.fo];
      }
#pragma unroll
      for (int l = 0; l <= NH; ++l) {
        const float s = add_xor32(S.b[l] + stage[2 * K + l][L.lh][L.fo]);
        if (L.lh == 0) part[(l == 0 ? H * in : at_hidden(in, l - 1) + H * H) + L.fo] = s;
      }
    }
    const float bo = wave_total(S.bo);
    if (L.lane == 0 && (int)(threadIdx.x >> 6) < out) part[at_hidden(in, NH) + out * H + (threadIdx.x >> 6)] = bo;
  }

  // Of the `blocks` blocks of 32 rows in the order of their rows, workgroup g of `groups` (at most one a
  // block) takes those from g blocks / groups on, two of a member together; what it has of a member goes to
  // slot g + m of the partials: g + m rises from each of its (g, m) to the next.
  static __device__ void run(const GenParams& p) {
    __shared__ __attribute__((aligned(1024))) Smem sm;
    const RoutedRows<32> rr(p);
    const int64_t groups = min(rr.tiles, (int64_t)gridDim.x);
    const int64_t g = (int64_t)(blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3);
    if (blockIdx.x == 0) rr.write_slots(p, groups);
    if (g >= groups) return;
    Me L;
    {
      const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
      const Lane A = make_lane(wave & 3, 0);
      L.lane = A.lane;
      L.lr = A.lr;
      L.lh = A.lh;
      L.wf = A.wf;
      L.we = wave >> 2;
      L.fo = 32 * L.wf + L.lr;
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        L.own[q] = (L.we ? A.w[2 + q] : A.w[q]) + (uint32_t)L.wf * 32 * RB;
        L.tr[q] = L.we ? A.tr[1][q] : A.tr[0][q];
      }
      L.woff = (uint32_t)(L.wf * KS * kTerms * 64 + L.lane) * 16u;
    }
    int64_t i = g * rr.tiles / groups;
    const int64_t end = (g + 1) * rr.tiles / groups;
    GenTile t;
    bool more = rr.find(p, i, t);                    // (there is one)
    while (more) {                                   // a member
      const int m = t.m;
      const Rsrc R = split_rsrc(p.split + (size_t)m * 2 * NH * (kCopy / 2), 2 * NH * kCopy);
      Ring w;
#pragma unroll
      for (int q = 0; q < PD; ++q) load_w(R, L.woff, q * kStep, w[q]);
      int rows = (int)min(t.end - t.row0, (int64_t)(i + 1 < end ? 64 : 32));
      Inputs given = inputs(p, t, rows);
      // all reads before the first is used
      const int f = threadIdx.x % H, j0 = threadIdx.x / H;   // 4 columns at a time
      const float *W0 = p.W[0] + (int64_t)m * H * p.in + f * p.in, *WL = p.W[NH + 1] + (int64_t)m * H * p.out + f;
      float e0[2], eo[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        e0[k] = W0[min(j0 + 4 * k, p.in - 1)];
        eo[k] = WL[min(j0 + 4 * k, p.out - 1) * H];
      }
      const float* bias = j0 == 0 ? p.b[0] : NH == 1 || j0 == 1 ? p.b[1] : NH == 2 || j0 == 2 ? p.b[2] : p.b[3];
      const float eb = bias[(int64_t)m * H + f], ebo = p.b[NH + 1][(int64_t)m * p.out + min(f, p.out - 1)];
      __syncthreads();                               // the member before is read
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        sm.w0[j0 + 4 * k][f] = j0 + 4 * k < p.in ? e0[k] : 0.0f;
        sm.wo[j0 + 4 * k][f] = j0 + 4 * k < p.out ? eo[k] : 0.0f;
      }
      if (j0 <= NH) sm.bias[j0][f] = eb;
      if (threadIdx.x < kGMaxIO) sm.bo[threadIdx.x] = ebo;
      Sums S = {};
      bool same;
      do {
        // the next tile, its inputs read while this one is worked on
        const int64_t row0 = t.row0;
        const int now = rows;
        const Inputs here = given;
        i += rows > 32 ? 2 : 1;
        t.row0 += rows;
        more = i < end;
        if (more && t.row0 >= t.end) more = rr.find(p, i, t);
        same = more && t.m == m;
        if (same) {
          rows = (int)min(t.end - t.row0, (int64_t)(i + 1 < end ? 64 : 32));
          given = inputs(p, t, rows);
        }
        __syncthreads();                             // the tile before is read
        tile(p, sm, L, row0, now, here, R, w, S);
      } while (same);
      flush(p, sm, L, p.part + (g + m) * p.PS, S);
    }
  }
};

template <int NH>
__global__ __launch_bounds__(kGThreads, 1) void k_gen_backward_routed(GenParams p) {
  GenBwd<NH>::run(p);
}

// Sum of the per-tile partials of member blockIdx.y in a fixed order, scattered
// to the caller's gradient arrays.
struct GenReduceArgs {
  const float* part;
  int64_t P;
  int tiles;
  int n_layers;
  int64_t poff_w[kMaxGenLayers], poff_b[kMaxGenLayers], wsz[kMaxGenLayers], bsz[kMaxGenLayers];
  float* dW[kMaxGenLayers];
  float* db[kMaxGenLayers];
};

// s += the values of tiles t, t + S, ..., up to N of them, loaded together.
template <int S, int N>
__device__ __forceinline__ void add_tiles(const float* src, int t, int tiles, int64_t P, float& s) {
  float x[N];
#pragma unroll
  for (int u = 0; u < N; ++u) x[u] = src[(int64_t)min(t + u * S, tiles - 1) * P];
#pragma unroll
  for (int u = 0; u < N; ++u) s += t + u * S < tiles ? x[u] : 0.f;
}

// S tile slices summed side by side, then combined in order: four, or one where there are
// no more tiles than that (the same sum; four slices then are blocks of mostly idle waves:
// 300 members of one tile 134 us against 69, 100 members 47 against 25).  Eight tiles'
// loads in flight (one by one, 16 tiles a slice are 16 round trips), and fewer for a last
// group that is shorter; a slice is a whole number of waves, so that no branch diverges.
template <int S>
__global__ __launch_bounds__(256) void k_gen_reduce(GenReduceArgs r) {
  constexpr int C = 256 / S;
  const int m = blockIdx.y;
  const int le = threadIdx.x % C, sl = threadIdx.x / C;
  const int64_t e = (int64_t)blockIdx.x * C + le;
  float v = 0.f;
  if (e < r.P) {
    const float* src = r.part + (int64_t)m * r.tiles * r.P + e;
    int t = sl;
    for (; t + 4 * S < r.tiles; t += 8 * S) add_tiles<S, 8>(src, t, r.tiles, r.P, v);
    if (t + 2 * S < r.tiles) add_tiles<S, 4>(src, t, r.tiles, r.P, v);
    else if (t < r.tiles) add_tiles<S, 2>(src, t, r.tiles, r.P, v);
  }
  if constexpr (S > 1) {
    __shared__ float red[S][C];
    red[sl][le] = v;
    __syncthreads();
    if (sl != 0) return;
    v = 0.f;
#pragma unroll
    for (int q = 0; q < S; ++q) v += red[q][le];
  }
  if (e >= r.P) return;
  for (int l = 0; l < r.n_layers; ++l) {
    if (e >= r.poff_w[l] && e < r.poff_w[l] + r.wsz[l]) { r.dW[l][m * r.wsz[l] + (e - r.poff_w[l])] = v; return; }
    if (e >= r.poff_b[l] && e < r.poff_b[l] + r.bsz[l]) { r.db[l][m * r.bsz[l] + (e - r.poff_b[l])] = v; return; }
  }
}

// The same for members on rows of their own: member blockIdx.y's partials are slots[m]'s.  A thread takes four
// values (partials are padded to 16 bytes), four slices of the partials side by side: with one value a thread
// the blocks of 100 members took 51 us, four times as many as these.
__global__ __launch_bounds__(256) void k_gen_reduce_routed(GenReduceArgs r, const int* __restrict__ slots, int64_t PS) {
  constexpr int S = 4, C = 256 / S;
  __shared__ f32x4 red[S][C];
  const int m = blockIdx.y, first = slots[2 * m], n = slots[2 * m + 1];
  const int le = threadIdx.x % C, sl = threadIdx.x / C;
  const int64_t e0 = ((int64_t)blockIdx.x * C + le) * 4;
  f32x4 v = {};
  if (e0 < r.P) {
    const float* src = r.part + (int64_t)first * PS + e0;
    for (int t = sl; t < n; t += 4 * S) {
      f32x4 x[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) x[u] = *reinterpret_cast<const f32x4*>(src + (int64_t)min(t + u * S, n - 1) * PS);
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (t + u * S < n) v += x[u];
    }
  }
  red[sl][le] = v;
  __syncthreads();
  // thread (value q of a group of four): all 256 write, one each
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (e >= r.P) return;
  float t = 0.f;
#pragma unroll
  for (int q = 0; q < S; ++q) t += reinterpret_cast<const float*>(&red[q][0])[threadIdx.x];
  for (int l = 0; l < r.n_layers; ++l) {
    if (e >= r.poff_w[l] && e < r.poff_w[l] + r.wsz[l]) { r.dW[l][m * r.wsz[l] + (e - r.poff_w[l])] = t; return; }
    if (e >= r.poff_b[l] && e < r.poff_b[l] + r.bsz[l]) { r.db[l][m * r.bsz[l] + (e - r.poff_b[l])] = t; return; }
  }
}

// Ensemble statistics of theta[M][k][out]: per (row, component) the member
// mean and the population standard deviation about it; rowstat[0][r][c] = mean,
// rowstat[1][r][c] = sigma.  A block has 16 (row, component) pairs side by side,
// so that a load is 64 contiguous bytes of a member, and 16 slices of the members:
// slice j takes members j, j + 16, ..., and the sixteen partial sums are added in
// a fixed tree.  A slice's first kEnsKeep members are loaded together and kept for
// the second pass, so that up to 128 members are one round trip to memory (100
// members on 1,024 rows, with k_ens_final's 1,024 threads: 79.7 -> 76.3 us a call
// of the ensemble response).
constexpr int kEnsCols = 16, kEnsSlices = 16, kEnsKeep = 8;

__global__ __launch_bounds__(256) void k_ens_rows(const float* __restrict__ theta, int M, int64_t k, int out,
                                                  float* __restrict__ rowstat) {
  __shared__ float red[2][4][kEnsCols];
  const int il = threadIdx.x % kEnsCols, j = threadIdx.x / kEnsCols, wave = threadIdx.x >> 6;
  const int64_t stride = k * out;
  const int64_t i = (int64_t)blockIdx.x * kEnsCols + il;
  const float* src = theta + min(i, stride - 1);
  // over the slices: 2 bits within a wave, 2 across the waves
  auto total = [&](float v, int pass) __attribute__((always_inline)) {
    v += __shfl_xor(v, 16, 64);
    v += __shfl_xor(v, 32, 64);
    if ((threadIdx.x & 63) < kEnsCols) red[pass][wave][il] = v;
    __syncthreads();
    return (red[pass][0][il] + red[pass][1][il]) + (red[pass][2][il] + red[pass][3][il]);
  };
  float x[kEnsKeep];
#pragma unroll
  for (int u = 0; u < kEnsKeep; ++u) x[u] = src[min(j + u * kEnsSlices, M - 1) * stride];
  float s = 0.f;
#pragma unroll
  for (int u = 0; u < kEnsKeep; ++u) s += j + u * kEnsSlices < M ? x[u] : 0.f;
#pragma unroll 4
  for (int m = j + kEnsKeep * kEnsSlices; m < M; m += kEnsSlices) s += src[m * stride];
  const float mean = total(s, 0) / (float)M;
  float q = 0.f;
#pragma unroll
  for (int u = 0; u < kEnsKeep; ++u) {
    const float dv = j + u * kEnsSlices < M ? x[u] - mean : 0.f;
    q = fmaf(dv, dv, q);
  }
#pragma unroll 4
  for (int m = j + kEnsKeep * kEnsSlices; m < M; m += kEnsSlices) {
    const float dv = src[m * stride] - mean;
    q = fmaf(dv, dv, q);
  }
  q = total(q, 1);
  if (i < stride && j == 0) {
    rowstat[i] = mean;
    rowstat[stride + i] = sqrtf(q / (float)M);
  }
}

// Batch averages of the row statistics (one workgroup): thread (component
// c, slice q) sums rows q, q + 128, ... of component c (out <= 8); the 128
// slices of a component are then added in a fixed tree.
constexpr int kEnsFinal = 1024;

__global__ __launch_bounds__(kEnsFinal) void k_ens_final(const float* __restrict__ rowstat, int64_t k, int out,
                                                   const float* __restrict__ p_true, float* __restrict__ p_hat,
                                                   float* __restrict__ sigma, float* __restrict__ r_hat) {
  constexpr int kSlices = kEnsFinal / kGMaxIO;   // 128
  __shared__ float red[2][kSlices][kGMaxIO];
  const int c = threadIdx.x % kGMaxIO, q = threadIdx.x / kGMaxIO;
  float a = 0.f, b = 0.f;
  if (c < out) {
    // unrolled so that eight rows' loads are in flight at once (the adds keep
    // their order)
#pragma unroll 8
    for (int64_t r = q; r < k; r += kSlices) {
      a += rowstat[r * out + c];
      b += rowstat[k * out + r * out + c];
    }
  }
  red[0][q][c] = a;
  red[1][q][c] = b;
  __syncthreads();
  for (int w = kSlices / 2; w > 0; w >>= 1) {
    if (q < w) {
      red[0][q][c] += red[0][q + w][c];
      red[1][q][c] += red[1][q + w][c];
    }
    __syncthreads();
  }
  if (q == 0 && c < out) {
    const float ph = red[0][0][c] / (float)k;
    p_hat[c] = ph;
    sigma[c] = red[1][0][c] / (float)k;
    if (r_hat) r_hat[c] = (p_true[c] - ph) / p_true[c];
  }
}

struct GenVariant {
  int H, NH;
  void (*fwd[2])(GenParams);   // 64-row, 16-row tiles
  void (*bwd[2])(GenParams);
  void (*fwd_routed[2])(GenParams);
  void (*bwd_routed[2])(GenParams);
};

#define SAGIPS_GEN_VARIANT(H_, NH_)                                               \
  {                                                                              \
    H_, NH_, {k_gen_forward<NH_, false>, k_gen_forward16<H_, NH_, false>},       \
        {k_gen_backward<H_, NH_, 64>, k_gen_backward<H_, NH_, 16> },             \
        {k_gen_forward<NH_, true>, k_gen_forward16<H_, NH_, true>},              \
        {k_gen_backward_routed<NH_>, k_gen_backward_routed16<H_, NH_>}            \
  }

const GenVariant kGenVariants[] = {SAGIPS_GEN_VARIANT(128, 1), SAGIPS_GEN_VARIANT(128, 2), SAGIPS_GEN_VARIANT(128, 3)};

const GenVariant* find_gen(const sagips_gen& G) {
  const int H = G.width[1], NH = G.n_layers - 2;
  for (const GenVariant& v : kGenVariants)
    if (v.H == H && v.NH == NH) return &v;
  return nullptr;
}

GenParams gen_params(const sagips_gen& G, const float* noise, int64_t k) {
  GenParams p;
  memset(&p, 0, sizeof(p));
  int64_t off = 0;
  for (int l = 0; l < G.n_layers; ++l) {
    p.W[l] = G.W[l];
    p.b[l] = G.b[l];
    p.wsz[l] = (int64_t)G.width[l + 1] * G.width[l];
    p.bsz[l] = G.width[l + 1];
    p.poff_w[l] = off;
    off += p.wsz[l];
    p.poff_b[l] = off;
    off += p.bsz[l];
  }
  p.P = off;
  p.in = G.width[0];
  p.out = G.width[G.n_layers];
  p.k = k;
  p.slope = G.leaky_slope;
  p.noise = noise;
  return p;
}

GenReduceArgs reduce_args(const sagips_gen& G, const GenParams& p, int tiles, float* const* dW, float* const* db) {
  GenReduceArgs r;
  memset(&r, 0, sizeof(r));
  r.part = p.part;
  r.P = p.P;
  r.tiles = tiles;
  r.n_layers = G.n_layers;
  for (int l = 0; l < G.n_layers; ++l) {
    r.poff_w[l] = p.poff_w[l];
    r.poff_b[l] = p.poff_b[l];
    r.wsz[l] = p.wsz[l];
    r.bsz[l] = p.bsz[l];
    r.dW[l] = dW[l];
    r.db[l] = db[l];
  }
  return r;
}

// Row tile: 64, unless 64-row tiles of all members would not cover the CUs.
inline int gen_rows(const sagips_gen& G, int64_t k, int n_cu) {
  return ((k + 63) / 64) * G.n_members >= n_cu ? 64 : 16;
}
inline int gen_tiles(int64_t k, int T) { return (int)((k + T - 1) / T); }

}  // namespace

bool gen_supported(const sagips_gen& G, const char** why) {
  if (G.n_layers < 3 || G.n_layers > kMaxGenLayers) { *why = "generator needs 3 to 5 layers"; return false; }
  if (G.width[0] < 1 || G.width[0] > kGMaxIO || G.width[G.n_layers] < 1 || G.width[G.n_layers] > kGMaxIO) {
    *why = "generator input and output widths must be in [1, 8]";
    return false;
  }
  for (int l = 1; l < G.n_layers; ++l)
    if (G.width[l] != G.width[1]) { *why = "all hidden widths must be equal"; return false; }
  if (!find_gen(G)) { *why = "unsupported generator shape (hidden width 128 with 1-3 hidden-to-hidden layers)"; return false; }
  return true;
}

size_t gen_backward_workspace(const sagips_gen& G, int64_t k, int n_cu) {
  const GenParams p = gen_params(G, nullptr, k);
  return sizeof(float) * (size_t)p.P * gen_tiles(k, gen_rows(G, k, n_cu)) * G.n_members;
}

size_t ensemble_workspace(const sagips_gen& G, int64_t k) {
  const size_t th = (sizeof(float) * (size_t)G.n_members * k * G.width[G.n_layers] + 255) & ~(size_t)255;
  return th + sizeof(float) * 2 * (size_t)k * G.width[G.n_layers];
}

hipError_t launch_gen_forward(const sagips_gen& G, const float* noise, int64_t k, float* theta, int n_cu,
                              hipStream_t st, Timer* tm) {
  GenParams p = gen_params(G, noise, k);
  p.theta = theta;
  const GenVariant* v = find_gen(G);
  const int T = gen_rows(G, k, n_cu);
  if (tm) tm->begin("gen_forward");
  hipLaunchKernelGGL(v->fwd[T == 64 ? 0 : 1], dim3(gen_tiles(k, T), G.n_members), dim3(T == 64 ? kFwdThreads : kGThreads),
                     0, st, p);
  if (tm) tm->end();
  return hipGetLastError();
}

hipError_t launch_gen_backward(const sagips_gen& G, const float* noise, int64_t k, const float* dtheta,
                               float* const* dW, float* const* db, void* ws, int n_cu, hipStream_t st, Timer* tm) {
  GenParams p = gen_params(G, noise, k);
  p.dtheta = dtheta;
  p.part = static_cast<float*>(ws);
  const GenVariant* v = find_gen(G);
  const int T = gen_rows(G, k, n_cu);
  const int tiles = gen_tiles(k, T);
  if (tm) tm->begin("gen_backward");
  hipLaunchKernelGGL(v->bwd[T == 64 ? 0 : 1], dim3(tiles, G.n_members), dim3(kGThreads), 0, st, p);
  if (tm) tm->end();
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const GenReduceArgs r = reduce_args(G, p, tiles, dW, db);
  if (tm) tm->begin("gen_reduce");
  if (tiles <= 4) hipLaunchKernelGGL(k_gen_reduce<1>, dim3((unsigned)((p.P + 255) / 256), G.n_members), dim3(256), 0, st, r);
  else hipLaunchKernelGGL(k_gen_reduce<4>, dim3((unsigned)((p.P + 63) / 64), G.n_members), dim3(256), 0, st, r);
  if (tm) tm->end();
  return hipGetLastError();
}

// Members on rows of their own: tiles of 64 rows where those alone would cover half of the
// compute units.
namespace {
// Tiles at most: every member's last one may be partly filled.
inline int64_t routed_tiles(const sagips_gen& G, int64_t k, int T) { return k / T + (G.n_members < k ? G.n_members : k); }
inline int routed_rows(int64_t k, int n_cu) { return k / 64 >= n_cu / 2 ? 64 : 16; }
// The backward pass: where tiles of 16 rows would take a second turn of the compute units (4,096 rows of 8
// members: 97 us in tiles of 16, 61 in tiles of 64).
inline int routed_rows_back(const sagips_gen& G, int64_t k, int n_cu) { return routed_tiles(G, k, 16) > n_cu ? 64 : 16; }

// Workgroups of the backward pass, a multiple of 8.
inline int routed_groups(const sagips_gen& G, int64_t k, int T, int n_cu) {
  const int64_t t = routed_tiles(G, k, T == 64 ? 32 : 16), most = (n_cu + 7) / 8 * 8;
  return (int)(t < most ? (t + 7) / 8 * 8 : most);
}
inline int64_t padded_partial(int64_t P) { return (P + 3) & ~(int64_t)3; }
// Bytes of the split copies.
inline size_t routed_split_bytes(const sagips_gen& G) {
  return (size_t)G.n_members * 2 * (G.n_layers - 2) * split_copy_bytes(128);
}
}  // namespace

size_t gen_backward_routed_workspace(const sagips_gen& G, int64_t k, int n_cu) {
  const GenParams p = gen_params(G, nullptr, k);
  const int T = routed_rows_back(G, k, n_cu);
  const size_t partials = routed_groups(G, k, T, n_cu) + (size_t)G.n_members;
  return (T == 64 ? routed_split_bytes(G) : 0) + sizeof(float) * (size_t)padded_partial(p.P) * partials + sizeof(int) * 2 * (size_t)G.n_members;
}

hipError_t launch_gen_forward_routed(const sagips_gen& G, const float* x, const int32_t* offsets, int64_t k, float* theta,
                                     int n_cu, hipStream_t st, Timer* tm) {
  GenParams p = gen_params(G, x, k);
  p.theta = theta;
  p.offsets = offsets;
  p.members = G.n_members;
  const GenVariant* v = find_gen(G);
  const int T = routed_rows(k, n_cu);
  if (tm) tm->begin("gen_forward_routed");
  hipLaunchKernelGGL(v->fwd_routed[T == 64 ? 0 : 1], dim3((unsigned)((routed_tiles(G, k, T) + 7) / 8 * 8)),
                     dim3(T == 64 ? kFwdThreads : kGThreads), 0, st, p);
  if (tm) tm->end();
  return hipGetLastError();
}

hipError_t launch_gen_backward_routed(const sagips_gen& G, const float* x, const int32_t* offsets, int64_t k,
                                      const float* dtheta, float* const* dW, float* const* db, float* dx, void* ws, int n_cu,
                                      hipStream_t st, Timer* tm) {
  GenParams p = gen_params(G, x, k);
  const int T = routed_rows_back(G, k, n_cu), groups = routed_groups(G, k, T, n_cu), NH = G.n_layers - 2;
  p.dtheta = dtheta;
  p.part = reinterpret_cast<float*>(static_cast<char*>(ws) + (T == 64 ? routed_split_bytes(G) : 0));
  p.offsets = offsets;
  p.members = G.n_members;
  p.dx = dx;
  const GenVariant* v = find_gen(G);
  if (T == 64) {
    u16* copies = static_cast<u16*>(ws);
    p.split = copies;
    if (tm) tm->begin("gen_split");
    hipLaunchKernelGGL(k_split_members, dim3(128 * 128 / 8 / 256, 2 * NH, G.n_members), dim3(256), 0, st, p, copies, NH);
    if (tm) tm->end();
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  p.PS = padded_partial(p.P);
  p.slots = reinterpret_cast<int*>(p.part + (size_t)p.PS * (groups + (size_t)G.n_members));
  if (tm) tm->begin("gen_backward_routed");
  hipLaunchKernelGGL(v->bwd_routed[T == 64 ? 0 : 1], dim3(groups), dim3(kGThreads), 0, st, p);
  if (tm) tm->end();
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const GenReduceArgs r = reduce_args(G, p, 0, dW, db);
  const dim3 grid((unsigned)((p.P + 255) / 256), G.n_members);
  if (tm) tm->begin("gen_reduce_routed");
  hipLaunchKernelGGL(k_gen_reduce_routed, grid, dim3(256), 0, st, r, p.slots, p.PS);
  if (tm) tm->end();
  return hipGetLastError();
}

hipError_t launch_ensemble(const sagips_gen& G, const float* noise, int64_t k, const float* p_true, float* p_hat,
                           float* sigma, float* r_hat, void* ws, int n_cu, hipStream_t st, Timer* tm) {
  const int out = G.width[G.n_layers];
  float* theta = static_cast<float*>(ws);
  const size_t th = (sizeof(float) * (size_t)G.n_members * k * out + 255) & ~(size_t)255;
  float* rowstat = reinterpret_cast<float*>(static_cast<char*>(ws) + th);
  hipError_t e = launch_gen_forward(G, noise, k, theta, n_cu, st, tm);
  if (e != hipSuccess) return e;
  if (tm) tm->begin("ensemble_rows");
  hipLaunchKernelGGL(k_ens_rows, dim3((unsigned)((k * out + kEnsCols - 1) / kEnsCols)), dim3(256), 0, st, theta,
                     G.n_members, k, out, rowstat);
  if (tm) tm->end();
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (tm) tm->begin("ensemble_final");
  hipLaunchKernelGGL(k_ens_final, dim3(1), dim3(kEnsFinal), 0, st, rowstat, k, out, p_true, p_hat, sigma, r_hat);
  if (tm) tm->end();
  return hipGetLastError();
}

}  // namespace sagips
