// Group norm with an activation and dropout, forward, over channels-last
// tensors (bf16 or fp32, fp32 arithmetic).
//
// A pass over a tensor costs the time HBM takes for it, so x is read once where
// a sample's tile (whole groups of channels, all pixels) stays in the registers
// of one workgroup (512 KB of registers a CU against 160 KB of LDS) or, for many
// small tiles, of one wavefront: mean, then the squares of the differences from
// it, then the output, all from registers.  The two sums keep a group whose mean
// is far from zero exact where sums of squares would cancel.  A tile too large
// for that is cut into chunks of pixels: one pass leaves mean and squared
// differences of every chunk, which combine exactly (T. Chan, G. Golub, R.
// LeVeque, 1979), and a second pass applies them.
#include "gn.h"
#include "common.h"

namespace ckpt {
namespace {

// The element pass: thread parameters of a vector column, then pixels.
template <typename XT, int V, bool FOLD>
struct Column {
  float mean[FOLD ? 1 : V], a[V], b[V];
  __device__ __forceinline__ void affine(const GnArgs &A, int c, const float (&rstd)[FOLD ? 1 : V]) {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      a[j] = A.gamma[c + j] * rstd[FOLD ? 0 : j];
      b[j] = A.beta[c + j];
    }
  }
  __device__ __forceinline__ void put(const GnArgs &A, const DropKey &key, const Vec<XT, V> &x, int64_t pix, int c) const {
    float v[V];
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = gn_act(A.act, gn_affine(float(x.v[j]), mean[FOLD ? 0 : j], a[j], b[j]));
    if (A.drop.rng) gn_drop<V>(A, key, uint64_t(pix), c, v);
    store_vec<XT, V>(static_cast<XT *>(A.out) + pix * A.ldo + c, v);
  }
};

// One team per (sample, tile); PART: per chunk of a sample's tile, leaving the
// chunk's mean and squared differences per group.
template <typename XT, int V, int NV, bool FOLD, bool WAVE, bool PART>
__global__ __launch_bounds__(1024) void k_gn_fwd(GnArgs A) {
  extern __shared__ float lds[];
  constexpr int NJ = FOLD ? 1 : V;
  const Team<WAVE> tm(A);
  const int teams = WAVE ? blockDim.x / 64 : 1;
  const int tile = blockIdx.x % A.tiles;
  const int64_t by = blockIdx.x / A.tiles;
  const int c = tile * A.W + tm.tx * V;
  const bool col = c < A.C && tm.ty < A.TY;
  const int buf = A.pow2 ? A.redbuf : 0;
  float *red = lds + tm.index * (A.pow2 ? 2 : 1) * A.redbuf;
  const DropKey key = drop_key(A.drop);
  const int64_t n0 = PART ? by / A.chunks : by * teams + tm.index;
  const int64_t step = PART ? A.n : int64_t(A.rows) * teams;
  const int64_t p0 = PART ? (by % A.chunks) * (int64_t(A.TY) * NV) : 0;
  const int64_t np = PART ? min(A.hw - p0, int64_t(A.TY) * NV) : A.hw;
  for (int64_t i = n0; i < A.n; i += step) {
    const int64_t pix0 = i * A.hw + p0;
    const XT *const x = static_cast<const XT *>(A.x) + (pix0 + tm.ty) * A.ldx + c;
    const int64_t dx = int64_t(A.TY) * A.ldx;
    Vec<XT, V> xr[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (col && tm.ty + k * A.TY < np) xr[k] = load_vec<XT, V>(x + k * dx);
    float s[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) s[j] = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (col && tm.ty + k * A.TY < np)
#pragma unroll
        for (int j = 0; j < V; ++j) s[FOLD ? 0 : j] += float(xr[k].v[j]);
    group_sums<1, NJ, WAVE>(A, tm, s, red);
    const float m = float(np * A.cg);  // exact: a team holds fewer than 2^24 values
    Column<XT, V, FOLD> cp;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      cp.mean[j] = s[j] / m;  // not times 1 / m: a constant group's mean is that constant
      s[j] = 0.f;
    }
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (col && tm.ty + k * A.TY < np)
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float t = float(xr[k].v[j]) - cp.mean[FOLD ? 0 : j];
          s[FOLD ? 0 : j] += t * t;
        }
    group_sums<1, NJ, WAVE>(A, tm, s, red + buf);
    if (!PART)
#pragma unroll
      for (int j = 0; j < NJ; ++j) s[j] = 1.f / sqrtf(s[j] / m + A.eps);
    // the first thread of each group writes its statistics
    if (tm.ty == 0 && c < A.C)
#pragma unroll
      for (int j = 0; j < NJ; ++j)
        if ((c + j) % A.cg == 0) {
          const int k = (c + j) / A.cg;
          if (PART) {
            float *const o = A.gpart + (by * A.G + k) * 2;
            o[0] = cp.mean[j];
            o[1] = s[j];
          } else {
            A.st[i * A.G + k] = cp.mean[j];
            A.st[(A.n + i) * A.G + k] = s[j];
          }
        }
    if (!PART && col) {
      cp.affine(A, c, s);
#pragma unroll
      for (int k = 0; k < NV; ++k)
        if (tm.ty + k * A.TY < np) cp.put(A, key, xr[k], pix0 + tm.ty + k * A.TY, c);
    }
  }
}

// Statistics of group blockIdx.x (of all n G) from its chunks' means and squared
// differences, one wavefront, in double: sum cnt mean / m, then sum (M2 + cnt
// (mean_i - mean)^2).
__global__ __launch_bounds__(64) void k_gn_merge(GnArgs A, int rows_per_chunk) {
  const int64_t i = blockIdx.x / A.G;
  const int k = blockIdx.x % A.G;
  const float *const part = A.gpart + (i * A.chunks * A.G + k) * 2;
  const double m = double(A.hw) * A.cg;
  double s = 0;
  for (int64_t q = threadIdx.x; q < A.chunks; q += 64) {
    const double cnt = double(min(int64_t(rows_per_chunk), A.hw - q * rows_per_chunk)) * A.cg;
    s += cnt * part[q * A.G * 2];
  }
  for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off);
  const double mean = s / m;
  s = 0;
  for (int64_t q = threadIdx.x; q < A.chunks; q += 64) {
    const double cnt = double(min(int64_t(rows_per_chunk), A.hw - q * rows_per_chunk)) * A.cg;
    const double t = part[q * A.G * 2] - mean;
    s += part[q * A.G * 2 + 1] + cnt * t * t;
  }
  for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off);
  if (threadIdx.x == 0) {
    A.st[i * A.G + k] = float(mean);
    A.st[(A.n + i) * A.G + k] = 1.f / sqrtf(float(s / m) + A.eps);
  }
}

// The output from known statistics, chunk by chunk.
template <typename XT, int V, int NV, bool FOLD>
__global__ __launch_bounds__(1024) void k_gn_apply(GnArgs A) {
  constexpr int NJ = FOLD ? 1 : V;
  const int tx = threadIdx.x % A.VC, ty = threadIdx.x / A.VC;
  const int tile = blockIdx.x % A.tiles;
  const int64_t by = blockIdx.x / A.tiles;
  const int c = tile * A.W + tx * V;
  if (c >= A.C || ty >= A.TY) return;
  const int64_t i = by / A.chunks, p0 = (by % A.chunks) * (int64_t(A.TY) * NV);
  const int64_t np = min(A.hw - p0, int64_t(A.TY) * NV), pix0 = i * A.hw + p0;
  const XT *const x = static_cast<const XT *>(A.x) + (pix0 + ty) * A.ldx + c;
  const int64_t dx = int64_t(A.TY) * A.ldx;
  Vec<XT, V> xr[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k)
    if (ty + k * A.TY < np) xr[k] = load_vec<XT, V>(x + k * dx);
  const DropKey key = drop_key(A.drop);
  const GnGroups<V, FOLD> grp(A, c);
  Column<XT, V, FOLD> cp;
  float rstd[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    cp.mean[j] = A.st[i * A.G + grp.k[j]];
    rstd[j] = A.st[(A.n + i) * A.G + grp.k[j]];
  }
  cp.affine(A, c, rstd);
#pragma unroll
  for (int k = 0; k < NV; ++k)
    if (ty + k * A.TY < np) cp.put(A, key, xr[k], pix0 + ty + k * A.TY, c);
}

template <typename XT, int V, int NV, bool FOLD>
void launch_fwd(hipStream_t s, const GnPlan &g, const GnArgs &a) {
  const dim3 grid(uint32_t(g.blocks)), block(g.threads);
  if (g.wave)
    hipLaunchKernelGGL((k_gn_fwd<XT, V, NV, FOLD, true, false>), grid, block, g.lds, s, a);
  else
    hipLaunchKernelGGL((k_gn_fwd<XT, V, NV, FOLD, false, false>), grid, block, g.lds, s, a);
}

template <typename XT, int V, bool FOLD>
void run_apply(hipStream_t s, const GnPlan &g, const GnArgs &a) {
  hipLaunchKernelGGL((k_gn_apply<XT, V, GN_EW_NV, FOLD>), dim3(uint32_t(g.blocks)), dim3(g.threads), 0, s, a);
}

template <typename XT, int V, bool FOLD>
void run_fwd(hipStream_t s, const GnPlan &g, const GnArgs &a) {
  if (g.split) {
    constexpr int NV = V == 1 ? 16 : 8;
    hipLaunchKernelGGL((k_gn_fwd<XT, V, NV, FOLD, false, true>), dim3(uint32_t(g.blocks)), dim3(g.threads), g.lds, s, a);
    hipLaunchKernelGGL(k_gn_merge, dim3(uint32_t(a.n * a.G)), dim3(64), 0, s, a, a.TY * NV);
    return;
  }
  if (g.NV <= 2) return launch_fwd<XT, V, 2, FOLD>(s, g, a);
  if (g.NV <= 4) return launch_fwd<XT, V, 4, FOLD>(s, g, a);
  if (g.NV <= 8) return launch_fwd<XT, V, 8, FOLD>(s, g, a);
  // fp32 vectors stop at 8 (gn_plan)
  if constexpr (V == 1 || sizeof(XT) == 2) launch_fwd<XT, V, 16, FOLD>(s, g, a);
}

}  // namespace

void gn_forward(hipStream_t s, const GnProblem &p, const void *x, const float *gamma, const float *beta,
                const DropArgs &drop, void *y, float *st, void *ws) {
  const GnPlan g = gn_plan(p, false);
  GnArgs a = gn_args(p, g, drop);
  a.x = x;
  a.out = y;
  a.ldo = p.ldy;
  a.gamma = gamma;
  a.beta = beta;
  a.st = st;
  a.gpart = static_cast<float *>(ws);
  if (g.V == 1)
    p.xf ? run_fwd<float, 1, true>(s, g, a) : run_fwd<__bf16, 1, true>(s, g, a);
  else if (g.fold)
    p.xf ? run_fwd<float, 8, true>(s, g, a) : run_fwd<__bf16, 8, true>(s, g, a);
  else
    p.xf ? run_fwd<float, 8, false>(s, g, a) : run_fwd<__bf16, 8, false>(s, g, a);
  if (g.split) gn_apply(s, p, x, st, gamma, beta, drop, y);
}

void gn_apply(hipStream_t s, const GnProblem &p, const void *x, const float *st, const float *gamma,
              const float *beta, const DropArgs &drop, void *y) {
  const GnPlan g = gn_plan_elements(p);
  GnArgs a = gn_args(p, g, drop);
  a.x = x;
  a.out = y;
  a.ldo = p.ldy;
  a.gamma = gamma;
  a.beta = beta;
  a.st = const_cast<float *>(st);
  if (g.V == 1)
    p.xf ? run_apply<float, 1, true>(s, g, a) : run_apply<__bf16, 1, true>(s, g, a);
  else if (g.fold)
    p.xf ? run_apply<float, 8, true>(s, g, a) : run_apply<__bf16, 8, true>(s, g, a);
  else
    p.xf ? run_apply<float, 8, false>(s, g, a) : run_apply<__bf16, 8, false>(s, g, a);
}

}  // namespace ckpt
