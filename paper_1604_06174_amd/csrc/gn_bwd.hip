// Group norm with an activation and dropout, backward, over channels-last
// tensors.  From x, the statistics, the counter and g alone (neither output nor
// mask is kept):
//
//   t = x - mean, u = t a + beta (a = gamma rstd), xhat = t rstd
//   du = dropout(g) act'(u), dbeta = sum du, dgamma = sum du xhat
//   S1 = sum gamma du, S2 = sum gamma du xhat over a group's m values
//   d = a du - rstd S1 / m - t rstd^2 S2 / m
//
// As in the forward, a tile that fits stays in registers (x as loaded, du in
// fp32): x and g are read once.  A larger one takes a pass for the sums and a
// pass that applies them.  Channel sums leave one record per workgroup (or
// chunk), added in a fixed order.
#include "common.h"
#include "gn.h"

namespace ckpt {
namespace {

template <typename XT, int V, bool FOLD>
struct Column {
  float mean[FOLD ? 1 : V], rstd[FOLD ? 1 : V], gamma[V], beta[V];
  __device__ __forceinline__ void params(const GnArgs &A, int c) {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      gamma[j] = A.gamma[c + j];
      beta[j] = A.beta[c + j];
    }
  }
  __device__ __forceinline__ void stats(const GnArgs &A, const GnGroups<V, FOLD> &grp, int64_t i) {
#pragma unroll
    for (int j = 0; j < (FOLD ? 1 : V); ++j) {
      mean[j] = A.st[i * A.G + grp.k[j]];
      rstd[j] = A.st[(A.n + i) * A.G + grp.k[j]];
    }
  }
  // du in place of g
  __device__ __forceinline__ void du(const GnArgs &A, const DropKey &key, const Vec<XT, V> &x, uint64_t pix, int c,
                                     float g[V]) const {
    if (A.drop.rng) gn_drop<V>(A, key, pix, c, g);
    if (A.act != GN_ACT_NONE)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int q = FOLD ? 0 : j;
        g[j] = gn_act_bwd(A.act, gn_affine(float(x.v[j]), mean[q], gamma[j] * rstd[q], beta[j]), g[j]);
      }
  }
  // d from du and the group's k1 = rstd S1 / m, k2 = rstd^2 S2 / m
  template <typename DT>
  __device__ __forceinline__ void put(const GnArgs &A, const Vec<XT, V> &x, const float (&k1)[FOLD ? 1 : V],
                                      const float (&k2)[FOLD ? 1 : V], int64_t pix, int c, const float du[V]) const {
    float v[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int q = FOLD ? 0 : j;
      v[j] = gamma[j] * rstd[q] * du[j] - k1[q] - (float(x.v[j]) - mean[q]) * k2[q];
    }
    store_vec<DT, V>(static_cast<DT *>(A.out) + pix * A.ldo + c, v);
  }
};

// One team per (sample, tile), looping over samples; PART: per chunk of a
// sample's tile, leaving the chunk's sums.
template <typename XT, typename GT_, typename DT, int V, int NV, bool FOLD, bool WAVE, bool PART>
__global__ __launch_bounds__(V == 8 ? 512 : 1024) void k_gn_bwd(GnArgs A) {
  extern __shared__ float lds[];
  constexpr int NJ = FOLD ? 1 : V;
  const Team<WAVE> tm(A);
  const int teams = WAVE ? blockDim.x / 64 : 1;
  const int tile = blockIdx.x % A.tiles;
  const int64_t by = blockIdx.x / A.tiles;
  const int c = tile * A.W + tm.tx * V;
  const bool col = c < A.C && tm.ty < A.TY;
  float *const red = lds + tm.index * (A.pow2 ? 2 : 1) * A.redbuf;
  int buf = 0;
  const DropKey key = drop_key(A.drop);
  const int64_t n0 = PART ? by / A.chunks : by * teams + tm.index;
  const int64_t step = PART ? A.n : int64_t(A.rows) * teams;
  const int64_t p0 = PART ? (by % A.chunks) * (int64_t(A.TY) * NV) : 0;
  const int64_t np = PART ? min(A.hw - p0, int64_t(A.TY) * NV) : A.hw;
  const GnGroups<V, FOLD> grp(A, col ? c : 0);
  Column<XT, V, FOLD> cp;
  cp.params(A, col ? c : 0);
  float ch[2 * V];  // sums of du xhat, then of du, per channel
#pragma unroll
  for (int j = 0; j < 2 * V; ++j) ch[j] = 0.f;
  for (int64_t i = n0; i < A.n; i += step) {
    const int64_t pix0 = i * A.hw + p0;
    const XT *const x = static_cast<const XT *>(A.x) + (pix0 + tm.ty) * A.ldx + c;
    const GT_ *const g = static_cast<const GT_ *>(A.g) + (pix0 + tm.ty) * A.ldg + c;
    const int64_t dx = int64_t(A.TY) * A.ldx, dg = int64_t(A.TY) * A.ldg;
    Vec<XT, V> xr[NV];
    float du[NV][V];
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (col && tm.ty + k * A.TY < np) {
        xr[k] = load_vec<XT, V>(x + k * dx);
        const Vec<GT_, V> gr = load_vec<GT_, V>(g + k * dg);
#pragma unroll
        for (int j = 0; j < V; ++j) du[k][j] = float(gr.v[j]);
      }
    cp.stats(A, grp, i);
    float s1[V], s2[V];
#pragma unroll
    for (int j = 0; j < V; ++j) s1[j] = s2[j] = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (col && tm.ty + k * A.TY < np) {
        cp.du(A, key, xr[k], uint64_t(pix0 + tm.ty + k * A.TY), c, du[k]);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          s1[j] += du[k][j];
          s2[j] += du[k][j] * ((float(xr[k].v[j]) - cp.mean[FOLD ? 0 : j]) * cp.rstd[FOLD ? 0 : j]);
        }
      }
    float s[2 * NJ];
#pragma unroll
    for (int j = 0; j < 2 * NJ; ++j) s[j] = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      ch[j] += s2[j];
      ch[V + j] += s1[j];
      s[FOLD ? 0 : j] += cp.gamma[j] * s1[j];
      s[NJ + (FOLD ? 0 : j)] += cp.gamma[j] * s2[j];
    }
    group_sums<2, NJ, WAVE>(A, tm, s, red + buf);
    if (A.pow2) buf = A.redbuf - buf;
    if (PART) {
      if (tm.ty == 0 && c < A.C)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
          if ((c + j) % A.cg == 0) {
            float *const o = A.gpart + (by * A.G + grp.k[j]) * 2;
            o[0] = s[j];
            o[1] = s[NJ + j];
          }
    } else if (col) {
      float k1[NJ], k2[NJ];
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        k1[j] = cp.rstd[j] * s[j] * A.inv_m;
        k2[j] = cp.rstd[j] * cp.rstd[j] * s[NJ + j] * A.inv_m;
      }
#pragma unroll
      for (int k = 0; k < NV; ++k)
        if (tm.ty + k * A.TY < np)
          cp.template put<DT>(A, xr[k], k1, k2, pix0 + tm.ty + k * A.TY, c, du[k]);
    }
  }
  // the channels' sums over the workgroup's pixels: record `by` of cpart
  __syncthreads();
  const int O = 2 * V * A.VC;
  float *const out0 = A.cpart ? A.cpart + by * 2 * A.C : A.dgamma;
  float *const out1 = A.cpart ? out0 + A.C : A.dbeta;
  if (A.pow2) {
    const int w = threadIdx.x >> 6, lane = threadIdx.x & 63, nw = blockDim.x >> 6;
    for (int off = A.VC; off < 64; off <<= 1)
#pragma unroll
      for (int k = 0; k < 2 * V; ++k) ch[k] += __shfl_xor(ch[k], off);
    if (lane < A.VC)
#pragma unroll
      for (int q = 0; q < 2; ++q)
#pragma unroll
        for (int j = 0; j < V; ++j) lds[w * O + q * A.W + tm.tx * V + j] = ch[q * V + j];
    __syncthreads();
    for (int o = threadIdx.x; o < O; o += blockDim.x) {
      const int q = o / A.W, cc = tile * A.W + o - q * A.W;
      float s = 0.f;
      for (int k = 0; k < nw; ++k) s += lds[k * O + o];
      if (cc < A.C) (q ? out1 : out0)[cc] = s;
    }
    return;
  }
  const int tree = (A.TY + (A.TY + 7) / 8) * O;
  if (tm.ty < A.TY)
#pragma unroll
    for (int k = 0; k < 2 * V; ++k) lds[tm.index * tree + tm.ty * O + k * A.VC + tm.tx] = ch[k];
  const float *const sums = row_tree<WAVE, 2 * V>(tm, A.TY, A.VC, lds + tm.index * tree);
  __syncthreads();
  const int at = int(sums - lds) - tm.index * tree;
  for (int o = threadIdx.x; o < O; o += blockDim.x) {
    const int k = o / A.VC, cc = tile * A.W + (o - k * A.VC) * V + k % V;
    float s = 0.f;
    for (int q = 0; q < teams; ++q) s += lds[q * tree + at + o];
    if (cc < A.C) (k < V ? out0 : out1)[cc] = s;
  }
}

// gsum[i][k][2] = the sum of group (i, k)'s chunk sums, one wavefront each
__global__ __launch_bounds__(64) void k_gn_bwd_merge(GnArgs A, float *gsum) {
  const int64_t i = blockIdx.x / A.G;
  const int k = blockIdx.x % A.G;
  const float *const part = A.gpart + (i * A.chunks * A.G + k) * 2;
  float s1 = 0.f, s2 = 0.f;
  for (int64_t q = threadIdx.x; q < A.chunks; q += 64) {
    s1 += part[q * A.G * 2];
    s2 += part[q * A.G * 2 + 1];
  }
  for (int off = 32; off > 0; off >>= 1) {
    s1 += __shfl_xor(s1, off);
    s2 += __shfl_xor(s2, off);
  }
  if (threadIdx.x == 0) {
    gsum[int64_t(blockIdx.x) * 2] = s1;
    gsum[int64_t(blockIdx.x) * 2 + 1] = s2;
  }
}

// dgamma | dbeta from `rows` records [2][C]: 16 columns a workgroup, 64 threads
// each, added in a fixed order
__global__ __launch_bounds__(1024) void k_gn_channel_sums(int64_t rows, int C, const float *part, float *dgamma,
                                                          float *dbeta) {
  __shared__ float red[64][17];
  const int e = blockIdx.x * 16 + threadIdx.x % 16, r0 = threadIdx.x / 16;
  float s = 0.f;
  if (e < 2 * C)
    for (int64_t r = r0; r < rows; r += 64) s += part[r * 2 * C + e];
  red[r0][threadIdx.x % 16] = s;
  __syncthreads();
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  s = red[lane][w];
  for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off);
  const int o = blockIdx.x * 16 + w;
  if (lane == 0 && o < 2 * C) (o < C ? dgamma : dbeta)[o < C ? o : o - C] = s;
}

// d from known group sums, chunk by chunk
template <typename XT, typename GT_, typename DT, int V, int NV, bool FOLD>
__global__ __launch_bounds__(256) void k_gn_bwd_apply(GnArgs A) {
  constexpr int NJ = FOLD ? 1 : V;
  const int tx = threadIdx.x % A.VC, ty = threadIdx.x / A.VC;
  const int tile = blockIdx.x % A.tiles;
  const int64_t by = blockIdx.x / A.tiles;
  const int c = tile * A.W + tx * V;
  if (c >= A.C || ty >= A.TY) return;
  const int64_t i = by / A.chunks, p0 = (by % A.chunks) * (int64_t(A.TY) * NV);
  const int64_t np = min(A.hw - p0, int64_t(A.TY) * NV), pix0 = i * A.hw + p0;
  const XT *const x = static_cast<const XT *>(A.x) + (pix0 + ty) * A.ldx + c;
  const GT_ *const g = static_cast<const GT_ *>(A.g) + (pix0 + ty) * A.ldg + c;
  const int64_t dx = int64_t(A.TY) * A.ldx, dg = int64_t(A.TY) * A.ldg;
  Vec<XT, V> xr[NV];
  Vec<GT_, V> gr[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k)
    if (ty + k * A.TY < np) {
      xr[k] = load_vec<XT, V>(x + k * dx);
      gr[k] = load_vec<GT_, V>(g + k * dg);
    }
  const DropKey key = drop_key(A.drop);
  const GnGroups<V, FOLD> grp(A, c);
  Column<XT, V, FOLD> cp;
  cp.params(A, c);
  cp.stats(A, grp, i);
  float k1[NJ], k2[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    const float *const s = A.gsum + (i * A.G + grp.k[j]) * 2;
    k1[j] = cp.rstd[j] * s[0] * A.inv_m;
    k2[j] = cp.rstd[j] * cp.rstd[j] * s[1] * A.inv_m;
  }
#pragma unroll
  for (int k = 0; k < NV; ++k)
    if (ty + k * A.TY < np) {
      float du[V];
#pragma unroll
      for (int j = 0; j < V; ++j) du[j] = float(gr[k].v[j]);
      const int64_t pix = pix0 + ty + k * A.TY;
      cp.du(A, key, xr[k], uint64_t(pix), c, du);
      cp.template put<DT>(A, xr[k], k1, k2, pix, c, du);
    }
}

template <typename XT, typename GT_, typename DT, int V, int NV, bool FOLD>
void launch_bwd(hipStream_t s, const GnPlan &g, const GnArgs &a) {
  const dim3 grid(uint32_t(g.blocks)), block(g.threads);
  if (g.wave)
    hipLaunchKernelGGL((k_gn_bwd<XT, GT_, DT, V, NV, FOLD, true, false>), grid, block, g.lds, s, a);
  else
    hipLaunchKernelGGL((k_gn_bwd<XT, GT_, DT, V, NV, FOLD, false, false>), grid, block, g.lds, s, a);
}

template <typename XT, typename GT_, typename DT, int V, bool FOLD>
void run_bwd(hipStream_t s, const GnProblem &p, const GnPlan &g, GnArgs a) {
  if (!g.split) {
    if (g.NV <= 2) return launch_bwd<XT, GT_, DT, V, 2, FOLD>(s, g, a);
    if (g.NV <= 4) return launch_bwd<XT, GT_, DT, V, 4, FOLD>(s, g, a);
    if (g.NV <= 8) return launch_bwd<XT, GT_, DT, V, 8, FOLD>(s, g, a);
    // vectors stop at 8 (gn_plan)
    if constexpr (V == 1) launch_bwd<XT, GT_, DT, V, 16, FOLD>(s, g, a);
    return;
  }
  constexpr int NV = V == 1 ? 16 : 8;
  hipLaunchKernelGGL((k_gn_bwd<XT, GT_, DT, V, NV, FOLD, false, true>), dim3(uint32_t(g.blocks)), dim3(g.threads),
                     g.lds, s, a);
  float *const gsum = const_cast<float *>(a.gsum);
  hipLaunchKernelGGL(k_gn_bwd_merge, dim3(uint32_t(a.n * a.G)), dim3(64), 0, s, a, gsum);
  const GnPlan e = gn_plan_elements(p);
  GnArgs ea = gn_args(p, e, a.drop);
  ea.x = a.x;
  ea.g = a.g;
  ea.out = a.out;
  ea.ldo = a.ldo;
  ea.gamma = a.gamma;
  ea.beta = a.beta;
  ea.st = a.st;
  ea.gsum = gsum;
  if (e.V == V)
    hipLaunchKernelGGL((k_gn_bwd_apply<XT, GT_, DT, V, GN_EW_NV, FOLD>), dim3(uint32_t(e.blocks)), dim3(e.threads),
                       0, s, ea);
  else  // a vector row whose groups only fit a team element by element
    hipLaunchKernelGGL((k_gn_bwd_apply<XT, GT_, DT, 8, GN_EW_NV, false>), dim3(uint32_t(e.blocks)), dim3(e.threads),
                       0, s, ea);
}

template <typename XT, typename GT_, typename DT>
void run_types(hipStream_t s, const GnProblem &p, const GnPlan &g, const GnArgs &a) {
  if (g.V == 1)
    run_bwd<XT, GT_, DT, 1, true>(s, p, g, a);
  else if (g.fold)
    run_bwd<XT, GT_, DT, 8, true>(s, p, g, a);
  else
    run_bwd<XT, GT_, DT, 8, false>(s, p, g, a);
}

}  // namespace

void gn_backward(hipStream_t s, const GnProblem &p, const void *g, const void *x, const float *st,
                 const float *gamma, const float *beta, const DropArgs &drop, void *d, float *dgamma,
                 float *dbeta, void *ws) {
  const GnPlan pl = gn_plan(p, true);
  GnArgs a = gn_args(p, pl, drop);
  a.x = x;
  a.g = g;
  a.out = d;
  a.ldo = p.ldd;
  a.gamma = gamma;
  a.beta = beta;
  a.st = const_cast<float *>(st);
  a.dgamma = dgamma;
  a.dbeta = dbeta;
  char *w = static_cast<char *>(ws);
  if (pl.split) {
    a.gpart = reinterpret_cast<float *>(w);
    w += align256(uint64_t(p.n) * pl.chunks * p.G * 8);
    a.gsum = reinterpret_cast<const float *>(w);
    w += align256(uint64_t(p.n) * p.G * 8);
  }
  const int64_t rows = pl.split ? p.n * pl.chunks : pl.rows;
  if (rows > 1) a.cpart = reinterpret_cast<float *>(w);
  if (p.xf)
    run_types<float, float, float>(s, p, pl, a);
  else if (p.gf)
    p.df ? run_types<__bf16, float, float>(s, p, pl, a) : run_types<__bf16, float, __bf16>(s, p, pl, a);
  else
    p.df ? run_types<__bf16, __bf16, float>(s, p, pl, a) : run_types<__bf16, __bf16, __bf16>(s, p, pl, a);
  if (rows > 1)
    hipLaunchKernelGGL(k_gn_channel_sums, dim3((2 * p.C + 15) / 16), dim3(1024), 0, s, rows, p.C, a.cpart, dgamma,
                       dbeta);
}

}  // namespace ckpt
