// Group norm with an activation and dropout, forward, over channels-last
// tensors (bf16 or fp32, fp32 arithmetic).
//
// A pass over a tensor costs the time HBM takes for it, so x is read once where
// a sample's tile (whole groups of channels, all pixels) stays in the registers
// of one workgroup (512 KB of registers a CU against 160 KB of LDS) or, for many
// small tiles, of one wavefront: mean, then the squares of the differences from
// it, then the output, all from registers.  The two sums keep a group whose mean
// is far from zero exact where sums of squares would cancel.  A tile too large
// for that is cut into chunks of pixels: a first pass leaves mean and squared
// differences of every chunk, which combine exactly (T. Chan, G. Golub, R.
// LeVeque, 1979); the second pass combines them and applies them.
#include "common.h"
#include "gn.h"

namespace ckpt {
namespace {

// A vector column's parameters and one vector's output.
template <typename XT, int V, int NJ>
struct Column {
  float mean[NJ], a[V], b[V];
  template <bool SILU, bool DROP>
  __device__ __forceinline__ void put(const GnArgs &A, const DropKey &key, const Vec<XT, V> &x, int64_t pix, int c) const {
    float v[V];
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = gn_act<SILU, sizeof(XT) == 4>(A.act == GN_ACT_RELU, gn_affine(float(x.v[j]), mean[NJ == 1 ? 0 : j], a[j], b[j]));
    if (DROP) gn_drop<V>(A, key, uint64_t(pix), c, v);
    store_vec<XT, V>(static_cast<XT *>(A.out) + pix * A.ldo + c, v);
  }
};

// Resident: one team per (sample, tile); a wavefront's loops over samples.
template <typename XT, int V, int NV, int NJ, bool WAVE, int RED, bool SILU, bool DROP>
__global__ __launch_bounds__(WAVE ? 256 : 1024) void k_gn_fwd(GnArgs A) {
  extern __shared__ float lds[];
  const Team<WAVE> tm(A);
  const int teams = WAVE ? blockDim.x / 64 : 1;
  const int by = A.by_tiles.of(blockIdx.x), tile = blockIdx.x - by * A.tiles;
  const int c = tile * A.W + tm.tx * V;
  const bool column = tm.tx < A.cols && c < A.C;
  float *const red = lds + tm.index * (RED == GN_RED_GROUPS ? 2 : 1) * A.redbuf;
  const DropKey key = drop_key(A.drop);
  const float m = float(A.hw * A.cg);  // exact: a team holds fewer than 2^24 values
  // a wavefront's rows are pixels, or samples of one
  const bool packed = WAVE && A.pack > 1;
  const int ty = packed ? 0 : tm.ty, step = A.rows * teams * (WAVE ? A.pack : 1);
  for (int i0 = (by * teams + tm.index) * (WAVE ? A.pack : 1); i0 < A.n; i0 = WAVE ? i0 + step : A.n) {
    const int i = packed ? i0 + tm.ty : i0;
    const bool own = column && (!packed || i < A.n), col = own && ty < A.TY;
    const int64_t pix0 = int64_t(i) * A.hw;
    const XT *const x = static_cast<const XT *>(A.x) + (pix0 + ty) * A.ldx + c;
    const int64_t dx = int64_t(A.TY) * A.ldx;
    Vec<XT, V> xr[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (col && ty + k * A.TY < A.hw) xr[k] = load_vec<XT, V>(x + k * dx);
    Column<XT, V, NJ> cp;
    float gamma[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      gamma[j] = A.gamma[col ? c + j : j];
      cp.b[j] = A.beta[col ? c + j : j];
    }
    float s[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) s[j] = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (col && ty + k * A.TY < A.hw)
#pragma unroll
        for (int j = 0; j < V; ++j) s[NJ == 1 ? 0 : j] += float(xr[k].v[j]);
    group_sums<1, NJ, V, WAVE, RED>(A, tm, s, red);
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      cp.mean[j] = s[j] / m;  // not times 1 / m: exact sums (as of a constant of few bits) give the exact mean
      s[j] = 0.f;
    }
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (col && ty + k * A.TY < A.hw) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float t = float(xr[k].v[j]) - cp.mean[NJ == 1 ? 0 : j];
          s[NJ == 1 ? 0 : j] += t * t;
        }
      }
    group_sums<1, NJ, V, WAVE, RED>(A, tm, s, red + (RED == GN_RED_GROUPS ? A.redbuf : 0));
#pragma unroll
    for (int j = 0; j < NJ; ++j) s[j] = rsqrtf(s[j] * A.inv_m + A.eps);
    // the first thread of each group writes its statistics
    if (ty == 0 && own)
#pragma unroll
      for (int j = 0; j < NJ; ++j)
        if (const int k = A.by_cg.of(c + j); k * A.cg == c + j) {
          A.st[i * A.G + k] = cp.mean[j];
          A.st[(A.n + i) * A.G + k] = s[j];
        }
    if (col) {
#pragma unroll
      for (int j = 0; j < V; ++j) cp.a[j] = gamma[j] * s[NJ == 1 ? 0 : j];
#pragma unroll
      for (int k = 0; k < NV; ++k)
        if (ty + k * A.TY < A.hw)
          cp.template put<SILU, DROP>(A, key, xr[k], pix0 + ty + k * A.TY, c);
    }
  }
}

// Split, first pass: a chunk's mean and squared differences per group.  Each
// thread sums differences from a pivot, and their squares, block by block of its
// rows; a block of n2 values joins the n1 before it, whose mean is its pivot, by
//   mean += s1 / (n1 + n2), M2 += s2 - s1^2 / (n1 + n2)
// which is Chan's formula (gn_apply) for such a pivot.  A block is as long as all
// before it, and 256 values at most: s1^2 / (n1 + n2) <= s2 n2 / (n1 + n2) is then at
// most half of s2, whatever the values.  (The first block's pivot is the mean of eight
// of its 32 values, or one of its 16: at most fifteen sixteenths.)  A single pivot for
// a whole chunk would cancel by the number of its values where the first of them is
// far from the others (1 / std off by 3e-4 at 784 values a thread, 1e-2 at 3136; 3e-7
// this way, in the same time).
template <typename XT, int V, int NJ, int RED>
__global__ __launch_bounds__(1024) void k_gn_stats(GnArgs A) {
  extern __shared__ float lds[];
  const Team<false> tm(A);
  const int by = A.by_tiles.of(blockIdx.x), tile = blockIdx.x - by * A.tiles;
  const int i = A.by_chunks.of(by), p0 = (by - i * A.chunks) * A.chunk, np = min(A.hw - p0, A.chunk);
  const int c = tile * A.W + tm.tx * V;
  const bool own = tm.tx < A.cols && c < A.C;
  const int rows = own && tm.ty < A.TY && tm.ty < np ? (np - tm.ty + A.TY - 1) / A.TY : 0;
  const XT *x = static_cast<const XT *>(A.x) + (int64_t(i) * A.hw + p0 + tm.ty) * A.ldx + c;
  const int64_t dx = int64_t(A.TY) * A.ldx;
  // mean: the pivot, `low` what its roundings left (one at every block)
  float mean[NJ], low[NJ], m2[NJ], s1[NJ], s2[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) mean[j] = low[j] = m2[j] = 0.f;
  // (eight single elements in flight: a load instruction moves an eighth of a vector's)
  constexpr int U = V == 1 ? 8 : 4;
  auto add = [&](const Vec<XT, V> &v) {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float t = float(v.v[j]) - mean[NJ == 1 ? 0 : j];
      s1[NJ == 1 ? 0 : j] += t;
      s2[NJ == 1 ? 0 : j] += t * t;
    }
  };
  if (rows > 0) {
    const Vec<XT, V> v = load_vec<XT, V>(x);
#pragma unroll
    for (int j = 0; j < V; ++j) mean[NJ == 1 ? 0 : j] += NJ == 1 ? float(v.v[j]) * (1.f / V) : float(v.v[j]);
  }
  constexpr int E = NJ == 1 ? V : 1;  // values a row adds to a sum
  for (int r = 0; r < rows;) {
    const int end = min(rows, r + (r ? min(r, 256 / E) : E == 8 ? 4 : 16));
#pragma unroll
    for (int j = 0; j < NJ; ++j) s1[j] = s2[j] = 0.f;
    for (; r + U <= end; r += U, x += U * dx) {
      Vec<XT, V> xr[U];
#pragma unroll
      for (int k = 0; k < U; ++k) xr[k] = load_vec<XT, V>(x + k * dx);
      // all of them before the first wait: to save registers the compiler would
      // take them one by one (128 x 3136 pixels x 72 channels in 24 groups: 50 us, 39)
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int k = 0; k < U; ++k) add(xr[k]);
    }
    for (; r < end; ++r, x += dx) add(load_vec<XT, V>(x));
    const float inv = 1.f / float(r * E);
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const float q = s1[j] * inv, step = q + low[j], sum = mean[j] + step, part = sum - mean[j];
      low[j] = (mean[j] - (sum - part)) + (step - part);
      mean[j] = sum;
      // squares past fp32's range stay so (finite ones are at least s1 q)
      m2[j] += s2[j] <= 3.4028234e38f ? fmaxf(s2[j] - s1[j] * q, 0.f) : s2[j];
    }
  }
  const float cnt = float(rows * E), m = float(int64_t(np) * A.cg);
  float s[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) s[j] = cnt * mean[j];
  group_sums<1, NJ, V, false, RED>(A, tm, s, lds);
  float all[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    all[j] = s[j] / m;
    const float t = mean[j] - all[j];
    s[j] = m2[j] + cnt * t * t;
  }
  group_sums<1, NJ, V, false, RED>(A, tm, s, lds + (RED == GN_RED_GROUPS ? A.redbuf : 0));
  if (tm.ty == 0 && own)
#pragma unroll
    for (int j = 0; j < NJ; ++j)
      if (const int k = A.by_cg.of(c + j); k * A.cg == c + j) {
        float *const o = A.gpart + (int64_t(by) * A.G + k) * 2;
        o[0] = all[j];
        o[1] = s[j];
      }
}

// The mean and squared differences of L chunks' (mean_q, M2_q), lanes of a
// wavefront side by side, in double: sum cnt mean_q / m, then sum (M2_q + cnt
// (mean_q - mean)^2).
template <int L, int PER>
__device__ __forceinline__ void merge_chunks(const GnArgs &A, int i, int k, int lane, float &mean, float &rstd) {
  const float2 *const part = reinterpret_cast<const float2 *>(A.gpart) + int64_t(i) * A.chunks1 * A.G + k;
  auto count = [&](int q) { return double(min(A.chunk1, A.hw - q * A.chunk1)) * A.cg; };
  const double m = double(A.hw) * A.cg;
  float2 v[PER];
  double s = 0;
  for (int q0 = 0; q0 < A.chunks1; q0 += L * PER)
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const int q = q0 + u * L + lane;
      if (q < A.chunks1) {
        v[u] = part[int64_t(q) * A.G];
        s += count(q) * v[u].x;
      }
    }
#pragma unroll
  for (int off = L / 2; off > 0; off >>= 1) s += __shfl_xor(s, off);
  const double mu = s / m;
  s = 0;
  for (int q0 = 0; q0 < A.chunks1; q0 += L * PER)
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const int q = q0 + u * L + lane;
      if (q < A.chunks1) {
        if (A.chunks1 > L * PER) v[u] = part[int64_t(q) * A.G];
        const double t = v[u].x - mu;
        s += v[u].y + count(q) * t * t;
      }
    }
#pragma unroll
  for (int off = L / 2; off > 0; off >>= 1) s += __shfl_xor(s, off);
  mean = float(mu);
  rstd = rsqrtf(float(s / m) + A.eps);
}

// Many chunks: one wavefront per group of a sample.
__global__ __launch_bounds__(64) void k_gn_merge(GnArgs A) {
  const int i = blockIdx.x / A.G, k = blockIdx.x % A.G;
  float mean, rstd;
  merge_chunks<64, 4>(A, i, k, threadIdx.x, mean, rstd);
  if (threadIdx.x == 0) {
    A.st[i * A.G + k] = mean;
    A.st[(A.n + i) * A.G + k] = rstd;
  }
}

// Split, second pass, and the re-run: the output of a chunk of one sample's
// pixels.  The channels' parameters are formed once in LDS; MERGE: from the
// first pass's chunks, whose statistics the first chunk's workgroups leave.
template <typename XT, int V, bool MERGE>
__global__ __launch_bounds__(256) void k_gn_apply(GnArgs A) {
  extern __shared__ float lds[];
  const int t = threadIdx.x, T = blockDim.x, ty = A.by_vc.of(t), tx = t - ty * A.VC;
  const int by = A.by_tiles.of(blockIdx.x), tile = blockIdx.x - by * A.tiles, c0 = tile * A.W, c = c0 + tx * V;
  const int i = A.by_chunks.of(by), p0 = (by - i * A.chunks) * A.chunk, np = min(A.hw - p0, A.chunk);
  const int64_t pix0 = int64_t(i) * A.hw + p0;
  const bool col = c < A.C && ty < A.TY;
  const XT *const x = static_cast<const XT *>(A.x) + pix0 * A.ldx + c;
  constexpr int U = 2;  // vectors worked on, and as many in flight
  Vec<XT, V> xr[U];
#pragma unroll
  for (int k = 0; k < U; ++k)
    if (col && ty + k * A.TY < np) xr[k] = load_vec<XT, V>(x + int64_t(ty + k * A.TY) * A.ldx);
  const DropKey key = drop_key(A.drop);
  const int nc = min(A.W, A.C - c0), g0 = A.by_cg.of(c0), ng = A.by_cg.of(c0 + nc - 1) - g0 + 1;
  if (MERGE) {
    float *const gs = lds + 3 * A.W;
    for (int g = t / 8; g - t / 8 < ng; g += T / 8) {
      float mean, rstd;
      merge_chunks<8, 8>(A, i, g0 + min(g, ng - 1), t % 8, mean, rstd);
      if (t % 8 == 0 && g < ng) {
        gs[2 * g] = mean;
        gs[2 * g + 1] = rstd;
        // the tile that a group begins in is the one that leaves its statistics
        if (p0 == 0 && (g0 + g) * A.cg >= c0) {
          A.st[i * A.G + g0 + g] = mean;
          A.st[(A.n + i) * A.G + g0 + g] = rstd;
        }
      }
    }
    __syncthreads();
  }
  for (int e = t; e < nc; e += T) {
    const int g = A.by_cg.of(c0 + e);
    const float *const gs = lds + 3 * A.W + 2 * (g - g0);
    lds[e] = MERGE ? gs[0] : A.st[i * A.G + g];
    lds[A.W + e] = A.gamma[c0 + e] * (MERGE ? gs[1] : A.st[(A.n + i) * A.G + g]);
    lds[2 * A.W + e] = A.beta[c0 + e];
  }
  __syncthreads();
  if (!col) return;
  Column<XT, V, V> cp;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    cp.mean[j] = lds[tx * V + j];
    cp.a[j] = lds[A.W + tx * V + j];
    cp.b[j] = lds[2 * A.W + tx * V + j];
  }
  gn_choose(A, [&](auto silu, auto drop) {
    int r = ty;
    // element by element, while every thread has all its pixels: without conditions the
    // wait for a load is for it alone, not for the stores before it as well (16 x 784
    // pixels x 333 channels 12.3 -> 8.7 us; vectors take the same time either way)
    for (int q = 2 * U * A.TY; V == 1 && q <= np; q += U * A.TY, r += U * A.TY) {
      Vec<XT, V> nx[U];
#pragma unroll
      for (int k = 0; k < U; ++k) nx[k] = load_vec<XT, V>(x + int64_t(r + (U + k) * A.TY) * A.ldx);
#pragma unroll
      for (int k = 0; k < U; ++k) cp.template put<silu.value, drop.value>(A, key, xr[k], pix0 + r + k * A.TY, c);
#pragma unroll
      for (int k = 0; k < U; ++k) xr[k] = nx[k];
    }
    for (; r < np; r += U * A.TY) {
      Vec<XT, V> nx[U];
#pragma unroll
      for (int k = 0; k < U; ++k)
        if (r + (U + k) * A.TY < np) nx[k] = load_vec<XT, V>(x + int64_t(r + (U + k) * A.TY) * A.ldx);
#pragma unroll
      for (int k = 0; k < U; ++k)
        if (r + k * A.TY < np) cp.template put<silu.value, drop.value>(A, key, xr[k], pix0 + r + k * A.TY, c);
#pragma unroll
      for (int k = 0; k < U; ++k) xr[k] = nx[k];
    }
  });
}

// The re-run where a sample's pixels are few: workgroups take pixels of any
// sample, and a vector's statistics are read with it.
template <typename XT, int V, int NJ>
__global__ __launch_bounds__(256) void k_gn_apply_rows(GnArgs A) {
  const int ty = A.by_vc.of(threadIdx.x), tx = threadIdx.x - ty * A.VC;
  const int by = A.by_tiles.of(blockIdx.x), c = (blockIdx.x - by * A.tiles) * A.W + tx * V;
  if (c >= A.C || ty >= A.TY) return;
  const DropKey key = drop_key(A.drop);
  const GnGroups<V, NJ> grp(A, c);
  Column<XT, V, NJ> cp;
  float gamma[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    gamma[j] = A.gamma[c + j];
    cp.b[j] = A.beta[c + j];
  }
  // below 2^30 pixels, samples of fewer than 64 (gn_few_pixels)
  const int p0 = by * A.chunk, p1 = min(A.n * A.hw, p0 + A.chunk);
  gn_choose(A, [&](auto silu, auto drop) {
    for (int p = p0 + ty; p < p1; p += A.TY) {
      const Vec<XT, V> x = load_vec<XT, V>(static_cast<const XT *>(A.x) + int64_t(p) * A.ldx + c);
      const int i = p / A.hw;
      float rstd[NJ];
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        cp.mean[j] = A.st[i * A.G + grp.k[j]];
        rstd[j] = A.st[(A.n + i) * A.G + grp.k[j]];
      }
#pragma unroll
      for (int j = 0; j < V; ++j) cp.a[j] = gamma[j] * rstd[NJ == 1 ? 0 : j];
      cp.template put<silu.value, drop.value>(A, key, x, p, c);
    }
  });
}

template <typename XT, int V, int NV, int NJ>
void launch_resident(hipStream_t s, const GnPlan &g, const GnArgs &a) {
  const dim3 grid(uint32_t(g.first.blocks)), block(g.first.threads);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, g.lds, s, a); };
  gn_choose(a, [&](auto silu, auto drop) {
    constexpr bool S = decltype(silu)::value, D = decltype(drop)::value;
    // a wavefront's tile ends at two vectors a thread (gn_plan)
    if constexpr (NV <= 2)
      if (g.wave)
        return g.red == GN_RED_GROUPS ? go(k_gn_fwd<XT, V, NV, NJ, true, GN_RED_GROUPS, S, D>)
                                      : go(k_gn_fwd<XT, V, NV, NJ, true, GN_RED_COLUMNS, S, D>);
    g.red == GN_RED_GROUPS    ? go(k_gn_fwd<XT, V, NV, NJ, false, GN_RED_GROUPS, S, D>)
    : g.red == GN_RED_COLUMNS ? go(k_gn_fwd<XT, V, NV, NJ, false, GN_RED_COLUMNS, S, D>)
                              : go(k_gn_fwd<XT, V, NV, NJ, false, GN_RED_TREE, S, D>);
  });
}

size_t apply_lds(const GnArgs &a, bool merge) {
  return 4 * (3 * size_t(a.W) + (merge ? 2 * (size_t(a.W) / a.cg + 2) : 0));
}

template <typename XT, int V, int NJ>
void run_fwd(hipStream_t s, const GnProblem &p, const GnPlan &g, GnArgs a) {
  if (g.resident) {
    if (g.NV <= 1) return launch_resident<XT, V, 1, NJ>(s, g, a);
    if (g.NV <= 2) return launch_resident<XT, V, 2, NJ>(s, g, a);
    if (g.NV <= 4) return launch_resident<XT, V, 4, NJ>(s, g, a);
    if (g.NV <= 8) return launch_resident<XT, V, 8, NJ>(s, g, a);
    // fp32 vectors stop at 8 (gn_plan)
    if constexpr (V == 1 || sizeof(XT) == 2) launch_resident<XT, V, 16, NJ>(s, g, a);
    return;
  }
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(uint32_t(g.first.blocks)), dim3(g.first.threads), g.lds, s, a);
  };
  g.red == GN_RED_GROUPS    ? go(k_gn_stats<XT, V, NJ, GN_RED_GROUPS>)
  : g.red == GN_RED_COLUMNS ? go(k_gn_stats<XT, V, NJ, GN_RED_COLUMNS>)
                            : go(k_gn_stats<XT, V, NJ, GN_RED_TREE>);
  GnArgs b = gn_args(p, g.second, a.drop);
  b.x = a.x;
  b.out = a.out;
  b.ldo = a.ldo;
  b.gamma = a.gamma;
  b.beta = a.beta;
  b.st = a.st;
  b.gpart = a.gpart;
  b.chunks1 = int(g.first.chunks);
  b.chunk1 = int(g.first.chunk);
  const dim3 grid(uint32_t(g.second.blocks)), block(g.second.threads);
  if (g.merge) {
    hipLaunchKernelGGL(k_gn_merge, dim3(uint32_t(p.n * p.G)), dim3(64), 0, s, b);
    hipLaunchKernelGGL((k_gn_apply<XT, V, false>), grid, block, apply_lds(b, false), s, b);
  } else {
    hipLaunchKernelGGL((k_gn_apply<XT, V, true>), grid, block, apply_lds(b, true), s, b);
  }
}

template <typename XT, int V, int NJ>
void run_apply(hipStream_t s, const GnCover &v, const GnArgs &a) {
  const dim3 grid(uint32_t(v.blocks)), block(v.threads);
  if (gn_few_pixels(a.hw))
    hipLaunchKernelGGL((k_gn_apply_rows<XT, V, NJ>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((k_gn_apply<XT, V, false>), grid, block, apply_lds(a, false), s, a);
}

}  // namespace

void gn_forward(hipStream_t s, const GnProblem &p, const GnPlan &g, const void *x, const float *gamma,
                const float *beta, const DropArgs &drop, void *y, float *st, void *ws) {
  GnArgs a = gn_args(p, g.first, drop);
  a.rows = int(g.rows);
  a.redbuf = g.redbuf;
  a.pack = g.pack;
  a.x = x;
  a.out = y;
  a.ldo = p.ldy;
  a.gamma = gamma;
  a.beta = beta;
  a.st = st;
  a.gpart = static_cast<float *>(ws);
  if (g.first.V == 1)
    p.xf ? run_fwd<float, 1, 1>(s, p, g, a) : run_fwd<__bf16, 1, 1>(s, p, g, a);
  else if (g.NJ == 1)
    p.xf ? run_fwd<float, 8, 1>(s, p, g, a) : run_fwd<__bf16, 8, 1>(s, p, g, a);
  else
    p.xf ? run_fwd<float, 8, 8>(s, p, g, a) : run_fwd<__bf16, 8, 8>(s, p, g, a);
}

void gn_apply(hipStream_t s, const GnProblem &p, const GnCover &v, const void *x, const float *st,
              const float *gamma, const float *beta, const DropArgs &drop, void *y) {
  GnArgs a = gn_args(p, v, drop);
  a.x = x;
  a.out = y;
  a.ldo = p.ldy;
  a.gamma = gamma;
  a.beta = beta;
  a.st = const_cast<float *>(st);
  if (v.V == 1)
    p.xf ? run_apply<float, 1, 1>(s, v, a) : run_apply<__bf16, 1, 1>(s, v, a);
  else if (p.cg % 8 == 0)
    p.xf ? run_apply<float, 8, 1>(s, v, a) : run_apply<__bf16, 8, 1>(s, v, a);
  else
    p.xf ? run_apply<float, 8, 8>(s, v, a) : run_apply<__bf16, 8, 8>(s, v, a);
}

}  // namespace ckpt
