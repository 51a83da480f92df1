// Group norm with an activation and dropout, backward, over channels-last
// tensors.  From x, the statistics, the counter and g alone (neither output nor
// mask is kept):
//
//   t = x - mean, u = t a + beta (a = gamma rstd), xhat = t rstd
//   du = dropout(g) act'(u), dbeta = sum du, dgamma = sum du xhat
//   k1 = sum a du / m, k2 = rstd sum a du xhat / m over a group's m values
//   d = a du - k1 - t k2
//
// As in the forward, a tile that fits stays in registers (x as loaded, du in
// fp32): x and g are read once.  A larger one takes a pass for the channels'
// sums per chunk of pixels and a second that adds up the chunks, folds the
// channels into their groups and forms d.  Channel sums leave one record per
// workgroup (or chunk), added in a fixed order.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>

#include "common.h"
#include "gn.h"

namespace ckpt {
namespace gnb {

// A vector column's parameters; du of one vector, in place of g.
template <typename XT, int V, int NJ>
struct Column {
  float mean[NJ], a[V], beta[V];
  template <bool SILU, bool DROP>
  __device__ __forceinline__ void du(const GnArgs &A, const DropKey &key, const Vec<XT, V> &x, uint64_t pix, int c,
                                     float g[V]) const {
    if (DROP) gn_drop<V>(A, key, pix, c, g);
    if (SILU || A.act == GN_ACT_RELU)
#pragma unroll
      for (int j = 0; j < V; ++j)
        g[j] = gn_act_bwd<SILU, sizeof(XT) == 4>(true, gn_affine(float(x.v[j]), mean[NJ == 1 ? 0 : j], a[j], beta[j]), g[j]);
  }
  template <typename DT>
  __device__ __forceinline__ void put(const GnArgs &A, const Vec<XT, V> &x, const float (&k1)[NJ],
                                      const float (&k2)[NJ], int64_t pix, int c, const float du[V]) const {
    float v[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int q = NJ == 1 ? 0 : j;
      v[j] = a[j] * du[j] - k1[q] - (float(x.v[j]) - mean[q]) * k2[q];
    }
    store_vec<DT, V>(static_cast<DT *>(A.out) + pix * A.ldo + c, v);
  }
};

// The channels' sums of a workgroup, ch[j] = sum du xhat and ch[V + j] = sum du of
// a thread's pixels: record `by` of cpart, or dgamma and dbeta themselves.
template <int V, bool WAVE, int RED>
__device__ __forceinline__ void channel_record(const GnArgs &A, const Team<WAVE> &tm, int teams, int tile, int by,
                                               float (&ch)[2 * V], float *lds) {
  const int O = 2 * V * A.VC;
  float *const out0 = A.cpart ? A.cpart + int64_t(by) * 2 * A.C : A.dgamma;
  float *const out1 = A.cpart ? out0 + A.C : A.dbeta;
  const float *sums = lds;
  int parts, pitch;
  if constexpr (RED != GN_RED_TREE) {
    const int w = threadIdx.x >> 6;
    wave_columns<2 * V>(ch, threadIdx.x & 63, A.VC, tm.tx, lds + w * O);
    parts = blockDim.x >> 6;
    pitch = O;
  } else {
    const int tree = (A.TY + (A.TY + 7) / 8) * O;
    float *const mine = lds + tm.index * tree;
    if (tm.ty < A.TY)
#pragma unroll
      for (int k = 0; k < 2 * V; ++k) mine[tm.ty * O + k * A.VC + tm.tx] = ch[k];
    sums = lds + (row_tree<WAVE, 2 * V>(tm, A.TY, A.VC, mine) - mine);
    parts = teams;
    pitch = tree;
  }
  __syncthreads();
  // thread by channel, so that the record is written in order
  for (int o = threadIdx.x; o < 2 * A.W; o += blockDim.x) {
    const int q = o >= A.W, e = o - q * A.W, k = q * V + e % V;
    float s = 0.f;
    for (int r = 0; r < parts; ++r) s += sums[r * pitch + k * A.VC + e / V];
    if (tile * A.W + e < A.C) (q ? out1 : out0)[tile * A.W + e] = s;
  }
}

// Resident teams: a workgroup with one sample, a wavefront that loops over samples,
// and a workgroup that does (gn_plan: more samples than fill the device).
enum { GNB_ONE = 0, GNB_WAVE = 1, GNB_LOOP = 2 };

// Wavefronts a SIMD that a resident kernel's registers leave room for: 4 (128
// registers), 2 where its vectors, or the sums of eight channels that a team keeps from
// sample to sample, take more (wavefronts, 2048 samples of 16 pixels x 64 channels in
// groups of four: 17.1 us held to 128 registers, 11.9 not).
template <int V, int NV, int NJ, int TEAM>
constexpr int gnb_waves() {
  return V == 8 && (NV >= 4 || (TEAM != GNB_ONE && NJ > 1) || (TEAM == GNB_LOOP && NV >= 2)) ? 2 : 4;
}

// Resident: one team per (sample, tile), or per tile of several samples in turn.
// GNB_LOOP chooses SiLU and dropout as it runs (from its second sample on, the code
// jumped to is in the instruction cache), the others are compiled for them.
template <typename XT, typename GT_, typename DT, int V, int NV, int NJ, int TEAM, int RED, bool SILU,
          bool DROP>
__global__ __launch_bounds__(TEAM == GNB_WAVE ? 256 : V == 8 ? 512 : 1024, (gnb_waves<V, NV, NJ, TEAM>())) void k_gn_bwd(GnArgs A) {
  constexpr bool WAVE = TEAM == GNB_WAVE;
  extern __shared__ float lds[];
  const Team<WAVE> tm(A);
  const int teams = WAVE ? blockDim.x / 64 : 1;
  const int by = A.by_tiles.of(blockIdx.x), tile = blockIdx.x - by * A.tiles;
  const int c = tile * A.W + tm.tx * V;
  const bool column = tm.tx < A.cols && c < A.C;
  float *const red = lds + tm.index * (RED == GN_RED_GROUPS ? 2 : 1) * A.redbuf;
  int buf = 0;
  const DropKey key = drop_key(A.drop);
  const GnGroups<V, NJ> grp(A, column ? c : 0);
  float ch[2 * V];
#pragma unroll
  for (int j = 0; j < 2 * V; ++j) ch[j] = 0.f;
  // a wavefront's rows are pixels, or samples of one
  const bool packed = WAVE && A.pack > 1;
  const int ty = packed ? 0 : tm.ty, step = A.rows * teams * (WAVE ? A.pack : 1);
  for (int i0 = (by * teams + tm.index) * (WAVE ? A.pack : 1); i0 < A.n; i0 = TEAM == GNB_ONE ? A.n : i0 + step) {
    const bool live = !packed || i0 + tm.ty < A.n, col = column && live && ty < A.TY;
    const int i = packed ? min(i0 + tm.ty, A.n - 1) : i0;
    const int64_t pix0 = int64_t(i) * A.hw;
    const XT *const x = static_cast<const XT *>(A.x) + (pix0 + ty) * A.ldx + c;
    const GT_ *const g = static_cast<const GT_ *>(A.g) + (pix0 + ty) * A.ldg + c;
    const int64_t dx = int64_t(A.TY) * A.ldx, dg = int64_t(A.TY) * A.ldg;
    Vec<XT, V> xr[NV];
    Vec<GT_, V> gr[NV];
    float du[NV][V];
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (col && ty + k * A.TY < A.hw) {
        xr[k] = load_vec<XT, V>(x + k * dx);
        gr[k] = load_vec<GT_, V>(g + k * dg);
      }
    Column<XT, V, NJ> cp;
    float rstd[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      cp.mean[j] = A.st[i * A.G + grp.k[j]];
      rstd[j] = A.st[(A.n + i) * A.G + grp.k[j]];
    }
#pragma unroll
    for (int j = 0; j < V; ++j) {
      cp.a[j] = A.gamma[col ? c + j : j] * rstd[NJ == 1 ? 0 : j];
      cp.beta[j] = A.beta[col ? c + j : j];
    }
    float s1[V], s2[V];  // sums of du and of du t
#pragma unroll
    for (int j = 0; j < V; ++j) s1[j] = s2[j] = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (col && ty + k * A.TY < A.hw) {
#pragma unroll
        for (int j = 0; j < V; ++j) du[k][j] = float(gr[k].v[j]);
        const uint64_t pix = uint64_t(pix0 + ty + k * A.TY);
        if constexpr (TEAM == GNB_LOOP)
          gn_choose(A, [&](auto silu, auto drop) { cp.template du<silu.value, drop.value>(A, key, xr[k], pix, c, du[k]); });
        else
          cp.template du<SILU, DROP>(A, key, xr[k], pix, c, du[k]);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          s1[j] += du[k][j];
          s2[j] += du[k][j] * (float(xr[k].v[j]) - cp.mean[NJ == 1 ? 0 : j]);
        }
      }
    float s[2 * NJ];
#pragma unroll
    for (int j = 0; j < 2 * NJ; ++j) s[j] = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int q = NJ == 1 ? 0 : j;
      s2[j] *= rstd[q];
      ch[j] += s2[j];
      ch[V + j] += s1[j];
      s[q] += cp.a[j] * s1[j];
      s[NJ + q] += cp.a[j] * s2[j];
    }
    group_sums<2, NJ, V, WAVE, RED>(A, tm, s, red + buf);
    if (RED == GN_RED_GROUPS) buf = A.redbuf - buf;
    if (col) {
      float k1[NJ], k2[NJ];
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        k1[j] = s[j] * A.inv_m;
        k2[j] = rstd[j] * s[NJ + j] * A.inv_m;
      }
#pragma unroll
      for (int k = 0; k < NV; ++k)
        if (ty + k * A.TY < A.hw) {
          cp.template put<DT>(A, xr[k], k1, k2, pix0 + ty + k * A.TY, c, du[k]);
        }
    }
  }
  __syncthreads();
  channel_record<V, WAVE, RED>(A, tm, teams, tile, by, ch, lds);
}

// The parameters of nc channels from c0 of sample i, in LDS: mean | a | beta, W each.
__device__ __forceinline__ void channel_params(const GnArgs &A, int i, int c0, int nc, float *lds) {
  for (int e = threadIdx.x; e < nc; e += blockDim.x) {
    const int g = A.by_cg.of(c0 + e);
    lds[e] = A.st[i * A.G + g];
    lds[A.W + e] = A.gamma[c0 + e] * A.st[(A.n + i) * A.G + g];
    lds[2 * A.W + e] = A.beta[c0 + e];
  }
}

template <typename XT, int V>
__device__ __forceinline__ void take_params(const GnArgs &A, int tx, const float *lds, Column<XT, V, V> &cp) {
#pragma unroll
  for (int j = 0; j < V; ++j) {
    cp.mean[j] = lds[tx * V + j];
    cp.a[j] = lds[A.W + tx * V + j];
    cp.beta[j] = lds[2 * A.W + tx * V + j];
  }
}

// Split, first pass: a chunk's channel sums.
template <typename XT, typename GT_, int V, int RED>
__global__ __launch_bounds__(V == 8 ? 512 : 1024) void k_gn_bwd_sums(GnArgs A) {
  extern __shared__ float lds[];
  const Team<false> tm(A);
  const int by = A.by_tiles.of(blockIdx.x), tile = blockIdx.x - by * A.tiles, c0 = tile * A.W, c = c0 + tm.tx * V;
  const int i = A.by_chunks.of(by), p0 = (by - i * A.chunks) * A.chunk, np = min(A.hw - p0, A.chunk);
  const int64_t pix0 = int64_t(i) * A.hw + p0;
  const bool col = tm.tx < A.cols && c < A.C && tm.ty < A.TY;
  const XT *const x = static_cast<const XT *>(A.x) + pix0 * A.ldx + c;
  const GT_ *const g = static_cast<const GT_ *>(A.g) + pix0 * A.ldg + c;
  // vectors in flight besides those worked on: more cost registers that hide the
  // arithmetic better (stage 1 with dropout: 58.6 us, 61.9 with two)
  constexpr int U = V == 1 ? 4 : 1;
  Vec<XT, V> xr[U];
  Vec<GT_, V> gr[U];
#pragma unroll
  for (int k = 0; k < U; ++k)
    if (col && tm.ty + k * A.TY < np) {
      xr[k] = load_vec<XT, V>(x + int64_t(tm.ty + k * A.TY) * A.ldx);
      gr[k] = load_vec<GT_, V>(g + int64_t(tm.ty + k * A.TY) * A.ldg);
    }
  const DropKey key = drop_key(A.drop);
  channel_params(A, i, c0, min(A.W, A.C - c0), lds);
  __syncthreads();
  float ch[2 * V];
#pragma unroll
  for (int j = 0; j < 2 * V; ++j) ch[j] = 0.f;
  if (col) {
    Column<XT, V, V> cp;
    take_params(A, tm.tx, lds, cp);
    auto add = [&](auto silu, auto drop, const Vec<XT, V> &xv, const Vec<GT_, V> &gv, int p) {
      float du[V];
#pragma unroll
      for (int j = 0; j < V; ++j) du[j] = float(gv.v[j]);
      cp.template du<silu.value, drop.value>(A, key, xv, uint64_t(pix0 + p), c, du);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        ch[j] += du[j] * (float(xv.v[j]) - cp.mean[j]);
        ch[V + j] += du[j];
      }
    };
    gn_choose(A, [&](auto silu, auto drop) {
      int r = tm.ty;
      // element by element, while every thread has all its pixels (k_gn_apply; vectors
      // lose by it: stage 1 with dropout 58.6 -> 62.7 us)
      for (int q = 2 * U * A.TY; V == 1 && q <= np; q += U * A.TY, r += U * A.TY) {
        Vec<XT, V> nx[U];
        Vec<GT_, V> ng[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
          nx[k] = load_vec<XT, V>(x + int64_t(r + (U + k) * A.TY) * A.ldx);
          ng[k] = load_vec<GT_, V>(g + int64_t(r + (U + k) * A.TY) * A.ldg);
        }
#pragma unroll
        for (int k = 0; k < U; ++k) add(silu, drop, xr[k], gr[k], r + k * A.TY);
#pragma unroll
        for (int k = 0; k < U; ++k) {
          xr[k] = nx[k];
          gr[k] = ng[k];
        }
      }
      for (; r < np; r += U * A.TY) {
        Vec<XT, V> nx[U];
        Vec<GT_, V> ng[U];
#pragma unroll
        for (int k = 0; k < U; ++k)
          if (r + (U + k) * A.TY < np) {
            nx[k] = load_vec<XT, V>(x + int64_t(r + (U + k) * A.TY) * A.ldx);
            ng[k] = load_vec<GT_, V>(g + int64_t(r + (U + k) * A.TY) * A.ldg);
          }
#pragma unroll
        for (int k = 0; k < U; ++k)
          if (r + k * A.TY < np) add(silu, drop, xr[k], gr[k], r + k * A.TY);
#pragma unroll
        for (int k = 0; k < U; ++k) {
          xr[k] = nx[k];
          gr[k] = ng[k];
        }
      }
    });
#pragma unroll
    for (int j = 0; j < V; ++j) ch[j] *= A.st[(A.n + i) * A.G + A.by_cg.of(c + j)];
  }
  __syncthreads();
  channel_record<V, false, RED>(A, tm, 1, tile, by, ch, lds);
}

// The sums of `rows` records [2][C] (dgamma | dbeta at the end): the 16 columns from
// 16 blk, a thread per column and row in turn, added in a fixed order.  A call of many
// samples may have a record for each: they are taken eight at a time without conditions
// (with one per load these waited for each other: the backward of 20000 samples of 49
// pixels x 64 channels took 130 us, without 107) and added as a tree.
// red: [blockDim / 16][17].
__device__ __forceinline__ void record_sums(const float *cpart, int rows, int C, int blk, float *out0, float *out1,
                                            float *red) {
  const int e = blk * 16 + threadIdx.x % 16, r0 = threadIdx.x / 16, R = blockDim.x / 16;
  float s = 0.f;
  if (e < 2 * C) {
    const float *const part = cpart + e;
    constexpr int U = 8;
    float v[U];
    int r = r0;
    for (; r + (U - 1) * R < rows; r += U * R) {
#pragma unroll
      for (int k = 0; k < U; ++k) v[k] = part[int64_t(r + k * R) * 2 * C];
      s += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
    }
    if (r < rows) {
#pragma unroll
      for (int k = 0; k < U; ++k) v[k] = r + k * R < rows ? part[int64_t(r + k * R) * 2 * C] : 0.f;
#pragma unroll
      for (int k = 0; k < U; ++k) s += v[k];
    }
  }
  red[r0 * 17 + threadIdx.x % 16] = s;
  __syncthreads();
  if (threadIdx.x < 16 && e < 2 * C) {
    s = 0.f;
    for (int r = 0; r < R; ++r) s += red[r * 17 + threadIdx.x];
    (e < C ? out0 : out1)[e < C ? e : e - C] = s;
  }
}

// Split, second pass: d of a chunk of one sample's pixels.  The first `sums`
// workgroups add up the records of dgamma and dbeta beside it.  MERGED: the
// groups' sums are in gsum; else the tile holds whole groups and forms them from
// the chunks' channel sums.
template <typename XT, typename GT_, typename DT, int V, bool MERGED>
__global__ __launch_bounds__(V == 8 ? 256 : 1024) void k_gn_bwd_apply(GnArgs A, int sums) {
  extern __shared__ float lds[];
  if (int(blockIdx.x) < sums) return record_sums(A.cpart, A.n * A.chunks1, A.C, blockIdx.x, A.dgamma, A.dbeta, lds);
  const int t = threadIdx.x, T = blockDim.x, ty = A.by_vc.of(t), tx = t - ty * A.VC;
  const int blk = blockIdx.x - sums, by = A.by_tiles.of(blk), c0 = (blk - by * A.tiles) * A.W, c = c0 + tx * V;
  const int i = A.by_chunks.of(by), p0 = (by - i * A.chunks) * A.chunk, np = min(A.hw - p0, A.chunk);
  const int64_t pix0 = int64_t(i) * A.hw + p0;
  const bool col = c < A.C && ty < A.TY;
  const XT *const x = static_cast<const XT *>(A.x) + pix0 * A.ldx + c;
  const GT_ *const g = static_cast<const GT_ *>(A.g) + pix0 * A.ldg + c;
  constexpr int U = V == 1 ? 4 : 1;
  Vec<XT, V> xr[U];
  Vec<GT_, V> gr[U];
#pragma unroll
  for (int k = 0; k < U; ++k)
    if (col && ty + k * A.TY < np) {
      xr[k] = load_vec<XT, V>(x + int64_t(ty + k * A.TY) * A.ldx);
      gr[k] = load_vec<GT_, V>(g + int64_t(ty + k * A.TY) * A.ldg);
    }
  const DropKey key = drop_key(A.drop);
  const int nc = min(A.W, A.C - c0);
  channel_params(A, i, c0, nc, lds);
  float *const kk = lds + 3 * A.W;  // k1 | k2, W each
  if (MERGED) {
    for (int e = t; e < nc; e += T) {
      const int k = i * A.G + A.by_cg.of(c0 + e);
      kk[e] = A.gsum[2 * k] * A.inv_m;
      kk[A.W + e] = A.st[A.n * A.G + k] * A.gsum[2 * k + 1] * A.inv_m;
    }
    __syncthreads();
  } else {
    // the tile's channel sums, du xhat then du: the chunks dealt to T / (2 W) threads each
    float *const part = kk + 2 * A.W;
    const int S = max(1, T / (2 * A.W));
    for (int o = t; o < 2 * A.W * S; o += T) {
      const int e = o % (2 * A.W), q = e >= A.W, cc = c0 + e - q * A.W;
      float s = 0.f;
      if (cc < A.C) {
        const float *const r = A.cpart + int64_t(i) * A.chunks1 * 2 * A.C + q * A.C + cc;
        constexpr int P = 8;
        for (int k = o / (2 * A.W); k < A.chunks1; k += P * S) {
          float v[P];
#pragma unroll
          for (int u = 0; u < P; ++u) v[u] = k + u * S < A.chunks1 ? r[int64_t(k + u * S) * 2 * A.C] : 0.f;
#pragma unroll
          for (int u = 0; u < P; ++u) s += v[u];
        }
      }
      part[o] = s;
    }
    __syncthreads();
    for (int e = t; e < 2 * A.W; e += T) {
      float s = 0.f;
      for (int k = 0; k < S; ++k) s += part[k * 2 * A.W + e];
      part[e] = s * lds[A.W + e % A.W];  // times a; only this thread reads what it overwrites
    }
    __syncthreads();
    for (int e = t; e < nc; e += T) {
      const int f = A.by_cg.of(e) * A.cg;
      float s1 = 0.f, s2 = 0.f;
      for (int k = 0; k < A.cg; ++k) {
        s2 += part[f + k];
        s1 += part[A.W + f + k];
      }
      kk[e] = s1 * A.inv_m;
      kk[A.W + e] = A.st[(A.n + i) * A.G + A.by_cg.of(c0 + e)] * s2 * A.inv_m;
    }
    __syncthreads();
  }
  if (!col) return;
  Column<XT, V, V> cp;
  take_params(A, tx, lds, cp);
  float k1[V], k2[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    k1[j] = kk[tx * V + j];
    k2[j] = kk[A.W + tx * V + j];
  }
  auto form = [&](auto silu, auto drop, const Vec<XT, V> &xv, const Vec<GT_, V> &gv, int p) {
    float du[V];
#pragma unroll
    for (int j = 0; j < V; ++j) du[j] = float(gv.v[j]);
    cp.template du<silu.value, drop.value>(A, key, xv, uint64_t(pix0 + p), c, du);
    cp.template put<DT>(A, xv, k1, k2, pix0 + p, c, du);
  };
  gn_choose(A, [&](auto silu, auto drop) {
    int r = ty;
    for (int q = 2 * U * A.TY; V == 1 && q <= np; q += U * A.TY, r += U * A.TY) {  // as in the first pass
      Vec<XT, V> nx[U];
      Vec<GT_, V> ng[U];
#pragma unroll
      for (int k = 0; k < U; ++k) {
        nx[k] = load_vec<XT, V>(x + int64_t(r + (U + k) * A.TY) * A.ldx);
        ng[k] = load_vec<GT_, V>(g + int64_t(r + (U + k) * A.TY) * A.ldg);
      }
#pragma unroll
      for (int k = 0; k < U; ++k) form(silu, drop, xr[k], gr[k], r + k * A.TY);
#pragma unroll
      for (int k = 0; k < U; ++k) {
        xr[k] = nx[k];
        gr[k] = ng[k];
      }
    }
    for (; r < np; r += U * A.TY) {
      Vec<XT, V> nx[U];
      Vec<GT_, V> ng[U];
#pragma unroll
      for (int k = 0; k < U; ++k)
        if (r + (U + k) * A.TY < np) {
          nx[k] = load_vec<XT, V>(x + int64_t(r + (U + k) * A.TY) * A.ldx);
          ng[k] = load_vec<GT_, V>(g + int64_t(r + (U + k) * A.TY) * A.ldg);
        }
#pragma unroll
      for (int k = 0; k < U; ++k)
        if (r + k * A.TY < np) form(silu, drop, xr[k], gr[k], r + k * A.TY);
#pragma unroll
      for (int k = 0; k < U; ++k) {
        xr[k] = nx[k];
        gr[k] = ng[k];
      }
    }
  });
}

// many chunks or wide groups: gsum[i][k] = sum a du | sum a du xhat of one group
void merge_groups(hipStream_t s, const GnArgs &a);
// dgamma | dbeta from the resident passes' records (gn_plan: in so many segments first)
void sum_records(hipStream_t s, const GnArgs &a, int segments);

template <typename XT, typename GT_, typename DT, int V, int NV, int NJ>
void launch_resident(hipStream_t s, const GnPlan &g, const GnArgs &a) {
  const dim3 grid(uint32_t(g.first.blocks)), block(g.first.threads);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, g.lds, s, a); };
  gn_choose(a, [&](auto silu, auto drop) {
    constexpr bool S = decltype(silu)::value, D = decltype(drop)::value;
    // a wavefront's tile ends at two vectors a thread (gn_plan)
    if constexpr (NV <= 2)
      if (g.wave)
        return g.red == GN_RED_GROUPS ? go(k_gn_bwd<XT, GT_, DT, V, NV, NJ, GNB_WAVE, GN_RED_GROUPS, S, D>)
                                      : go(k_gn_bwd<XT, GT_, DT, V, NV, NJ, GNB_WAVE, GN_RED_COLUMNS, S, D>);
    // a workgroup loops over samples of four pixels at most, or two (gn_plan); 64 columns
    // or fewer it takes only with three or four, two a thread
    if constexpr (NV <= (V == 8 ? 4 : 2))
      if (g.rows < a.n) {
        if constexpr (V == 8 && NV == 2) {
          if (g.red == GN_RED_COLUMNS) return go(k_gn_bwd<XT, GT_, DT, V, NV, NJ, GNB_LOOP, GN_RED_COLUMNS, false, false>);
          if constexpr (NJ == 1)
            if (g.red == GN_RED_GROUPS) return go(k_gn_bwd<XT, GT_, DT, V, NV, NJ, GNB_LOOP, GN_RED_GROUPS, false, false>);
        }
        return go(k_gn_bwd<XT, GT_, DT, V, NV, NJ, GNB_LOOP, GN_RED_TREE, false, false>);
      }
    g.red == GN_RED_GROUPS    ? go(k_gn_bwd<XT, GT_, DT, V, NV, NJ, GNB_ONE, GN_RED_GROUPS, S, D>)
    : g.red == GN_RED_COLUMNS ? go(k_gn_bwd<XT, GT_, DT, V, NV, NJ, GNB_ONE, GN_RED_COLUMNS, S, D>)
                              : go(k_gn_bwd<XT, GT_, DT, V, NV, NJ, GNB_ONE, GN_RED_TREE, S, D>);
  });
}

template <typename XT, typename GT_, typename DT, int V, int NJ>
void run(hipStream_t s, const GnProblem &p, const GnPlan &g, const GnArgs &a) {
  if (g.resident) {
    if (g.NV <= 1)
      launch_resident<XT, GT_, DT, V, 1, NJ>(s, g, a);
    else if (g.NV <= 2)
      launch_resident<XT, GT_, DT, V, 2, NJ>(s, g, a);
    else if (g.NV <= 4)
      launch_resident<XT, GT_, DT, V, 4, NJ>(s, g, a);
    else if (g.NV <= 8)
      launch_resident<XT, GT_, DT, V, 8, NJ>(s, g, a);
    else if constexpr (V == 1)  // vectors stop at 8 (gn_plan)
      launch_resident<XT, GT_, DT, V, 16, NJ>(s, g, a);
    if (g.rows > 1) sum_records(s, a, g.segments);
    return;
  }
  const GnCover &v = g.first, &w = g.second;
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(uint32_t(v.blocks)), dim3(v.threads), std::max(g.lds, size_t(12) * v.W), s, a);
  };
  g.red == GN_RED_TREE ? go(k_gn_bwd_sums<XT, GT_, V, GN_RED_TREE>) : go(k_gn_bwd_sums<XT, GT_, V, GN_RED_COLUMNS>);
  GnArgs b = gn_args(p, w, a.drop);
  b.x = a.x;
  b.g = a.g;
  b.out = a.out;
  b.ldo = a.ldo;
  b.gamma = a.gamma;
  b.beta = a.beta;
  b.st = a.st;
  b.cpart = a.cpart;
  b.gsum = a.gsum;
  b.dgamma = a.dgamma;
  b.dbeta = a.dbeta;
  b.chunks1 = int(v.chunks);
  b.chunk1 = int(v.chunk);
  const int sums = (2 * p.C + 15) / 16;
  const dim3 grid(uint32_t(w.blocks + sums)), block(w.threads);
  const size_t red = size_t(w.threads / 16) * 17;
  const size_t params = 5 * size_t(w.W);
  if (g.merge) {
    merge_groups(s, b);
    hipLaunchKernelGGL((k_gn_bwd_apply<XT, GT_, DT, V, true>), grid, block, 4 * std::max(red, params), s, b, sums);
  } else {
    const size_t part = 2 * size_t(w.W) * std::max(1, w.threads / (2 * w.W));
    hipLaunchKernelGGL((k_gn_bwd_apply<XT, GT_, DT, V, false>), grid, block, 4 * std::max(red, params + part), s, b,
                       sums);
  }
}

template <typename XT, typename GT_, typename DT>
void run_types(hipStream_t s, const GnProblem &p, const GnPlan &g, const GnArgs &a) {
  if (g.first.V == 1)
    run<XT, GT_, DT, 1, 1>(s, p, g, a);
  else if (g.NJ == 1)
    run<XT, GT_, DT, 8, 1>(s, p, g, a);
  else
    run<XT, GT_, DT, 8, 8>(s, p, g, a);
}

void run_f32(hipStream_t s, const GnProblem &p, const GnPlan &g, const GnArgs &a);
void run_bf16_f32(hipStream_t s, const GnProblem &p, const GnPlan &g, const GnArgs &a);
void run_bf16_bf16(hipStream_t s, const GnProblem &p, const GnPlan &g, const GnArgs &a);

}  // namespace gnb
}  // namespace ckpt
