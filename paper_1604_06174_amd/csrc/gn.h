// Group norm with an activation and dropout over channels-last tensors: the
// launch geometry (host), and the arguments and reductions its kernels share.
//
//   t = x - mean, u = t (gamma rstd) + beta, v = act(u), y = dropout(v)
//
// over groups of cg = C / G consecutive channels of one sample's hw pixels.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "lanes.h"
#include "philox.h"
#include "vec.h"

namespace ckpt {

enum { GN_ACT_NONE = 0, GN_ACT_RELU = 1, GN_ACT_SILU = 2 };

// One call's problem (ckpt_gn_desc with its defaults filled in).
struct GnProblem {
  int64_t n, hw;
  int C, G, cg, act;
  bool xf, gf, df;  // fp32 (else bf16): x and y; g; d
  int64_t ldx, ldy, ldg, ldd;
  float eps;
};

// How a pass covers it.  A tile is W consecutive channels (whole vectors of V) of
// one sample: VC threads cover a pixel (cols = W / V of them with a vector; the rest,
// where VC is rounded up to a power of two, idle), TY pixels are covered at once.
struct GnCover {
  int V, W, tiles, cols, VC, TY, threads;
  int64_t chunks, chunk;  // a sample's pixels: chunks of `chunk`
  int64_t blocks;
};

// How a team's sums are reduced: in LDS alone (VC above 64); within wavefronts first
// (VC a power of two, at most 64); and that with whole groups filling the columns, so
// that a group of vectors is a power of two of them (VC = cols).
enum { GN_RED_TREE = 0, GN_RED_COLUMNS = 1, GN_RED_GROUPS = 2 };

// The passes of a call.
struct GnPlan {
  // resident: a sample's tile (whole groups) stays in the registers of one team, NV
  // vectors a thread; `wave`: of one wavefront each, `teams` a workgroup, else the
  // workgroup is the team.  `rows` workgroups a tile, each with a record of channel sums:
  // below n they loop over samples
  bool resident, wave;
  int NV, teams;
  int pack;  // samples of one pixel that a wavefront takes at once (1: its rows are pixels)
  int64_t rows;
  int segments;  // their records are added up in so many segments first (1: at once)
  // split: `first` leaves every chunk's sums, `second` applies them, adding them up by
  // itself (`merge`: a launch between them does)
  bool merge;
  int NJ;      // values a vector's sums consist of: 1 (it lies within one group) or V
  int red;     // how sums are reduced: GN_RED_*
  int redbuf;  // floats of LDS of one reduction
  size_t lds;
  GnCover first, second;  // resident: `first` alone
  uint64_t ws_groups, ws_channels, ws_sums;  // bytes of the workspace's parts
};

// Throws CKPT_E_UNSUPPORTED for problems outside the kernels' range.
GnPlan gn_plan(const GnProblem &p, bool backward);
// the cover of a split call's second pass, in vectors of V, and of a re-run
GnCover gn_cover_elements(const GnProblem &p, int V, bool whole_groups);
GnCover gn_cover_rerun(const GnProblem &p);
// samples of so few pixels that the re-run's workgroups take those of several
inline bool gn_few_pixels(int64_t hw) { return hw < 64; }
inline uint64_t gn_workspace_bytes(const GnPlan &g) { return g.ws_groups + g.ws_channels + g.ws_sums; }
void gn_forward(hipStream_t s, const GnProblem &p, const GnPlan &g, const void *x, const float *gamma,
                const float *beta, const DropArgs &drop, void *y, float *st, void *ws);
void gn_apply(hipStream_t s, const GnProblem &p, const GnCover &v, const void *x, const float *st,
              const float *gamma, const float *beta, const DropArgs &drop, void *y);
void gn_backward(hipStream_t s, const GnProblem &p, const GnPlan &plan, const void *g, const void *x,
                 const float *st, const float *gamma, const float *beta, const DropArgs &drop, void *d,
                 float *dgamma, float *dbeta, void *ws);

// Division of numbers below 2^21 (block and thread numbers) by one below 2^21, and
// of channels (below 2^20) by a group's (at most 4096), as a multiplication:
// floor(a / d) = floor(a ceil(2^s / d) / 2^s) while a (d - 1) < 2^s.
struct GnDivide {
  uint64_t m;
  __host__ __device__ GnDivide(int64_t d = 1) : m(((uint64_t(1) << 42) + d - 1) / d) {}
  __device__ __forceinline__ int of(uint32_t a) const { return int((uint64_t(a) * m) >> 42); }
};

// what the kernels take
struct GnArgs {
  const void *x, *g;
  void *out;  // y or d
  const float *gamma, *beta;
  float *st;     // mean [n G] | rstd [n G]
  float *gpart;  // forward, split: [n][chunks][G] (mean, squared differences) of the first pass's chunks
  float *cpart;  // backward: [rows][2][C] of the channels (sum du xhat | sum du)
  float *gsum;   // backward, split and merged: [n][G] (sum a du, sum a du xhat)
  float *dgamma, *dbeta;
  int n, hw, rows;
  int chunks, chunk;    // this pass's
  int chunks1, chunk1;  // the first pass's
  int C, G, cg, act;
  GnDivide by_tiles, by_chunks, by_vc, by_cg;
  int64_t ldx, ldg, ldo;
  float eps, inv_m;
  int W, tiles, cols, VC, TY;
  int redbuf, pack;
  DropArgs drop;
};

// the arguments a problem and a pass's cover fix
inline GnArgs gn_args(const GnProblem &p, const GnCover &v, const DropArgs &drop) {
  GnArgs a{};
  a.n = int(p.n);
  a.hw = int(p.hw);
  a.chunks = int(v.chunks);
  a.chunk = int(v.chunk);
  a.by_tiles = GnDivide(v.tiles);
  a.by_chunks = GnDivide(v.chunks);
  a.by_vc = GnDivide(v.VC);
  a.by_cg = GnDivide(p.cg);
  a.C = p.C;
  a.G = p.G;
  a.cg = p.cg;
  a.act = p.act;
  a.ldx = p.ldx;
  a.ldg = p.ldg;
  a.eps = p.eps;
  a.inv_m = float(1.0 / (double(p.hw) * p.cg));
  a.W = v.W;
  a.tiles = v.tiles;
  a.cols = v.cols;
  a.VC = v.VC;
  a.TY = v.TY;
  a.drop = drop;
  return a;
}

// ------------------------------------------------------------- reductions --
// A team: T threads that hold one tile, a wavefront of its own (WAVE) or the
// workgroup.  tx, ty: the vector column and pixel row of a thread; threads with
// ty >= TY are idle.
template <bool WAVE>
struct Team {
  int t, T, tx, ty, index;
  __device__ __forceinline__ explicit Team(const GnArgs &a) {
    t = WAVE ? threadIdx.x & 63 : threadIdx.x;
    T = WAVE ? 64 : blockDim.x;
    index = WAVE ? threadIdx.x >> 6 : 0;
    ty = a.by_vc.of(t);
    tx = t - ty * a.VC;
  }
  // a wavefront's LDS accesses complete in order: keeping the compiler from
  // moving them is all that its own team needs
  __device__ __forceinline__ void sync() const {
    if (WAVE) {
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    } else {
      __syncthreads();
    }
  }
};

// floats of LDS one call of group_sums<NQ, NJ> uses per team of T threads
inline int gn_reduce_floats(const GnCover &v, int red, int T, int NQ, int NJ, int cg) {
  const int gt = NQ * (v.W / cg);
  if (red == GN_RED_GROUPS && NJ == 1) return T / 64 * gt;
  if (red != GN_RED_TREE) return (T > 64 ? T / 64 + 1 : 1) * NQ * v.VC * NJ + gt;
  return (v.TY + (v.TY + 7) / 8) * v.VC * NQ * NJ + gt;
}

// Sums of the rows of red[TY][O], O = VC NVAL, eight at a time (a fixed tree);
// returns where the O sums lie.  Every thread of the team calls it after its
// writes.
template <bool WAVE, int NVAL>
__device__ __forceinline__ float *row_tree(const Team<WAVE> &tm, int TY, int VC, float *red) {
  const int O = VC * NVAL;
  float *src = red, *dst = red + TY * O;
  tm.sync();
  for (int rows = TY; rows > 1;) {
    const int nr = (rows + 7) / 8;
    if (tm.ty < TY)
      for (int slot = tm.ty; slot < nr * NVAL; slot += TY) {
        const int r = slot / NVAL, o = (slot % NVAL) * VC + tm.tx;
        float v[8], s = 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = src[min(8 * r + k, rows - 1) * O + o];
#pragma unroll
        for (int k = 0; k < 8; ++k) s += 8 * r + k < rows ? v[k] : 0.f;
        dst[r * O + o] = s;
      }
    tm.sync();
    float *const f = src;
    src = dst;
    dst = f;
    rows = nr;
  }
  return src;
}

// The sum of n values `pitch` apart, the reads of four at a time in flight.
__device__ __forceinline__ float strided_sum(const float *p, int n, int pitch) {
  float s = 0.f;
  for (int i = 0; i < n; i += 4) {
    float v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = p[min(i + u, n - 1) * pitch];
#pragma unroll
    for (int u = 0; u < 4; ++u) s += i + u < n ? v[u] : 0.f;
  }
  return s;
}

// Sums over whole groups, VC a power of two: quantity q of the m-th of M groups in a
// vector at val[q M + m], or (M = 1) of a group of q1 vectors.  g0: the group (of the
// tile's GT) of the thread's first value; `first`: its vector is that group's first.
template <int NQ, int M, bool WAVE>
__device__ __forceinline__ void whole_groups(const GnArgs &a, const Team<WAVE> &tm, float (&val)[NQ * M], int q1,
                                             int g0, bool first, int GT, float *red) {
  const int lane = tm.t & 63, w = tm.t >> 6, nw = tm.T / 64;
  add_from<NQ * M>(WAVE && a.pack > 1 ? 64 : a.VC, val);  // packed: every row is a sample
  if (M == 1) add_below<NQ * M>(q1, val);
  if (nw == 1) return;
  if (lane < a.VC && first)
#pragma unroll
    for (int q = 0; q < NQ; ++q)
#pragma unroll
      for (int m = 0; m < M; ++m) red[(w * NQ + q) * GT + g0 + m] = val[q * M + m];
  tm.sync();
#pragma unroll
  for (int q = 0; q < NQ; ++q)
#pragma unroll
    for (int m = 0; m < M; ++m) val[q * M + m] = strided_sum(red + q * GT + g0 + m, nw, NQ * GT);
}

// val[q NJ + j], q < NQ: quantity q of the thread's pixels, of its vector (NJ = 1,
// the vector lies within one group) or of its channel j (NJ = V).  Replaced by the
// sum over the whole group it belongs to.  red: redbuf floats of LDS, where RED is
// GN_RED_GROUPS other ones than the call before's (one barrier may be all there is
// between a call's reads and the next one's writes; the others have two).
template <int NQ, int NJ, int V, bool WAVE, int RED>
__device__ __forceinline__ void group_sums(const GnArgs &a, const Team<WAVE> &tm, float (&val)[NQ * NJ],
                                           float *red) {
  constexpr int NVAL = NQ * NJ;
  const int GT = a.by_cg.of(a.W);            // groups of the tile
  const int q1 = NJ == 1 ? a.cg / V : a.cg;  // values of a group
  const int lane = tm.t & 63, w = tm.t >> 6, nw = tm.T / 64;
  if constexpr (RED == GN_RED_GROUPS && NJ == 1) {
    // VC = GT q1 is a power of two, so q1 is one
    const int grp = a.by_cg.of(tm.tx * V);
    whole_groups<NQ, 1, WAVE>(a, tm, val, q1, grp, grp * a.cg == tm.tx * V, GT, red);
    return;
  }
  if constexpr (RED == GN_RED_GROUPS && NJ == 8) {
    // groups of two or four channels: several whole ones in a vector
    auto fold = [&](auto cg) {
      constexpr int CG = decltype(cg)::value, M = NJ / CG;
      float v[NQ * M];
#pragma unroll
      for (int k = 0; k < NQ * M; ++k) {
        v[k] = val[k * CG];
#pragma unroll
        for (int j = 1; j < CG; ++j) v[k] += val[k * CG + j];
      }
      whole_groups<NQ, M, WAVE>(a, tm, v, 1, tm.tx * M, true, GT, red);
#pragma unroll
      for (int k = 0; k < NVAL; ++k) val[k] = v[k / CG];
    };
    if (a.cg == 2) return fold(std::integral_constant<int, 2>());
    if (a.cg == 4) return fold(std::integral_constant<int, 4>());
  }
  const int O = a.VC * NVAL;
  float *col;  // the columns' sums, value k of column tx at k VC + tx
  float *gt;
  if constexpr (RED != GN_RED_TREE) {
    wave_columns<NVAL>(val, lane, a.VC, tm.tx, red + w * O);
    tm.sync();
    col = red;
    gt = red + O;
    if (nw > 1) {
      gt = red + (nw + 1) * O;
      col = red + nw * O;
      for (int o = tm.t; o < O; o += tm.T) col[o] = strided_sum(red + o, nw, O);
      tm.sync();
    }
  } else {
    tm.sync();
    if (tm.ty < a.TY)
#pragma unroll
      for (int k = 0; k < NVAL; ++k) red[tm.ty * O + k * a.VC + tm.tx] = val[k];
    col = row_tree<WAVE, NVAL>(tm, a.TY, a.VC, red);
    gt = red + (a.TY + (a.TY + 7) / 8) * O;
  }
  // value i of the tile, of quantity q
  auto at = [&](int q, int i) { return col[(q * NJ + i % NJ) * a.VC + i / NJ]; };
  if (q1 <= 16) {
    for (int g = tm.t; g < GT * NQ; g += tm.T) {
      const int q = NQ == 2 && g >= GT, i0 = (g - q * GT) * q1;
      float s = 0.f;
      for (int i = 0; i < q1; i += 4) {
        float v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = at(q, i0 + min(i + u, q1 - 1));
#pragma unroll
        for (int u = 0; u < 4; ++u) s += i + u < q1 ? v[u] : 0.f;
      }
      gt[g] = s;
    }
  } else {
    for (int g = w; g < GT * NQ; g += nw) {
      const int q = NQ == 2 && g >= GT, i0 = (g - q * GT) * q1;
      float s[1] = {0.f};
      for (int i = lane; i < q1; i += 64) s[0] += at(q, i0 + i);
      add_from<1>(1, s);
      if (lane == 0) gt[g] = s[0];
    }
  }
  tm.sync();
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    const int grp = min(a.by_cg.of(tm.tx * V + j), GT - 1);  // an idle column's is nobody's
#pragma unroll
    for (int q = 0; q < NQ; ++q) val[q * NJ + j] = gt[q * GT + grp];
  }
}

// ------------------------------------------------------------ the elements --
// u = (x - mean) a + b, every operation rounded by itself (none fused into
// another, nor into the product that forms the mean): the same bits wherever it
// is formed, so that a re-run equals the first forward and a backward takes
// ReLU's decision as it did.
__device__ __forceinline__ float gn_affine(float x, float mean, float a, float b) {
#pragma clang fp contract(off)
  const float m = (x - mean) * a;
  return m + b;
}

// e^-u for fp32 activations, two steps off at most: 2^t with t the rounded product of -u
// and log2 e, times 1 + ln 2 (what the product's rounding and the constant's left).
// Past 200 either way it is 0 or infinite (there infinities would meet in that rest).
__device__ __forceinline__ float gn_exp_neg(float u) {
  const float v = __builtin_amdgcn_fmed3f(-u, -200.f, 200.f);
  const float t = v * 1.44269502f, rest = fmaf(v, 1.92596303e-8f, fmaf(v, 1.44269502f, -t));
  return __builtin_amdgcn_exp2f(t) * fmaf(rest, 0.693147181f, 1.f);
}

// FINE: fp32 activations.  bf16 ones take the exponential in two instructions: its
// relative error, 1.25 |u| half steps of fp32, is a thousandth of theirs and less for |u|
// up to 50.  (fp32 forward of 32 x 3136 pixels x 64 channels 19.8 us, 20.1 FINE; where
// code has yet to be fetched its 40 bytes an element count: 34 x 102 x 240 9.3 and 10.1.)
template <bool FINE>
__device__ __forceinline__ float gn_sigmoid(float u) {
  return __builtin_amdgcn_rcpf(1.f + (FINE ? gn_exp_neg(u) : __expf(-u)));
}

// v = act(u), not SiLU: ReLU (NaN passes through) or nothing by a uniform flag, which
// costs no jump
template <bool SILU, bool FINE>
__device__ __forceinline__ float gn_act(bool relu, float u) {
  if (SILU) return u * gn_sigmoid<FINE>(u);
  return relu && u < 0.f ? 0.f : u;
}

// dv act'(u)
template <bool SILU, bool FINE>
__device__ __forceinline__ float gn_act_bwd(bool relu, float u, float dv) {
  if (SILU) {
    const float q = gn_sigmoid<FINE>(u);
    return dv * (q * (1.f + u * (1.f - q)));
  }
  return u > 0.f || !relu ? dv : 0.f;
}

// f(SiLU or not, dropped out or not) with compile-time constants: the element code
// of a thread's vectors then runs straight through, where a choice per vector jumps
// to lines that the instruction cache has yet to fetch (0.15 us each).
template <class F>
__host__ __device__ __forceinline__ void gn_choose(const GnArgs &a, F &&f) {
  auto act = [&](auto drop) {
    if (a.act == GN_ACT_SILU)
      f(std::true_type(), drop);
    else
      f(std::false_type(), drop);
  };
  if (a.drop.rng)
    act(std::true_type());
  else
    act(std::false_type());
}

// the dropout of the V elements from channel c of pixel `pix` (of all n hw)
template <int V>
__device__ __forceinline__ void gn_drop(const GnArgs &a, const DropKey &key, uint64_t pix, int c, float v[V]) {
  const uint64_t e = pix * uint32_t(a.C) + c;
  if (V == 8)
    drop8(a.drop, key, uint32_t(e >> 3), v);
  else
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = drop1(a.drop, key, e + j, v[j]);
}

// groups (of the sample) of the vector at channel c, or of its channels (NJ = V)
template <int V, int NJ>
struct GnGroups {
  int k[NJ];
  __device__ __forceinline__ GnGroups(const GnArgs &a, int c) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) k[j] = a.by_cg.of(c + j);
  }
};

}  // namespace ckpt
