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

// How a pass covers it.  A tile is W consecutive channels (whole groups, whole
// vectors of V) of one sample, or of one chunk of its pixels; VC = W / V threads
// cover a pixel, TY pixels are covered at once, NV times in turn.
struct GnPlan {
  bool split;   // a sample's tile does not stay in one team's registers
  bool wave;    // teams of one wavefront each (else the workgroup)
  bool fold;    // a vector lies within one group
  bool pow2;    // VC is a power of two, at most 64: wavefronts reduce in registers
  int V, W, tiles, VC, TY, NV;
  int threads, teams;
  int rows;       // resident backward: records of channel sums (samples taken at a time)
  int64_t chunks; // split: chunks of TY NV pixels per sample
  int64_t blocks;
  int redbuf;  // floats of LDS of one reduction
  size_t lds;
};

// Throws CKPT_E_UNSUPPORTED for problems outside the kernels' range.
GnPlan gn_plan(const GnProblem &p, bool backward);
// The element passes' cover (known statistics or sums): tiles of vector columns,
// chunks of TY GN_EW_NV pixels.
constexpr int GN_EW_NV = 4;
GnPlan gn_plan_elements(const GnProblem &p);
// the device memory a forward or backward needs besides its tensors
uint64_t gn_workspace_bytes(const GnProblem &p, bool backward);
void gn_forward(hipStream_t s, const GnProblem &p, const void *x, const float *gamma, const float *beta,
                const DropArgs &drop, void *y, float *st, void *ws);
void gn_apply(hipStream_t s, const GnProblem &p, const void *x, const float *st, const float *gamma,
              const float *beta, const DropArgs &drop, void *y);
void gn_backward(hipStream_t s, const GnProblem &p, const void *g, const void *x, const float *st,
                 const float *gamma, const float *beta, const DropArgs &drop, void *d, float *dgamma,
                 float *dbeta, void *ws);

// what the kernels take
struct GnArgs {
  const void *x, *g;
  void *out;  // y or d
  const float *gamma, *beta;
  float *st;         // mean [n G] | rstd [n G]
  float *gpart;      // split: [n][chunks][G][2] of the groups
  float *cpart;      // backward: [rows][2][C] of the channels (sum du xhat | sum du)
  const float *gsum; // backward, split: [n][G][2] of whole groups
  float *dgamma, *dbeta;
  int64_t n, hw, chunks;
  int C, G, cg, act;
  int64_t ldx, ldg, ldo;
  float eps, inv_m;
  int W, tiles, VC, TY, rows;
  int redbuf;  // floats of LDS of one reduction (group_sums)
  bool pow2;
  DropArgs drop;
};

// the arguments a plan and problem fix
inline GnArgs gn_args(const GnProblem &p, const GnPlan &g, const DropArgs &drop) {
  GnArgs a{};
  a.n = p.n;
  a.hw = p.hw;
  a.chunks = g.chunks;
  a.C = p.C;
  a.G = p.G;
  a.cg = p.cg;
  a.act = p.act;
  a.ldx = p.ldx;
  a.ldg = p.ldg;
  a.eps = p.eps;
  a.inv_m = float(1.0 / (double(p.hw) * p.cg));
  a.W = g.W;
  a.tiles = g.tiles;
  a.VC = g.VC;
  a.TY = g.TY;
  a.rows = g.rows;
  a.redbuf = g.redbuf;
  a.pow2 = g.pow2;
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
    tx = t % a.VC;
    ty = t / a.VC;
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
inline size_t gn_reduce_floats(const GnPlan &p, int T, int NQ, int NJ, int cg) {
  const size_t gt = size_t(NQ) * (p.W / cg);
  if (p.pow2) return size_t(T / 64) * NQ * (p.fold ? p.W / cg : p.W) + gt;
  return (size_t(p.TY) + (p.TY + 7) / 8) * p.VC * NQ * NJ + gt;
}

// Sums of the rows of red[TY][O], eight at a time (a fixed tree); returns where
// the O sums lie.  Every thread of the team calls it after its writes.
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
        float s = 0.f;
        for (int k = 8 * r; k < min(8 * r + 8, rows); ++k) s += src[k * O + o];
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

// val[q NJ + j], q < NQ: quantity q of the thread's pixels, of its vector (NJ = 1,
// a vector within one group) or of its channel j.  Replaced by the sum over the
// whole group that the vector (channel j) belongs to.  red: gn_reduce_floats of
// LDS, where pow2 another one than the call before's.
template <int NQ, int NJ, bool WAVE>
__device__ __forceinline__ void group_sums(const GnArgs &a, const Team<WAVE> &tm, float (&val)[NQ * NJ],
                                           float *red) {
  constexpr int NVAL = NQ * NJ;
  constexpr bool FOLD = NJ == 1;
  const int GT = a.W / a.cg;            // groups of the tile
  const int V = a.W / a.VC;
  const int q1 = FOLD ? a.cg / V : a.cg;  // values a group consists of per row
  const int lane = tm.t & 63, w = tm.t >> 6, nw = tm.T / 64;
  if (a.pow2) {
    for (int off = a.VC; off < 64; off <<= 1)
#pragma unroll
      for (int k = 0; k < NVAL; ++k) val[k] += __shfl_xor(val[k], off);
    if (FOLD) {
      // VC = GT q1 is a power of two, so q1 is one
      for (int off = 1; off < q1; off <<= 1)
#pragma unroll
        for (int k = 0; k < NVAL; ++k) val[k] += __shfl_xor(val[k], off);
      if (nw == 1) return;
      const int grp = tm.tx / q1;
      if (lane < a.VC && tm.tx % q1 == 0)
#pragma unroll
        for (int k = 0; k < NVAL; ++k) red[(w * NQ + k) * GT + grp] = val[k];
      tm.sync();
#pragma unroll
      for (int k = 0; k < NVAL; ++k) {
        float s = 0.f;
        for (int i = 0; i < nw; ++i) s += red[(i * NQ + k) * GT + grp];
        val[k] = s;
      }
      return;
    }
    if (lane < a.VC)
#pragma unroll
      for (int q = 0; q < NQ; ++q)
#pragma unroll
        for (int j = 0; j < NJ; ++j) red[(w * NQ + q) * a.W + tm.tx * NJ + j] = val[q * NJ + j];
    float *const gt = red + nw * NQ * a.W;
    tm.sync();
    for (int g = tm.t; g < GT * NQ; g += tm.T) {
      const int q = g / GT, ch = (g - q * GT) * a.cg;
      float s = 0.f;
      for (int i = 0; i < nw; ++i)
        for (int c = 0; c < a.cg; ++c) s += red[(i * NQ + q) * a.W + ch + c];
      gt[g] = s;
    }
    tm.sync();
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int grp = (tm.tx * NJ + j) / a.cg;
#pragma unroll
      for (int q = 0; q < NQ; ++q) val[q * NJ + j] = gt[q * GT + grp];
    }
    return;
  }
  const int O = a.VC * NVAL;
  tm.sync();
  if (tm.ty < a.TY)
#pragma unroll
    for (int k = 0; k < NVAL; ++k) red[tm.ty * O + k * a.VC + tm.tx] = val[k];
  const float *const col = row_tree<WAVE, NVAL>(tm, a.TY, a.VC, red);
  float *const gt = red + (a.TY + (a.TY + 7) / 8) * O;
  // value i of group g of quantity q: column g q1 + i (FOLD), else channel g q1 + i
  auto at = [&](int q, int i) {
    return FOLD ? col[q * a.VC + i] : col[(q * NJ + i % NJ) * a.VC + i / NJ];
  };
  if (q1 <= 16) {
    for (int g = tm.t; g < GT * NQ; g += tm.T) {
      const int q = g / GT, i0 = (g - q * GT) * q1;
      float s = 0.f;
      for (int i = 0; i < q1; ++i) s += at(q, i0 + i);
      gt[g] = s;
    }
  } else {
    for (int g = w; g < GT * NQ; g += nw) {
      const int q = g / GT, i0 = (g - q * GT) * q1;
      float s = 0.f;
      for (int i = lane; i < q1; i += 64) s += at(q, i0 + i);
      for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off);
      if (lane == 0) gt[g] = s;
    }
  }
  tm.sync();
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    const int grp = (tm.tx * V + j) / a.cg;
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

__device__ __forceinline__ float gn_sigmoid(float u) { return __builtin_amdgcn_rcpf(1.f + __expf(-u)); }

// v = act(u); NaN passes through ReLU
__device__ __forceinline__ float gn_act(int act, float u) {
  if (act == GN_ACT_RELU) return u < 0.f ? 0.f : u;
  if (act == GN_ACT_SILU) return u * gn_sigmoid(u);
  return u;
}

// dv act'(u)
__device__ __forceinline__ float gn_act_bwd(int act, float u, float dv) {
  if (act == GN_ACT_RELU) return u > 0.f ? dv : 0.f;
  if (act == GN_ACT_SILU) {
    const float q = gn_sigmoid(u);
    return dv * (q * (1.f + u * (1.f - q)));
  }
  return dv;
}

// the dropout of the V elements from channel c of pixel `pix` (of all n hw)
template <int V>
__device__ __forceinline__ void gn_drop(const GnArgs &a, const DropKey &key, uint64_t pix, int c, float v[V]) {
  const uint64_t e = pix * uint64_t(a.C) + c;
  if (V == 8)
    drop8(a.drop, key, uint32_t(e >> 3), v);
  else
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = drop1(a.drop, key, e + j, v[j]);
}

// group (of the sample) of channel j of the vector at channel c
template <int V, bool FOLD>
struct GnGroups {
  int k[FOLD ? 1 : V];
  __device__ __forceinline__ GnGroups(const GnArgs &a, int c) {
#pragma unroll
    for (int j = 0; j < (FOLD ? 1 : V); ++j) k[j] = (c + j) / a.cg;
  }
};

}  // namespace ckpt
