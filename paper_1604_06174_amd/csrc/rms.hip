// RMS norm with the residual's addition: h = x + res (rounded to the stream's type),
// st = 1 / sqrt(mean h^2 + eps), y = h st w in 32, 16 or 8 bits; the re-run from kept h
// and st; the backward d = gh + st (g w - xhat mean(g w xhat)), dw = sum g xhat.
//
// One pass: a team (a wavefront for rows of up to 1024 columns, else a workgroup)
// holds a whole row in registers, so every tensor is read or written once.  Teams loop
// over rows with the weight kept in registers.  A thread's vectors are eight columns
// each, `TEAM` vectors apart, so a wavefront's accesses are contiguous.  The last vector
// of a row whose width 8 does not divide is loaded whole, into the next row, where there
// is one, and stored element by element.
//
// Bound by HBM (a copy of 256 MiB reaches 5.5 TB/s): 16384 x 4096 with a residual and an 8-bit output
// 91 us (5.2 TB/s), 16384 x 2048 backward 58 us (4.7 TB/s; its records of sums are 5% more, and their launch 5 us).
#include "common.h"
#include "lanes.h"
#include "seq.h"
#include "vec.h"

namespace ckpt {
namespace {

struct E4m3 {
  uint8_t bits;
};

// eight elements from p, or the first cnt of them (the others 0); over: all eight can be read
template <typename T>
__device__ __forceinline__ void load8(const T *p, int cnt, float v[8], bool over = false) {
  if (cnt >= 8 || over) {
    const Vec<T, 8> r = load_vec<T, 8>(p);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = k < cnt ? float(r.v[k]) : 0.f;
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = k < cnt ? float(p[k]) : 0.f;
  }
}

template <typename T>
__device__ __forceinline__ void store8(T *p, int cnt, const float v[8]) {
  if (cnt >= 8) {
    store_vec<T, 8>(p, v);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < cnt) p[k] = (T)v[k];
  }
}

// rounded to e4m3, to nearest even; |v| is at most 448 here, but for the last bit of a
// float, which rounds to 448
__device__ __forceinline__ void store8(E4m3 *p, int cnt, const float v[8]) {
  uint32_t w[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    int t = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * k], v[4 * k + 1], 0, false);
    w[k] = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * k + 2], v[4 * k + 3], t, true);
  }
  if (cnt >= 8) {
    typedef uint32_t pair __attribute__((ext_vector_type(2), aligned(1)));
    *reinterpret_cast<pair *>(p) = pair{w[0], w[1]};
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < cnt) p[k].bits = uint8_t(w[k / 4] >> (8 * (k % 4)));
  }
}

__device__ __forceinline__ float wave_sum(float v) {
  v = xor_add<1>(v);
  v = xor_add<2>(v);
  v = xor_add<4>(v);
  v = xor_add<8>(v);
  v = xor_add<16>(v);
  return xor_add<32>(v);
}

// The largest of magnitudes as their bits: a NaN's are above all others', so it stays.
template <int OFF>
__device__ __forceinline__ uint32_t xor_max(uint32_t v) {
  float o = __uint_as_float(v);
  if constexpr (OFF >= 16) {
    float w = o;
    swap_rows<OFF>(o, w);
    const uint32_t a = __float_as_uint(o), b = __float_as_uint(w);
    return a > b ? a : b;
  } else {
    const uint32_t b = __float_as_uint(lane_xor<OFF>(o));
    return v > b ? v : b;
  }
}

// over aligned runs of `lanes` lanes (a power of two)
__device__ __forceinline__ uint32_t run_max(uint32_t v, int lanes) {
  if (lanes > 1) v = xor_max<1>(v);
  if (lanes > 2) v = xor_max<2>(v);
  if (lanes > 4) v = xor_max<4>(v);
  if (lanes > 8) v = xor_max<8>(v);
  if (lanes > 16) v = xor_max<16>(v);
  if (lanes > 32) v = xor_max<32>(v);
  return v;
}

// A team's sum of one value a thread, the same bits in all of them.  `slot` alternates
// between calls, so one barrier a call is enough.
template <int TEAM>
__device__ __forceinline__ float team_sum(float v, float *red, int slot) {
  v = wave_sum(v);
  if constexpr (TEAM > 64) {
    constexpr int W = TEAM / 64;
    if ((threadIdx.x & 63) == 0) red[slot * W + threadIdx.x / 64] = v;
    __syncthreads();
    v = red[slot * W];
#pragma unroll
    for (int k = 1; k < W; ++k) v += red[slot * W + k];
  }
  return v;
}

template <int TEAM>
__device__ __forceinline__ uint32_t team_max(uint32_t v, uint32_t *red, int slot) {
  v = run_max(v, 64);
  if constexpr (TEAM > 64) {
    constexpr int W = TEAM / 64;
    if ((threadIdx.x & 63) == 0) red[slot * W + threadIdx.x / 64] = v;
    __syncthreads();
    v = red[slot * W];
#pragma unroll
    for (int k = 1; k < W; ++k) v = v > red[slot * W + k] ? v : red[slot * W + k];
  }
  return v;
}

constexpr int block_of(int team) { return team < 256 ? 256 : team; }

template <typename XT, typename HT, typename YT, bool RES, bool APPLY, int TEAM, int NV>
__global__ __launch_bounds__(block_of(TEAM)) void k_rms_fwd(RmsArgs A) {
  constexpr int TEAMS = block_of(TEAM) / TEAM;
  constexpr bool F8 = std::is_same<YT, E4m3>::value;
  __shared__ float red[TEAM > 64 ? 2 * TEAM / 64 : 1];
  __shared__ uint32_t redm[TEAM > 64 ? 2 * TEAM / 64 : 1];
  const int t = threadIdx.x % TEAM;
  float w[NV][8];
  int cnt[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    cnt[j] = min(8, A.c - (j * TEAM + t) * 8);
    if (cnt[j] > 0) load8(A.w + (j * TEAM + t) * 8, cnt[j], w[j]);
  }
  int slot = 0;
  for (int64_t row = blockIdx.x * int64_t(TEAMS) + threadIdx.x / TEAM; row < A.rows;
       row += int64_t(gridDim.x) * TEAMS, slot ^= 1) {
    const bool more = row + 1 < A.rows && A.c >= 8;
    float v[NV][8];
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[j][k] = 0.f;
      if (cnt[j] > 0)
        load8(static_cast<const XT *>(A.x) + row * (APPLY ? A.ldh : A.ldx) + (j * TEAM + t) * 8, cnt[j], v[j], more);
    }
    if constexpr (RES) {
#pragma unroll
      for (int j = 0; j < NV; ++j)
        if (cnt[j] > 0) {
          float r[8];
          load8(static_cast<const HT *>(A.res) + row * A.ldh + (j * TEAM + t) * 8, cnt[j], r, more);
          // the norm is of the sum as the stream keeps it
#pragma unroll
          for (int k = 0; k < 8; ++k) v[j][k] = float((HT)(v[j][k] + r[k]));
        }
#pragma unroll
      for (int j = 0; j < NV; ++j)
        if (cnt[j] > 0) store8(static_cast<HT *>(A.h) + row * A.ldh + (j * TEAM + t) * 8, cnt[j], v[j]);
    }
    float st;
    if constexpr (APPLY) {
      st = A.st[row];
    } else {
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int k = 0; k < 8; ++k) sum = fmaf(v[j][k], v[j][k], sum);
      sum = team_sum<TEAM>(sum, red, slot);
      st = 1.f / sqrtf(fmaf(sum, A.inv_c, A.eps));
      if (t == 0) A.st[row] = st;
    }
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < 8; ++k) v[j][k] = v[j][k] * st * w[j][k];
    if constexpr (F8) {
      uint32_t top[NV];
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        top[j] = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const uint32_t b = k < cnt[j] ? __float_as_uint(v[j][k]) & 0x7fffffffu : 0u;
          top[j] = top[j] > b ? top[j] : b;
        }
      }
      if (A.qgroup) {
#pragma unroll
        for (int j = 0; j < NV; ++j) top[j] = run_max(top[j], A.qgroup / 8);
      } else {
        uint32_t m = top[0];
#pragma unroll
        for (int j = 1; j < NV; ++j) m = m > top[j] ? m : top[j];
        m = team_max<TEAM>(m, redm, slot);
#pragma unroll
        for (int j = 0; j < NV; ++j) top[j] = m;
      }
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const uint32_t least = __float_as_uint(1e-30f);
        const float m = __uint_as_float(top[j] > least ? top[j] : least);
        const float inv = 448.f / m;
#pragma unroll
        for (int k = 0; k < 8; ++k) v[j][k] *= inv;
        if (cnt[j] > 0) {
          const int vec = j * TEAM + t;
          if (A.qgroup ? vec % (A.qgroup / 8) == 0 : vec == 0)
            A.ys[row * A.groups + (A.qgroup ? vec / (A.qgroup / 8) : 0)] = m / 448.f;
        }
      }
    }
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (cnt[j] > 0) store8(static_cast<YT *>(A.y) + row * A.ldy + (j * TEAM + t) * 8, cnt[j], v[j]);
  }
}

template <typename GT, typename HT, typename DT, int TEAM, int NV>
__global__ __launch_bounds__(block_of(TEAM)) void k_rms_bwd(RmsBwdArgs A) {
  constexpr int TEAMS = block_of(TEAM) / TEAM;
  __shared__ float red[TEAM > 64 ? 2 * TEAM / 64 : 1];
  __shared__ float dws[TEAMS > 1 ? (TEAMS - 1) * TEAM * NV * 8 : 1];
  const int t = threadIdx.x % TEAM;
  float w[NV][8], dw[NV][8];
  int cnt[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    cnt[j] = min(8, A.c - (j * TEAM + t) * 8);
#pragma unroll
    for (int k = 0; k < 8; ++k) w[j][k] = dw[j][k] = 0.f;
    if (cnt[j] > 0) load8(A.w + (j * TEAM + t) * 8, cnt[j], w[j]);
  }
  int slot = 0;
  for (int64_t row = blockIdx.x * int64_t(TEAMS) + threadIdx.x / TEAM; row < A.rows;
       row += int64_t(gridDim.x) * TEAMS, slot ^= 1) {
    const bool more = row + 1 < A.rows && A.c >= 8;
    float x[NV][8], g[NV][8], e[NV][8];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
#pragma unroll
      for (int k = 0; k < 8; ++k) x[j][k] = g[j][k] = e[j][k] = 0.f;
      const int64_t col = (j * TEAM + t) * 8;
      if (cnt[j] > 0) {
        load8(static_cast<const HT *>(A.h) + row * A.ldh + col, cnt[j], x[j], more);
        load8(static_cast<const GT *>(A.g) + row * A.ldg + col, cnt[j], g[j], more);
        if (A.gh) load8(static_cast<const DT *>(A.gh) + row * A.ldd + col, cnt[j], e[j], more);
      }
    }
    const float st = A.st[row];
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        x[j][k] *= st;
        dw[j][k] = fmaf(g[j][k], x[j][k], dw[j][k]);
        g[j][k] *= w[j][k];
        sum = fmaf(g[j][k], x[j][k], sum);
      }
    const float mean = team_sum<TEAM>(sum, red, slot) * A.inv_c;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
#pragma unroll
      for (int k = 0; k < 8; ++k) g[j][k] = fmaf(st, fmaf(-x[j][k], mean, g[j][k]), e[j][k]);
      if (cnt[j] > 0) store8(static_cast<DT *>(A.d) + row * A.ldd + (j * TEAM + t) * 8, cnt[j], g[j]);
    }
  }
  // the workgroup's teams in order, then one record of the workgroup
  if constexpr (TEAMS > 1) {
    const int team = threadIdx.x / TEAM;
    if (team > 0) {
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int k = 0; k < 8; ++k) dws[((team - 1) * NV * 8 + j * 8 + k) * TEAM + t] = dw[j][k];
    }
    __syncthreads();
    if (team > 0) return;
#pragma unroll
    for (int q = 0; q < TEAMS - 1; ++q)
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int k = 0; k < 8; ++k) dw[j][k] += dws[(q * NV * 8 + j * 8 + k) * TEAM + t];
  }
#pragma unroll
  for (int j = 0; j < NV; ++j)
    if (cnt[j] > 0) store8(A.part + int64_t(blockIdx.x) * A.cpad + (j * TEAM + t) * 8, cnt[j], dw[j]);
}

// dw = the workgroups' records added up: 32 columns a workgroup, each of 32 half wavefronts every 32nd
// record, sixteen in flight, then the 32 sums in order: a chain of at most rows / teams in a team, its workgroup's
// four teams, 48 records and 32 sums
__global__ __launch_bounds__(1024) void k_rms_dw(const float *part, int groups, int c, int cpad, float *dw) {
  constexpr int AHEAD = 16;
  __shared__ float red[32][32];
  const int lane = threadIdx.x & 31, half = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
  float s = 0.f;
  if (col < c) {
    for (int b = half; b < groups; b += 32 * AHEAD) {
      float v[AHEAD];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) v[u] = part[int64_t(min(b + 32 * u, groups - 1)) * cpad + col];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) s += b + 32 * u < groups ? v[u] : 0.f;
    }
  }
  red[half][lane] = s;
  __syncthreads();
  if (half == 0 && col < c) {
    float v = red[0][lane];
#pragma unroll
    for (int k = 1; k < 32; ++k) v += red[k][lane];
    dw[col] = v;
  }
}

// A row's team and vectors a thread.  At 134 MB a tensor of 16 bits: rows of 2048 by a wavefront with
// four vectors a thread 55 us forward and 79 backward, by a workgroup with one 51 and 58; rows of
// 8192 by 256 threads with four 54 and 84, by 1024 with one 49 and 61.  Rows above 8192 columns leave the backward
// 128 registers a thread, and with mixed types 2 to 38 more go to memory: 2048 x 16384, g fp32, h and d bf16 82 us
// (4.1 TB/s), g and h bf16, d fp32 94 (4.3); all of them bf16, with none, 58 (4.7).
template <typename F>
void with_team(int c, F &&f) {
  using std::integral_constant;
  const int vecs = (c + 7) / 8;
#define CKPT_TEAM(team, nv) f(integral_constant<int, team>(), integral_constant<int, nv>())
  if (vecs <= 64) CKPT_TEAM(64, 1);
  else if (vecs <= 128) CKPT_TEAM(64, 2);
  else if (vecs <= 256) CKPT_TEAM(256, 1);
  else if (vecs <= 512) CKPT_TEAM(256, 2);
  else if (vecs <= 1024) CKPT_TEAM(1024, 1);
  else CKPT_TEAM(1024, 2);
#undef CKPT_TEAM
}

template <typename XT, typename HT, typename YT, bool RES, bool APPLY>
void launch_fwd(hipStream_t s, const RmsArgs &a) {
  with_team(a.c, [&](auto team, auto nv) {
    constexpr int TEAM = team, NV = nv, TEAMS = block_of(TEAM) / TEAM;
    const int64_t need = (int64_t(a.rows) + TEAMS - 1) / TEAMS;
    // a few rows each: 16384 x 4096 with an 8-bit output 92 us, with four times as many each 102
    const int64_t fill = 1024 * 2048 / block_of(TEAM);
    hipLaunchKernelGGL((k_rms_fwd<XT, HT, YT, RES, APPLY, TEAM, NV>), dim3(uint32_t(need < fill ? need : fill)),
                       dim3(block_of(TEAM)), 0, s, a);
  });
}

template <typename XT, typename HT, bool RES, bool APPLY>
void forward_y(hipStream_t s, const RmsArgs &a, int ytype) {
  if (ytype == SEQ_F32) launch_fwd<XT, HT, float, RES, APPLY>(s, a);
  else if (ytype == SEQ_BF16) launch_fwd<XT, HT, __bf16, RES, APPLY>(s, a);
  else launch_fwd<XT, HT, E4m3, RES, APPLY>(s, a);
}

template <typename GT, typename HT, typename DT>
void launch_bwd(hipStream_t s, const RmsBwdArgs &a, int groups) {
  with_team(a.c, [&](auto team, auto nv) {
    constexpr int TEAM = team, NV = nv;
    hipLaunchKernelGGL((k_rms_bwd<GT, HT, DT, TEAM, NV>), dim3(groups), dim3(block_of(TEAM)), 0, s, a);
  });
  hipLaunchKernelGGL(k_rms_dw, dim3((a.c + 31) / 32), dim3(1024), 0, s, a.part, groups, a.c, a.cpad, a.dw);
}

template <typename GT, typename HT>
void backward_d(hipStream_t s, const RmsBwdArgs &a, int groups, int dtype) {
  dtype == SEQ_F32 ? launch_bwd<GT, HT, float>(s, a, groups) : launch_bwd<GT, HT, __bf16>(s, a, groups);
}

}  // namespace

void rms_forward(hipStream_t s, const RmsArgs &a, int xtype, int htype, int ytype, bool apply) {
  const bool xf = xtype == SEQ_F32, hf = htype == SEQ_F32;
  if (apply)
    hf ? forward_y<float, float, false, true>(s, a, ytype) : forward_y<__bf16, __bf16, false, true>(s, a, ytype);
  else if (!a.res)
    hf ? forward_y<float, float, false, false>(s, a, ytype) : forward_y<__bf16, __bf16, false, false>(s, a, ytype);
  else if (xf)
    hf ? forward_y<float, float, true, false>(s, a, ytype) : forward_y<float, __bf16, true, false>(s, a, ytype);
  else
    hf ? forward_y<__bf16, float, true, false>(s, a, ytype) : forward_y<__bf16, __bf16, true, false>(s, a, ytype);
}

// Workgroups of a backward, each with a record of c sums: as many as are resident together, for with
// fewer the loads in flight do not cover the memory's latency, and a second round of workgroups finds
// them all at the same place again (16384 x 2048: 512 take 79 us, 1024 64, 1536 60, 2048 73).
int rms_backward_groups(int64_t rows, int c) {
  int most = 0, teams = 0;
  with_team(c, [&](auto team, auto nv) {
    constexpr int TEAM = team, NV = nv;
    teams = block_of(TEAM) / TEAM;
    most = TEAM == 1024 ? (NV == 1 ? 512 : 256) : NV == 1 ? 1536 : 1024;
  });
  const int64_t need = (rows + teams - 1) / teams;
  return int(need < most ? need : most);
}

void rms_backward(hipStream_t s, const RmsBwdArgs &a, int groups, int gtype, int htype, int dtype) {
  const bool gf = gtype == SEQ_F32, hf = htype == SEQ_F32;
  if (gf)
    hf ? backward_d<float, float>(s, a, groups, dtype) : backward_d<float, __bf16>(s, a, groups, dtype);
  else
    hf ? backward_d<__bf16, float>(s, a, groups, dtype) : backward_d<__bf16, __bf16>(s, a, groups, dtype);
}

}  // namespace ckpt
