// Attention forward over packed sequences: o = softmax(scale q k^T) v and the logarithm of each
// row's sum, in one pass over the keys with the running maximum and sum of the softmax.
//
// The query rows that share a key head, (token, head of the group) in this order, are one
// matrix: a key tile is read once for all of them, and single tokens fill tiles as far as
// their heads go.  Each of a workgroup's wavefronts keeps 32 of these rows; the keys come by in
// tiles through LDS, the next one loading while one is worked on.
//   many rows (k_attn_fwd<D, 4>): four wavefronts with 32 rows each share tiles of 64 keys
//   few rows (k_attn_fwd<D, 1>): four wavefronts with the same 32 rows take a quarter each of tiles
//     of 128 keys and join their sums at the end
// Where there are too few workgroups for the chip, the keys are split over several, whose
// unfinished rows go to the workspace and are joined by k_attn_join.
#include "attn.h"
#include "common.h"

namespace ckpt {
namespace {

using namespace at;

template <int D, int WQ>
__global__ __launch_bounds__(256, 2) void k_attn_fwd(AttnArgs A, int tiles) {
  constexpr int WK = 4 / WQ, BM = 32 * WQ, BN = WQ == 4 ? 64 : 128, SUBS = BN / 32 / WK, T = D / 32, KK = D / 16;
  __shared__ __align__(16) unsigned char kt0[BN * D * 2], kt1[BN * D * 2], vt0[BN * D * 2], vt1[BN * D * 2];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wq = WQ == 4 ? wave : 0, wk = WQ == 4 ? 0 : wave;
  const int kvh = blockIdx.x % A.kv_heads, tile = tiles - 1 - int(blockIdx.x / A.kv_heads);
  Sequence sq;
  if (!find_tile(A, A.qoff, A.tq, A.rep, BM, tile, sq)) return;
  const int64_t rows = int64_t(sq.lq) * A.rep;

  // the lane's query
  const int64_t row = sq.first + wq * 32 + (lane & 31);
  const bool valid = row < rows;
  const int64_t r = valid ? row : rows - 1;
  const int token = int(r / A.rep), head = kvh * A.rep + int(r - int64_t(token) * A.rep);
  const int past = sq.lk - sq.lq;
  const int lim = A.causal ? min(sq.lk, max(0, token + past + 1)) : sq.lk;  // keys it sees
  const int lim_lo = __builtin_amdgcn_readfirstlane(lim), lim_hi = __builtin_amdgcn_readlane(lim, 31);  // the wavefront's least and most
  const int64_t last = min(sq.first + BM, rows) - 1;
  const int kend = A.causal ? min(sq.lk, max(0, int(last / A.rep) + past + 1)) : sq.lk;
  const int all = (kend + BN - 1) / BN;
  const int begin = int(int64_t(all) * blockIdx.y / gridDim.y), end = int(int64_t(all) * (blockIdx.y + 1) / gridDim.y);

  bf16x8 q[KK];
  {
    const __bf16 *p = A.q + (sq.q0 + token) * A.ldq + head * A.hsq;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) q[kk] = kept(p, kk, A.dim);
  }
  const Places<D> places;
  const __bf16 *const vp = A.v + sq.k0 * A.ldv + kvh * A.hsv;
  const Loader<D, BN, 256> kload(A.k + sq.k0 * A.ldk + kvh * A.hsk, A.ldk, A.dim), vload(vp, A.ldv, A.dim);

  f32x16 o[T];
  clear(o);
  float m = -INFINITY, l = 0.f;
  const float sc = A.scale * LOG2E;
  unsigned bad = 0;

  auto work = [&](int it, const unsigned char *kt, const unsigned char *vt, auto masked) __attribute__((always_inline)) {
    constexpr bool MASKED = decltype(masked)::value;
    const Places<D> at = places.here();
    // keys the lane's query sees from its half's first on
    const int left = lim - (it * BN + wk * SUBS * 32) - 4 * (lane >> 5);
    f32x16 s[SUBS];
    clear(s);
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
#pragma unroll
      for (int u = 0; u < SUBS; ++u) s[u] = mfma(at.rows(kt, (wk * SUBS + u) * 32, kk), q[kk], s[u]);
    float top = -INFINITY;
#pragma unroll
    for (int u = 0; u < SUBS; ++u)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        if (MASKED && u * 32 + 8 * (i / 4) + i % 4 >= left) s[u][i] = -INFINITY;
        top = fmaxf(top, s[u][i]);
      }
    top = halves_max(top);
    // The maximum is moved when it would let an exponential exceed 2^8: o and l stay far
    // inside fp32, and most tiles leave them as they are.
    if (__any((top - m) * sc > 8.f)) {
      top = fmaxf(m, top);
      const float f = exp2_fast((m - (top == -INFINITY ? 0.f : top)) * sc);
      m = top;
      l *= f;
#pragma unroll
      for (int t = 0; t < T; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] *= f;
    }
    const float base = (m == -INFINITY ? 0.f : m) * sc;
#pragma unroll
    for (int u = 0; u < SUBS; ++u)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[u][i] = exp2_fast(fmaf(s[u][i], sc, -base));
        l += s[u][i];
      }
#pragma unroll
    for (int u = 0; u < SUBS; ++u)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int first = (wk * SUBS + u) * 32 + c * 16;
        if constexpr (MASKED) add_rows_finite<D>(o, at, vt, first, operand(s[u], c), bad);
        else add_rows<D>(o, at, vt, first, operand(s[u], c));
      }
  };
  const int n = end - begin;
  // tiles whose keys every row of the wavefront sees
  const int whole = lim_lo - (wk + 1) * SUBS * 32 + BN;
  const int full = max(0, min(n, (whole > 0 ? whole / BN : 0) - begin));
  auto load = [&](int it, unsigned char *kt, unsigned char *vt) __attribute__((always_inline)) {
    kload.load(kt, int64_t(it) * BN, sq.lk - it * BN);
    vload.load(vt, int64_t(it) * BN, sq.lk - it * BN);
  };
  if (n > 0) load(begin, kt0, vt0);
  two_kinds(n, full, [&](int i, auto place, auto masked) __attribute__((always_inline)) {
    tile_barrier();
    if (i + 1 < n) load(begin + i + 1, place ? kt0 : kt1, place ? vt0 : vt1);
    work(begin + i, place ? kt1 : kt0, place ? vt1 : vt0, masked);
  });
  if (__any(bad != 0))
    for (int it = begin; it < end; ++it) {
      const int j0 = it * BN + wk * SUBS * 32;
      if (j0 + SUBS * 32 > lim_lo && j0 < lim_hi)
        add_special<D>(o, vp, A.ldv, A.dim, j0, min(j0 + SUBS * 32, sq.lk), false, [&](int j) { return j < lim; });
    }
  l = halves_add(l);

  if constexpr (WK > 1) {
    // the wavefronts' sums by their common maximum, one wavefront's o (fp32, [D][32]) in each
    // half of two of the tiles
    __shared__ float ms[WK][32], ls[WK][32];
    tile_barrier();
    float *const mine = reinterpret_cast<float *>(wave < 2 ? kt0 : vt0) + (wave & 1) * D * 32;
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) mine[(32 * t + d_row(i)) * 32 + (lane & 31)] = o[t][i];
    if (lane < 32) {
      ms[wave][lane] = m;
      ls[wave][lane] = l;
    }
    __syncthreads();
    const float m0 = fmaxf(fmaxf(ms[0][lane & 31], ms[1][lane & 31]), fmaxf(ms[2][lane & 31], ms[3][lane & 31]));
    float f[WK];
    l = 0.f;
#pragma unroll
    for (int w = 0; w < WK; ++w) {
      f[w] = exp2_fast((ms[w][lane & 31] - (m0 == -INFINITY ? 0.f : m0)) * sc);
      l += ls[w][lane & 31] * f[w];
    }
    m = m0;
    if (wave) return;
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int e = (32 * t + d_row(i)) * 32 + (lane & 31);
        const float *const a = reinterpret_cast<const float *>(kt0) + e, *const b = reinterpret_cast<const float *>(vt0) + e;
        // a wavefront without keys has a factor of 0 and nothing but zeros
        o[t][i] = a[0] * f[0] + a[D * 32] * f[1] + b[0] * f[2] + b[D * 32] * f[3];
      }
  }
  if (!valid) return;
  const int64_t at_row = head * A.tq + sq.q0 + token;
  if (gridDim.y > 1) {
    const int64_t p = int64_t(blockIdx.y) * A.heads * A.tq + at_row;
    if (lane < 32) {
      A.pml[2 * p] = m;
      A.pml[2 * p + 1] = l;
    }
    store_part<D>(A.po + p * A.dim, o, 1.f, A.dim);
    return;
  }
  if (lane < 32) A.lse[at_row] = l == 0.f ? -INFINITY : fmaf(m, A.scale, logf(l));
  store_row<D>(A.o + (sq.q0 + token) * A.ldo + head * A.hso, o, l == 0.f ? 0.f : 1.f / l, A.dim);
}

// a row's splits joined: sixteen lanes a row, eight columns each
__global__ __launch_bounds__(256) void k_attn_join(AttnArgs A) {
  const int64_t at = blockIdx.x * int64_t(16) + threadIdx.x / 16, n = A.heads * A.tq;
  if (at >= n) return;
  const int64_t token = at % A.tq;
  const int head = int(at / A.tq), col = (threadIdx.x & 15) * 8;
  // rows of no sequence have no splits either
  if (token < A.qoff[0] || token >= A.qoff[A.seqs]) return;
  const float sc = A.scale * LOG2E;
  float m = -INFINITY;
  for (int z = 0; z < A.splits; ++z) m = fmaxf(m, A.pml[2 * (z * n + at)]);
  const float base = m == -INFINITY ? 0.f : m;
  float l = 0.f, o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 2
  for (int z = 0; z < A.splits; ++z) {
    const float lz = A.pml[2 * (z * n + at) + 1];
    const float f = exp2_fast((A.pml[2 * (z * n + at)] - base) * sc);
    if (lz == 0.f) continue;
    l += lz * f;
    if (col < A.dim) {
      const float4 *const p = reinterpret_cast<const float4 *>(A.po + (z * n + at) * A.dim + col);
      const float4 a = p[0], b = p[1];
      o[0] += a.x * f, o[1] += a.y * f, o[2] += a.z * f, o[3] += a.w * f;
      o[4] += b.x * f, o[5] += b.y * f, o[6] += b.z * f, o[7] += b.w * f;
    }
  }
  if (col == 0) A.lse[at] = l == 0.f ? -INFINITY : fmaf(m, A.scale, logf(l));
  if (col < A.dim) {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    bf16x8 r;
#pragma unroll
    for (int k = 0; k < 8; ++k) r[k] = (__bf16)(o[k] * inv);
    *reinterpret_cast<bf16x8 *>(A.o + token * A.ldo + head * A.hso + col) = r;
  }
}

bool few_rows(const AttnArgs &a) { return a.tq * a.rep <= int64_t(32) * a.seqs; }

template <int D>
void forward(hipStream_t s, const AttnArgs &a) {
  const int bm = few_rows(a) ? 32 : 128;
  const int tiles = int(a.tq * a.rep / bm) + a.seqs;
  const dim3 grid(uint32_t(tiles) * a.kv_heads, a.splits);
  if (bm == 32)
    hipLaunchKernelGGL((k_attn_fwd<D, 1>), grid, dim3(256), 0, s, a, tiles);
  else
    hipLaunchKernelGGL((k_attn_fwd<D, 4>), grid, dim3(256), 0, s, a, tiles);
  if (a.splits > 1)
    hipLaunchKernelGGL(k_attn_join, dim3(uint32_t((a.heads * a.tq + 15) / 16)), dim3(256), 0, s, a);
}

}  // namespace

// Workgroups for one another's keys where the rows alone fill less than two for each compute
// unit; a split is 256 keys at least of a sequence of the average length.
int attn_splits(const AttnArgs &a) {
  const int bm = few_rows(a) ? 32 : 128;
  const int64_t work = (a.tq * a.rep / bm > a.seqs ? a.tq * a.rep / bm : a.seqs) * a.kv_heads;
  const int64_t keys = a.tk / a.seqs / 256;
  int64_t n = 512 / (work > 0 ? work : 1);
  n = n < keys ? n : keys;
  return int(n < 1 ? 1 : n > 64 ? 64 : n);
}

void attn_forward(hipStream_t s, const AttnArgs &a) {
  if (a.tq == 0) return;
  a.dim <= 64 ? forward<64>(s, a) : forward<128>(s, a);
}

}  // namespace ckpt
