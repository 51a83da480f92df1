// Attention backward over packed sequences, from the forward's o and lse:
//   p = exp(scale q k^T - lse), ds = p (g v^T - delta), delta = sum(g o),
//   dq = scale ds k, dk = scale ds^T q, dv = p^T g.
// Two passes, so that nothing is added by atomics: k_attn_dkv keeps 32 keys a wavefront and lets
// the queries come by, k_attn_dq keeps 32 queries and lets the keys come by (p and ds
// are formed in both: seven products instead of five).
#include "attn.h"
#include "common.h"

namespace ckpt {
namespace {

using namespace at;

// sixteen lanes a row, eight columns each
__global__ __launch_bounds__(256) void k_attn_delta(AttnArgs A) {
  const int64_t at = blockIdx.x * int64_t(16) + threadIdx.x / 16;
  if (at >= A.heads * A.tq) return;
  const int64_t token = at / A.heads;
  const int head = int(at - token * A.heads), col = (threadIdx.x & 15) * 8;
  if (token < A.qoff[0] || token >= A.qoff[A.seqs]) return;
  float s = 0.f;
  if (col < A.dim) {
    const int64_t e = token * A.ldo + head * A.hso + col;
    const bf16x8 g = *reinterpret_cast<const bf16x8 *>(A.g + e), o = *reinterpret_cast<const bf16x8 *>(A.out + e);
#pragma unroll
    for (int k = 0; k < 8; ++k) s = fmaf(float(g[k]), float(o[k]), s);
  }
  s = xor_add<1>(s);
  s = xor_add<2>(s);
  s = xor_add<4>(s);
  s = xor_add<8>(s);
  if (col == 0) A.delta[head * A.tq + token] = s;
}

template <int D>
__global__ __launch_bounds__(256, 2) void k_attn_dq(AttnArgs A, int tiles) {
  constexpr int BM = 128, BN = 64, SUBS = BN / 32, T = D / 32, KK = D / 16;
  __shared__ __align__(16) unsigned char kt0[BN * D * 2], kt1[BN * D * 2], vt0[BN * D * 2], vt1[BN * D * 2];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int kvh = blockIdx.x % A.kv_heads, tile = tiles - 1 - int(blockIdx.x / A.kv_heads);
  Sequence sq;
  if (!find_tile(A, A.qoff, A.tq, A.rep, BM, tile, sq)) return;
  const int64_t rows = int64_t(sq.lq) * A.rep;
  const int64_t row = sq.first + wave * 32 + (lane & 31);
  const bool valid = row < rows;
  const int64_t r = valid ? row : rows - 1;
  const int token = int(r / A.rep), head = kvh * A.rep + int(r - int64_t(token) * A.rep);
  const int past = sq.lk - sq.lq;
  const int lim = A.causal ? min(sq.lk, max(0, token + past + 1)) : sq.lk;
  const int lim_lo = __builtin_amdgcn_readfirstlane(lim), lim_hi = __builtin_amdgcn_readlane(lim, 31);
  const int64_t last = min(sq.first + BM, rows) - 1;
  const int kend = A.causal ? min(sq.lk, max(0, int(last / A.rep) + past + 1)) : sq.lk;
  const int end = (kend + BN - 1) / BN;

  bf16x8 q[KK], g[KK];
  {
    const __bf16 *p = A.q + (sq.q0 + token) * A.ldq + head * A.hsq, *pg = A.g + (sq.q0 + token) * A.ldo + head * A.hso;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      q[kk] = kept(p, kk, A.dim);
      g[kk] = kept(pg, kk, A.dim);
    }
  }
  const float lse2 = A.lse[head * A.tq + sq.q0 + token] * LOG2E, delta = A.delta[head * A.tq + sq.q0 + token];
  const Places<D> at;
  const __bf16 *const kp = A.k + sq.k0 * A.ldk + kvh * A.hsk, *const vp = A.v + sq.k0 * A.ldv + kvh * A.hsv;
  auto load = [&](int it, unsigned char *kt, unsigned char *vt) {
    load_tile<D, BN, 256>(kt, kp + int64_t(it) * BN * A.ldk, A.ldk, sq.lk - it * BN, A.dim);
    load_tile<D, BN, 256>(vt, vp + int64_t(it) * BN * A.ldv, A.ldv, sq.lk - it * BN, A.dim);
  };
  f32x16 dq[T];
  clear(dq);
  const float sc = A.scale * LOG2E;

  auto work = [&](int it, const unsigned char *kt, const unsigned char *vt, auto masked) {
    constexpr bool MASKED = decltype(masked)::value;
#pragma unroll
    for (int u = 0; u < SUBS; ++u) {
      f32x16 s[1], dp[1];
      clear(s);
      clear(dp);
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        s[0] = mfma(at.rows(kt, u * 32, kk), q[kk], s[0]);
        dp[0] = mfma(at.rows(vt, u * 32, kk), g[kk], dp[0]);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float p = exp2_fast(fmaf(s[0][i], sc, -lse2)), ds = p * (dp[0][i] - delta);
        s[0][i] = MASKED && it * BN + u * 32 + d_row(i) >= lim ? 0.f : ds;
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int first = u * 32 + c * 16;
        if constexpr (MASKED)
          add_rows_seen<D>(dq, at, kt, first, operand(s[0], c), [&](int k) { return it * BN + first + k < lim; });
        else
          add_rows<D>(dq, at, kt, first, operand(s[0], c));
      }
    }
  };
  auto step = [&](int it, const unsigned char *kt, const unsigned char *vt, unsigned char *kn, unsigned char *vn) {
    tile_barrier();
    if (it + 1 < end) load(it + 1, kn, vn);
    if (it * BN >= lim_hi) return;
    if (it * BN + BN > lim_lo) work(it, kt, vt, std::true_type());
    else work(it, kt, vt, std::false_type());
  };
  if (end > 0) load(0, kt0, vt0);
  for (int it = 0; it < end; it += 2) {
    step(it, kt0, vt0, kt1, vt1);
    if (it + 1 < end) step(it + 1, kt1, vt1, kt0, vt0);
  }
  if (valid) store_row<D>(A.dq + (sq.q0 + token) * A.ldq + head * A.hsq, dq, A.scale, A.dim);
}

template <int D>
__global__ __launch_bounds__(256, 2) void k_attn_dkv(AttnArgs A) {
  constexpr int BM = 128, BN = 64, T = D / 32, KK = D / 16;
  __shared__ __align__(16) unsigned char qt0[BN * D * 2], qt1[BN * D * 2], gt0[BN * D * 2], gt1[BN * D * 2];
  __shared__ float st0[2 * BN], st1[2 * BN];  // lse in base 2 | delta
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int kvh = blockIdx.x % A.kv_heads, tile = int(blockIdx.x / A.kv_heads);
  Sequence sq;
  if (!find_tile(A, A.koff, A.tk, 1, BM, tile, sq)) return;
  const int first = int(sq.first), key = first + wave * 32 + (lane & 31);
  const bool valid = key < sq.lk;
  const int past = sq.lk - sq.lq;
  // the first query that sees the key, the wavefront's and the workgroup's first
  const int from = A.causal ? max(0, key - past) : 0;
  const int from_lo = __builtin_amdgcn_readfirstlane(from), from_hi = __builtin_amdgcn_readlane(from, 31);
  const int begin = (A.causal ? max(0, first - past) : 0) / BN, end = (sq.lq + BN - 1) / BN;
  const int per = max(0, end - begin), n = per * A.rep;  // tiles of a head, of all

  bf16x8 k[KK], v[KK];
  {
    const int kr = min(key, sq.lk - 1);
    const __bf16 *p = A.k + (sq.k0 + kr) * A.ldk + kvh * A.hsk, *pv = A.v + (sq.k0 + kr) * A.ldv + kvh * A.hsv;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      k[kk] = kept(p, kk, A.dim);
      v[kk] = kept(pv, kk, A.dim);
    }
  }
  const Places<D> at;
  const float sc = A.scale * LOG2E;
  auto load = [&](int it, unsigned char *qt, unsigned char *gt, float *st) {
    const int head = kvh * A.rep + it / per, t0 = (begin + it % per) * BN;
    load_tile<D, BN, 256>(qt, A.q + (sq.q0 + t0) * A.ldq + head * A.hsq, A.ldq, sq.lq - t0, A.dim);
    load_tile<D, BN, 256>(gt, A.g + (sq.q0 + t0) * A.ldo + head * A.hso, A.ldo, sq.lq - t0, A.dim);
    if (threadIdx.x < BN) {
      // rows past the sequence's and rows that see nothing: p = exp(-inf)
      const int t = t0 + threadIdx.x;
      const int64_t e = head * A.tq + sq.q0 + min(t, sq.lq - 1);
      const float lse = A.lse[e];
      st[threadIdx.x] = t < sq.lq && lse != -INFINITY ? lse * LOG2E : INFINITY;
      st[BN + threadIdx.x] = t < sq.lq && lse != -INFINITY ? A.delta[e] : 0.f;
    }
  };
  f32x16 dk[T], dv[T];
  clear(dk);
  clear(dv);

  auto work = [&](int t0, const unsigned char *qt, const unsigned char *gt, const float *st, auto masked) {
    constexpr bool MASKED = decltype(masked)::value;
#pragma unroll
    for (int u = 0; u < BN / 32; ++u) {
      f32x16 s[1], dp[1];
      clear(s);
      clear(dp);
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        s[0] = mfma(at.rows(qt, u * 32, kk), k[kk], s[0]);
        dp[0] = mfma(at.rows(gt, u * 32, kk), v[kk], dp[0]);
      }
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const int first = u * 32 + 8 * b + 4 * (lane >> 5);
        const float4 ls = *reinterpret_cast<const float4 *>(st + first), de = *reinterpret_cast<const float4 *>(st + BN + first);
        const float lsa[4] = {ls.x, ls.y, ls.z, ls.w}, dea[4] = {de.x, de.y, de.z, de.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = 4 * b + e;
          const bool hidden = MASKED && t0 + first + e < from;
          const float p = exp2_fast(fmaf(s[0][i], sc, -lsa[e])), ds = p * (dp[0][i] - dea[e]);
          s[0][i] = hidden ? 0.f : p;
          dp[0][i] = hidden ? 0.f : ds;
        }
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int first = u * 32 + c * 16;
        if constexpr (MASKED) {
          auto sees = [&](int r) { return t0 + first + r >= from; };
          add_rows_seen<D>(dv, at, gt, first, operand(s[0], c), sees);
          add_rows_seen<D>(dk, at, qt, first, operand(dp[0], c), sees);
        } else {
          add_rows<D>(dv, at, gt, first, operand(s[0], c));
          add_rows<D>(dk, at, qt, first, operand(dp[0], c));
        }
      }
    }
  };
  auto step = [&](int it, const unsigned char *qt, const unsigned char *gt, const float *st, unsigned char *qn,
                  unsigned char *gn, float *sn) {
    tile_barrier();
    if (it + 1 < n) load(it + 1, qn, gn, sn);
    const int t0 = (begin + it % per) * BN;
    if (t0 + BN <= from_lo) return;
    if (t0 < from_hi) work(t0, qt, gt, st, std::true_type());
    else work(t0, qt, gt, st, std::false_type());
  };
  if (n > 0) load(0, qt0, gt0, st0);
  for (int it = 0; it < n; it += 2) {
    step(it, qt0, gt0, st0, qt1, gt1, st1);
    if (it + 1 < n) step(it + 1, qt1, gt1, st1, qt0, gt0, st0);
  }
  if (!valid) return;
  store_row<D>(A.dk + (sq.k0 + key) * A.ldk + kvh * A.hsk, dk, A.scale, A.dim);
  store_row<D>(A.dv + (sq.k0 + key) * A.ldv + kvh * A.hsv, dv, 1.f, A.dim);
}

template <int D>
void backward(hipStream_t s, const AttnArgs &a) {
  const int kt = int(a.tk / 128) + a.seqs, qt = int(a.tq * a.rep / 128) + a.seqs;
  if (a.tk > 0) hipLaunchKernelGGL(k_attn_dkv<D>, dim3(uint32_t(kt) * a.kv_heads), dim3(256), 0, s, a);
  if (a.tq > 0) hipLaunchKernelGGL(k_attn_dq<D>, dim3(uint32_t(qt) * a.kv_heads), dim3(256), 0, s, a, qt);
}

}  // namespace

int attn_splits(const AttnArgs &a);

uint64_t attn_plan(AttnArgs &a, bool backward, char *ws) {
  if (backward) {
    if (ws) a.delta = reinterpret_cast<float *>(ws);
    return 4 * uint64_t(a.heads) * a.tq;
  }
  a.splits = attn_splits(a);
  if (a.splits == 1) return 0;
  const uint64_t rows = uint64_t(a.splits) * a.heads * a.tq;
  if (ws) {
    a.pml = reinterpret_cast<float *>(ws);
    a.po = a.pml + (2 * rows + 3) / 4 * 4;
  }
  return 4 * ((2 * rows + 3) / 4 * 4 + rows * a.dim);
}

void attn_backward(hipStream_t s, const AttnArgs &a) {
  if (a.tq > 0)
    hipLaunchKernelGGL(k_attn_delta, dim3(uint32_t((a.heads * a.tq + 15) / 16)), dim3(256), 0, s, a);
  a.dim <= 64 ? backward<64>(s, a) : backward<128>(s, a);
}

}  // namespace ckpt
