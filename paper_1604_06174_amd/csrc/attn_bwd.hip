// Attention backward over packed sequences, from the forward's o and lse:
//   p = exp(scale q k^T - lse), ds = p (g v^T - delta), delta = sum(g o),
//   dq = scale ds k, dk = scale ds^T q, dv = p^T g.
// Two passes, so that nothing is added by atomics: k_attn_dq keeps 32 queries a wavefront and lets
// the keys come by, k_attn_dkv keeps 32 keys and lets the queries come by (p and ds are formed in
// both: seven products instead of five).
//
// Both are bound as the forward is, by the order within a wavefront, with two of them on a SIMD (wide heads): of
// the cycles that a compute unit is busy, matrix instructions take 56% in dq and 48% in dk and dv, vector ones 30% and
// more (exponentials), LDS reads 28% and 36%.  8192 causal tokens, 16/4 heads of 128: dq 409 us, dk and dv 613 and 23
// for the query heads' parts, 1018 in a stream of calls, 675 TFLOP/s of the five products or 945 of the seven that
// run (the library's largest bf16 products reach 1300); 8201 tokens in 19 sequences, 16 heads of 64: 51 and 51, 95
// in a stream of calls.
#include "attn.h"
#include "common.h"

namespace ckpt {
namespace {

using namespace at;

// dq.  The accumulators of scores, their gradients and dq, and q and g kept, of wide heads leave room for two
// wavefronts on a SIMD.  Tiles of 64 keys of narrow heads halve the barriers (dq, dk and dv 94 us, with 32
// 99), of wide ones they are no gain (1044 us, with 32 1025).  delta and the base-2 lse are formed here, where
// o and g are at hand, and left for k_attn_dkv, which saves a pass of its own over both.
template <int D>
__global__ __launch_bounds__(256, 2) void k_attn_dq(AttnArgs A, int tiles) {
  constexpr int BM = 128, BN = D == 64 ? 64 : 32, SUBS = BN / 32, T = D / 32, KK = D / 16;
  __shared__ __align__(16) unsigned char kt0[BN * D * 2], kt1[BN * D * 2], vt0[BN * D * 2], vt1[BN * D * 2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kvh = blockIdx.x % A.kv_heads, tile = int(blockIdx.x / A.kv_heads);
  Sequence sq;
  if (!find_tile<true>(A, A.rep, BM, tiles, tile, sq)) return;
  const int64_t rows = int64_t(sq.lq) * A.rep;
  const int64_t row = sq.first + wave * 32 + (lane & 31);
  const bool valid = row < rows;
  const int64_t r = valid ? row : rows - 1;
  const int token = int(r / A.rep), head = kvh * A.rep + int(r - int64_t(token) * A.rep);
  const int past = sq.lk - sq.lq;
  const int lim = A.causal ? min(sq.lk, max(0, token + past + 1)) : sq.lk;
  const int lim_hi = __builtin_amdgcn_readlane(lim, 31);  // the wavefront's most
  const int lim_lo = A.causal ? min(sq.lk, max(0, int(sq.first / A.rep) + past + 1)) : sq.lk;  // the workgroup's least
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
  // the row's sum of g o and its lse in base 2 (infinite for rows that see nothing, so that p = exp2(-inf)),
  // for here and for k_attn_dkv
  const int64_t at_row = head * A.tq + sq.q0 + token;
  float lse2 = A.lse[at_row], delta = 0.f;
  lse2 = lse2 == -INFINITY ? INFINITY : lse2 * LOG2E;
  {
    const __bf16 *p = A.out + (sq.q0 + token) * A.ldo + head * A.hso;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      const bf16x8 o = kept(p, kk, A.dim);
#pragma unroll
      for (int e = 0; e < 8; ++e) delta = fmaf(float(g[kk][e]), float(o[e]), delta);
    }
    delta = halves_add(delta);
    if (valid && lane < 32) {
      A.lse2[at_row] = lse2;
      A.delta[at_row] = delta;
    }
  }
  const Places<D> places;
  const __bf16 *const kp = A.k + sq.k0 * A.ldk + kvh * A.hsk;
  const Loader<D, BN, 256> kload(kp, A.ldk, A.dim), vload(A.v + sq.k0 * A.ldv + kvh * A.hsv, A.ldv, A.dim);
  auto load = [&](int it, unsigned char *kt, unsigned char *vt) __attribute__((always_inline)) {
    kload.load(kt, int64_t(it) * BN, sq.lk - it * BN);
    vload.load(vt, int64_t(it) * BN, sq.lk - it * BN);
  };
  __shared__ int special;
  if (threadIdx.x == 0) special = 0;
  f32x16 dq[T];
  clear(dq);
  const float sc = A.scale * LOG2E;

  auto work = [&](int it, const unsigned char *kt, const unsigned char *vt, auto masked) __attribute__((always_inline)) {
    constexpr bool MASKED = decltype(masked)::value;
    const Places<D> at = places.here();
    const int left = lim - it * BN - 4 * (lane >> 5);  // keys the lane's query sees from its half's first on
#pragma unroll
    for (int u = 0; u < SUBS; ++u) {
      if (MASKED && it * BN + u * 32 >= lim_hi) break;  // nothing for the wavefront's rows
      f32x16 s[1], dp[1];
      clear(s);
      clear(dp);
      in_turn<2 * KK, 4>([&](int i) { return at.rows(i & 1 ? vt : kt, u * 32, i / 2); },
                         [&](int i, bf16x8 a) {
                           if (i & 1) dp[0] = mfma(a, g[i / 2], dp[0]);
                           else s[0] = mfma(a, q[i / 2], s[0]);
                         });
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float p = exp2_fast(fmaf(s[0][i], sc, -lse2)), ds = p * (dp[0][i] - delta);
        s[0][i] = MASKED && u * 32 + 8 * (i / 4) + i % 4 >= left ? 0.f : ds;
      }
      const bf16x8 ds[2] = {operand(s[0], 0), operand(s[0], 1)};
      in_turn<2 * T, 4>([&](int i) { return at.columns(kt, u * 32 + i / T * 16, i % T); },
                        [&](int i, bf16x8 a) { dq[i % T] = mfma(a, ds[i / T], dq[i % T]); });
    }
  };
  if (end > 0) load(0, kt0, vt0);
  const int full = min(end, lim_lo / BN) & ~1;  // tiles that every row sees whole
  two_kinds(end, full, [&](int it, auto place, auto masked) __attribute__((always_inline)) {
    tile_barrier();
    if constexpr (decltype(masked)::value) {
      scrub<BN * D * 2>(place ? kt1 : kt0, special);
      __syncthreads();
    }
    if (it + 1 < end) load(it + 1, place ? kt0 : kt1, place ? vt0 : vt1);
    work(it, place ? kt1 : kt0, place ? vt1 : vt0, masked);
  });
  if (end > 0 && special)
    add_special(dq, kp, A.ldk, A.dim, full * BN, min(end * BN, sq.lk), true, [&](int j) { return j < lim; });
  if (valid) store_row(A.dq + (sq.q0 + token) * A.ldq + head * A.hsq, dq, A.scale, A.dim);
}

static __device__ __align__(16) const float g_infinity[64] = {
#define CKPT_INF4 INFINITY, INFINITY, INFINITY, INFINITY
#define CKPT_INF16 CKPT_INF4, CKPT_INF4, CKPT_INF4, CKPT_INF4
    CKPT_INF16, CKPT_INF16, CKPT_INF16, CKPT_INF16};

// dk and dv: the wavefront's keys stay in registers and the workgroup's values in LDS, read as they are
// needed, for dk, dv, p and ds fill the registers (of wide heads five go to memory, none of them in the loop
// over whole tiles); queries, g, lse and delta come by in tiles of 32.
// A key head's query heads are taken one after the other, or dealt to `parts` workgroups.
template <int D>
__global__ __launch_bounds__(256, D == 64 ? 3 : 2) void k_attn_dkv(AttnArgs A) {
  constexpr int BM = 128, BN = 32, T = D / 32, KK = D / 16;
  __shared__ __align__(16) unsigned char qt0[BN * D * 2], qt1[BN * D * 2], gt0[BN * D * 2], gt1[BN * D * 2];
  __shared__ __align__(16) unsigned char vt[BM * D * 2];
  __shared__ __align__(16) float st0[128], st1[128];  // lse in base 2 | delta, 64 places each
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // a tile's heads and their parts side by side: workgroups start in the order of their work
  const int part = blockIdx.x % A.parts, kvh = blockIdx.x / A.parts % A.kv_heads, tile = int(blockIdx.x / A.parts / A.kv_heads);
  Sequence sq;
  if (!find_tile<false>(A, 1, BM, 0, tile, sq)) return;
  const int first = int(sq.first), key = first + wave * 32 + (lane & 31);
  const bool valid = key < sq.lk;
  const int past = sq.lk - sq.lq;
  // the first query that sees the key, and the workgroup's first tile
  const int from = A.causal ? max(0, key - past) : 0;
  const int from_lo = __builtin_amdgcn_readfirstlane(from);  // the wavefront's least
  const int begin = (A.causal ? max(0, first - past) : 0) / BN, end = (sq.lq + BN - 1) / BN;
  const int heads = A.rep / A.parts, head0 = kvh * A.rep + part * heads;
  const int per = max(0, end - begin), n = per * heads;  // tiles of a head, of all

  bf16x8 k[KK];
  {
    const __bf16 *p = A.k + (sq.k0 + min(key, sq.lk - 1)) * A.ldk + kvh * A.hsk;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) k[kk] = kept(p, kk, A.dim);
  }
  const Places<D> places;
  const float sc = A.scale * LOG2E;
  const Loader<D, BN, 256> qload(A.q + sq.q0 * A.ldq + head0 * A.hsq, A.ldq, A.dim),
      gload(A.g + sq.q0 * A.ldo + head0 * A.hso, A.ldo, A.dim);
  auto load = [&](int h, int t, unsigned char *qt, unsigned char *gt, float *st) __attribute__((always_inline)) {
    const int t0 = t * BN;
    qload.load(qt, t0, sq.lq - t0, 2 * h * A.hsq);
    gload.load(gt, t0, sq.lq - t0, 2 * h * A.hso);
    // lse and delta, a wavefront each
    if (wave < 2) {
      const float *src = (wave ? A.delta : A.lse2) + (head0 + h) * A.tq + sq.q0 + t0;
      if (t0 + BN <= sq.lq) {
        asm("" : "+s"(src));
        const char *const p = reinterpret_cast<const char *>(src);
        __builtin_amdgcn_global_load_lds(p + unsigned(4 * (lane & (BN - 1))), (lds_void *)(st + 64 * wave), 4, 0, 0);
      } else {  // rows past the sequence's: p = exp2(-inf)
        int at = lane;
        asm volatile("" : "+v"(at));
        const float *const none = (wave ? reinterpret_cast<const float *>(g_zeros) : g_infinity) + at;
        const float *const p = t0 + at < sq.lq ? src + at : none;
        __builtin_amdgcn_global_load_lds(p, (lds_void *)(st + 64 * wave), 4, 0, 0);
      }
    }
  };
  f32x16 dk[T], dv[T];
  clear(dk);
  clear(dv);
  __shared__ int special;
  if (threadIdx.x == 0) special = 0;

  auto work = [&](int t0, const unsigned char *qt, const unsigned char *gt, const float *st, auto masked) __attribute__((always_inline)) {
    constexpr bool MASKED = decltype(masked)::value;
    const Places<D> at = places.here();
    const int unseen = from - t0 - 4 * (lane >> 5);  // queries that do not see the lane's key, from its half's first on
#pragma unroll
    for (int u = 0; u < BN / 32; ++u) {
      if (MASKED && t0 + u * 32 + 32 <= from_lo) continue;  // no query that sees the wavefront's keys
      f32x16 s[1], dp[1];
      clear(s);
      clear(dp);
      in_turn<KK, 4>([&](int i) { return at.rows(qt, u * 32, i); },
                     [&](int i, bf16x8 a) { s[0] = mfma(a, k[i], s[0]); });
      struct Pair {
        bf16x8 g, v;
      };
      in_turn<KK, 2>([&](int i) { return Pair{at.rows(gt, u * 32, i), at.rows(vt, wave * 32, i)}; },
                     [&](int i, const Pair &a) { dp[0] = mfma(a.g, a.v, dp[0]); });
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const int row = u * 32 + 8 * b + 4 * (lane >> 5);
        const float4 ls = *reinterpret_cast<const float4 *>(st + row), de = *reinterpret_cast<const float4 *>(st + 64 + row);
        const float lsa[4] = {ls.x, ls.y, ls.z, ls.w}, dea[4] = {de.x, de.y, de.z, de.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = 4 * b + e;
          const bool hidden = MASKED && u * 32 + 8 * b + e < unseen;
          const float p = exp2_fast(fmaf(s[0][i], sc, -lsa[e])), ds = p * (dp[0][i] - dea[e]);
          s[0][i] = hidden ? 0.f : p;
          dp[0][i] = hidden ? 0.f : ds;
        }
      }
      const bf16x8 pb[2] = {operand(s[0], 0), operand(s[0], 1)}, ds[2] = {operand(dp[0], 0), operand(dp[0], 1)};
      in_turn<2 * T, 4>([&](int i) { return at.columns(gt, u * 32 + i / T * 16, i % T); },
                        [&](int i, bf16x8 a) { dv[i % T] = mfma(a, pb[i / T], dv[i % T]); });
      in_turn<2 * T, 4>([&](int i) { return at.columns(qt, u * 32 + i / T * 16, i % T); },
                        [&](int i, bf16x8 a) { dk[i % T] = mfma(a, ds[i / T], dk[i % T]); });
    }
  };
  // Tiles from the last query back: workgroups that start together read the same tiles together
  // (through one L2), and the tiles with queries before some key's first come last, after all heads'
  // others.
  const int seen = min(end, max(begin, A.causal ? (max(0, min(first + BM, sq.lk) - 1 - past) + BN - 1) / BN : 0));
  struct Cursor {
    int h, t, lo, hi;  // head, tile, its kind's tiles
  };
  auto advance = [&](Cursor &c) __attribute__((always_inline)) {
    if (--c.t >= c.lo) return;
    if (++c.h == heads) c = Cursor{0, 0, begin, seen};
    c.t = c.hi - 1;
  };
  const Cursor start = seen < end ? Cursor{0, end - 1, seen, end} : Cursor{0, seen - 1, begin, seen};
  Cursor ahead = start, now = start;
  auto next = [&](unsigned char *qt, unsigned char *gt, float *st) __attribute__((always_inline)) {
    load(ahead.h, ahead.t, qt, gt, st);
    advance(ahead);
  };
  if (n > 0) {
    Loader<D, BM, 256>(A.v + sq.k0 * A.ldv + kvh * A.hsv, A.ldv, A.dim).load(vt, first, sq.lk - first);
    next(qt0, gt0, st0);
  }
  const int whole = (end - seen) * heads;  // tiles that see all of the workgroup's keys
  two_kinds(n, whole & ~1, [&](int it, auto place, auto masked) __attribute__((always_inline)) {
    tile_barrier();
    if constexpr (decltype(masked)::value) {
      scrub<BN * D * 2>(place ? qt1 : qt0, special);
      scrub<BN * D * 2>(place ? gt1 : gt0, special);
      __syncthreads();
    }
    if (it + 1 < n) next(place ? qt0 : qt1, place ? gt0 : gt1, place ? st0 : st1);
    work(now.t * BN, place ? qt1 : qt0, place ? gt1 : gt0, place ? st1 : st0, masked);
    advance(now);
  });
  if (n > 0 && special)
    for (int h = 0; h < heads; ++h) {
      auto sees = [&](int r) { return r >= from; };
      // the tiles with tests: an odd one of the others, which comes just before them, is taken so too
      const int row0 = begin * BN, row1 = min(sq.lq, (seen + (h == heads - 1 && (whole & 1))) * BN);
      add_special(dv, A.g + sq.q0 * A.ldo + (head0 + h) * A.hso, A.ldo, A.dim, row0, row1, false, sees);
      add_special(dk, A.q + sq.q0 * A.ldq + (head0 + h) * A.hsq, A.ldq, A.dim, row0, row1, true, sees);
    }
  if (!valid) return;
  if (A.parts > 1) {
    // fp32, for k_attn_heads: dk's parts, then dv's
    float *const p = A.pkv + ((int64_t(part) * A.tk + sq.k0 + key) * A.kv_heads + kvh) * A.dim;
    store_row(p, dk, A.scale, A.dim);
    store_row(p + A.parts * A.tk * A.kv_heads * A.dim, dv, 1.f, A.dim);
    return;
  }
  store_row(A.dk + (sq.k0 + key) * A.ldk + kvh * A.hsk, dk, A.scale, A.dim);
  store_row(A.dv + (sq.k0 + key) * A.ldv + kvh * A.hsv, dv, 1.f, A.dim);
}

// the parts of the query heads that share a key head, added up in order; a thread has eight columns
// of dk (blockIdx.y 0) or dv
__global__ __launch_bounds__(256) void k_attn_heads(AttnArgs A) {
  const int vecs = A.dim / 8;
  const int64_t at = blockIdx.x * int64_t(256) + threadIdx.x, row = at / vecs, n = A.tk * A.kv_heads;
  if (row >= n) return;
  const int64_t token = row / A.kv_heads;
  if (token < A.koff[0] || token >= A.koff[A.seqs]) return;
  const int head = int(row - token * A.kv_heads), col = int(at - row * vecs) * 8;
  const float *p = A.pkv + ((blockIdx.y ? int64_t(A.parts) * n : 0) + row) * A.dim + col;
  float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 2
  for (int k = 0; k < A.parts; ++k, p += n * A.dim) {
    const float4 a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
    s[0] += a.x, s[1] += a.y, s[2] += a.z, s[3] += a.w;
    s[4] += b.x, s[5] += b.y, s[6] += b.z, s[7] += b.w;
  }
  bf16x8 r;
#pragma unroll
  for (int k = 0; k < 8; ++k) r[k] = (__bf16)s[k];
  __bf16 *const to = blockIdx.y ? A.dv + token * A.ldv + head * A.hsv : A.dk + token * A.ldk + head * A.hsk;
  *reinterpret_cast<bf16x8 *>(to + col) = r;
}

template <int D>
void backward(hipStream_t s, const AttnArgs &a) {
  const int kt = int(a.tk / 128) + a.seqs, qt = int(a.tq * a.rep / 128) + a.seqs;
  if (a.tq > 0) hipLaunchKernelGGL(k_attn_dq<D>, dim3(uint32_t(qt) * a.kv_heads), dim3(256), 0, s, a, qt);
  if (a.tk == 0) return;
  hipLaunchKernelGGL(k_attn_dkv<D>, dim3(uint32_t(kt) * a.kv_heads * a.parts), dim3(256), 0, s, a);
  if (a.parts > 1)
    hipLaunchKernelGGL(k_attn_heads, dim3(uint32_t((a.tk * a.kv_heads * (a.dim / 8) + 255) / 256), 2), dim3(256), 0, s, a);
}

}  // namespace

int attn_splits(const AttnArgs &a);

// Workgroups that a key head's query heads are dealt to, a divisor of their number: as many as
// make two workgroups for each place on the chip, so that the causal ones, of all lengths, even out.
static int parts_of(const AttnArgs &a) {
  const int64_t work = (a.tk / 128 > a.seqs ? a.tk / 128 : a.seqs) * a.kv_heads;
  int n = 1;
  while (n < a.rep && (a.rep % n || work * n < 1024)) ++n;
  return n;
}

uint64_t attn_plan(AttnArgs &a, bool backward, char *ws) {
  auto align4 = [](uint64_t v) { return (v + 3) / 4 * 4; };
  if (backward) {
    a.parts = parts_of(a);
    const uint64_t rows = align4(uint64_t(a.heads) * a.tq);
    if (ws) {
      a.delta = reinterpret_cast<float *>(ws);
      a.lse2 = a.delta + rows;
      a.pkv = a.lse2 + rows;
    }
    return 4 * (2 * rows + (a.parts > 1 ? 2 * uint64_t(a.parts) * a.tk * a.kv_heads * a.dim : 0));
  }
  a.splits = attn_splits(a);
  if (a.splits == 1) return 0;
  const uint64_t rows = uint64_t(a.splits) * a.heads * a.tq;
  if (ws) {
    a.pml = reinterpret_cast<float *>(ws);
    a.po = a.pml + align4(2 * rows);
  }
  return 4 * (align4(2 * rows) + rows * a.dim);
}

void attn_backward(hipStream_t s, const AttnArgs &a) {
  a.dim <= 64 ? backward<64>(s, a) : backward<128>(s, a);
}

}  // namespace ckpt
