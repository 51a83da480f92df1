// Attention forward over packed sequences: o = softmax(scale q k^T) v and the logarithm of each
// row's sum, in one pass over the keys with the running maximum and sum of the softmax.
//
// The query rows that share a key head, (token, head of the group) in this order, are one
// matrix: a key tile is read once for all of them, and single tokens fill tiles as far as
// their heads go.  Each of a workgroup's wavefronts keeps 32 of these rows; the keys come by in
// tiles through LDS, later ones loading while one is worked on (k_attn_many, k_attn_few).
// Where there are too few workgroups for the chip, the keys are split over several, whose
// unfinished rows go to the workspace and are joined by k_attn_join.
#include "attn.h"
#include "common.h"

namespace ckpt {
namespace {

using namespace at;

// A row's softmax as it goes on: exponentials are powers of two relative to `base`, times 2^-ROOM, and l is
// their sum.  The base is a whole number, so that moving it scales by a power of two, which rounds
// nothing; it is moved only when an exponential would exceed 1.  So exponentials are never above
// exp(score - the row's largest), and a product with values near the type's largest overflows only where
// that one would.  The products with the values take the exponentials rounded to bf16, so o is divided by the
// sum of these, lr: it is a mean of the values by weights that add up to 1, exact where a row sees one key
// (with l it would be off by half a step of bf16), and lse takes l.
//
// ROOM: 16384 tokens, 16/4 heads of 128 in seven sequences take 235 us, 237 with 2 and 250 with 0, for the base then
// moves more often.  An exponent of -8 is rounded to 2^-21, so lse of rows with few keys is off by 1.4e-7 on
// the average, and by 0.5e-7 with 0; of rows with hundreds by 3.7e-7 and 3.4e-7, the scores' own rounding.
constexpr float ROOM = 8.f;

// The base of a row that sees keys is never below this, that of one that sees none is -infinity: both have l = 0 if
// all scores are -infinity, but the first is no zero, it is 0 / 0.
constexpr float LEAST = -3.402823466e38f;

// lse of a row, and what its o is to be multiplied by for the mean of the values, f / l as a rule
static_assert(ROOM == 8.f, "l is 2^-8 times the sum relative to the base");
__device__ __forceinline__ float lse_of(float base, float l) {
  return l != 0.f ? fmaf(base, LN2, logf(l * 0x1p8f)) : base == -INFINITY ? -INFINITY : NAN;
}
__device__ __forceinline__ float over(float f, float base, float l) {
  return l != 0.f ? f / l : base == -INFINITY ? 0.f : NAN;
}

// An exponent is score sc + add, in one operation.  Where the base is large that will not do: the product
// score sc, which the base comes from, and the one inside the fused operation differ by half a step of fp32 (1/4 at
// 2^22, 128 at 2^31), so an exponential may overflow or all of a row's be zeros.  If it is so for a row of the
// wavefront, exponents are formed apart (a test of a scalar for others).
struct Sums {
  float sc;  // of scores to exponents
  float base = -INFINITY, l = 0.f, lr = 0.f, top = 0.f;
  float add = 0.f;
  bool large = false;

  __device__ __forceinline__ explicit Sums(float scale) : sc(scale) {}
  // does a row of the wavefront have to move its base for scores up to `score`?
  __device__ __forceinline__ bool rises(float score) {
    top = score * sc;
    return __any(top - base > ROOM);
  }
  // moves it, and says what the sums so far are to be scaled by
  __device__ __forceinline__ float move() {
    const float to = fmaxf(base, ceilf(top));
    const float f = to == base ? 1.f : exp2_fast(base - to);
    base = to;
    l *= f;
    lr *= f;
    const float from = base == -INFINITY ? 0.f : base;
    large = __any(fabsf(from) >= 0x1p22f);
    add = large ? 0.f : -ROOM - from;
    return f;
  }
  __device__ __forceinline__ float apart(float score) const {
#pragma clang fp contract(off)
    const float e = score * sc;
    return e - (base == -INFINITY ? 0.f : base) - ROOM;
  }
  __device__ __forceinline__ float exponential(float score) const { return exp2_fast(fmaf(score, large ? 1.f : sc, add)); }
  // to lr: eight rounded exponentials
  __device__ __forceinline__ void add_rounded(bf16x8 p) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 ones = {(__bf16)1.f, (__bf16)1.f};
#pragma unroll
    for (int e = 0; e < 8; e += 2) lr = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{p[e], p[e + 1]}, ones, lr, false);
  }
  // after the last key: l of the whole row, and the factor of o that goes with it.  sees: the row sees a key (of a
  // row's parts, one says so)
  __device__ __forceinline__ float end(bool sees) {
    if (sees) base = fmaxf(base, LEAST);
    l = halves_add(l);
    lr = halves_add(lr);
    return l == 0.f ? 0.f : l / lr;
  }
};

// A workgroup's rows and the keys they see: what a lane needs of its query.
template <int BM>
struct Query {
  Sequence sq;
  int64_t rows;
  int token, head, lim;  // lim: keys it sees
  int lim_lo, kend;      // the workgroup's least and most
  bool valid;

  // the lane's row is `row` of the tile; false: the tile has none
  __device__ __forceinline__ bool find(const AttnArgs &A, int tiles, int tile, int kvh, int row) {
    if (!find_tile<true>(A, A.rep, BM, tiles, tile, sq)) return false;
    rows = int64_t(sq.lq) * A.rep;
    valid = sq.first + row < rows;
    const int64_t r = valid ? sq.first + row : rows - 1;
    token = int(r / A.rep);
    head = kvh * A.rep + int(r - int64_t(token) * A.rep);
    const int past = sq.lk - sq.lq;
    lim = A.causal ? min(sq.lk, max(0, token + past + 1)) : sq.lk;
    const int64_t last = min(sq.first + BM, rows) - 1;
    lim_lo = A.causal ? min(sq.lk, max(0, int(sq.first / A.rep) + past + 1)) : sq.lk;
    kend = A.causal ? min(sq.lk, max(0, int(last / A.rep) + past + 1)) : sq.lk;
    return true;
  }
};

// What a workgroup does: a tile's heads and their splits lie side by side, so that workgroups start in
// the order of their work.
struct Block {
  int split, kvh, tile;

  __device__ __forceinline__ explicit Block(const AttnArgs &A) {
    split = int(blockIdx.x % A.splits);
    kvh = int(blockIdx.x / A.splits % A.kv_heads);
    tile = int(blockIdx.x / A.splits / A.kv_heads);
  }
  // the split's share of n tiles
  __device__ __forceinline__ void share(const AttnArgs &A, int n, int &begin, int &end) const {
    begin = int(int64_t(n) * split / A.splits);
    end = int(int64_t(n) * (split + 1) / A.splits);
  }
};

// Where a lane's row goes: factor o / l and lse, or, of a split, factor o and its sums.  `part` says what of
// o: part(row, scale) with a row of bf16 or of floats.
template <typename F>
__device__ __forceinline__ void finish(const AttnArgs &A, int split, int head, int64_t token, float base, float l,
                                       float factor, bool sums, F &&part) {
  const int64_t at_row = head * A.tq + token;
  sums = sums && (threadIdx.x & 63) < 32;
  if (A.splits > 1) {
    const int64_t p = int64_t(split) * A.heads * A.tq + at_row;
    if (sums) {
      A.pml[2 * p] = base;
      A.pml[2 * p + 1] = l;
    }
    part(A.po + p * A.dim, factor);
    return;
  }
  if (sums) A.lse[at_row] = lse_of(base, l);
  part(A.o + token * A.ldo + head * A.hso, over(factor, base, l));
}

// A wavefront's 32 rows as 32 keys after the other go by; of o it forms 32 N columns.
template <int D, int N>
struct Rows {
  static constexpr int KK = D / 16;
  bf16x8 q[KK];
  f32x16 o[N];
  Sums z;

  __device__ __forceinline__ Rows(const AttnArgs &A, const __bf16 *query) : z(A.scale * LOG2E) {
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) q[kk] = kept(query, kk, A.dim);
    clear(o);
  }
  // the 32 keys and values from row `first` of the tiles on; `seen`: how many of them the lane's row sees
  // (MASKED: it may be less than all)
  template <bool MASKED>
  __device__ __forceinline__ void turn(const Places<D> &at, const unsigned char *kt, const unsigned char *vt, int first,
                                       int seen) {
    f32x16 s[1];
    clear(s);
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) s[0] = mfma(at.rows(kt, first, kk), q[kk], s[0]);
    const int left = seen - 4 * ((threadIdx.x & 63) >> 5);  // from the first key of the lane's half on
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if (MASKED && 8 * (i / 4) + i % 4 >= left) s[0][i] = -INFINITY;
      top = fmaxf(top, s[0][i]);
    }
    if (z.rises(halves_max(top))) {
      const float f = z.move();
#pragma unroll
      for (int t = 0; t < N; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] *= f;
    }
    if (z.large) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[0][i] = z.apart(s[0][i]);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[0][i] = z.exponential(s[0][i]);
      z.l += s[0][i];
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const bf16x8 p = operand(s[0], c);
      z.add_rounded(p);
      add_rows(o, at, vt, first + 16 * c, p);
    }
  }
};

// The loop over tiles [begin, end) of BN keys that both kernels share: work(tile, kt, vt, masked) on each,
// the next loading meanwhile.  Tiles that not every row sees whole have their values scrubbed; the first
// of them is returned.
template <int D, int BN, typename F>
__device__ __forceinline__ int each_tile(const Loader<D, BN, 256> &kload, const Loader<D, BN, 256> &vload, int begin,
                                         int end, int lim_lo, int lk, unsigned char *kt0, unsigned char *kt1,
                                         unsigned char *vt0, unsigned char *vt1, int &special, F &&work) {
  auto load = [&](int it, unsigned char *kt, unsigned char *vt) __attribute__((always_inline)) {
    kload.load(kt, int64_t(it) * BN, lk - it * BN);
    vload.load(vt, int64_t(it) * BN, lk - it * BN);
  };
  const int n = end - begin, full = max(0, min(n, lim_lo / BN - begin)) & ~1;
  if (threadIdx.x == 0) special = 0;
  if (n > 0) load(begin, kt0, vt0);
  two_kinds(n, full, [&](int i, auto place, auto masked) __attribute__((always_inline)) {
    tile_barrier();
    if constexpr (decltype(masked)::value) {
      scrub<BN * D * 2>(place ? vt1 : vt0, special);
      __syncthreads();
    }
    if (i + 1 < n) load(begin + i + 1, place ? kt0 : kt1, place ? vt0 : vt1);
    work(begin + i, place ? kt1 : kt0, place ? vt1 : vt0, masked);
  });
  return begin + full;
}

// Four wavefronts of 32 rows share tiles of 32 keys, which leaves room for three of them on each SIMD.
// 16384 tokens, 16/4 heads of 128 in seven sequences: 235 us, 860 TFLOP/s of the visible products (the library's
// largest bf16 products reach 1300).  Bound by a wavefront's own order, scores, exponentials, values, which three on
// a SIMD cover in part: of the cycles that a compute unit is busy, vector instructions take 64%, matrix ones 45%,
// LDS reads 23%, without a conflict.  Tiles of 64 keys with two wavefronts took 4% longer, and so did the scores, exponentials
// and values of three turns side by side; 64 rows a wavefront, one a SIMD, 25%.
template <int D>
__global__ __launch_bounds__(256, 3) void k_attn_many(AttnArgs A, int tiles) {
  constexpr int BM = 128, BN = 32;
  __shared__ __align__(16) unsigned char kt0[BN * D * 2], kt1[BN * D * 2], vt0[BN * D * 2], vt1[BN * D * 2];
  __shared__ int special;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Block b(A);
  Query<BM> y;
  if (!y.find(A, tiles, b.tile, b.kvh, wave * 32 + (lane & 31))) return;
  const int lk = y.sq.lk, lim_hi = __builtin_amdgcn_readlane(y.lim, 31);  // the wavefront's most
  const bool idle = y.sq.first + wave * 32 >= y.rows;
  int begin, end;
  b.share(A, (y.kend + BN - 1) / BN, begin, end);

  Rows<D, D / 32> r(A, A.q + (y.sq.q0 + y.token) * A.ldq + y.head * A.hsq);
  const Places<D> places;
  const __bf16 *const vp = A.v + y.sq.k0 * A.ldv + b.kvh * A.hsv;
  const Loader<D, BN, 256> kload(A.k + y.sq.k0 * A.ldk + b.kvh * A.hsk, A.ldk, A.dim), vload(vp, A.ldv, A.dim);
  const int scrubbed =
      each_tile(kload, vload, begin, end, y.lim_lo, lk, kt0, kt1, vt0, vt1, special,
                [&](int it, const unsigned char *kt, const unsigned char *vt, auto masked) __attribute__((always_inline)) {
                  constexpr bool MASKED = decltype(masked)::value;
                  if (idle || (MASKED && it * BN >= lim_hi)) return;  // nothing for the wavefront's rows
                  r.template turn<MASKED>(places.here(), kt, vt, 0, y.lim - it * BN);
                });
  if (begin < end && special)
    add_special(r.o, vp, A.ldv, A.dim, scrubbed * BN, min(end * BN, lk), false, [&](int j) { return j < y.lim; });
  const float factor = r.z.end(b.split == 0 && y.lim > 0);
  if (y.valid)
    finish(A, b.split, y.head, y.sq.q0 + y.token, r.z.base, r.z.l, factor, true,
           [&](auto *row, float scale) { store_row(row, r.o, scale, A.dim); });
}

// Four wavefronts with the same 32 rows and tiles of 64 keys: two take 32 of the keys each, and half of o's
// columns (forming the same scores twice, which costs a call that HBM bounds nothing), and the sums over the keys
// are joined at the end.  Bound by HBM: 16 single tokens, 32/8 heads of 128, up to 8192 keys, 64 us in
// all, 4.7 TB/s.  With tiles of 128 keys, a quarter of them a wavefront's, one workgroup fits a compute unit,
// and its start and end (7 us) are not covered: 3 us more.
template <int D>
__global__ __launch_bounds__(256) void k_attn_few(AttnArgs A, int tiles) {
  constexpr int BM = 32, BN = 64, T = D / 32, N = T / 2;
  __shared__ __align__(16) unsigned char kt0[BN * D * 2], kt1[BN * D * 2], vt0[BN * D * 2], vt1[BN * D * 2];
  __shared__ int special;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Block b(A);
  Query<BM> y;
  if (!y.find(A, tiles, b.tile, b.kvh, lane & 31)) return;
  const int lk = y.sq.lk;
  int begin, end;
  b.share(A, (y.kend + BN - 1) / BN, begin, end);

  const int part = wave & 1, columns = (wave >> 1) * N;  // its keys of a tile and its columns / 32
  Rows<D, N> r(A, A.q + (y.sq.q0 + y.token) * A.ldq + y.head * A.hsq);
  const Places<D> places(columns);
  const __bf16 *const vp = A.v + y.sq.k0 * A.ldv + b.kvh * A.hsv;
  const Loader<D, BN, 256> kload(A.k + y.sq.k0 * A.ldk + b.kvh * A.hsk, A.ldk, A.dim), vload(vp, A.ldv, A.dim);
  const int scrubbed =
      each_tile(kload, vload, begin, end, y.lim_lo, lk, kt0, kt1, vt0, vt1, special,
                [&](int it, const unsigned char *kt, const unsigned char *vt, auto masked) __attribute__((always_inline)) {
                  r.template turn<decltype(masked)::value>(places.here(), kt, vt, part * 32, y.lim - it * BN - part * 32);
                });
  if (begin < end && special)
    for (int it = scrubbed; it < end; ++it)
      add_special(r.o, vp + 32 * columns, A.ldv, A.dim - 32 * columns, it * BN + part * 32,
                  min(it * BN + part * 32 + 32, lk), false, [&](int j) { return j < y.lim; });

  // The sums by their larger base: o (fp32, four values of a lane a place) goes through two of the tiles,
  // and each wavefront adds up, and stores, 32 columns.
  __shared__ float bases[2][32], ls[2][32], factors[2][32];
  tile_barrier();
  auto place = [&](int w, int t, int c) { return reinterpret_cast<float4 *>(w ? vt0 : kt0) + (t * 4 + c) * 64 + lane; };
#pragma unroll
  for (int t = 0; t < N; ++t)
#pragma unroll
    for (int c = 0; c < 4; ++c)
      *place(part, columns + t, c) = make_float4(r.o[t][4 * c], r.o[t][4 * c + 1], r.o[t][4 * c + 2], r.o[t][4 * c + 3]);
  const float factor = r.z.end(b.split == 0 && part == 0 && y.lim > 0);
  if (columns == 0 && lane < 32) {
    bases[part][lane] = r.z.base;
    ls[part][lane] = r.z.l;
    factors[part][lane] = factor;
  }
  __syncthreads();
  if (wave >= T) return;
  const float base = fmaxf(bases[0][lane & 31], bases[1][lane & 31]);
  float sum = 0.f;
  f32x16 out;
#pragma unroll
  for (int i = 0; i < 16; ++i) out[i] = 0.f;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    // a wavefront without keys has a factor of 0 and nothing but zeros
    const float f = exp2_fast(bases[w][lane & 31] - (base == -INFINITY ? 0.f : base));
    const float fo = f * factors[w][lane & 31];
    sum += ls[w][lane & 31] * f;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const float4 v = *place(w, wave, c);
      out[4 * c] = fmaf(v.x, fo, out[4 * c]);
      out[4 * c + 1] = fmaf(v.y, fo, out[4 * c + 1]);
      out[4 * c + 2] = fmaf(v.z, fo, out[4 * c + 2]);
      out[4 * c + 3] = fmaf(v.w, fo, out[4 * c + 3]);
    }
  }
  if (y.valid)
    finish(A, b.split, y.head, y.sq.q0 + y.token, base, sum, 1.f, wave == 0,
           [&](auto *row, float scale) { store_tile(row, out, wave, scale, A.dim); });
}

// A row's splits joined: a wavefront a row, lane z with the sums of split z (there are at most 64), then
// sixteen lanes with eight columns each for every fourth split.  Every split is added, however small
// its factor: an infinity or a NaN that its keys' values left in its columns stands nowhere else.
__global__ __launch_bounds__(256) void k_attn_join(AttnArgs A) {
  const int64_t at = blockIdx.x * int64_t(4) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = A.heads * A.tq;
  if (at >= n) return;
  const int64_t token = at % A.tq;
  const int lane = threadIdx.x & 63, head = int(at / A.tq), col = (lane & 15) * 8, quarter = lane >> 4;
  // rows of no sequence have no splits either
  if (token < A.qoff[0] || token >= A.qoff[A.seqs]) return;
  float base = -INFINITY, l = 0.f;
  if (lane < A.splits) {
    base = A.pml[2 * (lane * n + at)];
    l = A.pml[2 * (lane * n + at) + 1];
  }
  float top = base;
#pragma unroll
  for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
  const float f = exp2_fast(base - (top == -INFINITY ? 0.f : top));  // 0 for a split without keys, which left zeros
  l *= f;                                 // a NaN of a split stays one
#pragma unroll
  for (int o = 32; o; o >>= 1) l += __shfl_xor(l, o);
  float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  const bool ok = col < A.dim;
  for (int z0 = 0; z0 < A.splits; z0 += 4) {
    const int z = z0 + quarter;
    const float fz = __shfl(f, z);
    if (!ok || z >= A.splits) continue;
    const float4 *const p = reinterpret_cast<const float4 *>(A.po + (z * n + at) * A.dim + col);
    const float4 a = p[0], b = p[1];
    s[0] = fmaf(a.x, fz, s[0]), s[1] = fmaf(a.y, fz, s[1]), s[2] = fmaf(a.z, fz, s[2]), s[3] = fmaf(a.w, fz, s[3]);
    s[4] = fmaf(b.x, fz, s[4]), s[5] = fmaf(b.y, fz, s[5]), s[6] = fmaf(b.z, fz, s[6]), s[7] = fmaf(b.w, fz, s[7]);
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) s[k] = xor_add<32>(xor_add<16>(s[k]));
  if (lane == 0) A.lse[at] = lse_of(top, l);
  if (ok && quarter == 0) {
    const float inv = over(1.f, top, l);
    bf16x8 r;
#pragma unroll
    for (int k = 0; k < 8; ++k) r[k] = (__bf16)(s[k] * inv);
    *reinterpret_cast<bf16x8 *>(A.o + token * A.ldo + head * A.hso + col) = r;
  }
}

// Up to 32 rows a sequence on the average go to k_attn_few.  64 sequences of 1024 keys, 16 heads of 64: 8 or 32
// rows each 61 us (by k_attn_many 57), 64 each 103 (61); one token, 8 heads of 128 against 2048 keys 13 (16),
// 16 tokens of 32/8 heads against up to 8192 56 (62).
bool few_rows(const AttnArgs &a) { return a.tq * a.rep <= int64_t(32) * a.seqs; }

template <int D>
void forward(hipStream_t s, const AttnArgs &a) {
  const int bm = few_rows(a) ? 32 : 128;
  const int tiles = int(a.tq * a.rep / bm) + a.seqs;
  const dim3 grid(uint32_t(tiles) * a.kv_heads * a.splits);
  if (bm == 32)
    hipLaunchKernelGGL(k_attn_few<D>, grid, dim3(256), 0, s, a, tiles);
  else
    hipLaunchKernelGGL(k_attn_many<D>, grid, dim3(256), 0, s, a, tiles);
  if (a.splits > 1)
    hipLaunchKernelGGL(k_attn_join, dim3(uint32_t((a.heads * a.tq + 3) / 4)), dim3(256), 0, s, a);
}

}  // namespace

// Workgroups for one another's keys where the rows alone make less than three for each compute
// unit; a split is 256 keys at least of a sequence of the average length.  768: 16 single tokens,
// 32/8 heads of 128, against up to 8192 keys (three batches) 56, 56 and 58 us; 512: 68, 66 and 68, for the longest
// sequences end last; 1024: 59, 59 and 61.  Against 4096 keys each it is 64, 60 and 62, but lengths are seldom
// equal.  256 keys: one token of 8 heads against 2048 13 us, of 32/8 heads against 16384 26; 512 keys: 17 and 23.
int attn_splits(const AttnArgs &a) {
  const int bm = few_rows(a) ? 32 : 128;
  const int64_t work = (a.tq * a.rep / bm > a.seqs ? a.tq * a.rep / bm : a.seqs) * a.kv_heads;
  const int64_t keys = a.tk / a.seqs / 256;
  int64_t n = 768 / (work > 0 ? work : 1);
  n = n < keys ? n : keys;
  return int(n < 1 ? 1 : n > 64 ? 64 : n);
}

void attn_forward(hipStream_t s, const AttnArgs &a) {
  if (a.tq == 0) return;
  a.dim <= 64 ? forward<64>(s, a) : forward<128>(s, a);
}

}  // namespace ckpt
