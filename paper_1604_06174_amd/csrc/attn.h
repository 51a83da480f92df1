// What the attention kernels share: packed sequences, tiles in LDS, matrix operands.
//
// All products run on v_mfma_f32_32x32x16_bf16: D[m][n] += sum over k of A[m][k] B[k][n],
// m, n < 32, k < 16.  Lane l holds A[l % 32][8 (l / 32) + e] and B[8 (l / 32) + e][l % 32]
// for e < 8, and of D the rows 8 (i / 4) + 4 (l / 32) + i % 4, i < 16, of column l % 32.
//
// A product's rows m are those of the tile that comes by in LDS and its columns n those that the
// wavefront keeps in registers, so a lane has one kept row (a query in the forward and
// dq, a key in dk and dv) and softmax's sums, masks and scales of it are the lane's own.
// Probabilities then are D of one product and, without leaving their lanes, B of the
// next: its k runs over the tile's rows in the order in which D holds them, k = 8 h + e being row
// 8 (e / 4) + 4 h + e % 4 of sixteen, and A (values by rows of the tile, so transposed) is
// read from LDS in that order by gfx950's transposing read.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "lanes.h"
#include "seq.h"

namespace ckpt {
namespace at {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef short short8v __attribute__((ext_vector_type(8)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) short4v lds_short4;

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;

static __device__ __align__(16) const unsigned g_zeros[1024] = {};

__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// the tile's loads of this wavefront have landed and its LDS reads returned; then every
// wavefront's have
__device__ __forceinline__ void tile_barrier() {
  __builtin_amdgcn_s_waitcnt(0x70);  // vmcnt 0, lgkmcnt 0
  __syncthreads();
}

// ---- sequences -------------------------------------------------------------
struct Sequence {
  int64_t q0, k0;  // first rows
  int lq, lk;
  int64_t first;   // first row of the tile, within the sequence
};

__device__ __forceinline__ int64_t clamp_row(int64_t v, int64_t lo, int64_t hi) { return v < lo ? lo : v > hi ? hi : v; }

__device__ __forceinline__ void rows_of(const AttnArgs &A, int s, Sequence &q) {
  q.q0 = clamp_row(A.qoff[s], 0, A.tq);
  q.lq = int(clamp_row(A.qoff[s + 1], q.q0, A.tq) - q.q0);
  q.k0 = clamp_row(A.koff[s], 0, A.tk);
  q.lk = int(clamp_row(A.koff[s + 1], q.k0, A.tk) - q.k0);
}

// sum over the wavefront's lanes
__device__ __forceinline__ int wave_add(int v) {
  v += __float_as_int(lane_xor<1>(__int_as_float(v)));
  v += __float_as_int(lane_xor<2>(__int_as_float(v)));
  v += __float_as_int(lane_xor<4>(__int_as_float(v)));
  v += __float_as_int(lane_xor<8>(__int_as_float(v)));
  float a = __int_as_float(v), b = a;
  swap_rows<16>(a, b);
  v = __float_as_int(a) + __float_as_int(b);
  a = b = __int_as_float(v);
  swap_rows<32>(a, b);
  return __builtin_amdgcn_readfirstlane(__float_as_int(a) + __float_as_int(b));
}

// The `index`-th tile of `size` rows, `per` rows to each token of the queries (QUERIES) or of the keys.
// false: there is none.
//
// Up to 64 sequences, a lane each, are ordered by their tiles' work, longest first: a causal tile's
// is its place in its sequence (of queries with the keys before them, of keys with the queries
// behind them), so the tiles of a level w or above are counted, sum over the sequences of how far they
// reach past w, and the level is searched for.  Then no long tile is left to the end.  A launch has
// workgroups for one more tile a sequence than its rows may fill; those without a tile come last.
// More sequences take the tiles from off[s] per / size + s on each: as many as its rows can take
// whatever their number, so a tile's sequence is found without adding lengths up.  Tiles then come in
// their sequences' order, those that rows do not fill among them.
template <bool QUERIES>
__device__ __forceinline__ bool find_tile(const AttnArgs &A, int per, int size, int tiles, int index, Sequence &q) {
  const int lane = threadIdx.x & 63;
  if (A.seqs <= 64) {
    Sequence mine{0, 0, 0, 0, 0};
    if (lane < A.seqs) rows_of(A, lane, mine);
    const int n = int((int64_t(QUERIES ? mine.lq : mine.lk) * per + size - 1) / size);
    // (it orders and no more: so long a past that 32 bits do not hold its tiles counts as a shorter one)
    const int low = QUERIES && A.causal ? int(min(int64_t(max(0, mine.lk - mine.lq)) * per / size, int64_t(1) << 29)) : 0;
    const bool single = !__any(n > 1);  // then a level's tiles are counted without adding up
    auto above = [&](int w) {
      return single ? int(__popcll(__ballot(n > 0 && low >= w))) : wave_add(max(0, min(n, low + n - w)));
    };
    const int total = above(0);
    if (index >= total) return false;
    int lo = 0, hi = 1;
    while (above(hi) > index) lo = hi, hi *= 2;
    while (hi - lo > 1) {
      const int mid = lo + (hi - lo) / 2;
      if (above(mid) > index) lo = mid;
      else hi = mid;
    }
    // the sequences with a tile at this level, in order
    const int rank = index - above(lo + 1);
    const bool has = lo >= low && lo < low + n;
    const uint64_t all = __ballot(has);
    const int who = __ffsll((unsigned long long)__ballot(has && __popcll(all & ((1ull << lane) - 1)) == rank)) - 1;
    auto of = [&](int v) { return __builtin_amdgcn_readlane(v, who); };
    q = Sequence{of(int(mine.q0)), of(int(mine.k0)), of(mine.lq), of(mine.lk), 0};  // rows fit 32 bits
    const int t = lo - __builtin_amdgcn_readlane(low, who);
    q.first = int64_t(QUERIES ? t : __builtin_amdgcn_readlane(n, who) - 1 - t) * size;
    return true;
  }
  const int *const off = QUERIES ? A.qoff : A.koff;
  const int tile = QUERIES ? tiles - 1 - index : index;  // later queries see more, earlier keys are seen more
  int lo = 0, n = A.seqs;
  while (true) {  // 64 sequences at a time, then 64 ranges of them ...
    const int step = (n + 63) / 64, s = lo + lane * step;
    const bool ok = lane * step < n && int64_t(off[s]) * per / size + s <= tile;
    const int c = __popcll(__ballot(ok));
    if (c == 0) return false;
    lo += (c - 1) * step;
    n = min(step, n - (c - 1) * step);
    if (step == 1) break;
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  rows_of(A, lo, q);
  q.first = (tile - (int64_t(off[lo]) * per / size + lo)) * size;
  return q.first >= 0 && q.first < int64_t(QUERIES ? q.lq : q.lk) * per;
}

// ---- tiles in LDS ----------------------------------------------------------
// Rows of D values without padding, their 16-byte chunks in an order of the row's own, so that
// neither 32 rows' equal chunks (A by rows) nor four rows' runs of chunks (A transposed)
// fall on the same banks.
template <int D>
__device__ __forceinline__ int swizzle(int row) {
  return D == 128 ? ((row & 3) << 2) | ((row >> 2) & 3) : (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
}

// The loader of a tile of ROWS rows, `ld` elements apart, straight into LDS: zeros for rows
// from `valid` on and columns from `dim` on.  A thread loads the same columns of each of its
// rows, whose order of chunks is the same (they are sixteen rows apart, or 32).  Whole tiles take
// addresses of a scalar and the lane's own 32 bits, so they cost the vector unit nothing.
template <int D, int ROWS, int THREADS>
struct Loader {
  static constexpr int C = D / 8, STEP = THREADS / C, N = ROWS / STEP;
  static_assert(STEP % 16 == 0 && ROWS % STEP == 0, "rows with the same order of chunks");
  const char *src;  // row 0
  int64_t pitch;    // bytes from row to row
  unsigned place;   // the lane's first chunk from the tile's first row, in bytes
  int dim;
  bool whole;       // all columns are below dim, and 32 bits hold the places

  __device__ __forceinline__ Loader(const __bf16 *base, int64_t ld, int dim_)
      : src(reinterpret_cast<const char *>(base)), pitch(2 * ld), dim(dim_) {
    const int row = threadIdx.x / C, col = ((threadIdx.x % C) ^ swizzle<D>(row)) * 8;
    place = unsigned(row) * unsigned(pitch) + 2 * col;
    whole = dim == D && pitch < (1 << 24);
  }
  // the tile from row `first` on, `offset` bytes further
  __device__ __forceinline__ void load(unsigned char *lds, int64_t first, int valid, int64_t offset = 0) const {
    const char *const p = src + first * pitch + offset;
    unsigned char *const to = lds + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 1024;
    if (whole && valid >= ROWS) {
#pragma unroll
      for (int c = 0; c < N; ++c) {
        const char *q = p + c * STEP * pitch;
        asm("" : "+s"(q));  // the scalar sum first
        __builtin_amdgcn_global_load_lds(q + place, (lds_void *)(to + c * THREADS * 16), 16, 0, 0);
      }
    } else {
      int tid = threadIdx.x;
      asm volatile("" : "+v"(tid));  // what follows is rare: it is worked out here, not kept in registers
      const int row = tid / C, col = ((tid % C) ^ swizzle<D>(row)) * 8;
#pragma unroll
      for (int c = 0; c < N; ++c) {
        const bool ok = col < dim && row + c * STEP < valid;
        const void *const q = ok ? static_cast<const void *>(p + (row + c * STEP) * pitch + 2 * col)
                                 : g_zeros + 4 * (tid & 255);
        __builtin_amdgcn_global_load_lds(q, (lds_void *)(to + c * THREADS * 16), 16, 0, 0);
      }
    }
  }
};

// a lane's places in a tile: of its row's chunks, and of the transposing reads
template <int D>
struct Places {
  int row;     // byte offset of chunk lane / 32 of row lane % 32; chunk 2 kk further on: ^ kk << 5
  int lo, hi;  // of the transposing reads of columns 0 .. 31; 32 b columns further on: ^ b << 6

  __device__ __forceinline__ explicit Places(int columns = 0) {  // (a power of two, or 0) times 32 columns further on
    const int lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5;
    row = r * D * 2 + ((swizzle<D>(r) ^ h) << 4);
    const int chunk = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1), r0 = 4 * h + ((lane >> 2) & 3), r1 = r0 + 8;
    lo = r0 * D * 2 + ((chunk ^ swizzle<D>(r0)) << 4) + (lane & 1) * 8;
    hi = r1 * D * 2 + ((chunk ^ swizzle<D>(r1)) << 4) + (lane & 1) * 8;
    lo ^= columns << 6;
    hi ^= columns << 6;
  }
  // A copy that the compiler takes for new values.  A tile's address in LDS is then an offset
  // within the reads; otherwise its sum with every place is formed before the loop, and
  // four tiles' sums take the registers of an accumulator.
  __device__ __forceinline__ Places here() const {
    Places p = *this;
    asm volatile("" : "+v"(p.row), "+v"(p.lo), "+v"(p.hi));
    return p;
  }

  // A by rows: columns 16 kk .. 16 kk + 15 of the 32 rows from `first` (a multiple of 32) on
  __device__ __forceinline__ bf16x8 rows(const unsigned char *tile, int first, int kk) const {
    return *reinterpret_cast<const bf16x8 *>(tile + first * D * 2 + (row ^ (kk << 5)));
  }
  // A transposed: m = columns 32 b .. 32 b + 31, k = the 16 rows from `first` (a multiple of 16) on
  __device__ __forceinline__ bf16x8 columns(const unsigned char *tile, int first, int b) const {
    const short4v x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4 *)(tile + first * D * 2 + (lo ^ (b << 6))));
    const short4v y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4 *)(tile + first * D * 2 + (hi ^ (b << 6))));
    const short8v v = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
    return __builtin_bit_cast(bf16x8, v);
  }
};

// eight values of a kept row from column 16 kk + 8 (lane / 32) on, zeros from dim on
__device__ __forceinline__ bf16x8 kept(const __bf16 *row, int kk, int dim) {
  const int col = 16 * kk + 8 * ((threadIdx.x & 63) >> 5);
  u32x4 v = {0u, 0u, 0u, 0u};
  if (col < dim) v = *reinterpret_cast<const u32x4 *>(row + col);
  return __builtin_bit_cast(bf16x8, v);
}

// B of a product over sixteen rows of a tile: eight of a D's sixteen values, rounded
__device__ __forceinline__ bf16x8 operand(const f32x16 &d, int half) {
  bf16x8 r;
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = (__bf16)d[8 * half + e];
  return r;
}

// use(i, load(i)) for i < N, each load AHEAD uses before its own and none earlier: left to itself
// the compiler starts all of them first, and the registers they land in push accumulators
// out to memory
template <int N, int AHEAD, typename L, typename U>
__device__ __forceinline__ void in_turn(L &&load, U &&use) {
  decltype(load(0)) f[N];
#pragma unroll
  for (int i = 0; i < AHEAD && i < N; ++i) f[i] = load(i);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (i + AHEAD < N) f[i + AHEAD] = load(i + AHEAD);
    use(i, f[i]);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// Magnitudes above the largest finite one in a tile as that one (as pairs of 16 bits without the
// sign, infinities and NaNs are the larger numbers); `special` is set if there were any.  A product
// with a tile of which a row does not see all takes zeros for what is hidden, and an infinity or a NaN would
// make a NaN of them; add_special then gives them to the rows that see them.  All of the workgroup, between
// barriers.
template <int BYTES>
__device__ __forceinline__ void scrub(unsigned char *tile, int &special) {
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  const u16x2 most = {0x7f7f, 0x7f7f};
#pragma unroll
  for (int c = 0; c < BYTES / 4096; ++c) {
    u32x4 *const at = reinterpret_cast<u32x4 *>(tile) + c * 256 + threadIdx.x;
    u32x4 w = *at;
    unsigned changed = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const u16x2 m = __builtin_bit_cast(u16x2, w[k] & 0x7fff7fffu);
      const unsigned f = __builtin_bit_cast(unsigned, __builtin_elementwise_min(m, most)) | (w[k] & 0x80008000u);
      changed |= f ^ w[k];
      w[k] = f;
    }
    if (changed) {
      *at = w;
      special = 1;
    }
  }
}

// acc += (values of the 16 rows of the tile from `first` on, transposed) b
template <int D, int N>
__device__ __forceinline__ void add_rows(f32x16 (&acc)[N], const Places<D> &at, const unsigned char *tile, int first,
                                         bf16x8 b) {
#pragma unroll
  for (int t = 0; t < N; ++t) acc[t] = mfma(at.columns(tile, first, t), b, acc[t]);
}

// What scrub took out of rows row0 .. row1 - 1 of a matrix whose row r is at src + r ld; sees(r): does
// the lane's row see it?  A probability times an infinity or a NaN is that
// infinity or NaN (it is positive, however small); a score's gradient times one is a NaN, for
// the score itself is then infinite or NaN (nan = true).
template <int N, typename F>
__device__ __forceinline__ void add_special(f32x16 (&acc)[N], const __bf16 *src, int64_t ld, int dim, int row0, int row1,
                                            bool nan, F &&sees) {
  for (int r = row0; r < row1; ++r) {
    if (!sees(r)) continue;
#pragma unroll
    for (int t = 0; t < N; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int col = 32 * t + 8 * (i / 4) + 4 * ((threadIdx.x & 63) >> 5) + i % 4;
        const float v = col < dim ? float(src[r * ld + col]) : 0.f;
        if (!(fabsf(v) < INFINITY)) acc[t][i] += nan ? NAN : v;
      }
  }
}

// row of D value i of 32: 8 (i / 4) + 4 (lane / 32) + i % 4
__device__ __forceinline__ int d_row(int i) { return 8 * (i / 4) + 4 * ((threadIdx.x & 63) >> 5) + i % 4; }

// Tiles [0, n) through two places in LDS, as step(tile, place, masked) with place and masked constants:
// the first `n1` without tests of every score, the others with.  Each kind's steps are a loop
// of their own without branches around them, which keeps the accumulators in their registers;
// the kind with tests serves any tile, so it takes an odd one too.
template <typename F>
__device__ __forceinline__ void two_kinds(int n, int n1, F &&step) {
  using std::integral_constant;
  constexpr integral_constant<int, 0> p0{};
  constexpr integral_constant<int, 1> p1{};
  int it = 0;
  for (; it + 1 < n1; it += 2) {
    step(it, p0, std::false_type());
    step(it + 1, p1, std::false_type());
  }
  for (; it < n; it += 2) {
    step(it, p0, std::true_type());
    if (it + 1 < n) step(it + 1, p1, std::true_type());
  }
}

// columns 32 t .. 32 t + 31 of a lane's row from an accumulator, scaled
__device__ __forceinline__ void store_tile(__bf16 *row, const f32x16 &acc, int t, float scale, int dim) {
  typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
#pragma unroll
  for (int b = 0; b < 4; ++b) {
    const int col = 32 * t + 8 * b + 4 * ((threadIdx.x & 63) >> 5);
    if (col >= dim) continue;
    bf16x4 v;
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = (__bf16)(acc[4 * b + k] * scale);
    *reinterpret_cast<bf16x4 *>(row + col) = v;
  }
}

__device__ __forceinline__ void store_tile(float *row, const f32x16 &acc, int t, float scale, int dim) {
#pragma unroll
  for (int b = 0; b < 4; ++b) {
    const int col = 32 * t + 8 * b + 4 * ((threadIdx.x & 63) >> 5);
    if (col < dim)
      *reinterpret_cast<float4 *>(row + col) =
          make_float4(acc[4 * b] * scale, acc[4 * b + 1] * scale, acc[4 * b + 2] * scale, acc[4 * b + 3] * scale);
  }
}

template <typename T, int N>
__device__ __forceinline__ void store_row(T *row, const f32x16 (&acc)[N], float scale, int dim) {
#pragma unroll
  for (int t = 0; t < N; ++t) store_tile(row, acc[t], t, scale, dim);
}

template <int N>
__device__ __forceinline__ void clear(f32x16 (&acc)[N]) {
#pragma unroll
  for (int t = 0; t < N; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[t][i] = 0.f;
}

// with the value of the other half's lane
__device__ __forceinline__ float halves_max(float v) {
  float a = v, b = v;
  swap_rows<32>(a, b);
  return fmaxf(a, b);
}
__device__ __forceinline__ float halves_add(float v) { return xor_add<32>(v); }

}  // namespace at
}  // namespace ckpt
