// Embedding: rows of a table looked up by id and scaled; the table's gradient, each id's
// rows added up in the order of its tokens.
//
// The gradient takes three launches.
//   k_embed_sort  orders the tokens by id, each id's in their order.  A workgroup
//     takes a range of ids, reads all ids (from L2: they are few against the rows),
//     counts those of its range for each of sixteen sections of the tokens, one a
//     wavefront, lists them, and places them.  The first position of a range is the number of
//     smaller ids, which the workgroup counts as it goes, so workgroups need nothing of
//     each other.
//   k_embed_sum   a wavefront takes a chunk of sorted positions, 512 columns, and adds up
//     the ids that begin in it, up to their ends.  An id with more tokens than a chunk is taken in
//     pieces of a chunk's length from its first on, each by the wavefront in whose chunk the
//     piece begins, which leaves its sum.  The first workgroups write the rows of absent ids:
//     their stores go out while the others look up what they have to add.
//   k_embed_join  adds the pieces of such an id, in order.
// Nothing is added by atomics (the counts are whole numbers), so the same bits come
// out on every run.
//
// Lookups are bound by HBM (32768 rows of 1024 columns, 16 bits: 22 us, 67 MB written and the table's
// 65 read, 6.1 TB/s with what the caches hold of it).  The gradient of 65536 unevenly distributed tokens, 50000
// ids, 1024 columns of 16 bits into 32: sort 18 us, bound by its most frequent range (with a loop over the ids in
// place of the vote on their bits 34), sum 84 (346 MB at 4.1 TB/s, rows in no order), join 12, latency.  The
// zeros written by the sort's workgroups: sum 62, but sort 17 more and few tokens slower as well.
#include "common.h"
#include "seq.h"
#include "vec.h"

#include <type_traits>

namespace ckpt {
namespace {

constexpr int SECTIONS = 16;    // wavefronts of a sorting workgroup
constexpr int LIST = 512;       // tokens of a section that are kept from the first reading
// ids that a wavefront writes zeros for (16384 tokens of 32000 ids, 2048 columns: 98 us, with 64 128)
constexpr int ABSENT = 16;
constexpr int MAX_RANGE = 1024; // ids of one: [SECTIONS][MAX_RANGE] counts take 64 KB of LDS

template <typename T>
__device__ __forceinline__ void load8(const T *p, int cnt, float v[8]) {
  if (cnt >= 8) {
    const Vec<T, 8> r = load_vec<T, 8>(p);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = float(r.v[k]);
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

// id i, or -1 outside the vocabulary
__device__ __forceinline__ int id_at(const EmbedArgs &A, int64_t i) {
  const int64_t id = A.ids64 ? static_cast<const int64_t *>(A.ids)[i] : static_cast<const int *>(A.ids)[i];
  return id >= 0 && id < A.vocab ? int(id) : -1;
}

// a thread takes a vector of eight columns of four rows, a quarter of the tokens apart
template <typename WT, typename YT>
__global__ __launch_bounds__(256) void k_embed_forward(EmbedArgs A, int nvec, int64_t quarter) {
  const int64_t i = blockIdx.x * int64_t(256) + threadIdx.x;
  const int64_t row = i >> 32 ? i / nvec : int64_t(uint32_t(i) / uint32_t(nvec));
  if (row >= quarter) return;
  const int col = int(i - row * nvec) * 8, cnt = min(8, A.c - col);
  int id[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) id[u] = row + u * quarter < A.tokens ? id_at(A, row + u * quarter) : -1;
  float v[4][8];
#pragma unroll
  for (int u = 0; u < 4; ++u) {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[u][k] = 0.f;
    if (id[u] >= 0) load8(static_cast<const WT *>(A.src) + int64_t(id[u]) * A.lds + col, cnt, v[u]);
  }
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    if (row + u * quarter >= A.tokens) continue;
    if (id[u] >= 0) {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[u][k] *= A.scale;
    }
    store8(static_cast<YT *>(A.dst) + (row + u * quarter) * A.ldd + col, cnt, v[u]);
  }
}

// four ids from token i on as 32 bits: -1 for those past the end and for wide ones that 32 bits
// do not hold (as unsigned numbers all of these lie above every vocabulary)
template <bool WIDE>
__device__ __forceinline__ void four_ids(const EmbedArgs &A, int64_t i, int64_t last, int id[4]) {
  typedef typename std::conditional<WIDE, int64_t, int>::type I;
  typedef I four __attribute__((ext_vector_type(4), aligned(sizeof(I))));
  const I *const p = static_cast<const I *>(A.ids) + i;
  four v = {-1, -1, -1, -1};
  if (i + 4 <= last) {
    v = *reinterpret_cast<const four *>(p);
  } else {
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (i + u < last) v[u] = p[u];
  }
#pragma unroll
  for (int u = 0; u < 4; ++u) id[u] = WIDE && (int64_t(v[u]) >> 31) ? -1 : int(v[u]);
}

// f(first token of 256, the lane's four ids) over tokens [first, last): 1024 tokens' ids are in
// flight at once
template <bool WIDE, typename F>
__device__ __forceinline__ void each_ids(const EmbedArgs &A, int64_t first, int64_t last, F &&f) {
  const int lane = threadIdx.x & 63;
  for (int64_t i = first; i < last; i += 1024) {
    int id[4][4];
#pragma unroll
    for (int g = 0; g < 4; ++g) four_ids<WIDE>(A, i + g * 256 + lane * 4, last, id[g]);
#pragma unroll
    for (int g = 0; g < 4; ++g) f(i + g * 256, id[g]);
  }
}

template <bool WIDE>
__global__ __launch_bounds__(64 * SECTIONS) void k_embed_sort(EmbedArgs A, int range) {
  __shared__ int cnt[SECTIONS * MAX_RANGE];  // [section][id of the range]
  __shared__ int wsum[SECTIONS];
  __shared__ unsigned lists[SECTIONS][LIST];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lo = int(min(int64_t(blockIdx.x) * range, A.vocab));
  const int n = int(min(int64_t(range), A.vocab - lo));
  const int64_t per = ((A.tokens + SECTIONS - 1) / SECTIONS + 255) / 256 * 256;
  const int64_t first = min(wave * per, A.tokens), last = min(first + per, A.tokens);
  for (int i = threadIdx.x; i < SECTIONS * range; i += 64 * SECTIONS) cnt[i] = 0;
  __syncthreads();

  // the range's tokens go to the wavefront's list as they are met, in order
  unsigned *const list = lists[wave];
  int less = 0, listed = 0;
  each_ids<WIDE>(A, first, last, [&](int64_t i, const int (&id)[4]) {
    bool in[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      less += unsigned(id[u]) < unsigned(lo);
      in[u] = unsigned(id[u]) - unsigned(lo) < unsigned(n);
    }
    if (!__any(in[0] | in[1] | in[2] | in[3])) return;
    uint64_t m[4];
    int at = listed;  // of the lane's first
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      m[u] = __ballot(in[u]);
      at += __popcll(m[u] & ((1ull << lane) - 1));
      listed += __popcll(m[u]);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (in[u]) {
        atomicAdd(&cnt[wave * range + id[u] - lo], 1);
        if (at < LIST) list[at] = unsigned(i - first + lane * 4 + u) | unsigned(id[u] - lo) << 22;
        ++at;
      }
  });
#pragma unroll
  for (int o = 32; o; o >>= 1) less += __shfl_xor(less, o);
  if (lane == 0) wsum[wave] = less;
  __syncthreads();
  int base = 0;
#pragma unroll
  for (int k = 0; k < SECTIONS; ++k) base += wsum[k];
  __syncthreads();  // wsum is written again below

  // cnt becomes the first position of each section's tokens of an id: an exclusive sum over
  // the ids, then over the sections; a thread has one id
  static_assert(MAX_RANGE <= 64 * SECTIONS, "an id a thread");
  const int i0 = threadIdx.x;
  int mine = 0;
  if (i0 < n) {
#pragma unroll
    for (int k = 0; k < SECTIONS; ++k) mine += cnt[k * range + i0];
  }
  int incl = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int t = __shfl_up(incl, o);
    if (lane >= o) incl += t;
  }
  if (lane == 63) wsum[wave] = incl;
  __syncthreads();
  int pos = base + incl - mine;
  for (int k = 0; k < wave; ++k) pos += wsum[k];
  if (i0 < n) {
    A.start[lo + i0] = pos;
#pragma unroll
    for (int k = 0; k < SECTIONS; ++k) {
      const int t = cnt[k * range + i0];
      cnt[k * range + i0] = pos;
      pos += t;
    }
  }
  // the last range's end is the end of all
  if (lo + n == A.vocab && n > 0 && threadIdx.x == 0) {
    int total = base;
    for (int k = 0; k < SECTIONS; ++k) total += wsum[k];
    A.start[A.vocab] = total;
  }
  __syncthreads();

  // 64 tokens in order, a lane each: their places are those of the id's tokens so far and of the lower
  // lanes with the same id, found by a vote on each bit of the ids
  const int bits = 32 - __clz(range - 1);
  auto put = [&](bool in, int id, int token) __attribute__((always_inline)) {
    uint64_t same = __ballot(in);
    if (!same) return;
    for (int k = 0; k < bits; ++k) {
      const bool one = id >> k & 1;
      const uint64_t ones = __ballot(one);
      same &= one ? ones : ~ones;
    }
    if (!in) return;
    // one wavefront's: its accesses are in order, and volatile keeps them in the code's
    volatile int *const at = &cnt[wave * range + id];
    const int p = *at + __popcll(same & ((1ull << lane) - 1));
    A.perm[p] = token;
    A.key[p] = lo + id;
    if (same >> lane == 1) *at = p + 1;  // the last of them
  };
  if (listed <= LIST && per <= (1 << 22)) {
    for (int i = 0; i < listed; i += 64) {
      const bool in = i + lane < listed;
      const unsigned entry = in ? list[i + lane] : 0u;
      put(in, int(entry >> 22), int(first) + int(entry & ((1u << 22) - 1)));
    }
    return;
  }
  // a longer list, or a section that 22 bits do not number, is read again
  for (int64_t i = first; i < last; i += 1024) {
    int id[16];
#pragma unroll
    for (int g = 0; g < 16; ++g) id[g] = i + g * 64 + lane < last ? id_at(A, i + g * 64 + lane) : -1;
#pragma unroll
    for (int g = 0; g < 16; ++g)
      put(unsigned(id[g]) - unsigned(lo) < unsigned(n), id[g] - lo, int(i) + g * 64 + lane);
  }
}

// row `v` of the gradient = the sum, or the sum added to it
template <typename DT>
__device__ __forceinline__ void put_row(const EmbedArgs &A, int v, int col, int cnt, float s[8]) {
  DT *const p = static_cast<DT *>(A.dst) + int64_t(v) * A.ldd + col;
#pragma unroll
  for (int k = 0; k < 8; ++k) s[k] *= A.scale;
  if (A.accumulate) {
    float old[8];
    load8(p, cnt, old);
#pragma unroll
    for (int k = 0; k < 8; ++k) s[k] += old[k];
  }
  store8(p, cnt, s);
}

template <typename GT, typename DT>
__global__ __launch_bounds__(256) void k_embed_sum(EmbedArgs A, int tiles, int zeros) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (int(blockIdx.x) < zeros) {
    const float zero[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int64_t v0 = (blockIdx.x * int64_t(4) + wave) * ABSENT; v0 < A.vocab; v0 += int64_t(zeros) * 4 * ABSENT) {
      const int64_t v = v0 + lane;
      for (uint64_t absent = __ballot(lane < ABSENT && v < A.vocab && A.start[v] == A.start[v + 1]); absent;
           absent &= absent - 1) {
        DT *const row = static_cast<DT *>(A.dst) + (v0 + __ffsll((unsigned long long)absent) - 1) * A.ldd;
        for (int col = lane * 8; col < A.c; col += 512) store8(row + col, min(8, A.c - col), zero);
      }
    }
    return;
  }
  const int64_t unit = (blockIdx.x - zeros) * int64_t(4) + wave;
  const int64_t chunk = unit / tiles;
  if (chunk >= A.chunks) return;
  const int col = int(unit - chunk * tiles) * 512 + lane * 8, cnt = min(8, A.c - col);
  // all positions that may have to be added up here (what lies past the last, `total`, is not looked at)
  const int total = A.start[A.vocab], P = A.chunk;
  int tok[2] = {0, 0}, key[2] = {0, 0};
#pragma unroll
  for (int u = 0; u < 2; ++u)
    if (const int64_t at = chunk * P + u * 64 + lane; at < A.tokens) {
      tok[u] = A.perm[at];
      key[u] = A.key[at];
    }
  const int p0 = int(min(chunk * P, int64_t(total))), p1 = min(p0 + P, total);
  if (p0 == p1) {
    if (lane == 0) A.tail[chunk] = -1;
    return;
  }
  auto token_at = [&](int q) { return q < 64 ? __builtin_amdgcn_readlane(tok[0], q) : __builtin_amdgcn_readlane(tok[1], q - 64); };
  auto key_at = [&](int q) { return q < 64 ? __builtin_amdgcn_readlane(key[0], q) : __builtin_amdgcn_readlane(key[1], q - 64); };
  const int k0 = key_at(0), k1 = key_at(p1 - p0 - 1);
  const int begin0 = A.start[k0], end0 = A.start[k0 + 1], begin1 = A.start[k1], end1 = A.start[k1 + 1];
  const bool long0 = end0 - begin0 > P, long1 = end1 - begin1 > P;
  // the first id or piece that begins in the chunk, and the end of the last
  int from = p0;
  if (begin0 < p0) {
    const int piece = begin0 + (p0 - begin0 + P - 1) / P * P;
    from = min(p1, long0 && piece < end0 ? piece : end0);
  }
  const int last = long1 ? begin1 + (p1 - 1 - begin1) / P * P : begin1;
  const int to = last < p0 ? from : long1 ? min(end1, last + P) : end1;
  const bool piece0 = long0 && from < min(end0, p1);  // the first is a piece,
  const bool piece1 = long1 && k1 != k0;              // or the last
  const int slot0 = from == begin0;                   // an id's first piece has a place of its own
  if (lane == 0) A.tail[chunk] = piece0 && slot0 ? k0 : piece1 ? k1 : -1;
  if (from == to) return;
  const int q0 = from - p0, q1 = to - p0;  // at most two chunks' length, less one
  float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  bool head = piece0;
  typedef Vec<GT, 8> Raw;
  auto fetch = [&](int q, Raw (&v)[8]) {
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int64_t row = token_at(min(q + u, q1 - 1));
      const GT *const p = static_cast<const GT *>(A.src) + row * A.lds + col;
      if (cnt >= 8 || (cnt > 0 && row + 1 < A.tokens && A.c >= 8)) {  // past an odd row's end lies the next row
        v[u] = load_vec<GT, 8>(p);
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[u].v[k] = k < cnt ? p[k] : (GT)0.f;
      }
    }
  };
  auto add = [&](int q, const Raw (&v)[8]) {
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if (q + u >= q1) break;
      const int id = key_at(q + u);
#pragma unroll
      for (int k = 0; k < 8; ++k) s[k] += float(v[u].v[k]);
      const bool end = q + u + 1 == q1;
      if (end || key_at(q + u + 1) != id) {
        if (cnt > 0) {
          if (head || (end && piece1))
            store8(A.part + (2 * chunk + (head ? slot0 : 1)) * A.cpad + col, cnt, s);
          else
            put_row<DT>(A, id, col, cnt, s);
        }
        head = false;
#pragma unroll
        for (int k = 0; k < 8; ++k) s[k] = 0.f;
      }
    }
  };
  // eight rows are added while the next eight load
  Raw r0[8], r1[8];
  fetch(q0, r0);
  for (int q = q0; q < q1; q += 16) {
    if (q + 8 < q1) fetch(q + 8, r1);
    add(q, r0);
    if (q + 16 < q1) fetch(q + 16, r0);
    if (q + 8 < q1) add(q + 8, r1);
  }
}

// The ids in pieces: a wavefront looks at a chunk, 512 columns, and adds up the pieces of the id that
// began there if they are few.  Many are dealt to the workgroup's eight wavefronts in runs, whose
// sums are then added in order.  Piece i begins in the i-th chunk after the id's first.
constexpr int JOIN = 8, FEW = 16;

template <typename DT>
__global__ __launch_bounds__(64 * JOIN) void k_embed_join(EmbedArgs A) {
  __shared__ float red[JOIN][8][64];
  __shared__ int ids[JOIN], pieces[JOIN];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = blockIdx.y * 512 + lane * 8, cnt = min(8, A.c - col);
  auto sum = [&](int64_t chunk, int a, int b, float (&s)[8]) {
    if (cnt <= 0) return;
#pragma unroll 8
    for (int i = a; i < b; ++i) {
      float v[8];
      load8(A.part + (2 * (chunk + i) + (i ? 0 : 1)) * A.cpad + col, cnt, v);
#pragma unroll
      for (int k = 0; k < 8; ++k) s[k] += v[k];
    }
  };
  const int64_t mine = blockIdx.x * int64_t(JOIN) + wave;
  const int key = mine < A.chunks ? A.tail[mine] : -1;
  int n = 0;
  if (key >= 0) {
    n = (A.start[key + 1] - A.start[key] + A.chunk - 1) / A.chunk;
    if (n <= FEW) {
      float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      sum(mine, 0, n, s);
      if (cnt > 0) put_row<DT>(A, key, col, cnt, s);
      n = 0;
    }
  }
  if (lane == 0) {
    ids[wave] = key;
    pieces[wave] = n;
  }
  __syncthreads();
  for (int w = 0; w < JOIN; ++w) {
    const int m = pieces[w];
    if (!m) continue;
    const int per = (m + JOIN - 1) / JOIN, a = min(wave * per, m), b = min(a + per, m);
    float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    sum(blockIdx.x * int64_t(JOIN) + w, a, b, s);
#pragma unroll
    for (int k = 0; k < 8; ++k) red[wave][k][lane] = s[k];
    __syncthreads();
    if (wave == 0 && cnt > 0) {
      const int waves = (m + per - 1) / per;
      for (int q = 1; q < waves; ++q)
#pragma unroll
        for (int k = 0; k < 8; ++k) s[k] += red[q][k][lane];
      put_row<DT>(A, ids[w], col, cnt, s);
    }
    __syncthreads();
  }
}

template <typename WT, typename YT>
void forward(hipStream_t s, const EmbedArgs &a) {
  const int nvec = (a.c + 7) / 8;
  const int64_t quarter = (a.tokens + 3) / 4;
  hipLaunchKernelGGL((k_embed_forward<WT, YT>), dim3(uint32_t((quarter * nvec + 255) / 256)), dim3(256), 0, s, a, nvec,
                     quarter);
}

template <typename GT, typename DT>
void backward(hipStream_t s, const EmbedArgs &a) {
  // a range for each compute unit, as far as the counts fit
  const int64_t even = (a.vocab + 255) / 256;
  const int range = int(even < MAX_RANGE ? even : MAX_RANGE);
  const dim3 ranges(uint32_t((a.vocab + range - 1) / range));
  if (a.ids64)
    hipLaunchKernelGGL(k_embed_sort<true>, ranges, dim3(64 * SECTIONS), 0, s, a, range);
  else
    hipLaunchKernelGGL(k_embed_sort<false>, ranges, dim3(64 * SECTIONS), 0, s, a, range);
  const int64_t need = (a.vocab + 4 * ABSENT - 1) / (4 * ABSENT);
  const int tiles = (a.c + 511) / 512, zeros = a.accumulate ? 0 : int(need < 65536 ? need : 65536);
  hipLaunchKernelGGL((k_embed_sum<GT, DT>), dim3(uint32_t(zeros + (int64_t(a.chunks) * tiles + 3) / 4)), dim3(256), 0, s,
                     a, tiles, zeros);
  if (a.tokens > a.chunk)
    hipLaunchKernelGGL(k_embed_join<DT>, dim3(uint32_t((a.chunks + JOIN - 1) / JOIN), uint32_t(tiles)), dim3(64 * JOIN),
                       0, s, a);
}

uint64_t align16(uint64_t v) { return (v + 15) & ~uint64_t(15); }

}  // namespace

void embed_forward(hipStream_t s, const EmbedArgs &a, int wtype, int ytype) {
  const bool yf = ytype == SEQ_F32;
  if (wtype == SEQ_F32)
    yf ? forward<float, float>(s, a) : forward<float, __bf16>(s, a);
  else
    yf ? forward<__bf16, float>(s, a) : forward<__bf16, __bf16>(s, a);
}

uint64_t embed_plan(EmbedArgs &a, char *ws) {
  // positions a wavefront begins with: 16 wavefronts for each compute unit, if there are as many (65536 tokens,
  // 1024 columns: 32 positions 117 us, 16 119, 64 120), but 16 at least, so that up to 16 tokens of an id are
  // one running sum (4099 tokens of 97 ids, 333 columns: 27 us, with 8 positions 23)
  const int64_t tiles = (a.c + 511) / 512;
  a.chunk = 64;
  while (a.chunk > 16 && (a.tokens + a.chunk - 1) / a.chunk * tiles < 4096) a.chunk /= 2;
  a.chunks = int((a.tokens + a.chunk - 1) / a.chunk);
  a.cpad = (a.c + 7) / 8 * 8;
  uint64_t at = 0;
  auto take = [&](uint64_t bytes) {
    const uint64_t p = at;
    at += align16(bytes);
    return p;
  };
  const uint64_t start = take(4 * uint64_t(a.vocab + 1)), perm = take(4 * uint64_t(a.tokens)),
                 key = take(4 * uint64_t(a.tokens)), tail = take(4 * uint64_t(a.chunks)), part = take(8 * uint64_t(a.chunks) * a.cpad);
  if (ws) {
    a.start = reinterpret_cast<int *>(ws + start);
    a.perm = reinterpret_cast<int *>(ws + perm);
    a.key = reinterpret_cast<int *>(ws + key);
    a.tail = reinterpret_cast<int *>(ws + tail);
    a.part = reinterpret_cast<float *>(ws + part);
  }
  return at;
}

void embed_backward(hipStream_t s, const EmbedArgs &a, int gtype, int dtype) {
  if (gtype == SEQ_F32)
    dtype == SEQ_F32 ? backward<float, float>(s, a) : backward<float, __bf16>(s, a);
  else
    dtype == SEQ_F32 ? backward<__bf16, float>(s, a) : backward<__bf16, __bf16>(s, a);
}

}  // namespace ckpt
