// Embedding: rows of a table looked up by id and scaled; the table's gradient, each id's
// rows added up in the order of its tokens.
//
// The gradient takes three launches.
//   k_embed_sort  orders the tokens by id, each id's in their order.  A workgroup
//     takes a range of ids, reads all ids (from L2: they are few against the rows),
//     counts those of its range for each of sixteen sections of the tokens, one a
//     wavefront, and places them.  The first position of a range is the number of
//     smaller ids, which the workgroup counts as it goes, so workgroups need nothing of
//     each other.
//   k_embed_sum   a wavefront adds up the rows of a chunk of sorted positions, 512
//     columns; an id whose tokens lie within the chunk is done, one that crosses an
//     end leaves its part.  Other workgroups write the rows of absent ids.
//   k_embed_join  adds the parts of an id that crosses chunks, in order.
// Nothing is added by atomics (the counts are whole numbers), so the same bits come
// out on every run.
#include "common.h"
#include "seq.h"
#include "vec.h"

namespace ckpt {
namespace {

constexpr int SECTIONS = 16;    // wavefronts of a sorting workgroup
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

__global__ __launch_bounds__(64 * SECTIONS) void k_embed_sort(EmbedArgs A, int range) {
  __shared__ int cnt[SECTIONS * MAX_RANGE];  // [section][id of the range]
  __shared__ int wsum[SECTIONS];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int lo = int(min(int64_t(blockIdx.x) * range, A.vocab));
  const int n = int(min(int64_t(range), A.vocab - lo));
  const int64_t per = ((A.tokens + SECTIONS - 1) / SECTIONS + 63) / 64 * 64;
  const int64_t first = min(wave * per, A.tokens), last = min(first + per, A.tokens);
  for (int i = threadIdx.x; i < SECTIONS * range; i += 64 * SECTIONS) cnt[i] = 0;
  __syncthreads();

  int less = 0;
#pragma unroll 4
  for (int64_t i = first; i < last; i += 64) {
    const int id = i + lane < last ? id_at(A, i + lane) : -1;
    less += id >= 0 && id < lo;
    if (id >= lo && id < lo + n) atomicAdd(&cnt[wave * range + id - lo], 1);
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) less += __shfl_xor(less, o);
  if (lane == 0) wsum[wave] = less;
  __syncthreads();
  int base = 0;
#pragma unroll
  for (int k = 0; k < SECTIONS; ++k) base += wsum[k];
  __syncthreads();  // wsum is written again below

  // cnt becomes the first position of each section's tokens of an id: an exclusive sum over
  // the ids, then over the sections; a thread has range / threads consecutive ids
  const int each = (range + 64 * SECTIONS - 1) / (64 * SECTIONS);  // 1
  int mine = 0;
  const int i0 = threadIdx.x * each;
  for (int i = i0; i < min(i0 + each, n); ++i)
    for (int k = 0; k < SECTIONS; ++k) mine += cnt[k * range + i];
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
  for (int i = i0; i < min(i0 + each, n); ++i) {
    A.start[lo + i] = pos;
    for (int k = 0; k < SECTIONS; ++k) {
      const int t = cnt[k * range + i];
      cnt[k * range + i] = pos;
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

  for (int64_t i = first; i < last; i += 64) {
    const int id = i + lane < last ? id_at(A, i + lane) : -1;
    uint64_t left = __ballot(id >= lo && id < lo + n);
    while (left) {
      const int key = __shfl(id, __ffsll((unsigned long long)left) - 1);
      const uint64_t same = __ballot(id == key);
      // one wavefront's: its accesses are in order, and volatile keeps them in the code's
      volatile int *const at = &cnt[wave * range + key - lo];
      const int p = *at;
      if (id == key) {
        const int rank = __popcll(same & ((1ull << lane) - 1));
        A.perm[p + rank] = int(i + lane);
        A.key[p + rank] = key;
        if (rank == 0) *at = p + __popcll(same);
      }
      left &= ~same;
    }
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

// Workgroups below `sums` add up chunks, a wavefront each; the others write the
// absent ids' rows.
template <typename GT, typename DT>
__global__ __launch_bounds__(256) void k_embed_sum(EmbedArgs A, int tiles, int sums) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (int(blockIdx.x) >= sums) {
    const int64_t rows = int64_t(gridDim.x - sums) * 4;
    const int64_t nvec = (A.c + 7) / 8;
    for (int64_t v = (blockIdx.x - sums) * int64_t(4) + wave; v < A.vocab; v += rows) {
      if (A.start[v] != A.start[v + 1]) continue;
      const float zero[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      for (int64_t j = lane; j < nvec; j += 64)
        store8(static_cast<DT *>(A.dst) + v * A.ldd + j * 8, min(8, A.c - int(j) * 8), zero);
    }
    return;
  }
  const int64_t unit = blockIdx.x * int64_t(4) + wave;
  const int64_t chunk = unit / tiles;
  if (chunk >= A.chunks) return;
  const int col = int(unit - chunk * tiles) * 512 + lane * 8, cnt = min(8, A.c - col);
  const int total = A.start[A.vocab];
  const int64_t p0 = chunk * A.chunk;
  const int len = int(min(int64_t(A.chunk), total - p0));
  if (len <= 0) return;
  int tok = 0, key = -1;
  if (lane < len) {
    tok = A.perm[p0 + lane];
    key = A.key[p0 + lane];
  }
  const bool before = p0 > 0 && A.key[p0 - 1] == __shfl(key, 0);
  const bool after = p0 + len < total && A.key[p0 + len] == __shfl(key, len - 1);
  float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  bool head = before;  // the rows so far belong to an id that began before the chunk
  for (int q = 0; q < len; q += 8) {
    float v[8][8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int64_t row = __builtin_amdgcn_readlane(tok, min(q + u, len - 1));
      if (cnt > 0) load8(static_cast<const GT *>(A.src) + row * A.lds + col, cnt, v[u]);
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if (q + u >= len) break;
      const int k0 = __builtin_amdgcn_readlane(key, q + u);
#pragma unroll
      for (int k = 0; k < 8; ++k) s[k] += v[u][k];
      const bool end = q + u + 1 == len;
      if (end || __builtin_amdgcn_readlane(key, min(q + u + 1, 63)) != k0) {
        if (cnt > 0) {
          if (head || (end && after))
            store8(A.part + (2 * chunk + (head ? 0 : 1)) * A.cpad + col, cnt, s);
          else
            put_row<DT>(A, k0, col, cnt, s);
        }
        head = false;
#pragma unroll
        for (int k = 0; k < 8; ++k) s[k] = 0.f;
      }
    }
  }
}

// the ids that cross the end of chunk blockIdx.x and began in it: 64 vectors of columns a
// workgroup, the parts dealt to sixteen wavefronts in runs, which are then added in order
template <typename DT>
__global__ __launch_bounds__(1024) void k_embed_join(EmbedArgs A) {
  __shared__ float red[16][8][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int total = A.start[A.vocab];
  const int64_t chunk = blockIdx.x, end = (chunk + 1) * A.chunk;
  if (end >= total) return;
  const int key = A.key[end - 1];
  if (A.key[end] != key || A.start[key] < chunk * A.chunk) return;
  const int64_t last = (A.start[key + 1] - 1) / A.chunk;  // the chunk that holds its last token
  const int n = int(last - chunk) + 1;                    // parts: this chunk's tail, the others' heads
  const int col = blockIdx.y * 512 + lane * 8, cnt = min(8, A.c - col);
  const int per = (n + 15) / 16, a = min(wave * per, n), b = min(a + per, n);
  float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (cnt > 0) {
#pragma unroll 4
    for (int i = a; i < b; ++i) {
      float v[8];
      load8(A.part + (2 * (chunk + i) + (i ? 0 : 1)) * A.cpad + col, cnt, v);
#pragma unroll
      for (int k = 0; k < 8; ++k) s[k] += v[k];
    }
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) red[wave][k][lane] = s[k];
  __syncthreads();
  if (wave == 0 && cnt > 0) {
    const int waves = (n + per - 1) / per;
    for (int w = 1; w < waves; ++w)
#pragma unroll
      for (int k = 0; k < 8; ++k) s[k] += red[w][k][lane];
    put_row<DT>(A, key, col, cnt, s);
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
  const int tiles = (a.c + 511) / 512;
  const int sums = int((int64_t(a.chunks) * tiles + 3) / 4);
  const int64_t rows = (a.vocab + 3) / 4;
  const int zeros = a.accumulate ? 0 : int(rows < 2048 ? rows : 2048);
  hipLaunchKernelGGL((k_embed_sum<GT, DT>), dim3(uint32_t(sums + zeros)), dim3(256), 0, s, a, tiles, sums);
  if (a.chunks > 1)
    hipLaunchKernelGGL(k_embed_join<DT>, dim3(uint32_t(a.chunks - 1), uint32_t(tiles)), dim3(1024), 0, s, a);
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
  a.chunk = 64;
  a.chunks = int((a.tokens + a.chunk - 1) / a.chunk);
  a.cpad = (a.c + 7) / 8 * 8;
  uint64_t at = 0;
  auto take = [&](uint64_t bytes) {
    const uint64_t p = at;
    at += align16(bytes);
    return p;
  };
  const uint64_t start = take(4 * uint64_t(a.vocab + 1)), perm = take(4 * uint64_t(a.tokens)),
                 key = take(4 * uint64_t(a.tokens)), part = take(8 * uint64_t(a.chunks) * a.cpad);
  if (ws) {
    a.start = reinterpret_cast<int *>(ws + start);
    a.perm = reinterpret_cast<int *>(ws + perm);
    a.key = reinterpret_cast<int *>(ws + key);
    a.part = reinterpret_cast<float *>(ws + part);
  }
  return at;
}

void embed_backward(hipStream_t s, const EmbedArgs &a, int gtype, int dtype) {
  // a range for each compute unit, as far as the counts fit
  const int64_t even = (a.vocab + 255) / 256;
  const int range = int(even < MAX_RANGE ? even : MAX_RANGE);
  hipLaunchKernelGGL(k_embed_sort, dim3(uint32_t((a.vocab + range - 1) / range)), dim3(64 * SECTIONS), 0, s, a, range);
  if (gtype == SEQ_F32)
    dtype == SEQ_F32 ? backward<float, float>(s, a) : backward<float, __bf16>(s, a);
  else
    dtype == SEQ_F32 ? backward<__bf16, float>(s, a) : backward<__bf16, __bf16>(s, a);
}

}  // namespace ckpt
