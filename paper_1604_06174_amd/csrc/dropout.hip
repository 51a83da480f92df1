// Dropout of a matrix, optionally added to a residual: y = res + (keep ? s x : 0)
// (s = 1 / (1 - p)), the mask from the counter-based generator of philox.h.  The
// backward is the same call on the gradient without a residual.
//
// A thread takes one generator block, eight consecutive elements of the row-major
// matrix: one access (16 bytes of bf16) where they lie in one row, which need not
// start anywhere in particular; a block across the end of a row goes element by
// element.  Bound by HBM: 100352 x 256 bf16 with a residual 28.9 us (5.3 TB/s, as a
// copy of that size); the generator, 20 products of 32 bits an eight, adds 2.6 us to
// the 15.9 us that the same rows take without it.
#include "common.h"
#include "dropout.h"
#include "vec.h"

namespace ckpt {
namespace {

struct Args {
  const void *x, *res;
  void *y;
  int64_t blocks;      // of eight elements
  int64_t count, cols; // elements; per row
  int64_t ldx, ldr, ldy;
  DropArgs drop;
};

template <typename XT, typename YT>
__global__ __launch_bounds__(256) void k_dropout(Args A) {
  const int64_t stride = int64_t(gridDim.x) * 256;
  const DropKey key = drop_key(A.drop);
  for (int64_t b = blockIdx.x * int64_t(256) + threadIdx.x; b < A.blocks; b += stride) {
    const int64_t e = b * 8;
    // 32-bit division where it is enough, none for a single row
    const int64_t row = A.cols == A.count ? 0 : A.count >> 32 ? e / A.cols : int64_t(uint32_t(e) / uint32_t(A.cols));
    const int64_t c = e - row * A.cols;
    float v[8];
    if (c + 8 <= A.cols) {
      const Vec<XT, 8> x = load_vec<XT, 8>(static_cast<const XT *>(A.x) + row * A.ldx + c);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = float(x.v[k]);
      if (A.drop.rng) drop8(A.drop, key, uint32_t(b), v);
      if (A.res) {
        const Vec<YT, 8> r = load_vec<YT, 8>(static_cast<const YT *>(A.res) + row * A.ldr + c);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] += float(r.v[k]);
      }
      store_vec<YT, 8>(static_cast<YT *>(A.y) + row * A.ldy + c, v);
    } else {
      int64_t rk[8], ck[8];
      rk[0] = row;
      ck[0] = c;
#pragma unroll
      for (int k = 1; k < 8; ++k) {
        const bool wrap = ck[k - 1] + 1 == A.cols;
        rk[k] = rk[k - 1] + wrap;
        ck[k] = wrap ? 0 : ck[k - 1] + 1;
      }
#pragma unroll
      for (int k = 0; k < 8; ++k)
        v[k] = e + k < A.count ? float(static_cast<const XT *>(A.x)[rk[k] * A.ldx + ck[k]]) : 0.f;
      if (A.drop.rng) drop8(A.drop, key, uint32_t(b), v);
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (e + k < A.count) {
          if (A.res) v[k] += float(static_cast<const YT *>(A.res)[rk[k] * A.ldr + ck[k]]);
          static_cast<YT *>(A.y)[rk[k] * A.ldy + ck[k]] = (YT)v[k];
        }
    }
  }
}

template <typename XT, typename YT>
void launch(hipStream_t s, const Args &a) {
  const int64_t g = (a.blocks + 255) / 256;
  hipLaunchKernelGGL((k_dropout<XT, YT>), dim3(uint32_t(g < 16384 ? g : 16384)), dim3(256), 0, s, a);
}

}  // namespace

void dropout(hipStream_t s, int64_t rows, int64_t cols, bool xf, const void *x, int64_t ldx, const void *res,
             int64_t ldr, bool yf, void *y, int64_t ldy, const DropArgs &drop) {
  Args a{x, res, y, 0, rows * cols, cols, ldx, ldr, ldy, drop};
  if (!res) a.ldr = cols;
  // rows without gaps are one row
  if (ldx == cols && a.ldr == cols && ldy == cols) {
    a.cols = a.ldx = a.ldr = a.ldy = a.count;
  }
  a.blocks = (a.count + 7) / 8;
  if (xf)
    yf ? launch<float, float>(s, a) : launch<float, __bf16>(s, a);
  else
    yf ? launch<__bf16, float>(s, a) : launch<__bf16, __bf16>(s, a);
}

}  // namespace ckpt
