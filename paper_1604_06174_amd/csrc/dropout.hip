// Dropout of a matrix, optionally added to a residual: y = res + (keep ? s x : 0)
// (s = 1 / (1 - p)), the mask from the counter-based generator of philox.h.  The
// backward is the same call on the gradient without a residual.
//
// A thread takes one generator block, eight consecutive elements of the
// row-major matrix: 16 bytes of bf16 in one access where the eight lie so.
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

// VECT: the eight elements of a block lie in one row
template <typename XT, typename YT, bool VECT>
__global__ __launch_bounds__(256) void k_dropout(Args A) {
  const int64_t stride = int64_t(gridDim.x) * 256;
  const DropKey key = drop_key(A.drop);
  for (int64_t b = blockIdx.x * int64_t(256) + threadIdx.x; b < A.blocks; b += stride) {
    const int64_t e = b * 8, row = e / A.cols, c = e - row * A.cols;
    float v[8];
    if (VECT) {
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
void launch(hipStream_t s, const Args &a, bool vect) {
  const int64_t g = (a.blocks + 255) / 256;
  const dim3 grid(uint32_t(g < 16384 ? g : 16384));
  if (vect)
    hipLaunchKernelGGL((k_dropout<XT, YT, true>), grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((k_dropout<XT, YT, false>), grid, dim3(256), 0, s, a);
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
  const bool vect = a.cols % 8 == 0;
  if (xf)
    yf ? launch<float, float>(s, a, vect) : launch<float, __bf16>(s, a, vect);
  else
    yf ? launch<__bf16, float>(s, a, vect) : launch<__bf16, __bf16>(s, a, vect);
}

}  // namespace ckpt
