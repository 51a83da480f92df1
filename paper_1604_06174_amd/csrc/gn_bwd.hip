// Group-norm backward: the launches that all types share, and the fp32 ones.
#include "gn_bwd.h"

namespace ckpt {
namespace gnb {
namespace {

// One workgroup per group of a sample: its channels across the threads, eight chunks
// at a time in flight.
__global__ __launch_bounds__(1024) void k_gn_bwd_merge(GnArgs A) {
  __shared__ float red[32];
  const int i = blockIdx.x / A.G, k = blockIdx.x - i * A.G;
  const float *const part = A.cpart + int64_t(i) * A.chunks1 * 2 * A.C + k * A.cg;
  // S threads a channel, each every S-th chunk
  const int S = max(1, int(blockDim.x) / A.cg);
  float s[2] = {0.f, 0.f};
  for (int e = threadIdx.x; e < A.cg * S; e += blockDim.x) {
    const int r0 = e / A.cg, c = e - r0 * A.cg;
    const float ga = A.gamma[k * A.cg + c];
    float t1 = 0.f, t2 = 0.f;
    constexpr int U = 8;
    for (int r = r0; r < A.chunks1; r += U * S) {
      float v[2 * U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float *const q = part + int64_t(min(r + u * S, A.chunks1 - 1)) * 2 * A.C + c;
        v[2 * u] = q[0];
        v[2 * u + 1] = q[A.C];
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        t2 += r + u * S < A.chunks1 ? v[2 * u] : 0.f;
        t1 += r + u * S < A.chunks1 ? v[2 * u + 1] : 0.f;
      }
    }
    s[0] += ga * t1;
    s[1] += ga * t2;
  }
  add_from<2>(1, s);
  const int w = threadIdx.x >> 6, nw = blockDim.x >> 6;
  if ((threadIdx.x & 63) == 0) {
    red[w] = s[0];
    red[16 + w] = s[1];
  }
  __syncthreads();
  if (threadIdx.x < 2) {
    float t = 0.f;
    for (int q = 0; q < nw; ++q) t += red[16 * threadIdx.x + q];
    A.gsum[2 * int64_t(blockIdx.x) + threadIdx.x] = A.st[(A.n + i) * A.G + k] * t;
  }
}

// dgamma and dbeta, or (`part`) the record of a segment of `per` of the records
__global__ __launch_bounds__(1024) void k_gn_records(GnArgs A, int per, float *part) {
  __shared__ float red[64 * 17];
  const int r0 = blockIdx.y * per;
  float *const out = part + int64_t(blockIdx.y) * 2 * A.C;
  record_sums(A.cpart + int64_t(r0) * 2 * A.C, min(per, A.rows - r0), A.C, blockIdx.x, part ? out : A.dgamma,
              part ? out + A.C : A.dbeta, red);
}

}  // namespace

void merge_groups(hipStream_t s, const GnArgs &a) {
  // as many wavefronts as hold about a chunk's row each
  const int64_t work = int64_t(a.chunks1) * a.cg / 8;
  const int threads = work >= 1024 ? 1024 : work >= 256 ? 256 : 64;
  hipLaunchKernelGGL(k_gn_bwd_merge, dim3(uint32_t(a.n * a.G)), dim3(threads), 0, s, a);
}

void sum_records(hipStream_t s, const GnArgs &a, int segments) {
  const uint32_t columns = (2 * a.C + 15) / 16;
  GnArgs b = a;
  if (segments > 1) {
    float *const part = a.cpart + int64_t(a.rows) * 2 * a.C;
    const int per = (a.rows + segments - 1) / segments;
    b.rows = (a.rows + per - 1) / per;
    hipLaunchKernelGGL(k_gn_records, dim3(columns, b.rows), dim3(1024), 0, s, a, per, part);
    b.cpart = part;
  }
  hipLaunchKernelGGL(k_gn_records, dim3(columns), dim3(1024), 0, s, b, b.rows, static_cast<float *>(nullptr));
}

void run_f32(hipStream_t s, const GnProblem &p, const GnPlan &g, const GnArgs &a) {
  run_types<float, float, float>(s, p, g, a);
}

}  // namespace gnb

void gn_backward(hipStream_t s, const GnProblem &p, const GnPlan &plan, const void *g, const void *x,
                 const float *st, const float *gamma, const float *beta, const DropArgs &drop, void *d,
                 float *dgamma, float *dbeta, void *ws) {
  GnArgs a = gn_args(p, plan.first, drop);
  a.rows = int(plan.rows);
  a.redbuf = plan.redbuf;
  a.pack = plan.pack;
  a.x = x;
  a.g = g;
  a.out = d;
  a.ldo = p.ldd;
  a.gamma = gamma;
  a.beta = beta;
  a.st = const_cast<float *>(st);
  a.dgamma = dgamma;
  a.dbeta = dbeta;
  char *const w = static_cast<char *>(ws);
  if (plan.ws_channels) a.cpart = reinterpret_cast<float *>(w);
  if (plan.ws_sums) a.gsum = reinterpret_cast<float *>(w + plan.ws_channels);
  if (p.xf)
    gnb::run_f32(s, p, plan, a);
  else if (p.gf)
    gnb::run_bf16_f32(s, p, plan, a);
  else
    gnb::run_bf16_bf16(s, p, plan, a);
}

}  // namespace ckpt
