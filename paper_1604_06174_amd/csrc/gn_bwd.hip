// Group-norm backward: the launches that all types share, and the fp32 ones.
#include "gn_bwd.h"

namespace ckpt {
namespace gnb {
namespace {

__global__ __launch_bounds__(64) void k_gn_bwd_merge(GnArgs A) {
  const int i = blockIdx.x / A.G, k = blockIdx.x % A.G;
  const float *const part = A.cpart + int64_t(i) * A.chunks1 * 2 * A.C + k * A.cg;
  const int64_t count = int64_t(A.chunks1) * A.cg;
  float s1 = 0.f, s2 = 0.f;
  for (int64_t e = threadIdx.x; e < count; e += 64) {
    const int64_t q = e / A.cg;
    const int c = int(e - q * A.cg);
    const float ga = A.gamma[k * A.cg + c];
    s2 += ga * part[q * 2 * A.C + c];
    s1 += ga * part[q * 2 * A.C + A.C + c];
  }
  float s[2] = {s1, s2};
  add_from<2>(1, s);
  if (threadIdx.x == 0) {
    const float rstd = A.st[(A.n + i) * A.G + k];
    A.gsum[2 * int64_t(blockIdx.x)] = rstd * s[0];
    A.gsum[2 * int64_t(blockIdx.x) + 1] = rstd * s[1];
  }
}

__global__ __launch_bounds__(1024) void k_gn_records(GnArgs A) {
  __shared__ float red[64 * 17];
  record_sums(A, A.rows, blockIdx.x, red);
}

}  // namespace

void merge_groups(hipStream_t s, const GnArgs &a) {
  hipLaunchKernelGGL(k_gn_bwd_merge, dim3(uint32_t(a.n * a.G)), dim3(64), 0, s, a);
}

void sum_records(hipStream_t s, const GnArgs &a) {
  hipLaunchKernelGGL(k_gn_records, dim3((2 * a.C + 15) / 16), dim3(1024), 0, s, a);
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
