// extern "C" group-norm and dropout calls (declared in include/ckpt.h, "operator
// calls").  Every argument is validated before anything is launched.
#include <hip/hip_runtime.h>

#include <cmath>
#include <string>

#include "capi_internal.h"
#include "dropout.h"
#include "gn.h"

static_assert(CKPT_ACT_NONE == ckpt::GN_ACT_NONE && CKPT_ACT_RELU == ckpt::GN_ACT_RELU &&
                  CKPT_ACT_SILU == ckpt::GN_ACT_SILU,
              "activation codes of the C ABI and the kernels agree");

namespace {

using ckpt::fail;

// a device buffer of elements of `size` bytes (a power of two); the message is put
// together only for a bad one
void need_ptr(const void *p, const char *fn, const char *arg, uintptr_t size = 1) {
  if (p && !(reinterpret_cast<uintptr_t>(p) & (size - 1))) return;
  const std::string what = std::string(fn) + "(" + arg + ")";
  if (!p) fail(CKPT_E_INVALID, what + ": null pointer");
  fail(CKPT_E_INVALID, what + ": misaligned address");
}

[[noreturn]] void refuse(int code, const char *fn, const char *what) { fail(code, std::string(fn) + what); }

uintptr_t size_of(bool f32) { return f32 ? 4 : 2; }

void launched(const char *fn) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) fail(CKPT_E_HIP, std::string(fn) + ": " + hipGetErrorString(e));
}

bool is_f32(int32_t type, const char *fn) {
  if (type != CKPT_TYPE_F32 && type != CKPT_TYPE_BF16) refuse(CKPT_E_INVALID, fn, ": unknown type");
  return type == CKPT_TYPE_F32;
}

// elements the generator can number (its block number is 32 bits)
constexpr int64_t kMaxElements = int64_t(1) << 35;

// a * b, both positive, below 2^62; -1 past it
int64_t product(int64_t a, int64_t b) {
  return a > (int64_t(1) << 62) / b ? -1 : a * b;
}

ckpt::DropArgs drop_args(const ckpt_dropout *d, const char *fn) {
  ckpt::DropArgs a{nullptr, 0, 0, 1.f};
  if (!d) return a;
  if (!(d->p >= 0.0 && d->p <= 1.0)) refuse(CKPT_E_INVALID, fn, ": dropout p must lie in [0, 1]");
  need_ptr(d->rng, fn, "dropout.rng", 8);
  const uint32_t t = uint32_t(std::floor(65536.0 * d->p + 0.5));
  if (t == 0) return a;
  a.rng = d->rng;
  a.site = d->site;
  a.thr = t == 65536 ? 0xffffffffu : (t << 16) - 1;
  a.scale = t == 65536 ? 0.f : float(65536.0 / double(65536 - t));
  return a;
}

ckpt::GnProblem problem_of(const ckpt_gn_desc *d, const char *fn) {
  need_ptr(d, fn, "desc");
  if (d->n < 1 || d->hw < 1 || d->c < 1 || d->groups < 1)
    refuse(CKPT_E_INVALID, fn, ": n, hw, c and groups must be positive");
  if (d->c % d->groups) refuse(CKPT_E_INVALID, fn, ": groups must divide c");
  if (d->act != CKPT_ACT_NONE && d->act != CKPT_ACT_RELU && d->act != CKPT_ACT_SILU)
    refuse(CKPT_E_INVALID, fn, ": unknown activation");
  if (!(d->eps > 0.f) || !std::isfinite(d->eps)) refuse(CKPT_E_INVALID, fn, ": eps must be positive");
  ckpt::GnProblem p{};
  p.n = d->n;
  p.hw = d->hw;
  p.C = d->c;
  p.G = d->groups;
  p.cg = d->c / d->groups;
  p.act = d->act;
  p.xf = is_f32(d->xtype, fn);
  p.gf = is_f32(d->gtype, fn);
  p.df = is_f32(d->dtype, fn);
  p.ldx = d->ldx ? d->ldx : d->c;
  p.ldy = d->ldy ? d->ldy : d->c;
  p.ldg = d->ldg ? d->ldg : d->c;
  p.ldd = d->ldd ? d->ldd : d->c;
  for (int64_t ld : {p.ldx, p.ldy, p.ldg, p.ldd}) {
    if (ld < d->c) refuse(CKPT_E_INVALID, fn, ": a pixel stride is smaller than c");
    const int64_t px = product(p.n, p.hw), e = px < 0 ? -1 : product(px, ld);
    if (e < 0 || e > (int64_t(1) << 60)) refuse(CKPT_E_UNSUPPORTED, fn, ": tensor too large");
  }
  if (p.C > (1 << 20)) refuse(CKPT_E_UNSUPPORTED, fn, ": c must not exceed 2^20");
  if (p.n * p.hw >= (int64_t(1) << 30)) refuse(CKPT_E_UNSUPPORTED, fn, ": n*hw must stay below 2^30");
  if (p.n * p.hw * p.C >= kMaxElements) refuse(CKPT_E_UNSUPPORTED, fn, ": n*hw*c must stay below 2^35");
  if (p.n * p.G >= (int64_t(1) << 25)) refuse(CKPT_E_UNSUPPORTED, fn, ": n*groups must stay below 2^25");
  p.eps = d->eps;
  return p;
}

// block numbers the kernels divide (GnDivide)
void grid_fits(const ckpt::GnCover &v, const char *fn) {
  if (v.blocks >= (int64_t(1) << 21) || v.chunks >= (int64_t(1) << 21)) refuse(CKPT_E_UNSUPPORTED, fn, ": tensor too large");
}

// a call's plan, its grids and workspace checked
ckpt::GnPlan plan_of(const ckpt::GnProblem &p, bool backward, const void *workspace, uint64_t workspace_bytes,
                     const char *fn) {
  const ckpt::GnPlan g = ckpt::gn_plan(p, backward);
  grid_fits(g.first, fn);
  grid_fits(g.second, fn);
  // what a forward of the same samples would be refused for (a backward's may loop)
  if (g.resident && !g.wave && p.n * g.first.tiles >= (int64_t(1) << 21)) refuse(CKPT_E_UNSUPPORTED, fn, ": tensor too large");
  const uint64_t want = ckpt::gn_workspace_bytes(g);
  if (want) {
    need_ptr(workspace, fn, "workspace", 16);
    if (workspace_bytes < want) refuse(CKPT_E_WORKSPACE, fn, ": workspace smaller than op_gn_workspace_bytes");
  }
  return g;
}

}  // namespace

extern "C" {

int op_gn_workspace_bytes(const ckpt_gn_desc *desc, int32_t backward, uint64_t *bytes) {
  return ckpt::guarded([&] {
    need_ptr(bytes, "op_gn_workspace_bytes", "bytes");
    const ckpt::GnProblem p = problem_of(desc, "op_gn_workspace_bytes");
    *bytes = ckpt::gn_workspace_bytes(ckpt::gn_plan(p, backward != 0));
  });
}

int op_gn_forward(const ckpt_gn_desc *desc, const void *x, const float *gamma, const float *beta,
                  const ckpt_dropout *drop, void *y, float *st, void *workspace, uint64_t workspace_bytes,
                  void *stream) {
  return ckpt::guarded([&] {
    const char *const fn = "op_gn_forward";
    const ckpt::GnProblem p = problem_of(desc, fn);
    need_ptr(x, fn, "x", size_of(p.xf));
    need_ptr(gamma, fn, "gamma", 4);
    need_ptr(beta, fn, "beta", 4);
    need_ptr(y, fn, "y", size_of(p.xf));
    need_ptr(st, fn, "st", 4);
    const ckpt::DropArgs da = drop_args(drop, fn);
    const ckpt::GnPlan plan = plan_of(p, false, workspace, workspace_bytes, fn);
    ckpt::gn_forward(static_cast<hipStream_t>(stream), p, plan, x, gamma, beta, da, y, st, workspace);
    launched("op_gn_forward");
  });
}

int op_gn_apply(const ckpt_gn_desc *desc, const void *x, const float *st, const float *gamma,
                const float *beta, const ckpt_dropout *drop, void *y, void *stream) {
  return ckpt::guarded([&] {
    const char *const fn = "op_gn_apply";
    const ckpt::GnProblem p = problem_of(desc, fn);
    need_ptr(x, fn, "x", size_of(p.xf));
    need_ptr(st, fn, "st", 4);
    need_ptr(gamma, fn, "gamma", 4);
    need_ptr(beta, fn, "beta", 4);
    need_ptr(y, fn, "y", size_of(p.xf));
    const ckpt::DropArgs da = drop_args(drop, fn);
    const ckpt::GnCover v = ckpt::gn_cover_rerun(p);
    grid_fits(v, fn);
    ckpt::gn_apply(static_cast<hipStream_t>(stream), p, v, x, st, gamma, beta, da, y);
    launched("op_gn_apply");
  });
}

int op_gn_backward(const ckpt_gn_desc *desc, const void *g, const void *x, const float *st,
                   const float *gamma, const float *beta, const ckpt_dropout *drop, void *d, float *dgamma,
                   float *dbeta, void *workspace, uint64_t workspace_bytes, void *stream) {
  return ckpt::guarded([&] {
    const char *const fn = "op_gn_backward";
    const ckpt::GnProblem p = problem_of(desc, fn);
    if (p.xf && !(p.gf && p.df))
      refuse(CKPT_E_UNSUPPORTED, fn, ": an fp32 x takes fp32 g and d");
    need_ptr(g, fn, "g", size_of(p.gf));
    need_ptr(x, fn, "x", size_of(p.xf));
    need_ptr(st, fn, "st", 4);
    need_ptr(gamma, fn, "gamma", 4);
    need_ptr(beta, fn, "beta", 4);
    need_ptr(d, fn, "d", size_of(p.df));
    need_ptr(dgamma, fn, "dgamma", 4);
    need_ptr(dbeta, fn, "dbeta", 4);
    const ckpt::DropArgs da = drop_args(drop, fn);
    const ckpt::GnPlan plan = plan_of(p, true, workspace, workspace_bytes, fn);
    ckpt::gn_backward(static_cast<hipStream_t>(stream), p, plan, g, x, st, gamma, beta, da, d, dgamma, dbeta, workspace);
    launched("op_gn_backward");
  });
}

int op_dropout(int64_t rows, int64_t cols, int32_t xtype, const void *x, int64_t ldx, const void *res,
               int64_t ldr, int32_t ytype, void *y, int64_t ldy, const ckpt_dropout *drop, void *stream) {
  return ckpt::guarded([&] {
    const char *const fn = "op_dropout";
    if (rows < 1 || cols < 1) refuse(CKPT_E_INVALID, fn, ": rows and cols must be positive");
    const bool xf = is_f32(xtype, fn), yf = is_f32(ytype, fn);
    need_ptr(x, fn, "x", size_of(xf));
    need_ptr(y, fn, "y", size_of(yf));
    if (res) need_ptr(res, fn, "res", size_of(yf));
    need_ptr(drop, fn, "drop");
    if (!ldx) ldx = cols;
    if (!ldr) ldr = cols;
    if (!ldy) ldy = cols;
    for (int64_t ld : {ldx, ldr, ldy}) {
      if (ld < cols) refuse(CKPT_E_INVALID, fn, ": a row stride is smaller than cols");
      const int64_t e = product(rows, ld);
      if (e < 0 || e > (int64_t(1) << 60)) refuse(CKPT_E_UNSUPPORTED, fn, ": tensor too large");
    }
    if (rows * cols >= kMaxElements) refuse(CKPT_E_UNSUPPORTED, fn, ": rows*cols must stay below 2^35");
    const ckpt::DropArgs da = drop_args(drop, fn);
    ckpt::dropout(static_cast<hipStream_t>(stream), rows, cols, xf, x, ldx, res, ldr, yf, y, ldy, da);
    launched("op_dropout");
  });
}

}  // extern "C"
