// How the group-norm passes cover a problem: tile, team and chunk sizes (host).
#include <algorithm>
#include <numeric>

#include "common.h"
#include "gn.h"

namespace ckpt {
namespace {

bool is_pow2(int64_t v) { return v > 0 && (v & (v - 1)) == 0; }
int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// LDS of the reductions (two buffers taken in turn where pow2)
void set_lds(const GnProblem &p, GnPlan &g, bool backward) {
  g.redbuf = int(gn_reduce_floats(g, g.wave ? 64 : g.threads, backward ? 2 : 1, g.fold ? 1 : g.V, p.cg));
  size_t f = size_t(g.pow2 ? 2 : 1) * g.teams * g.redbuf;
  if (backward) {
    // the channels' sums at the end
    const size_t e = g.pow2 ? size_t(g.threads / 64) * 2 * g.W
                            : size_t(g.teams) * (g.TY + (g.TY + 7) / 8) * g.VC * 2 * g.V;
    f = std::max(f, e);
  }
  g.lds = 4 * f;
}

}  // namespace

GnPlan gn_plan(const GnProblem &p, bool backward) {
  GnPlan g{};
  g.V = p.C % 8 == 0 ? 8 : 1;
  int64_t unit = std::lcm(int64_t(p.cg), int64_t(g.V));
  if (unit > 8 * 512) {
    // one element a thread (fails below for groups that are too wide for that)
    g.V = 1;
    unit = p.cg;
  }
  const int cap = backward && g.V == 8 ? 512 : 1024;
  if (unit / g.V > cap)
    fail(CKPT_E_UNSUPPORTED, "group norm: more than 1024 channels per group (4096 where 8 divides it)");
  // 128 bytes of a pixel at least, so that no two tiles share a cache line of
  // contiguous rows; more where a sample's pixels are too few for a wavefront
  const int64_t line = 128 / (p.xf ? 4 : 2);
  const int64_t want = std::max(line, ceil_div(64 * g.V, p.hw));
  int64_t W = std::min(unit * ceil_div(want, unit), unit * std::max<int64_t>(1, cap * g.V / unit));
  W = std::min<int64_t>(W, p.C);
  g.W = int(W);
  g.tiles = int(ceil_div(p.C, W));
  g.VC = g.W / g.V;
  g.fold = p.cg % g.V == 0;
  g.pow2 = is_pow2(g.VC) && g.VC <= 64;
  const int64_t vecs = int64_t(g.VC) * p.hw;
  // vectors a thread keeps: 4 registers each for bf16, 8 for fp32 (and 8 more for
  // the gradient)
  const int nv_max = g.V == 1 ? 16 : (backward || p.xf ? 8 : 16);
  const int64_t slabs = p.n * g.tiles;
  // a wavefront per sample and tile where there are enough of them to fill the
  // device (4 a SIMD); else more threads share one
  if (g.VC <= 64 && ceil_div(p.hw, 64 / g.VC) <= 8 && slabs >= 4096) {
    g.wave = true;
    g.teams = 4;
    g.threads = 256;
    g.TY = 64 / g.VC;
    g.NV = int(ceil_div(p.hw, g.TY));
    // the workgroups loop over samples, so that few records of channel sums are left
    g.rows = int(std::min<int64_t>(ceil_div(p.n, g.teams), std::max(1, 1024 / g.tiles)));
    g.blocks = int64_t(g.rows) * g.tiles;
    set_lds(p, g, backward);
    return g;
  }
  g.teams = 1;
  g.threads = int(std::min<int64_t>(cap, up(g.VC * ceil_div(p.hw, 4), 64)));
  if (g.threads < g.VC) g.threads = int(up(g.VC, 64));
  g.TY = g.threads / g.VC;
  const int64_t nv = ceil_div(p.hw, g.TY);
  // resident: few slabs only while one is read in a few microseconds by its one
  // compute unit
  if (nv <= nv_max && (slabs >= 128 || vecs <= 4096)) {
    g.NV = int(nv);
    g.rows = int(std::min<int64_t>(p.n, std::max(1, 4096 / g.tiles)));
    g.blocks = int64_t(g.rows) * g.tiles;
    set_lds(p, g, backward);
    return g;
  }
  g.split = true;
  g.threads = int(std::max<int64_t>(256, up(g.VC, 64)));
  g.TY = g.threads / g.VC;
  g.NV = g.V == 1 ? 16 : 8;
  g.chunks = ceil_div(p.hw, int64_t(g.TY) * g.NV);
  g.blocks = p.n * g.chunks * g.tiles;
  set_lds(p, g, backward);
  return g;
}

GnPlan gn_plan_elements(const GnProblem &p) {
  GnPlan g{};
  g.V = p.C % 8 == 0 ? 8 : 1;
  const int64_t vc = p.C / g.V;
  g.tiles = int(ceil_div(vc, 256));
  g.VC = int(ceil_div(vc, g.tiles));
  g.W = g.VC * g.V;
  g.fold = p.cg % g.V == 0;
  g.teams = 1;
  g.TY = int(std::min<int64_t>(256 / g.VC, p.hw));
  g.threads = int(up(int64_t(g.TY) * g.VC, 64));
  g.NV = GN_EW_NV;
  g.chunks = ceil_div(p.hw, int64_t(g.TY) * g.NV);
  g.blocks = p.n * g.chunks * g.tiles;
  return g;
}

uint64_t gn_workspace_bytes(const GnProblem &p, bool backward) {
  const GnPlan g = gn_plan(p, backward);
  uint64_t b = 0;
  if (g.split) b += align256(uint64_t(p.n) * g.chunks * p.G * 2 * 4);
  if (backward) {
    if (g.split) b += align256(uint64_t(p.n) * p.G * 2 * 4);
    const uint64_t rows = g.split ? uint64_t(p.n) * g.chunks : uint64_t(g.rows);
    if (rows > 1) b += align256(rows * 2 * p.C * 4);
  }
  return b;
}

}  // namespace ckpt
