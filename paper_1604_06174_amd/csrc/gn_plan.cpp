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

int vec_of(const GnProblem &p) { return p.C % 8 == 0 ? 8 : 1; }

// Tiles of whole groups and whole vectors, about `want` channels each, at most
// `cap` threads wide; V drops to 1 where a group is too wide for that.
void group_tiles(const GnProblem &p, int64_t want, int cap8, GnCover &v) {
  v.V = vec_of(p);
  int64_t unit = std::lcm(int64_t(p.cg), int64_t(v.V));
  if (unit > 8 * 512) {
    v.V = 1;
    unit = p.cg;
  }
  const int64_t cap = v.V == 8 ? cap8 : 1024;
  if (unit / v.V > cap)
    fail(CKPT_E_UNSUPPORTED, "group norm: more than 1024 channels per group (4096 where 8 divides it)");
  int64_t W = std::min(unit * ceil_div(want, unit), unit * std::max<int64_t>(1, cap * v.V / unit));
  W = std::min<int64_t>(W, p.C);
  v.W = int(W);
  v.tiles = int(ceil_div(p.C, W));
  v.VC = v.W / v.V;
}

// chunks of a sample's pixels, about `blocks` workgroups in all, at least `least` rows
// of threads each
void cut(const GnProblem &p, int64_t blocks, int64_t least, GnCover &v) {
  const int64_t want = std::max<int64_t>(1, ceil_div(blocks, p.n * v.tiles));
  v.chunk = up(std::max(ceil_div(p.hw, want), least * v.TY), v.TY);
  v.chunks = ceil_div(p.hw, v.chunk);
  v.blocks = p.n * v.tiles * v.chunks;
}

void reductions(const GnProblem &p, bool backward, int NQ, GnPlan &g) {
  const GnCover &v = g.first;
  g.pow2 = is_pow2(v.VC) && v.VC <= 64;
  g.NJ = p.cg % v.V == 0 ? 1 : v.V;
  const int T = g.wave ? 64 : v.threads;
  g.redbuf = NQ ? gn_reduce_floats(v, g.pow2, T, NQ, g.NJ, p.cg) : 0;
  size_t f = size_t(g.pow2 ? 2 : 1) * g.teams * g.redbuf;
  if (backward)  // the channels' sums
    f = std::max(f, g.pow2 ? size_t(v.threads / 64) * 2 * v.W
                           : size_t(g.teams) * (v.TY + (v.TY + 7) / 8) * v.VC * 2 * v.V);
  g.lds = 4 * f;
}

}  // namespace

GnCover gn_cover_elements(const GnProblem &p, int V, bool whole_groups) {
  GnCover v{};
  if (whole_groups) {
    // few enough channels for their parameters to stay in LDS
    group_tiles(p, 512, 64, v);
  } else {
    v.V = V;
    const int64_t vc = p.C / v.V;
    v.tiles = int(ceil_div(vc, 64));
    v.VC = int(ceil_div(vc, v.tiles));
    v.W = v.VC * v.V;
  }
  v.threads = int(std::max<int64_t>(256, up(v.VC, 64)));
  v.TY = v.threads / v.VC;
  v.TY = int(std::min<int64_t>(v.TY, p.hw));
  v.threads = int(up(int64_t(v.TY) * v.VC, 64));
  cut(p, 1024, 4, v);
  return v;
}

GnCover gn_cover_rerun(const GnProblem &p) {
  GnCover v = gn_cover_elements(p, vec_of(p), false);
  if (gn_few_pixels(p.hw)) {
    v.threads = 256;
    v.TY = v.threads / v.VC;
    const int64_t pixels = p.n * p.hw;
    v.chunk = up(std::max<int64_t>(ceil_div(pixels, std::max(1, 4096 / v.tiles)), 4 * v.TY), v.TY);
    v.blocks = v.tiles * ceil_div(pixels, v.chunk);
  }
  return v;
}

GnPlan gn_plan(const GnProblem &p, bool backward) {
  GnPlan g{};
  GnCover &v = g.first;
  g.teams = 1;
  // 128 bytes of a pixel at least, so that no two tiles share a cache line of
  // contiguous rows; more where a sample's pixels are too few for a wavefront
  const int64_t line = 128 / (p.xf ? 4 : 2);
  group_tiles(p, std::max(line, ceil_div(64 * vec_of(p), p.hw)), backward ? 512 : 1024, v);
  const int cap = backward && v.V == 8 ? 512 : 1024;
  const int64_t vecs = int64_t(v.VC) * p.hw, slabs = p.n * v.tiles;
  // vectors a thread keeps: 4 registers each for bf16, 8 for fp32 (and 8 more for
  // the gradient)
  const int nv_max = v.V == 1 ? 16 : (backward || p.xf ? 8 : 16);
  v.chunks = 1;
  v.chunk = p.hw;
  // a wavefront per sample and tile where there are enough of them to fill the
  // device (4 a SIMD); else more threads share one
  if (v.VC <= 64 && ceil_div(p.hw, 64 / v.VC) <= 8 && slabs >= 4096) {
    g.resident = g.wave = true;
    g.teams = 4;
    v.threads = 256;
    v.TY = 64 / v.VC;
    g.NV = int(ceil_div(p.hw, v.TY));
    // the workgroups loop over samples, so that few records of channel sums are left
    g.rows = std::min<int64_t>(ceil_div(p.n, g.teams), std::max(1, 1024 / v.tiles));
  } else {
    v.threads = int(std::min<int64_t>(cap, up(v.VC * ceil_div(p.hw, 2), 64)));
    if (v.threads < v.VC) v.threads = int(up(v.VC, 64));
    v.TY = v.threads / v.VC;
    const int64_t nv = ceil_div(p.hw, v.TY);
    // few slabs only while one is read in a few microseconds by its one compute unit
    if (nv <= nv_max && (slabs >= 128 || vecs <= 4096)) {
      g.resident = true;
      g.NV = int(nv);
      g.rows = p.n;
    }
  }
  if (g.resident) {
    v.blocks = g.rows * v.tiles;
    reductions(p, backward, backward ? 2 : 1, g);
    if (backward && g.rows > 1) g.ws_channels = align256(uint64_t(g.rows) * 2 * p.C * 4);
    return g;
  }
  v.threads = int(std::max<int64_t>(256, up(v.VC, 64)));
  v.TY = v.threads / v.VC;
  cut(p, 512, 4, v);
  reductions(p, backward, backward ? 0 : 1, g);
  if (backward) {
    g.merge = v.chunks > 32 || p.cg > 64;
    g.ws_channels = align256(uint64_t(p.n) * v.chunks * 2 * p.C * 4);
    if (g.merge) g.ws_sums = align256(uint64_t(p.n) * p.G * 8);
  } else {
    g.merge = v.chunks > 64;
    g.ws_groups = align256(uint64_t(p.n) * v.chunks * p.G * 8);
  }
  g.second = gn_cover_elements(p, v.V, backward && !g.merge);
  return g;
}

}  // namespace ckpt
