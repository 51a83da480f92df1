// How the group-norm passes cover a problem: tile, team and chunk sizes (host).
#include <algorithm>
#include <numeric>

#include "common.h"
#include "gn.h"

namespace ckpt {
namespace {

int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

int vec_of(const GnProblem &p) { return p.C % 8 == 0 ? 8 : 1; }

int pow2_up(int v) {
  int p = 1;
  while (p < v) p *= 2;
  return p;
}

// Tiles of whole groups and whole vectors, `want` channels or more each, at most
// cap8 threads wide (1024 element by element); V drops to 1 where a group is too wide.
// `lanes`: VC is rounded up to a power of two where it is at most 64, and the tile
// taken (of up to four times the channels) whose columns fill it best, 7/8 or more
// if any does.
void group_tiles(const GnProblem &p, int64_t want, int cap8, bool lanes, GnCover &v) {
  v.V = vec_of(p);
  int64_t unit = std::lcm(int64_t(p.cg), int64_t(v.V));
  if (unit > 8 * 512) {
    v.V = 1;
    unit = p.cg;
  }
  const int64_t cap = v.V == 8 ? cap8 : 1024;
  if (unit / v.V > cap)
    fail(CKPT_E_UNSUPPORTED, "group norm: more than 1024 channels per group (4096 where 8 divides it)");
  const int64_t units = p.C / unit;  // whole: C is a multiple of cg and of V
  int64_t m = std::min(std::min(ceil_div(want, unit), std::max<int64_t>(1, cap * v.V / unit)), units);
  auto cols = [&](int64_t k) { return k * unit / v.V; };
  if (lanes && cols(m) <= 64) {
    int64_t best = m;
    auto fill = [&](int64_t k) { return double(cols(k)) / pow2_up(int(cols(k))); };
    for (int64_t k = m; k <= std::min(4 * m, units) && cols(k) <= 64 && fill(best) < 0.875; ++k)
      if (fill(k) > fill(best)) best = k;
    m = best;
  }
  v.W = int(m * unit);
  v.tiles = int(ceil_div(p.C, v.W));
  v.cols = v.W / v.V;
  v.VC = lanes && v.cols <= 64 ? pow2_up(v.cols) : v.cols;
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
  g.red = v.VC > 64 ? GN_RED_TREE : v.VC == v.cols ? GN_RED_GROUPS : GN_RED_COLUMNS;
  g.NJ = p.cg % v.V == 0 ? 1 : v.V;
  const int T = g.wave ? 64 : v.threads;
  g.redbuf = NQ ? gn_reduce_floats(v, g.red, T, NQ, g.NJ, p.cg) : 0;
  size_t f = size_t(g.red == GN_RED_GROUPS ? 2 : 1) * g.teams * g.redbuf;
  if (backward)  // the channels' sums
    f = std::max(f, g.red != GN_RED_TREE ? size_t(v.threads / 64) * 2 * v.V * v.VC
                           : size_t(g.teams) * (v.TY + (v.TY + 7) / 8) * v.VC * 2 * v.V);
  g.lds = 4 * f;
}

}  // namespace

GnCover gn_cover_elements(const GnProblem &p, int V, bool whole_groups) {
  GnCover v{};
  if (whole_groups) {
    // few enough channels for their parameters to stay in LDS
    group_tiles(p, 512, 64, false, v);
  } else {
    v.V = V;
    const int64_t vc = p.C / v.V;
    v.tiles = int(ceil_div(vc, 64));
    v.VC = int(ceil_div(vc, v.tiles));
    v.W = v.VC * v.V;
    v.cols = v.VC;
  }
  v.threads = int(std::max<int64_t>(256, up(v.VC, 64)));
  v.TY = v.threads / v.VC;
  v.TY = int(std::min<int64_t>(v.TY, p.hw));
  v.threads = int(up(int64_t(v.TY) * v.VC, 64));
  // four workgroups a CU, one turn: each forms its channels' parameters once (the stem's
  // forward: 32.2 us, 32.7 at 2048, 33.9 at 4096)
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
  g.teams = g.pack = 1;
  // 128 bytes of a pixel at least, so that no two tiles share a cache line of
  // contiguous rows; more where a sample's pixels are too few for a wavefront
  const int64_t line = 128 / (p.xf ? 4 : 2);
  group_tiles(p, std::max(line, ceil_div(64 * vec_of(p), p.hw)), backward ? 512 : 1024, true, v);
  const int cap = backward && v.V == 8 ? 512 : 1024;
  const int64_t vecs = int64_t(v.VC) * p.hw, slabs = p.n * v.tiles;
  // vectors a thread keeps: 4 registers each for bf16, 8 for fp32 (and 8 more for
  // the gradient)
  const int nv_max = v.V == 1 ? 16 : (backward || p.xf ? 8 : 16);
  v.chunks = 1;
  v.chunk = p.hw;
  // short samples, many of them: a wavefront per sample and tile, or for several
  // samples of one pixel.  At four vectors a thread and more the workgroup form is
  // faster (49 pixels x 64 channels, 2048 tiles: 16.8 us backward against 19.6).
  if (v.VC <= 64 && ceil_div(p.hw, 64 / v.VC) <= 2 && slabs >= 1024) {
    g.resident = g.wave = true;
    g.teams = 4;
    v.threads = 256;
    v.TY = 64 / v.VC;
    g.NV = int(ceil_div(p.hw, v.TY));
    reductions(p, backward, backward ? 2 : 1, g);
    g.pack = p.hw == 1 && g.red == GN_RED_GROUPS && (g.NJ == 1 || p.cg == 2 || p.cg == 4) ? v.TY : 1;
    const int64_t turns = ceil_div(p.n, int64_t(g.teams) * g.pack);  // of one workgroup
    // the workgroups loop over samples: 1024 fill the device (2048 of 16384 rows of 1024
    // channels: 31 us backward against 28), and a backward leaves at most half as many
    // records of channel sums as it has turns
    g.rows = std::min<int64_t>(turns, std::max(1, 1024 / v.tiles));
    if (backward) g.rows = std::min(g.rows, std::max<int64_t>(std::min<int64_t>(turns, 64), ceil_div(turns, 2)));
  } else {
    // two vectors a thread while the workgroup may grow (one sample of 49 pixels x 512
    // channels, forward: 3.7 us; at four vectors 4.5, at eight 5.7)
    v.threads = int(std::min<int64_t>(cap, up(v.VC * ceil_div(p.hw, 2), 64)));
    if (v.threads < v.VC) v.threads = int(up(v.VC, 64));
    v.TY = v.threads / v.VC;
    const int64_t nv = ceil_div(p.hw, v.TY);
    // few slabs only while one is read in a few microseconds by its one compute unit
    // (bf16 forward, microseconds resident and split: 4 slabs of 3200 vectors 7.4 and
    // 8.7, of 6272 vectors 10.7 and 8.8; 32 of them 11.1 and 9.6, 64 11.9 and 12.4; 256
    // 20.0 and 24.8).  fp32 and the backward follow: 16 to 512 slabs of up to 3200 vectors
    // all lose by splitting (64 of 3200, bf16 backward 10.1 and 10.5, 512 of them 24.0 and
    // 26.3; of 1600 fp32 ones forward 8.1 and 9.6, backward 10.3 and 11.5)
    if (nv <= nv_max && (slabs >= 64 || vecs <= 4096)) {
      g.resident = true;
      g.NV = int(nv);
      g.rows = p.n;
      // a backward's workgroups loop over samples of so few pixels that a record of channel
      // sums for each (8 bytes a channel) would outweigh the sample: as many of them as the
      // device holds at once, 1024 at most (microseconds, a record per sample and this way:
      // 16384 rows of 1024 channels 115 and 41, 2048 of them 20 and 16, 4000 samples of 2 x
      // 4096 113 and 72, 8000 of 4 x 512 51 and 35; of 8 pixels some sizes lose: 8000 x 504
      // channels in twelves 77 and 84; element by element 8000 of 2 x 515 58 and 36, with
      // SiLU and dropout 77 and 60, of 3 pixels 91 and 112), and two samples each where
      // the records would take 12 MB (1000 rows of 2048 17.6 and 15.8, 500 of 4096 18.1 and
      // 15.8; of 10 MB and less some lose: 400 samples of 4 x 3000 17.8 and 18.3)
      if (backward && p.hw <= (v.V == 8 ? 4 : 2)) {
        const int64_t held = std::max(1, std::min(1024, (1 << 18) / v.threads) / v.tiles);
        g.rows = std::min(held, p.n * p.C >= (3 << 19) ? ceil_div(p.n, 2) : p.n);
      }
    }
  }
  if (g.resident) {
    v.blocks = g.rows * v.tiles;
    if (!g.wave) reductions(p, backward, backward ? 2 : 1, g);
    if (backward && g.rows > 1) {
      // 64 threads a column add up the records: more workgroups take part where that is
      // more than 64 records each (100000 of eight channels, one workgroup: 287 us, 177 in 25
      // segments; 16384 of 64: 53.6 and 39.7; 8000: 44.6 and 42.1; below, the launch costs what
      // it gives)
      g.segments = int(std::min<int64_t>(64, ceil_div(g.rows, 4096)));
      g.ws_channels = align256(uint64_t(g.rows + (g.segments > 1 ? g.segments : 0)) * 2 * p.C * 4);
    }
    return g;
  }
  v.threads = int(std::max<int64_t>(256, up(v.VC, 64)));
  v.TY = v.threads / v.VC;
  // two workgroups a CU: fewer chunks to add up outweigh the latency that four would
  // hide (stage-1 backward with dropout: 58.6 us, 60.1 at 1024, 66.0 at 256)
  cut(p, 512, 4, v);
  reductions(p, backward, backward ? 0 : 1, g);
  if (backward) {
    // adding up the chunks costs every workgroup of the second pass more the more there
    // are (a sample of 50176 pixels x 64 channels, 392 chunks: 27.6 us, 16.9 with a launch
    // for it; four of them, 121 chunks each: 32.7 and 31.2), and groups wider than a tile
    // have to be formed outside
    g.merge = v.chunks > 32 || p.cg > 64;
    g.ws_channels = align256(uint64_t(p.n) * v.chunks * 2 * p.C * 4);
    if (g.merge) g.ws_sums = align256(uint64_t(p.n) * p.G * 8);
  } else {
    // (392 chunks: 29.5 us, 14.7 with a launch; 98: 13.3 and 10.4; 64 or fewer are read
    // at once)
    g.merge = v.chunks > 64;
    g.ws_groups = align256(uint64_t(p.n) * v.chunks * p.G * 8);
  }
  g.second = gn_cover_elements(p, v.V, backward && !g.merge);
  return g;
}

}  // namespace ckpt
