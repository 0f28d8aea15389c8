// Which kernel a product of the gated feed-forward block takes (gated_ffn.hip), by its sizes: host code, which a CPU test
// compiles to hold the tests' shapes against what the rules can choose.
#pragma once
#include <cstddef>
#include <cstdint>

namespace mlc {
namespace {

// Whether M tokens take the kernel for few tokens (ffn_few_kernel) for a product with N x K weights.  Every workgroup reads all
// of x, so that beside the weights the L2 serves as much again for every 16 tokens: to 8 tokens that is hidden (2048 / 5632, both products: 23.3 us for one
// token, 24.5 for eight; the tiles 26.1 and 26.3), and of small weights, whose time is the launches', to 32 (512 / 2048, 16 tokens:
// 12.8 and 17.7; 2048 / 5632, 16 and 32 tokens: 27.8 and 35.2, the tiles 26.5 and 27.2).  Few rows of long weights are too
// few workgroups (20480 / 64, one token: 27 us, cut tiles 21).
bool few(int64_t M, int64_t N, int64_t K) {
  if (N < 512 && K > 4096) return false;
  return M <= 8 || (M <= 32 && N * K <= (int64_t)1 << 21);
}

constexpr int BK = 64;                              // depth of a K tile
constexpr int UNITS = 256;                          // compute units
// per_unit: workgroups a compute unit: one, whose ring fills its LDS (with a small tile four K tiles ahead), or two with half of
// it each.
struct Plan { int bm, bn, per_unit, whole, splits; };
struct Size { int64_t M, N; };                      // of a product; N: columns of accumulators (2 f of UP)

// The tile, and whether the tiles of the last, partly filled round are cut along K (only where can_split), by an estimate of the
// time: the compute units' share of tiles times what a tile's kt K tiles and its ends take, and the joining of cut tiles.
// The constants are fitted to the block's times on 13 shapes from 77 x 2560 x 10240 to 8192 x 2048 x 5632, each form's tile and
// cuts varied with the others held: the choice takes 1.065 of the best one's time at most, over 1.02 in three of 65 (one tile
// for all: 1.5 times and more in some of them).  `few` and `all`: a K tile's time with few tiles and with every unit busy,
// all[0] of products whose operands are both K-contiguous (UP, NT), all[1] with K-strided ones; in between by the units that
// have work, and of two workgroups a unit once there are two.  `ends`: of a tile's start and epilogue, one number for five forms
// that differ (DH's epilogue of a 256 tile is the longest); the fit's 1.065 holds for each of them.
struct TileCost { int bm, bn, per_unit; double few, all[2], ends; };      // us
constexpr TileCost TILE_COSTS[] = {{256, 256, 1, 0.76, {1.20, 1.10}, 9.9}, {128, 128, 1, 0.53, {0.42, 0.43}, 3.1},
                                   {128, 128, 2, 0.51, {0.39, 0.37}, 2.6}, {64, 128, 1, 0.42, {0.45, 0.35}, 2.4},
                                   {64, 128, 2, 0.54, {0.33, 0.32}, 1.9}};
constexpr double JOIN = 7.4, JOIN_BYTES = 3.7e6;    // us, and bytes a us
Plan pick(const Size* s, int n, int64_t kt, bool strided, bool can_split) {
  Plan best{};
  double least = 1e300;
  for (const TileCost& c : TILE_COSTS) {
    int64_t tiles = 0;
    for (int i = 0; i < n; ++i) tiles += ((s[i].M + c.bm - 1) / c.bm) * ((s[i].N + c.bn - 1) / c.bn);
    const int64_t slots = (int64_t)UNITS * c.per_unit, rest = tiles % slots, whole = tiles - rest;
    const double full = (double)(whole / UNITS) * (kt * c.all[strided] + c.ends);
    for (int splits = 1; splits <= 16; ++splits) {
      if (splits > 1 && (!can_split || rest * splits > slots || kt / splits < 4)) break;
      const int64_t items = rest * splits, share = (items + UNITS - 1) / UNITS;
      const double busy = c.per_unit == 2 ? share > 1 : items < UNITS ? (double)items / UNITS : 1.0;
      const double k_time = c.few + (c.all[strided] - c.few) * busy;
      const double join = splits > 1 ? JOIN + (double)items * c.bm * c.bn * 8 / JOIN_BYTES : 0.0;
      const double t = full + (double)share * ((double)kt / splits * k_time + c.ends) + join;
      if (t < least) {
        least = t;
        best = Plan{c.bm, c.bn, c.per_unit, splits > 1 ? (int)whole : 0, splits};
      }
    }
  }
  return best;
}
// (at most one round of items are split ones)
size_t partial_bytes(const Plan& p) { return p.splits > 1 ? (size_t)UNITS * p.per_unit * p.bm * p.bn * 4 : 0; }

int64_t k_tiles(int64_t K) { return (K + BK - 1) / BK; }
Plan plan_up(int64_t t, int64_t d, int64_t f) { const Size z{t, 2 * f}; return pick(&z, 1, k_tiles(d), false, false); }
Plan plan_down(int64_t t, int64_t d, int64_t f) { const Size z{t, d}; return pick(&z, 1, k_tiles(f), false, true); }
Plan plan_inner(int64_t t, int64_t d, int64_t f) { const Size z{t, f}; return pick(&z, 1, k_tiles(d), true, false); }
Plan plan_dx(int64_t t, int64_t d, int64_t f) { const Size z{t, d}; return pick(&z, 1, 2 * k_tiles(f), true, true); }
Plan plan_dw(int64_t t, int64_t d, int64_t f) { const Size z[3] = {{f, d}, {f, d}, {d, f}}; return pick(z, 3, k_tiles(t), true, true); }

}  // namespace
}  // namespace mlc
