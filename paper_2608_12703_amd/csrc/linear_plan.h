// How the products of linear.hip are cut into workgroups: rules on sizes, on whether the operands allow
// direct loads, and on measured times.  Host code alone, without the HIP headers.
#pragma once

#include <algorithm>
#include <cstddef>
#include <cstdint>

namespace ad {

constexpr int kBK = 64;                          // reduction elements of one LDS stage
// few rows: waves of a workgroup, and 32-wide steps that a wave has in flight
constexpr int kFewWaves = 8, kFewSteps = 5;

// How a product is cut.  Tiles that fill whole rounds of the chip are computed by one workgroup
// each; the tiles of the last, partly filled round in S parts of the reduction, so that the
// chip is about full there too.
struct Plan {
  int tile;              // 128 (four waves) or 256 (eight waves, one workgroup a CU)
  bool deep;             // 128: one workgroup a CU with a ring of four stages, not two with two
  int tiles_p, tiles_q, whole, S, steps;
  double cost;           // microseconds, to compare plans
};
constexpr int kCUs = 256;

// Workgroups at once, and measured microseconds: of a 64-wide step, and of a round of workgroups besides
// (its first loads, its epilogues).  14336 rows, width 1280 to 5120 (20 steps) and 5120 to 1280 (80):
// large 185 and 174, pairs 202 and 204, deep 241 and 211; 1536 rows, 1280 to 2560: 45, 27, 23.  The
// plan of least cost was within 0.6% of the best of the three over 147 products of 1 to 14336 rows.
struct Shape {
  int tile;
  bool deep;
  int slots;
  double step, round;
};
constexpr Shape kLarge = {256, false, kCUs, 1.6, 13.0}, kPairs = {128, false, 2 * kCUs, 1.05, 5.0},
                kDeep = {128, true, kCUs, 0.52, 5.6}, kAny = {128, false, 2 * kCUs, 1.6, 5.0};
// A checkpoint with rows of any alignment: its registers leave room for one workgroup a CU (1500 x 1283 x
// 1001 in two parts 31.6 us, in more 33 to 36).
constexpr Shape kAnyCkpt = {128, false, kCUs, 1.6, 5.0};

inline Plan plan_of(int P, int Q, int K, Shape sh) {
  Plan r;
  r.tile = sh.tile;
  r.deep = sh.deep;
  r.tiles_p = (P + sh.tile - 1) / sh.tile;
  r.tiles_q = (Q + sh.tile - 1) / sh.tile;
  const int all = (K + kBK - 1) / kBK;
  const int64_t T = (int64_t)r.tiles_p * r.tiles_q;
  const int rest = (int)(T % sh.slots);
  r.whole = (int)T;
  r.S = 1;
  r.steps = all;
  const double whole = sh.round + sh.step * all;
  r.cost = whole * (double)((T + sh.slots - 1) / sh.slots);
  for (int S = 2; rest && S <= 64 && rest * S <= sh.slots && all / S >= 4; ++S) {
    // the parts, their way through memory twice, and another launch
    const int steps = (all + S - 1) / S, parts = (all + steps - 1) / steps;
    const double cost = whole * (double)(T / sh.slots) + sh.round + sh.step * steps + 5.0 +
                        2e-6 * sh.tile * sh.tile * parts * rest;
    if (cost < r.cost) {
      r.whole = (int)(T - rest);
      r.S = parts;
      r.steps = steps;
      r.cost = cost;
    }
  }
  return r;
}

// From the sizes, whether the operands allow direct loads, and whether P is a checkpoint.
inline Plan plan(int P, int Q, int K, bool direct, bool ckpt) {
  if (!direct) return plan_of(P, Q, K, ckpt ? kAnyCkpt : kAny);
  Plan best = plan_of(P, Q, K, kPairs);
  for (const Shape& sh : {kLarge, kDeep}) {
    if (sh.deep && ckpt) continue;
    const Plan r = plan_of(P, Q, K, sh);
    if (r.cost < best.cost) best = r;
  }
  return best;
}

inline size_t part_floats(const Plan& r) {
  return r.S > 1 ? (size_t)r.S * (r.tiles_p * r.tiles_q - r.whole) * ((size_t)r.tile * r.tile + r.tile) : 0;
}

// Floats of workspace that a product may need, asked for before its operands are known.  wgrad: P may be a
// checkpoint.
inline size_t plan_floats(bool wgrad, int P, int Q, int K) {
  const size_t n = std::max(part_floats(plan(P, Q, K, true, false)), part_floats(plan(P, Q, K, false, false)));
  if (!wgrad) return n;
  return std::max({n, part_floats(plan(P, Q, K, true, true)), part_floats(plan(P, Q, K, false, true))});
}

// The forward product of few rows straight from registers: how it is cut, and its microseconds, to
// compare with a plan's: what the weight's loads take one after the other or at the memory's rate,
// and the rows, which every workgroup reads from L2 (measured from 1 to 32 rows at 1280 x 1280 to
// 51864 x 1280 and 1280 x 5120, within 20%; a 51864-wide head takes 27 us for a row, 42 for 16
// and 62 for 32, against 31, 31 and 32 in tiles).
struct FewPlan {
  bool narrow;   // 8 columns a workgroup where 16 would leave CUs without one
  int grid;
  double cost;
};
constexpr int kFewRows = 32;
inline FewPlan few_plan(int P, int Q, int K) {
  FewPlan f;
  f.narrow = (P + 15) / 16 < kCUs;
  f.grid = f.narrow ? (P + 7) / 8 : (P + 15) / 16;
  const int turns = ((K + 31) / 32 + kFewWaves * kFewSteps - 1) / (kFewWaves * kFewSteps);
  f.cost = std::max(3.0 + 1.2 * turns, 2.0 * P * K / 4.9e6) + 2.0 * f.grid * Q * K / 8e6;
  return f;
}
// (tiles read the weight at 4.2 TB/s at best)
inline bool few_wins(const FewPlan& f, const Plan& tiles, int P, int K) {
  return f.cost < std::max(tiles.cost, 2.0 * P * K / 4.2e6);
}

}  // namespace ad
