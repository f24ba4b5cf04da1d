// Into how many key ranges a walk over selected blocks is cut: plain functions of sizes, without HIP.
#pragma once

#include "launch_rules.hpp"

namespace astro {

constexpr int kMaxSelectSplits = 8;

// A tile of 32 keys in us: where a workgroup is alone on its CU, what each further one adds, and how many a CU holds.  Fitted to walks
// of 6 to 371 tiles by 2 to 1776 workgroups on 256 CUs, every number of ranges at 12 shapes of each kind; what the rule then picks is
// within 4 % of the best count but for launches of about 50 us, 10 %.
struct WalkCost {
  double alone, more;
  int per_cu;
  double tile(int workgroups) const { return workgroups ? alone + (workgroups - 1) * more : 0.; }
};
constexpr WalkCost select_fwd_cost(int D, int queries) {
  return D == 128 ? (queries == 128 ? WalkCost{1.02, 0.46, 2} : WalkCost{0.79, 0.16, 2}) : (queries == 128 ? WalkCost{0.74, 0.23, 3} : WalkCost{0.66, 0.10, 3});
}
constexpr WalkCost select_dq_cost(int D) { return D == 128 ? WalkCost{0.75, 0.30, 3} : WalkCost{0.62, 0.12, 3}; }

// items: workgroups without a cut, of `tiles` tiles each in the mean; part_bytes: what one range of all of them leaves.  A cut has to
// gain more than a launch and writing and reading the parts (5 bytes per ps each way) cost: 444 walks of 370 tiles at D = 64 364 us in
// one, 300 in four; 48 of 236 at D = 128 213 in one, 64 in five; 168 of 42 72 in one, 54 in three, 78 in eight.
inline int select_splits(const WalkCost& c, int n_cus, int items, double tiles, double part_bytes) {
  auto cost = [&](int n) {
    const int64_t wgs = (int64_t)items * n, round = (int64_t)c.per_cu * n_cus, rest = wgs % round;
    const int last = (int)((rest + n_cus - 1) / n_cus);  // workgroups on the fullest CU behind the full rounds
    return ((double)(wgs / round) * c.tile(c.per_cu) + c.tile(last)) * tiles / n + (n > 1 ? 5. + 2. * n * part_bytes / 5e6 : 0.);
  };
  int best = 1;
  for (int n = 2; n <= kMaxSelectSplits && n <= tiles / 2; ++n)
    if (cost(n) < 0.97 * cost(best)) best = n;
  return best;
}
// Calls of few rows (queries times heads) form their scores from three pieces of every operand and six products (24 bits), others from two
// and three (16 bits).  A score's error is that of a probability, 5e-6: over many rows the gradients' 2-norms are 5e-6 to 7e-6 off, hardly
// more for any inputs (the worst of 150 was 7.3e-6 at 400 rows, 7.0e-6 at 800 and more), but over a few, where one probability may make most of
// a gradient, up to 1.2e-5 (one in 40 to 140 over 1e-5 at 2 to 48 rows); with three pieces 7e-6.  A log-sum-exp is as near unless it is near 0, which it is in
// all rows only where there are very few of them.  Few rows wait for latencies: at 128 rows a forward takes 11.3 us from two pieces and 12.6
// from three.  At the long sizes three would take a third more.
constexpr bool select_fine(bool bwd, int64_t rows) { return rows <= (bwd ? 512 : 64); }
// whether a launch of this many rows and pairs may be cut at all (its workspace then has room for the parts)
inline bool select_may_split(int n_cus, int pairs, int Nq) { return (int64_t)blocks_of(Nq, 128) * pairs < 4 * n_cus; }

}  // namespace astro
