// Which kernel takes a linear layer in 8-bit integers with token scales, and how its rows are cut.  Plain C++.
#pragma once
#include <stdint.h>

#include "even_plan.h"
#include "launch_rules.h"

namespace gpusq {

// Most channels: the kernel for many rows has a row of Y in 32-bit offsets, 16 of them below 2^31 bytes.
constexpr int64_t kMostTokens8N = (int64_t)1 << 24;

// The tiles of the kernel for many rows (linear8_tiles.hip): 256 channels x chunks of whole 32-row units, all of the same height or one unit more, as
// many chunks as fill whole rounds over the CUs.  A step of 64 k of u units takes kStepFixed + kStepUnit u and no less than kStepLeast (microseconds).
constexpr double kStep8Fixed = 0.06, kStep8Unit = 0.075, kStep8Least = 0.17, kEpilogue8Unit = 0.5, kTile8Fixed = 1.0;
inline double tile8_cost(double units, int ksteps) {
  const double step = kStep8Fixed + kStep8Unit * units;
  return ksteps * (step > kStep8Least ? step : kStep8Least) + kTile8Fixed + kEpilogue8Unit * units;
}
struct Tokens8Plan {
  EvenPlan even;
  double cost;
};
inline Tokens8Plan tokens8_plan(int64_t M, int64_t N, int64_t K, int cus) {
  constexpr int kTallest = 8;
  const int tiles_n = (int)plan_div(N, kTileBN), ksteps = (int)plan_div(K, 64);
  const int64_t units = plan_div(M, 32), least = plan_div(plan_div(units, kTallest) * tiles_n, cus);
  Tokens8Plan best{};
  best.cost = -1;
  for (int64_t rounds = least; rounds <= least + 3; ++rounds) {
    int64_t chunks = rounds * cus / tiles_n;
    if (chunks < plan_div(units, kTallest)) chunks = plan_div(units, kTallest);
    if (chunks > units) chunks = units;
    const int64_t r = plan_div(chunks * tiles_n, cus);
    const int64_t most = r * (units / chunks) + plan_div((units % chunks) * tiles_n, cus);  // units of the workgroup with the most
    const double cost = r * tile8_cost((double)most / r, ksteps);
    if (best.cost >= 0 && cost >= best.cost) continue;
    best.cost = cost;
    best.even.tiles_n = tiles_n;
    best.even.chunks = (int)chunks;
    best.even.units = (int)(units / chunks);
    best.even.higher = (int)(units % chunks);
  }
  EvenPlan& p = best.even;
  const int64_t total = even_total(p);
  p.grid8 = (int)plan_div(total < cus ? total : cus, 8);
  p.rounds = (int)(total / (8 * p.grid8));
  p.last_round = (int)(total % (8 * p.grid8));
  int log2 = 1;
  while (((int64_t)1 << log2) < tiles_n) ++log2;
  p.shift = log2 - 1;
  p.inv = tiles_n > 1 ? (uint32_t)(((uint64_t)1 << (31 + log2)) / tiles_n + ((((uint64_t)1 << (31 + log2)) % tiles_n) != 0)) : 0u;
  return best;
}

}  // namespace gpusq
