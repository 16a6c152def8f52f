// Which kernel takes a linear layer in 8-bit integers with token scales, and how its rows are cut.  Plain C++.
#pragma once
#include <stdint.h>

#include "launch_rules.h"

namespace gpusq {

// Most channels: the kernel for many rows has a row of Y in 32-bit offsets, 16 of them below 2^31 bytes.
constexpr int64_t kMostTokens8N = (int64_t)1 << 24;
inline bool tokens8_countable(int64_t M, int64_t N) { return ceil_div(M, 32) * ceil_div(N, 64) <= INT32_MAX; }

// The tiles of the kernel for many rows (linear8_tiles.h): 32 tn channels (tn = 8, 4 or 2) x chunks of whole 32-row units, all of the same height or
// one unit more.  Tiles are numbered in bands of `band` chunks, inside a band chunks first: round i takes the tiles from i * grid on, in runs of
// grid / 8 to an XCD, whose L2 then holds the weights of some blocks of channels and the rows of some chunks, about as much of either.
struct Tokens8Plan {
  int tn, tiles_n, chunks, units, higher, band;
  int rounds, last_round;  // whole rounds of tiles; tiles behind them
  int grid8;               // grid / 8
};
struct Tokens8Tile {
  int n_blk, slabs;  // height in slabs of 16 rows
  int64_t m0;
};
__host__ __device__ inline Tokens8Tile tokens8_tile(const Tokens8Plan& p, int idx) {
  const int b = idx / (p.band * p.tiles_n), rest = idx - b * (p.band * p.tiles_n), left = p.chunks - b * p.band, wide = left < p.band ? left : p.band;
  Tokens8Tile t;
  t.n_blk = rest / wide;
  const int chunk = b * p.band + rest - t.n_blk * wide;
  t.slabs = 2 * (p.units + (chunk < p.higher ? 1 : 0));
  t.m0 = (int64_t)(chunk * p.units + (chunk < p.higher ? chunk : p.higher)) * 32;  // (units of 32 rows: below 2^18)
  return t;
}
__host__ __device__ inline int tokens8_units(const Tokens8Plan& p) { return p.units + (p.higher > 0); }  // of the highest tile
// Microseconds of a tile of 32 tn channels x `units` units: a step of 64 k as timed at 1 to 8 units on weights that come from memory (its copies, its
// instructions, its products, none of them alone), and what a tile takes besides.
inline double tile8_cost(int tn, double units, int ksteps) {
  const double step = tn == 8 ? 0.45 + 0.045 * units : tn == 4 ? 0.30 + 0.033 * units : 0.20 + 0.031 * units;
  return ksteps * step + 1.5 + 0.1 * tn * units;
}
inline Tokens8Plan tokens8_plan_of(int64_t M, int64_t N, int64_t chunks, int tn, int cus) {
  const int64_t units = ceil_div(M, 32);
  Tokens8Plan p;
  p.tn = tn;
  p.tiles_n = (int)ceil_div(N, 32 * tn);
  p.chunks = (int)chunks;
  p.units = (int)(units / chunks);
  p.higher = (int)(units % chunks);
  const int64_t total = chunks * p.tiles_n;
  p.grid8 = (int)ceil_div(total < cus ? total : cus, 8);
  p.rounds = (int)(total / (8 * p.grid8));
  p.last_round = (int)(total % (8 * p.grid8));
  // an XCD's grid8 tiles: band chunks of `units` units of rows, grid8 / band blocks of tn units of channels
  int band = 1;
  while (band < chunks && (int64_t)(band + 1) * (band + 1) * p.units <= (int64_t)p.grid8 * tn) ++band;
  p.band = band;
  return p;
}
// The plan whose busiest workgroup ends first, of every kind of tile and number of rounds near the fewest.
inline Tokens8Plan tokens8_plan(int64_t M, int64_t N, int64_t K, int cus) {
  constexpr int kTallest = 8;
  const int ksteps = (int)ceil_div(K, 64);
  const int64_t units = ceil_div(M, 32), fewest = ceil_div(units, kTallest);
  Tokens8Plan best{};
  double best_cost = -1;
  for (int tn = 8; tn >= 2; tn /= 2) {
    const int64_t tiles_n = ceil_div(N, 32 * tn), least = ceil_div(fewest * tiles_n, cus);
    for (int64_t rounds = least; rounds <= least + 3; ++rounds) {
      int64_t chunks = rounds * cus / tiles_n;
      chunks = chunks < fewest ? fewest : chunks > units ? units : chunks;
      const int64_t r = ceil_div(chunks * tiles_n, cus);
      const int64_t most = r * (units / chunks) + ceil_div((units % chunks) * tiles_n, cus);  // units of the workgroup with the most
      const double cost = r * tile8_cost(tn, (double)most / r, ksteps);
      if (best_cost >= 0 && cost >= best_cost) continue;
      best_cost = cost;
      best = tokens8_plan_of(M, N, chunks, tn, cus);
    }
  }
  return best;
}

}  // namespace gpusq
