// Walks the sizes of the calls that answer with drafted tokens: how a product of 8-bit weights is cut into tiles, a row of logits into parts, layers' caches
// into launches, and which kernel a tree's attention takes.  Prints what is wrong, or ok.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdio.h>

#include <random>
#include <vector>

#include "attend_plan.h"
#include "drafts_plan.h"
#include "linear8_plan.h"
#include "sample_plan.h"

using namespace gpusq;

// every part of a row has a place of its own in the workspace, in front of the next row's
static const char* samples(int64_t rows, int64_t vocabulary) {
  const int parts = sample_parts(rows, vocabulary);
  if (parts < 1 || parts > kSampleParts || (parts & (parts - 1)) != 0) return "parts";
  if (parts > 1 && (parts * rows > 256 || vocabulary / parts < 16384)) return "more parts than are worth it";
  const SampleSpace s = sample_space(parts);
  const int64_t ends[][2] = {{s.tops, 4LL * parts}, {s.maxima, 4LL * parts * kSampleThreads}, {s.masses, 8LL * parts * kSampleBins}, {s.counts, 4LL * parts * kSampleBins}, {s.sums, 8LL * parts * kSampleWaves},
                             {s.listed, 8LL * parts}, {s.list, 8LL * parts * kSampleListed}, {s.zones, 64}, {s.bytes, 0}};
  for (int i = 0; i + 1 < (int)(sizeof(ends) / sizeof(ends[0])); ++i)
    if (ends[i][0] % 16 != 0 || ends[i][0] + ends[i][1] > ends[i + 1][0]) return "workspace";
  return s.bytes % 16 == 0 ? nullptr : "alignment of a row's workspace";
}

// a workgroup has a token of its heads on its way, launches take every cache once and count their threads
static const char* accepted(int64_t batch, int64_t kv_heads, int DP) {
  const int64_t heads = heads_of_workgroup(kv_heads, DP);
  if (heads < 1 || heads > kv_heads || heads * token_units(DP) > kUnitsOfWorkgroup) return "heads of a workgroup";
  const int64_t groups = ceil_div(kv_heads, heads), most = caches_of_launch(batch, groups);
  if (most > kCachesOfLaunch || most < 0) return "caches of a launch";
  if (most > 0 && (1 + most * groups > 65535 || batch * (1 + most * groups) * 256 > UINT32_MAX)) return "threads beyond what is counted";
  return nullptr;
}

static const char* trees(int DP, int64_t pairs, int64_t cols) {
  const AttendShape s = attend_shape(true, DP, cols, true, pairs);
  if (s.many) return cols > kTreeColumns ? nullptr : DP == 256 && cols > kFewColumns ? nullptr : "kernel for many columns";
  if (s.columns % 16 != 0 || s.columns < 16 || (DP < 256 && s.columns > 16 * tree_blocks(DP))) return "columns";
  if (s.threads != 512 && s.threads != 256) return "threads";
  // even shares: no workgroup could be left out, none of fewer blocks would do
  const int64_t blocks = ceil_div(cols, 16), groups = ceil_div(cols, s.columns);
  if (DP < 256 && groups != ceil_div(blocks, tree_blocks(DP))) return "workgroups";
  return attend_launchable(pairs, cols, s) || pairs > 1000000 ? nullptr : "refused";
}

// every block of channels of every 32 rows is one workgroup's, once, in tiles no higher than the kernel has
static const char* tokens8(int64_t M, int64_t N, int64_t K, int cus) {
  const Tokens8Plan p = tokens8_plan(M, N, K, cus);
  if (p.tn != 8 && p.tn != 4 && p.tn != 2) return "channels of a tile";
  if (tokens8_units(p) > 8 || p.chunks < 1 || p.band < 1 || p.band > p.chunks) return "heights";
  const int64_t units = ceil_div(M, 32), tiles_n = ceil_div(N, 32 * p.tn), total = p.chunks * tiles_n, places = 8 * (int64_t)p.grid8;
  if (tiles_n != p.tiles_n || p.rounds * places + p.last_round != total || places > cus + 7) return "rounds";
  std::vector<char> taken(units * tiles_n);
  for (int64_t place = 0; place < places; ++place)
    for (int64_t i = 0; i < p.rounds + (place < p.last_round ? 1 : 0); ++i) {
      const Tokens8Tile t = tokens8_tile(p, (int)(i * places + place));
      if (t.n_blk < 0 || t.n_blk >= tiles_n || t.m0 % 32 != 0 || t.slabs < 2 || t.slabs > 2 * tokens8_units(p)) return "a tile";
      for (int64_t u = t.m0 / 32; u < t.m0 / 32 + t.slabs / 2; ++u) {
        if (u >= units) return "rows that are none";
        if (taken[u * tiles_n + t.n_blk]++) return "a tile twice";
      }
    }
  for (char c : taken)
    if (!c) return "a tile left out";
  return nullptr;
}

int main() {
  std::mt19937_64 rng(1);
  auto log = [&](double bits) { return (int64_t)exp2(std::uniform_real_distribution<double>(0, bits)(rng)); };
  for (int i = 0; i < 200000; ++i) {
    const int64_t rows = log(22), vocabulary = log(18.1);
    if (const char* wrong = samples(rows, vocabulary)) return printf("%s: %lld rows of %lld\n", wrong, (long long)rows, (long long)vocabulary), 1;
    const int64_t batch = log(24), heads = log(16);
    const int DP = 64 << rng() % 3;
    if (const char* wrong = accepted(batch, heads, DP)) return printf("%s: %lld sequences, %lld heads of %d\n", wrong, (long long)batch, (long long)heads, DP), 1;
    const int64_t pairs = log(14), cols = log(15);
    if (const char* wrong = trees(DP, pairs, cols)) return printf("%s: %lld pairs, %lld columns, heads of %d\n", wrong, (long long)pairs, (long long)cols, DP), 1;
  }
  for (int i = 0; i < 4000; ++i) {
    const int64_t M = log(16), N = 4 * log(15), K = 16 * log(10);
    const int cus = i % 4 == 0 ? 1 + (int)(rng() % 300) : 256;
    if (ceil_div(M, 32) * ceil_div(N, 64) > 200000) continue;
    if (const char* wrong = tokens8(M, N, K, cus)) return printf("%s: %lld rows, %lld channels, K %lld, %d CUs\n", wrong, (long long)M, (long long)N, (long long)K, cus), 1;
  }
  printf("ok\n");
}
