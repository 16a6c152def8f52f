// Sizes of the calls for trees of drafted tokens.  Plain C++.
#pragma once
#include <stdint.h>

#include "launch_rules.h"

namespace gpusq {

constexpr int kMostDrafts = 512;       // nodes of a tree: its sets twice are 64 KB of LDS
constexpr int kCachesOfLaunch = 128;   // layers' caches that one launch moves tokens in: their addresses are kernel arguments

struct DraftArgs {
  const int32_t *kv_lens, *cu_q;
  int tokens, batch, max_q;
};
// 16-bit units of a cache that a workgroup of 256 has on its way, and heads of a layer that it takes: one token of theirs at least
constexpr int kUnitsOfWorkgroup = 2048;
constexpr int token_units(int DP) { return DP / 2 + DP / 16; }
inline int64_t heads_of_workgroup(int64_t kv_heads, int DP) {
  const int64_t most = kUnitsOfWorkgroup / token_units(DP);
  return kv_heads < most ? kv_heads : most;
}
// How many caches a launch takes (grid: batch x 1 + caches * groups of heads workgroups of 256, the second dimension counted up to 65535); 0: not one
inline int64_t caches_of_launch(int64_t batch, int64_t groups) {
  const int64_t counted = UINT32_MAX / 256 / batch, rows = (counted < 65535 ? counted : 65535) - 1, n = rows / groups;
  return n < kCachesOfLaunch ? n : kCachesOfLaunch;
}
struct CacheList {
  void* of[kCachesOfLaunch];
};

}  // namespace gpusq
