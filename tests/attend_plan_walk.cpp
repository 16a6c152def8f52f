// Walks the plans of attention as its workgroups do (csrc/attend_plan.h), columns and keys, over sizes that no test launches.  Prints "ok", or what fails.
#include <math.h>
#include <stdio.h>

#include <random>

#include <hip/hip_runtime_api.h>

#include "attend_plan.h"

using namespace gpusq;

// the blocks of 16 columns of one (batch, key head) over workgroups of up to `most`: each met once, in order, in shares that are alike
static const char* columns(int64_t cols, int most) {
  const int64_t col_tiles = ceil_div(cols, 16), groups = ceil_div(col_tiles, most);
  int next = 0;
  for (int64_t b = 0; b < groups; ++b) {
    const ColumnShare s = column_share((int)col_tiles, (int)groups, (int)b);
    if (s.first != next) return "blocks of columns left out or met twice";
    if (s.last - s.first < col_tiles / groups || s.last - s.first > ceil_div(col_tiles, groups) || s.last - s.first > most) return "share";
    next = s.last;
  }
  return next == col_tiles ? nullptr : "blocks of columns not covered";
}

// `most` keys over parts of part_tiles tiles: each key in one part, and what a loop looks ahead of its last tile is a number
static const char* keys(int most, int part_tiles, int parts) {
  int64_t next = 0;
  for (int p = 0; p < parts; ++p) {
    const KeyRange k = keys_of_part(p, part_tiles, most);
    if (k.begin >= most) {
      if (k.end > k.begin) return "keys that are not there";
      continue;
    }
    if (k.begin != next || k.end <= k.begin || k.end - (int64_t)k.begin > (int64_t)part_tiles * 32) return "keys of a part";
    if (k.end != most && k.end % 64 != 0) return "half a page";
    if ((int64_t)k.end - 1 + kMostAhead > INT32_MAX) return "keys ahead";
    next = k.end;
  }
  return next == (most > 0 ? most : 0) ? nullptr : "keys not covered";
}

// every vector of tokens * per_token in a launch that counts its threads, and vectors in 31 bits
static const char* norms(int64_t per_token, int64_t in_workgroup) {
  const int64_t most = qk_norm_tokens(per_token, in_workgroup);
  if (most < 1) return "no token";
  const int64_t workgroups = ceil_div(most * per_token, in_workgroup);
  if (workgroups * 256 > UINT32_MAX || workgroups * in_workgroup > INT32_MAX) return "threads or vectors beyond what is counted";
  const int64_t more = ceil_div((most + 1) * per_token, in_workgroup);
  return more * 256 <= UINT32_MAX && (most + 1) * per_token <= INT32_MAX - 256 ? "fewer tokens than a launch takes" : nullptr;
}

// workgroups that are launched: enough for every block of columns of every unit, and their numbers and columns in 31 bits
static const char* launches(bool kv4, int DP, int64_t units, int64_t cols, bool reach) {
  const AttendShape s = attend_shape(kv4, DP, cols, reach);
  const int64_t col_blocks = ceil_div(cols, s.columns);
  if (!attend_launchable(units, cols, s)) return units * 1.0 * col_blocks * s.threads > 4.0e9 ? nullptr : "refused";
  const int64_t workgroups = attend_workgroups(units, col_blocks);
  if (workgroups < units * col_blocks || workgroups > units * col_blocks + 8 * col_blocks) return "number of workgroups";
  if (workgroups * s.threads > UINT32_MAX) return "threads beyond what a launch counts";
  return col_blocks * s.columns > INT32_MAX - 15 ? "columns beyond 31 bits" : nullptr;
}

int main() {
  // around where products with the number of blocks pass 2^31 and 2^32, and up to what 31 bits of columns allow
  for (const int most : {4, 8, 16})
    for (const int64_t near : {(int64_t)1, (int64_t)1 << 10, (int64_t)1 << 20, (int64_t)1 << 21, (int64_t)3 << 20, (int64_t)1 << 22, (int64_t)1 << 23,  (int64_t)1 << 26, (int64_t)1 << 31})
      for (int64_t cols = near - 300; cols < near + 300; cols += near < 1 << 24 ? 7 : 293) {
        if (cols < 1 || cols > INT32_MAX - 127) continue;
        if (const char* wrong = columns(cols, most)) return printf("%s: %lld columns, %d a workgroup\n", wrong, (long long)cols, 16 * most), 1;
      }
  std::mt19937_64 rng(1);
  // lengths up to the longest that is taken, columns that see none of them
  for (int i = 0; i < 100000; ++i) {
    const int length = i < 2000 ? kMostStates - i : (int)exp2(std::uniform_real_distribution<double>(0, 30.999)(rng));
    const int64_t tiles = ceil_div(length, 32), part_tiles = ceil_div(ceil_div(tiles, 1 + (int64_t)(rng() % 256)), 2) * 2;
    const int seen[] = {length, (int)(rng() % length), 0, -(int)(rng() % length)};
    for (const int most : seen)
      if (const char* wrong = keys(most, (int)part_tiles, (int)ceil_div(tiles, part_tiles)))
        return printf("%s: %d of %d keys, parts of %d tiles\n", wrong, most, length, (int)part_tiles), 1;
  }
  for (int i = 0; i < 2000; ++i) {
    const int64_t cols = (int64_t)exp2(std::uniform_real_distribution<double>(0, 24)(rng));
    if (const char* wrong = columns(cols, 4 << (rng() % 3))) return printf("%s: %lld columns\n", wrong, (long long)cols), 1;
  }
  for (int64_t per_token = 2; per_token <= 3 * 65536; per_token += per_token < 100 ? 1 : 97)
    for (const int64_t in_workgroup : {8, 12, 32, 64, 256})
      if (const char* wrong = norms(per_token, in_workgroup)) return printf("%s: %lld vectors a token\n", wrong, (long long)per_token), 1;
  for (int i = 0; i < 200000; ++i) {
    const int64_t units = (int64_t)exp2(std::uniform_real_distribution<double>(0, 32)(rng)), cols = (int64_t)exp2(std::uniform_real_distribution<double>(0, 31)(rng));
    if (const char* wrong = launches(rng() % 2, 64 << (rng() % 3), units, cols, rng() % 4 != 0)) return printf("%s: %lld units, %lld columns\n", wrong, (long long)units, (long long)cols), 1;
  }
  for (const int64_t cols : {INT32_MAX, INT32_MAX - 15, INT32_MAX - 127, INT32_MAX - 255, INT32_MAX - 2047})
    for (int k = 0; k < 12; ++k)
      if (const char* wrong = launches(k & 1, 64 << (k >> 2), 1, cols, k & 2)) return printf("%s: %lld columns\n", wrong, (long long)cols), 1;
  const int64_t pages = INT32_MAX / 64 - 1;  // of a sequence, at most; a loop is at one's beginning
  if (64 * (pages - 1) + kMostAhead > INT32_MAX) return printf("pages ahead\n"), 1;
  printf("ok\n");
}
