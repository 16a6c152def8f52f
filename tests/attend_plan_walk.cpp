// Walks the plans of attention as its workgroups do (csrc/attend_plan.h), over sizes that no test launches.  Prints "ok", or what fails.
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

int main() {
  // around where products with the number of blocks pass 2^31 and 2^32, and up to what 31 bits of columns allow
  for (const int most : {4, 8, 16})
    for (const int64_t near : {(int64_t)1, (int64_t)1 << 10, (int64_t)1 << 20, (int64_t)1 << 21, (int64_t)3 << 20, (int64_t)1 << 22, (int64_t)1 << 23,  (int64_t)1 << 26, (int64_t)1 << 31})
      for (int64_t cols = near - 300; cols < near + 300; cols += near < 1 << 24 ? 7 : 293) {
        if (cols < 1 || cols > INT32_MAX - 127) continue;
        if (const char* wrong = columns(cols, most)) return printf("%s: %lld columns, %d a workgroup\n", wrong, (long long)cols, 16 * most), 1;
      }
  std::mt19937_64 rng(1);
  for (int i = 0; i < 2000; ++i) {
    const int64_t cols = (int64_t)exp2(std::uniform_real_distribution<double>(0, 24)(rng));
    if (const char* wrong = columns(cols, 4 << (rng() % 3))) return printf("%s: %lld columns\n", wrong, (long long)cols), 1;
  }
  printf("ok\n");
}
