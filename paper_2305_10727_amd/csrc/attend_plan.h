// How attention deals out its columns, as the host plans it and as the kernels read it.  Plain C++, so that a host program can walk sizes that no
// test would launch.
#pragma once
#include <stdint.h>

#include "launch_rules.h"

namespace gpusq {

// The blocks of 16 columns that workgroup `block` of `groups` takes, 4 or more each but for a rest: first .. last - 1, in order, shares that are alike.
// Products with the number of blocks are taken while they fit 32 bits (up to 2^17 blocks: 65536 queries of 32 heads over one); beyond, the
// first workgroups have the rest, as a division in 64 bits would be code that every workgroup fetches.
struct ColumnShare {
  int first, last;
};
__host__ __device__ inline ColumnShare column_share(int col_tiles, int groups, int block) {
  ColumnShare s;
  if (col_tiles < 0x20000 || groups < 0x4000) {
    s.first = (int)((unsigned)block * (unsigned)col_tiles / (unsigned)groups);
    s.last = (int)((unsigned)(block + 1) * (unsigned)col_tiles / (unsigned)groups);
  } else {
    const int each = col_tiles / groups, rest = col_tiles - each * groups;
    s.first = block * each + (block < rest ? block : rest);
    s.last = s.first + each + (block < rest ? 1 : 0);
  }
  return s;
}

// The keys of part `part` of part_tiles tiles of 32 keys, of columns that see `most` keys.  (The sum of a part's beginning and its length
// passes 31 bits, not 32.)
struct KeyRange {
  int begin, end;
};
__host__ __device__ inline KeyRange keys_of_part(int part, int part_tiles, int most) {
  KeyRange k;
  k.begin = part * part_tiles * 32;
  const unsigned end = (unsigned)k.begin + (unsigned)part_tiles * 32;
  k.end = most < 0 || end > (unsigned)most ? most : (int)end;
  return k;
}
// A loop over the keys looks kMostAhead keys beyond a tile's first (four tiles of 32, two of 64), so fp16 states are kMostStates at most; a cache's
// are whole pages of 64, fewer than that.
constexpr int kMostAhead = 128, kMostStates = INT32_MAX - kMostAhead;

}  // namespace gpusq
