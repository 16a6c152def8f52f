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

// The kernels: few columns of a (batch, key head) with the keys dealt out over a workgroup's wavefronts, many with columns of their own for each.
constexpr int kFewColumns = 32;
constexpr int tiles_columns(bool kv4, int DP) { return (DP > 128 ? 64 : 128) * (kv4 ? 2 : 1); }
constexpr int tiles_threads(bool kv4) { return kv4 ? 512 : 256; }
// The kernel for many has the keys of a tile in 32-bit offsets: strides from token to token, in values, that it takes
inline bool tiles_reach(int64_t k_token, int64_t v_token) { return k_token < (1 << 24) && v_token < (1 << 24); }
struct AttendShape {
  bool many;
  int columns, threads;  // of a workgroup
};
inline AttendShape attend_shape(bool kv4, int DP, int64_t cols, bool reach) {
  if (cols > kFewColumns && reach) return AttendShape{true, tiles_columns(kv4, DP), tiles_threads(kv4)};
  // (two blocks of 16 columns of heads of 256 do not fit the registers of a wavefront)
  return cols <= 16 || DP == 256 ? AttendShape{false, 16, 512} : AttendShape{false, 32, 256};
}

// Workgroups: `units` are (batch, key head, part of the keys).  Many units are dealt out over the 8 XCDs in turn, few in equal shares.
__host__ __device__ inline bool attend_in_turn(int64_t units) { return units >= 64 || units % 8 == 0; }
inline int64_t attend_workgroups(int64_t units, int64_t col_blocks) {
  return attend_in_turn(units) ? ceil_div(units, 8) * 8 * col_blocks : ceil_div(units * col_blocks, 8) * 8;
}
// Whether a launch counts them, at `columns` columns a block (the product is formed of what fits)
inline bool attend_launchable(int64_t units, int64_t cols, const AttendShape& shape) {
  const int64_t col_blocks = ceil_div(cols, shape.columns);
  return units <= INT32_MAX && col_blocks <= INT32_MAX && launchable(attend_workgroups(units, col_blocks), shape.threads);
}
// The launch that joins `parts` parts of `rows` rows: for few of them a workgroup for as many rows as have 256 quads of channels, else one each
constexpr int kFewParts = 8;
inline int64_t join_workgroups(int64_t rows, int64_t D, int parts) { return parts <= kFewParts ? ceil_div(rows, 256 / (D / 4)) : rows; }

}  // namespace gpusq
