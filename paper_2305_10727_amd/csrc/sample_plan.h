// How the rows of sample_tokens are cut over workgroups, and their workspace.  Plain C++.
#pragma once
#include <stdint.h>

#include "launch_rules.h"

namespace gpusq {

constexpr int kSampleThreads = 1024, kSampleWaves = kSampleThreads / 64, kSampleBins = 2048, kSampleListed = 4096, kSampleParts = 8;

// Parts of a row, a workgroup each.  One is one launch, more are four: worth it where the rows leave most of the device idle and a part has work for
// longer than a launch takes.  (Top-k and top-p of one row, us, in 1, 2, 4, 8 parts: 32000 tokens 27, 34, 35, 41; 131072 47, 46, 40, 43, and with top-p
// alone 78, 59, 44, 40; 64 rows of 100003 tokens 69, 60, 54, 82.)
inline int sample_parts(int64_t rows, int64_t vocabulary) {
  int parts = 1;
  if (vocabulary < 65536) return parts;
  while (parts < kSampleParts && 2 * parts * rows <= 256 && vocabulary / (2 * parts) >= 16384) parts *= 2;
  return parts;
}

// What the workgroups of a row leave for each other, in bytes from the row's beginning (each a multiple of 16)
struct SampleSpace {
  int64_t tops;    // uint32 [parts]: the greatest logit's order
  int64_t maxima;  // float [parts][threads]: each thread's greatest logit
  int64_t masses;  // uint64 [parts][bins]
  int64_t counts;  // uint32 [parts][bins]
  int64_t sums;    // uint64 [parts * waves]
  int64_t listed;  // uint32 [parts][2]: tokens of the list, those of the k-th's bin
  int64_t list;    // uint64 [parts][listed]
  int64_t zones;   // what the histogram says
  int64_t bytes;
};
__host__ __device__ inline SampleSpace sample_space(int parts) {
  SampleSpace s;
  s.tops = 0;
  s.maxima = 4 * kSampleParts;
  s.masses = s.maxima + (int64_t)parts * kSampleThreads * 4;
  s.counts = s.masses + (int64_t)parts * kSampleBins * 8;
  s.sums = s.counts + (int64_t)parts * kSampleBins * 4;
  s.listed = s.sums + (int64_t)parts * kSampleWaves * 8;
  s.list = s.listed + 8 * kSampleParts;
  s.zones = s.list + (int64_t)parts * kSampleListed * 8;
  s.bytes = s.zones + 64;
  return s;
}

}  // namespace gpusq
