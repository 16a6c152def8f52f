// Tokens drawn from logits by temperature, top-k, top-p and min-p, with random numbers that are given.
//
//   w_i = exp((x_i - max x) / T), 0 below 2^-40;  the tokens in the order of their logits, ties by their index, are cut behind the first k, behind the
//   first whose weights reach p of the first k's, and in front of the first whose weight is below min_p;  drawn is the first token, in the
//   vocabulary's order, up to which the kept weights pass u of their sum.
//
// Where two tokens' shares meet is closer to a neighbour's than 32 bits tell apart, so weights are formed to 2^-31 of themselves, rounded to whole
// numbers of 2^-44 of the greatest's (one of 2^-40 to 2^-5 of itself; in their sum that is 2^-45 a token) and summed as these, of which no order changes
// the sum.  A token's place in the order is one number, its logit's bits made monotone and its index counted down: a cut is the least such number that
// is kept.
//
// A row is read three times: for its greatest logit; for a histogram of the logits' distances from it, in 2048 bins of 28 / 2048 of the temperature, from
// which the bin of the k-th token and the bins between which the p-th share ends are known; for the sums, and the tokens of those bins, which are sorted
// and decide.  A wavefront sums a stretch of the vocabulary; the token lies in the stretch that passes the random share, which is looked at once more.
// What bounds it is the instructions of the weights, 22 a token and pass, and of the histogram's atomics in LDS; the first reading is memory's.  So few rows
// are cut into parts, a workgroup each, in a launch for each reading and one that decides; and a thread whose greatest logit is behind the bins that are
// asked reads nothing more.  256 rows of 131072 fp32 logits (134 MB, 27 us at a copy's rate): 60 us without a cut, 70 with top-k, 106 with top-p, 102 with
// all; 256 of 32000 fp16 19, 30, 37, 39; one of 32000 16, 21, 31, 26, of 131072 18, 33, 40, 43; greedy ones, of one reading, 5.3, of 131072 over several workgroups 12.7.
#include "common.h"
#include "sample_plan.h"

#include <type_traits>

namespace gpusq {

namespace {

constexpr int kThreads = kSampleThreads, kWaves = kSampleWaves, kBins = kSampleBins, kListed = kSampleListed;
constexpr float kBinsOfUnit = kBins / 28.0f;  // (2^-40 is 27.73 below the greatest)
typedef unsigned long long u64;

// The logits' order: greater numbers first; -0 is 0, what is no number is -infinity
__device__ __forceinline__ unsigned key_of(float x) {
  x = x == x ? x + 0.0f : -__builtin_inff();
  const unsigned u = __float_as_uint(x);
  return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(unsigned key) { return __uint_as_float(key >> 31 ? key & 0x7fffffffu : ~key); }
__device__ __forceinline__ u64 place_of(float x, int i) { return (u64)key_of(x) << 32 | (unsigned)~i; }
__device__ __forceinline__ int index_of(u64 place) { return (int)~(unsigned)place; }
__device__ __forceinline__ float logit_of(u64 place) { return value_of((unsigned)(place >> 32)); }

// A step of a scan over the wavefront's lanes: the value of the lane that CTRL names, 0 where there is none or ROWS leaves the lane out
template <int CTRL, int ROWS>
__device__ __forceinline__ u64 from_lane(u64 v) {
  const int lo = __builtin_amdgcn_update_dpp(0, (int)(unsigned)v, CTRL, ROWS, 0xF, false), hi = __builtin_amdgcn_update_dpp(0, (int)(v >> 32), CTRL, ROWS, 0xF, false);
  return (u64)(unsigned)hi << 32 | (unsigned)lo;
}
// Of the lanes up to this one; op of 0 changes nothing.  (row_shr 1, 2, 4, 8, then the rows' last lanes: a fifth of the time of ds_bpermute's trips)
template <class Op>
__device__ __forceinline__ u64 scan(u64 v, Op op) {
  v = op(v, from_lane<0x111, 0xF>(v));
  v = op(v, from_lane<0x112, 0xF>(v));
  v = op(v, from_lane<0x114, 0xF>(v));
  v = op(v, from_lane<0x118, 0xF>(v));
  v = op(v, from_lane<0x142, 0xA>(v));
  return op(v, from_lane<0x143, 0xC>(v));
}
__device__ __forceinline__ u64 last_lane(u64 v) {
  return (u64)(unsigned)__builtin_amdgcn_readlane((int)(v >> 32), 63) << 32 | (unsigned)__builtin_amdgcn_readlane((int)(unsigned)v, 63);
}
__device__ __forceinline__ u64 sum_of(u64 a, u64 b) { return a + b; }
__device__ __forceinline__ u64 max_of(u64 a, u64 b) { return a > b ? a : b; }

struct Block {
  u64 part[kWaves];
  template <class Op>
  __device__ __forceinline__ u64 all(u64 v, Op op) {  // of all threads, to all threads
    v = last_lane(scan(v, op));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int i = 1; i < kWaves; ++i) v = op(v, part[i]);
    return v;
  }
  // sum of the threads in front of this one, and of all
  __device__ __forceinline__ u64 before(u64 v, u64* total = nullptr) {
    const int wave = threadIdx.x >> 6;
    const u64 upto = scan(v, sum_of);
    __syncthreads();
    if ((threadIdx.x & 63) == 63) part[wave] = upto;
    __syncthreads();
    u64 sum = upto - v, whole = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
      const u64 p = part[i];
      sum += i < wave ? p : 0;
      whole += p;
    }
    if (total != nullptr) *total = whole;
    return sum;
  }
  // how many of the threads' two answers are true
  __device__ __forceinline__ int count(bool a, bool b) {
    const int n = __popcll(__builtin_amdgcn_ballot_w64(a)) + __popcll(__builtin_amdgcn_ballot_w64(b));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = n;
    __syncthreads();
    int sum = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) sum += (int)part[i];
    return sum;
  }
  // the first thread for which it is so, or where none is the last for which `otherwise` is; -1: none
  __device__ __forceinline__ int first(bool is, bool otherwise) {
    const u64 yes = __builtin_amdgcn_ballot_w64(is), other = __builtin_amdgcn_ballot_w64(otherwise);
    const unsigned wave = threadIdx.x >> 6, lowest = yes != 0 ? 64 * wave + __builtin_ctzll(yes) : 0xFFFFu, highest = other != 0 ? 64 * wave + 64 - __builtin_clzll(other) : 0;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[wave] = lowest << 16 | highest;
    __syncthreads();
    unsigned lo = 0xFFFFu, hi = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
      const unsigned p = (unsigned)part[i];
      lo = lo < p >> 16 ? lo : p >> 16;
      hi = hi > (p & 0xFFFFu) ? hi : p & 0xFFFFu;
    }
    return lo != 0xFFFFu ? (int)lo : (int)hi - 1;
  }
};

struct Shared {
  Block block;
  double table[128];  // 2^(j / 128)
  u64 masses[kBins];
  unsigned counts[kBins];
  u64 list[kListed];
  u64 sums[kSampleParts * kWaves], found[2];
  unsigned listed, of_k_bin;
};

// exp(y) is 2^e times 2^(j / 128), from a table, times 2^(f / 128), 0 <= f < 1, of one fused step: 128 y / ln 2 in whole numbers of 2^-24 stands in the last
// places of a number of 64 bits, f in 24 of them, j in the next 7, e behind.  2^(f / 128) - 1, at most 0.0054, is three terms of its series in 32 bits: off by
// 2^-31 of the weight, by nothing for the greatest.
struct Weights {
  float top, limit, scale;  // the greatest logit; the distance of 2^-40 from it; bins of a distance
  double steps;             // 128 / (T ln 2)
  const double* table;
  __device__ __forceinline__ Weights(float top_, float temperature, const double* table_)
      : top(top_), limit(fminf(27.725887f * temperature, 3.4028235e38f)), scale(kBinsOfUnit / temperature), steps(184.664965233787314 / (double)temperature), table(table_) {}
  // (not so for what is no number, or -infinity)
  __device__ __forceinline__ bool has(float x) const { return top - x <= limit; }
  // of a logit that has one (of another any number): whole numbers of 2^-44, and kNone
  __device__ __forceinline__ u64 beyond_none(float x) const {
    const double s = __builtin_fma((double)x - (double)top, steps, 0x1.8p28);  // the last place is 2^-24
    const unsigned lo = (unsigned)__double2loint(s), hi = (unsigned)__double2hiint(s);
    const float f = (float)(lo & 0xFFFFFFu), q = f * __builtin_fmaf(f, __builtin_fmaf(f, 0x1.c6b08ep-98f, 0x1.ebfbep-65f), 0x1.62e430p-32f);
    const double c = table[lo >> 24 & 127], w = __builtin_fma(c, (double)q, c);
    const double scaled = __hiloint2double(__double2hiint(w) + (int)(__builtin_amdgcn_alignbit(hi, lo, 31) << 20), __double2loint(w));  // times 2^e
    return (u64)__double_as_longlong(scaled + 256.0);  // the last place is 2^-44
  }
  static constexpr u64 kNone = 0x4070000000000000ull;  // 256 in 64 bits
  __device__ __forceinline__ u64 of(float x) const { return beyond_none(x) - kNone; }
  __device__ __forceinline__ u64 operator()(float x) const { return has(x) ? of(x) : 0; }
  // ... a logit's bin, in the logits' order
  __device__ __forceinline__ float distance(float x) const { return (top - x) * scale; }
};

// A row of logits by vectors of 16 bytes, wherever it begins; of a part of it a wavefront has a stretch, its lanes a vector each at a time.
// each(value, index) is called of a lane's values one after the other, unrolled; indices in front of the row and behind it have -infinity.
template <typename T>
struct Row {
  static constexpr int VEC = 16 / (int)sizeof(T), AHEAD = 4;
  typedef T vec __attribute__((ext_vector_type(VEC)));
  const T* x;
  int V, off, vecs, per_wave;  // values in front of the row in its first vector; vectors of it, of a wavefront
  int begin;                   // the wavefront's first vector
  __device__ __forceinline__ Row(const SampleArgs& a, int row, int part, int parts)
      : x((const T*)a.logits + (int64_t)row * a.row_stride), V(a.V), off((int)(((uintptr_t)x & 15) / sizeof(T))), vecs((V + off + VEC - 1) / VEC) {
    per_wave = ((vecs + parts * kWaves - 1) / (parts * kWaves) + 63) & ~63;
    // (Wavefronts whose stretches begin a multiple of 16 KB apart ask the same channels of the memory at once: 256 rows of 131072 31 us a reading, 25 so)
    per_wave += per_wave % 1024 == 0 ? 64 : 0;
    begin = (part * kWaves + (threadIdx.x >> 6)) * per_wave;
  }
  __device__ __forceinline__ vec load(int v) const {
    const int i = v * VEC - off;
    if (i >= 0 && i + VEC <= V) return *(const vec*)(x + i);
    vec r;
#pragma unroll
    for (int e = 0; e < VEC; ++e) r[e] = i + e >= 0 && i + e < V ? x[i + e] : (T)-__builtin_inff();
    return r;
  }
  // For much work a value: each(values, index of the first) a vector at a time, the next two on their way
  template <class Each>
  __device__ __forceinline__ void step(Each each) const {
    const int end = begin + per_wave < vecs ? begin + per_wave : vecs;
    int v = begin + (threadIdx.x & 63);
    if (v >= end) return;
    vec now = load(v), next = load(v + 64 < end ? v + 64 : v);
#pragma unroll 1
    for (; v < end; v += 64) {
      const vec later = load(v + 128 < end ? v + 128 : v);
      float x[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) x[e] = (float)now[e];
      each(x, v * VEC - off);
      now = next;
      next = later;
    }
  }
  template <class Each>
  __device__ __forceinline__ void walk(Each each) const {
    const int end = begin + per_wave < vecs ? begin + per_wave : vecs;
    for (int v0 = begin + (threadIdx.x & 63); v0 < end; v0 += 64 * AHEAD) {
      vec r[AHEAD];
#pragma unroll
      for (int j = 0; j < AHEAD; ++j) {
        if (v0 + 64 * j < end) {
          r[j] = load(v0 + 64 * j);
        } else {
#pragma unroll
          for (int e = 0; e < VEC; ++e) r[j][e] = (T)-__builtin_inff();
        }
      }
#pragma unroll
      for (int j = 0; j < AHEAD; ++j)
#pragma unroll
        for (int e = 0; e < VEC; ++e) each((float)r[j][e], (v0 + 64 * j) * VEC - off + e);
    }
  }
  __device__ __forceinline__ int stretch_of(int i) const { return (i + off) / (per_wave * VEC); }
  __device__ __forceinline__ int first_of(int stretch) const {
    const int64_t i = (int64_t)stretch * per_wave * VEC - off;
    return i < 0 ? 0 : i < V ? (int)i : V;
  }
  // begins with another wavefront of the row
  __device__ __forceinline__ void to_part(int part) { begin = (part * kWaves + (threadIdx.x >> 6)) * per_wave; }
};

// What a row asks for
struct Asked {
  float temperature;
  int k;        // 0: all
  bool shares;  // whether a share of the weight is cut
  double p;
  u64 least;  // weight that min_p asks for
  float random;
  __device__ __forceinline__ Asked(const SampleArgs& a, int row) {
    temperature = 1.0f;
    int k_given = 0;
    float p_given = 1.0f, m = 0.0f;
    random = a.random[row];  // (all of them requested before one is looked at)
    if (a.temperature != nullptr) temperature = a.temperature[row];
    if (a.top_k != nullptr) k_given = a.top_k[row];
    if (a.top_p != nullptr) p_given = a.top_p[row];
    if (a.min_p != nullptr) m = a.min_p[row];
    k = k_given > 0 && k_given < a.V ? k_given : 0;
    shares = p_given < 1.0f;
    p = p_given > 0.0f ? (double)p_given : 0.0;
    least = m > 0.0f ? (u64)ceil((m < 1.0f ? (double)m : 1.0) * 0x1p44) : 0;
  }
  __device__ __forceinline__ bool greedy() const { return !(temperature > 0.0f); }
  __device__ __forceinline__ bool cuts() const { return k != 0 || shares; }
  __device__ __forceinline__ float heat() const { return fmaxf(temperature, 0x1p-100f); }
};

__device__ __forceinline__ void clear(Shared& sh, bool histogram) {
  const int tid = threadIdx.x;
  if (tid < 128) sh.table[tid] = exp2(tid * (1.0 / 128));
  if (histogram) {
#pragma unroll
    for (int i = 0; i < kBins; i += kThreads) {
      sh.masses[tid + i] = 0;
      sh.counts[tid + i] = 0;
    }
  }
  if (tid == 0) sh.listed = sh.of_k_bin = 0;
  __syncthreads();
}

template <typename T>
__device__ __forceinline__ float greatest_of_thread(const Row<T>& row) {
  float mine = -__builtin_inff();
  row.walk([&](float x, int) { mine = fmaxf(mine, x); });  // (a NaN is left out)
  return mine;
}

// The first bin for which it is so, and so for all behind it; kBins: none
template <class Reached>
__device__ __forceinline__ int first_bin(Shared& sh, Reached reached) {
  return sh.block.count(!reached(2 * threadIdx.x), !reached(2 * threadIdx.x + 1));
}
__device__ __forceinline__ void cumulate_counts(Shared& sh) {
  const int b = 2 * threadIdx.x;
  __syncthreads();
  const unsigned c0 = sh.counts[b], c1 = sh.counts[b + 1], before = (unsigned)sh.block.before(c0 + c1);
  sh.counts[b] = before + c0;
  sh.counts[b + 1] = before + c0 + c1;
  __syncthreads();
}

// Of the greatest logits of the threads (maxima(i), n of this one) the k-th lies in the row's k-th's bin or behind it: behind it nothing is asked.
template <class Maxima>
__device__ __forceinline__ int bins_asked(Shared& sh, const Asked& asked, const Weights& weight, int n, Maxima maxima) {
  if (asked.k == 0 || asked.k > n * kThreads) return kBins;
  for (int i = 0; i < n; ++i) {
    const float d = weight.distance(maxima(i));
    if (d < (float)kBins) atomicAdd(&sh.counts[(int)d], 1u);
  }
  cumulate_counts(sh);
  const int last = first_bin(sh, [&](int b) { return sh.counts[b] >= (unsigned)asked.k; });
  sh.counts[2 * threadIdx.x] = sh.counts[2 * threadIdx.x + 1] = 0;
  __syncthreads();
  return last < kBins ? last + 1 : kBins;
}

// (mine: the thread's greatest; a thread whose greatest is behind what is asked reads nothing, here and below)
template <typename T>
__device__ __forceinline__ void histogram(Shared& sh, const Row<T>& row, const Asked& asked, const Weights& weight, float mine, int behind) {
  constexpr int VEC = Row<T>::VEC;
  const float most = (float)behind;
  if (!(weight.distance(mine) < most)) return;
  if (asked.k != 0) {
    row.step([&](const float (&x)[VEC], int) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float d = weight.distance(x[e]);
        if (d < most) {
          atomicAdd(&sh.counts[(int)d], 1u);
          if (asked.shares && weight.has(x[e])) atomicAdd(&sh.masses[(int)d], weight.of(x[e]));
        }
      }
    });
  } else {
    row.step([&](const float (&x)[VEC], int) {
      u64 w[VEC];  // (formed side by side, without a branch)
#pragma unroll
      for (int e = 0; e < VEC; ++e) w[e] = weight.of(x[e]);
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (weight.has(x[e])) atomicAdd(&sh.masses[(int)weight.distance(x[e])], w[e]);
    });
  }
}

// What the whole row's histogram says
struct Zones {
  int k_bin, z0, z1;  // the k-th token's bin (kBins: none); the bins that the share's end may lie in
  int sure;           // tokens of bins in front of this one are kept, of those behind it those of the list alone
  int before_k;       // tokens in front of the k-th's bin
  u64 front, between, all;  // weight in front of `sure`, between the share's bins and the k-th's, of all
  __device__ __forceinline__ bool lists(int b) const { return b == k_bin || (b >= z0 && b <= z1); }
};
__device__ __forceinline__ Zones zones_of(Shared& sh, const Asked& asked) {
  Zones z{kBins, kBins, -1, kBins, 0, 0, 0, 0};
  if (asked.k != 0) {
    cumulate_counts(sh);
    z.k_bin = first_bin(sh, [&](int b) { return sh.counts[b] >= (unsigned)asked.k; });
    z.before_k = z.k_bin < kBins && z.k_bin > 0 ? (int)sh.counts[z.k_bin - 1] : 0;
  }
  if (asked.shares) {
    __syncthreads();
    const int b = 2 * threadIdx.x;
    const u64 m0 = sh.masses[b], m1 = sh.masses[b + 1], before = sh.block.before(m0 + m1);
    sh.masses[b] = before + m0;
    sh.masses[b + 1] = before + m0 + m1;
    __syncthreads();
    // the k tokens' weight lies between what is in front of the k-th's bin and what is up to it
    const u64 most = sh.masses[z.k_bin < kBins ? z.k_bin : kBins - 1], fewest = z.k_bin == kBins ? most : z.k_bin > 0 ? sh.masses[z.k_bin - 1] : 0;
    const double t0 = fmax(asked.p * (double)fewest, 1.0), t1 = fmax(asked.p * (double)most, 1.0);  // (a share of nothing: the greatest's bin)
    z.z0 = first_bin(sh, [&](int i) { return (double)sh.masses[i] >= t0; });
    z.z1 = first_bin(sh, [&](int i) { return (double)sh.masses[i] >= t1; });
    z.z0 = z.z0 < z.k_bin ? z.z0 : z.k_bin;
    z.z1 = z.z1 < z.k_bin ? z.z1 : z.k_bin;
  }
  z.sure = z.z0 < z.k_bin ? z.z0 : z.k_bin;
  if (asked.shares) {
    z.front = z.sure > 0 ? sh.masses[z.sure - 1] : 0;
    z.between = z.k_bin < kBins && z.k_bin > 0 && z.z1 < z.k_bin ? sh.masses[z.k_bin - 1] - sh.masses[z.z1] : 0;
    z.all = sh.masses[kBins - 1];
  }
  return z;
}

// The sum of the wavefront's stretch, of the tokens that are sure; the tokens of the list's bins to the list
template <typename T>
__device__ __forceinline__ u64 gather(Shared& sh, const Row<T>& row, const Asked& asked, const Weights& weight, float mine, const Zones& z) {
  constexpr int VEC = Row<T>::VEC;
  u64 sum = 0;
  const u64 least = asked.least;
  const float sure = (float)z.sure, last = (float)((z.k_bin < kBins ? z.k_bin : z.z1) + 1);
  auto list = [&](float x, int bin, int i) {
    if (bin == z.k_bin) atomicAdd(&sh.of_k_bin, 1u);
    const unsigned at = atomicAdd(&sh.listed, 1u);
    if (at < kListed) sh.list[at] = place_of(x, i);
  };
  const float nearest = weight.distance(mine);
  if (z.k_bin == kBins) {  // Most tokens weigh: their weights side by side, without a branch, and what each has too much is taken off at the end
    const u64 enough = least + Weights::kNone;
    u64 none = 0;
    if (z.sure == kBins) {
      if (nearest < sure) row.step([&](const float (&x)[VEC], int) {
        none += VEC * Weights::kNone;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const u64 w = weight.beyond_none(x[e]);
          sum += (int)weight.has(x[e]) & (int)(w >= enough) ? w : Weights::kNone;
        }
      });
    } else {
      if (nearest < last) row.step([&](const float (&x)[VEC], int i0) {
        none += VEC * Weights::kNone;
        bool some = false;
        float d[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          d[e] = weight.distance(x[e]);
          const u64 w = weight.beyond_none(x[e]);
          sum += (int)(d[e] < sure) & (int)(w >= enough) ? w : Weights::kNone;
          some |= (int)(d[e] >= sure) & (int)(d[e] < last);
        }
        if (some) {
#pragma unroll
          for (int e = 0; e < VEC; ++e)
            if (d[e] >= sure && d[e] < last && z.lists((int)d[e])) list(x[e], (int)d[e], i0 + e);
        }
      });
    }
    sum -= none;
  } else {
    if (nearest < last) row.step([&](const float (&x)[VEC], int i0) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float d = weight.distance(x[e]);
        if (d < last) {
          if (d < sure) {
            const u64 w = weight(x[e]);
            sum += w >= least ? w : 0;
          } else if (z.lists((int)d)) {
            list(x[e], (int)d, i0 + e);
          }
        }
      }
    });
  }
  return last_lane(scan(sum, sum_of));
}

// The value of lane ^ STEP
template <int STEP>
__device__ __forceinline__ unsigned across(unsigned v, int lane) {
  auto dpp = [](unsigned x, auto ctrl) { return (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, decltype(ctrl)::value, 0xF, 0xF, false); };
  if constexpr (STEP == 1) return dpp(v, std::integral_constant<int, 0xB1>());  // quad_perm 1 0 3 2
  if constexpr (STEP == 2) return dpp(v, std::integral_constant<int, 0x4E>());  // quad_perm 2 3 0 1
  if constexpr (STEP == 4) return dpp(dpp(v, std::integral_constant<int, 0x141>()), std::integral_constant<int, 0x1B>());  // row_half_mirror, quad_perm 3 2 1 0
  if constexpr (STEP == 8) return dpp(v, std::integral_constant<int, 0x128>());  // row_ror 8
  if constexpr (STEP == 16) {
    const auto s = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return lane & 16 ? s[0] : s[1];
  }
  if constexpr (STEP == 32) {
    const auto s = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return lane & 32 ? s[0] : s[1];
  }
}
template <int STEP>
__device__ __forceinline__ void sort_step(u64& v, int span) {
  const int tid = threadIdx.x;
  const u64 other = (u64)across<STEP>((unsigned)(v >> 32), tid) << 32 | across<STEP>((unsigned)v, tid);
  v = ((tid & span) == 0) == ((tid & STEP) == 0) ? max_of(v, other) : v < other ? v : other;
}
// Descending; n tokens, the rest of a power of two zeros.  Up to 1024 a thread has one, and only the steps from 64 on go through LDS (250 tokens: 5 us with all
// of them there, 2.5 so).  Beyond, a wavefront has 128 places in a row of its own, so only the steps beyond 64 need all wavefronts to meet.
__device__ __forceinline__ void sort_list(u64* list, int n) {
  const int tid = threadIdx.x;
  int size = 128;
  while (size < n) size *= 2;
  if (size <= kThreads) {
    u64 v = tid < n ? list[tid] : 0;
    for (int span = 2; span <= size; span *= 2) {
      for (int step = span / 2; step >= 64; step /= 2) {
        __syncthreads();
        if (tid < size) list[tid] = v;
        __syncthreads();
        if (tid < size) {
          const u64 other = list[tid ^ step];
          v = ((tid & span) == 0) == ((tid & step) == 0) ? max_of(v, other) : v < other ? v : other;
        }
      }
      if (span >= 64) sort_step<32>(v, span);
      if (span >= 32) sort_step<16>(v, span);
      if (span >= 16) sort_step<8>(v, span);
      if (span >= 8) sort_step<4>(v, span);
      if (span >= 4) sort_step<2>(v, span);
      sort_step<1>(v, span);
    }
    __syncthreads();
    if (tid < size) list[tid] = v;
    __syncthreads();
    return;
  }
  for (int i = n + threadIdx.x; i < size; i += kThreads) list[i] = 0;
  __syncthreads();
  for (int span = 2; span <= size; span *= 2)
    for (int step = span / 2; step > 0; step /= 2) {
      if (step > 32 && (step > 64 || span > 128)) __syncthreads();
      for (int i = threadIdx.x; i < size / 2; i += kThreads) {
        const int lo = 2 * i - (i & (step - 1)), hi = lo + step;
        const u64 a = list[lo], b = list[hi];
        if ((a < b) == ((lo & span) == 0)) {
          list[lo] = b;
          list[hi] = a;
        }
      }
      asm volatile("" ::: "memory");
    }
  __syncthreads();
}

// The cut, from the list's n tokens (at most kListed); the kept ones of them to the sums of the stretches that they lie in
template <typename T>
__device__ __forceinline__ u64 cut_of_list(Shared& sh, const Row<T>& row, const Asked& asked, const Weights& weight, const Zones& z, int n, int of_k_bin) {
  sort_list(sh.list, n);
  constexpr int EACH = kListed / kThreads;  // tokens of a thread, in order
  const int i0 = threadIdx.x * EACH;
  int end = z.k_bin < kBins ? n - of_k_bin + (asked.k - z.before_k) - 1 : n - 1;  // the last that is kept
  if (asked.shares) {
    u64 w[EACH], upto = 0;
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
      w[j] = i0 + j <= end ? weight(logit_of(sh.list[i0 + j])) : 0;
      upto += w[j];
    }
    u64 listed;
    const u64 before = sh.block.before(upto, &listed);
    const double target = asked.p * (double)(z.k_bin < kBins ? z.front + listed + z.between : z.all);
    int short_of = 0;  // the thread's tokens in front of which the share has not ended, and which do not end it
    upto = z.front + before;
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
      upto += w[j];
      short_of += i0 + j <= end && (double)upto < target ? 1 : 0;
    }
    const int at = (int)sh.block.all((u64)short_of, sum_of);
    if (at < end) end = at;
  }
  const u64 cut = sh.list[end];
  for (int i = threadIdx.x; i <= end; i += kThreads) {
    const u64 place = sh.list[i], w = weight(logit_of(place));
    if (w >= asked.least) atomicAdd(&sh.sums[row.stretch_of(index_of(place))], w);
  }
  return cut;
}

// By histograms of the places' digits, one after the other, over the whole row: of rows whose bins hold too many tokens to sort (ties; nearly flat rows, which
// take 0.5 to 1.1 ms for 64 rows of 100003 and are no model's).  The least
// place of the smallest front part of the order from `from` on that has `target` tokens, or so much weight.
template <typename T>
__device__ __attribute__((noinline)) u64 cut_by_digits(Shared& sh, const Row<T>& row, const Weights& weight, bool by_mass, double target, u64 from) {
  const int tid = threadIdx.x;
  u64 prefix = 0, above = 0;  // above: what the order has in front of the range that the digits so far leave
  int shift = 64;
  while (shift > 0) {
    const int digit = shift > 11 ? 11 : shift, low = shift - digit;
    __syncthreads();
    for (int i = tid; i < kBins; i += kThreads) {
      sh.counts[i] = 0;
      sh.masses[i] = 0;
    }
    __syncthreads();
    for (int i = tid; i < row.V; i += kThreads) {
      const float v = (float)row.x[i];
      const u64 place = place_of(v, i);
      if (place >= from && (shift == 64 || place >> shift == prefix)) {
        const int bin = (int)(place >> low & ((1u << digit) - 1));
        atomicAdd(&sh.counts[bin], 1u);
        if (by_mass) atomicAdd(&sh.masses[bin], weight(v));
      }
    }
    __syncthreads();
    // two bins a thread, the highest first
    const int hi = kBins - 1 - 2 * tid, lo = hi - 1;
    const u64 m1 = by_mass ? sh.masses[hi] : sh.counts[hi], m0 = by_mass ? sh.masses[lo] : sh.counts[lo];
    const u64 upto = above + sh.block.before(m1 + m0);
    // (the first bin that reaches it; where rounding leaves none, the last one with tokens)
    u64 mine = 0;
    if (sh.counts[hi] != 0 && (double)(upto + m1) >= target) mine = (u64)(hi + 1);
    else if (sh.counts[lo] != 0 && (double)(upto + m1 + m0) >= target) mine = (u64)(lo + 1);
    u64 bin = sh.block.all(mine, max_of);
    if (bin == 0) {
      u64 last = 0;
      if (sh.counts[lo] != 0) last = (u64)(kBins - lo);
      else if (sh.counts[hi] != 0) last = (u64)(kBins - hi);
      bin = kBins + 1 - sh.block.all(last, max_of);
    }
    const int chosen = (int)bin - 1;
    if (chosen == hi) sh.found[1] = upto;
    if (chosen == lo) sh.found[1] = upto + m1;
    __syncthreads();
    above = sh.found[1];
    prefix = prefix << digit | (unsigned)chosen;
    shift = low;
    if (sh.counts[chosen] == 1) break;  // (uniform) one token: it is the last one kept
  }
  return prefix << shift;
}
// The cut of a row whose list is too long, and the sums of all its stretches
template <typename T>
__device__ __attribute__((noinline)) u64 cut_without_list(Shared& sh, const Row<T>& row, const Asked& asked, const Weights& weight, const Zones& z, int stretches) {
  u64 cut = 0;
  const int tid = threadIdx.x;
  if (z.k_bin < kBins) cut = cut_by_digits<T>(sh, row, weight, false, (double)asked.k, 0);
  if (asked.shares) {
    u64 sum = 0;
    for (int i = tid; i < row.V; i += kThreads) sum += place_of((float)row.x[i], i) >= cut ? weight((float)row.x[i]) : 0;
    cut = max_of(cut, cut_by_digits<T>(sh, row, weight, true, asked.p * (double)sh.block.all(sum, sum_of), cut));
  }
  __syncthreads();
  for (int s = tid >> 6; s < stretches; s += kWaves) {
    u64 sum = 0;
    for (int i = row.first_of(s) + (tid & 63); i < row.first_of(s + 1); i += 64) {
      const u64 w = place_of((float)row.x[i], i) >= cut ? weight((float)row.x[i]) : 0;
      sum += w >= asked.least ? w : 0;
    }
    sum = last_lane(scan(sum, sum_of));
    if ((tid & 63) == 0) sh.sums[s] = sum;
  }
  return cut;
}

// Of `vecs` vectors from `first` on, some of them a thread in a row: the first value up to which what they have passes `share`, counted from `before` on;
// where none does the last that has any.  To the results, with its part of the total.
template <typename T, class Has>
__device__ __forceinline__ void answer(Shared& sh, const SampleArgs& a, int row_number, const Row<T>& row, int first, int vecs, u64 before, double share, u64 total, Has has) {
  constexpr int VEC = Row<T>::VEC;
  const int tid = threadIdx.x, each = (vecs + kThreads - 1) / kThreads, v0 = first + tid * each, most = first + vecs < row.vecs ? first + vecs : row.vecs;
  const int v1 = v0 + each < most ? v0 + each : most;
  u64 own = 0, w[VEC];
  auto look = [&](int v) {
    const auto x = row.load(v);
#pragma unroll
    for (int e = 0; e < VEC; ++e) w[e] = has((float)x[e], v * VEC - row.off + e);
  };
#pragma unroll 1
  for (int v = v0; v < v1; ++v) {
    look(v);
#pragma unroll
    for (int e = 0; e < VEC; ++e) own += w[e];
  }
  before += sh.block.before(own);
  const int who = sh.block.first(own != 0 && !((double)(before + own) <= share), own != 0);
  if (tid != who) return;
  int token = -1;
  u64 of_token = 0;
  bool on = true;
#pragma unroll 1
  for (int v = v0; v < v1; ++v) {
    if (each > 1) look(v);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const bool is = (int)on & (int)(w[e] != 0);
      token = is ? v * VEC - row.off + e : token;
      of_token = is ? w[e] : of_token;
      before += w[e];
      on = (int)on & (int)(w[e] == 0 || (double)before <= share);
    }
  }
  a.tokens[row_number] = token;
  a.probs[row_number] = (float)((double)of_token / (double)total);
}

// From the sums of the stretches: the one that the random share ends in (of 1 and more the last one with a token, of what is no number the first)
template <typename T>
__device__ __forceinline__ void draw(Shared& sh, const SampleArgs& a, int row_number, const Row<T>& row, const Asked& asked, const Weights& weight, u64 cut, int stretches) {
  const int tid = threadIdx.x;
  __syncthreads();
  const u64 own = tid < stretches ? sh.sums[tid] : 0;
  u64 total;
  const u64 before = sh.block.before(own, &total);
  const double share = (double)asked.random * (double)total;
  const int at = sh.block.first(own != 0 && !((double)(before + own) <= share), own != 0);
  if (tid == at) sh.found[0] = before;
  __syncthreads();
  const u64 least = asked.least;
  answer<T>(sh, a, row_number, row, at * row.per_wave, row.per_wave, sh.found[0], share, total, [&](float x, int i) {
    const u64 w = place_of(x, i) >= cut ? weight(x) : 0;
    return w >= least ? w : 0;
  });
}

// Rows that need no weights: of a greatest logit of -infinity (none is drawn) or +infinity (its tokens have 1 each, the others none), greedy ones.
// (part: the row, or the first part of it that has the greatest logit)
template <typename T>
__device__ __forceinline__ void draw_plain(Shared& sh, const SampleArgs& a, int row_number, const Row<T>& part, const Asked& asked, float top) {
  const int tid = threadIdx.x;
  if (top == -__builtin_inff() || asked.greedy()) {
    u64 first = 0;  // the lowest index, counted down
    part.walk([&](float x, int i) { first = x == top && i >= 0 && i < part.V ? max_of(first, (u64)(unsigned)~i) : first; });
    first = sh.block.all(first, max_of);
    if (tid == 0) {
      a.tokens[row_number] = top == -__builtin_inff() ? -1 : (int)~(unsigned)first;
      a.probs[row_number] = top == -__builtin_inff() ? 0.0f : 1.0f;
    }
    return;
  }
  u64 count = 0;
  for (int i = tid; i < part.V; i += kThreads) count += (float)part.x[i] == top;
  // kept are the first of them, by index
  u64 kept = sh.block.all(count, sum_of);
  if (asked.k != 0 && kept > (u64)asked.k) kept = asked.k;
  if (asked.shares) kept = (u64)fmax(1.0, ceil(asked.p * (double)kept));
  // (as weights of 1: a random share of the kept ones does not pass the last of them)
  const double share = fmin((double)asked.random * (double)kept, (double)kept - 0.5);
  answer<T>(sh, a, row_number, part, 0, part.vecs, 0, share, kept, [&](float x, int) { return (u64)(x == top); });
}

__device__ __forceinline__ bool is_plain(const Asked& asked, float top) { return top == -__builtin_inff() || top == __builtin_inff() || asked.greedy(); }

// The greedy answer of one reading: the first of the greatest
template <typename T>
__device__ __forceinline__ void draw_greatest(Shared& sh, const SampleArgs& a, int row_number, const Row<T>& row) {
  float best = -__builtin_inff();
  int at = 0;
  row.walk([&](float x, int i) {  // (a thread's indices grow; a NaN is not greater)
    at = x > best ? i : at;
    best = x > best ? x : best;
  });
  const u64 place = sh.block.all(place_of(best, at), max_of);
  if (threadIdx.x == 0) {
    const bool none = logit_of(place) == -__builtin_inff();
    a.tokens[row_number] = none ? -1 : index_of(place);
    a.probs[row_number] = none ? 0.0f : 1.0f;
  }
}

// ---- a workgroup a row ------------------------------------------------------------------------------------------------------------------
template <typename T>
__global__ void __launch_bounds__(kThreads) sample_rows_kernel(const SampleArgs a) {
  __shared__ Shared sh;
  const Row<T> row(a, blockIdx.x, 0, 1);
  const Asked asked(a, blockIdx.x);
  if (asked.greedy()) return draw_greatest<T>(sh, a, blockIdx.x, row);
  clear(sh, asked.cuts());
  const float mine = greatest_of_thread(row), top = value_of((unsigned)sh.block.all((u64)key_of(mine), max_of));
  if (is_plain(asked, top)) return draw_plain<T>(sh, a, blockIdx.x, row, asked, top);
  const Weights weight(top, asked.heat(), sh.table);
  Zones z{kBins, kBins, -1, kBins, 0, 0, 0, 0};
  if (asked.cuts()) {
    histogram(sh, row, asked, weight, mine, bins_asked(sh, asked, weight, 1, [&](int) { return mine; }));
    z = zones_of(sh, asked);
  }
  const u64 sum = gather(sh, row, asked, weight, mine, z);
  if ((threadIdx.x & 63) == 0) sh.sums[threadIdx.x >> 6] = sum;
  __syncthreads();
  u64 cut = 0;
  if (z.sure < kBins) {
    const int n = (int)sh.listed;
    cut = n <= kListed ? cut_of_list<T>(sh, row, asked, weight, z, n, (int)sh.of_k_bin) : cut_without_list<T>(sh, row, asked, weight, z, kWaves);
  }
  draw<T>(sh, a, blockIdx.x, row, asked, weight, cut, kWaves);
}

// ---- several workgroups a row: a launch a reading, what they leave for each other in the workspace -----------------------------------------
struct Parts {
  uint8_t* space;
  int parts;
};
struct Space {
  uint32_t* tops;
  float* maxima;
  u64 *masses, *sums, *list;
  unsigned *counts, *listed;
  Zones* zones;
  __device__ __forceinline__ Space(const Parts& p, int row) {
    const SampleSpace s = sample_space(p.parts);
    uint8_t* at = p.space + row * s.bytes;
    tops = (uint32_t*)(at + s.tops);
    maxima = (float*)(at + s.maxima);
    masses = (u64*)(at + s.masses);
    counts = (unsigned*)(at + s.counts);
    sums = (u64*)(at + s.sums);
    listed = (unsigned*)(at + s.listed);
    list = (u64*)(at + s.list);
    zones = (Zones*)(at + s.zones);
  }
};
static_assert(sizeof(Zones) <= 64, "as the workspace has it");

__device__ __forceinline__ float top_of(const Space& s, int parts) {
  unsigned keys[kSampleParts], key = 0;
#pragma unroll
  for (int i = 0; i < kSampleParts; ++i) keys[i] = s.tops[i < parts ? i : 0];  // (side by side)
#pragma unroll
  for (int i = 0; i < kSampleParts; ++i) key = key > keys[i] ? key : keys[i];
  return value_of(key);
}

template <typename T>
__global__ void __launch_bounds__(kThreads) sample_tops_kernel(const SampleArgs a, const Parts p) {
  __shared__ Block block;
  const Row<T> row(a, blockIdx.y, blockIdx.x, p.parts);
  const Space s(p, blockIdx.y);
  const float mine = greatest_of_thread(row);
  s.maxima[blockIdx.x * kThreads + threadIdx.x] = mine;
  const u64 key = block.all((u64)key_of(mine), max_of);
  if (threadIdx.x == 0) s.tops[blockIdx.x] = (unsigned)key;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) sample_histograms_kernel(const SampleArgs a, const Parts p) {
  __shared__ Shared sh;
  const Row<T> row(a, blockIdx.y, blockIdx.x, p.parts);
  const Space s(p, blockIdx.y);
  const Asked asked(a, blockIdx.y);
  const float top = top_of(s, p.parts);
  if (is_plain(asked, top) || !asked.cuts()) return;
  clear(sh, true);
  const Weights weight(top, asked.heat(), sh.table);
  const float mine = s.maxima[blockIdx.x * kThreads + threadIdx.x];
  histogram(sh, row, asked, weight, mine, bins_asked(sh, asked, weight, p.parts, [&](int i) { return s.maxima[i * kThreads + threadIdx.x]; }));
  __syncthreads();
  for (int i = threadIdx.x; i < kBins; i += kThreads) {
    if (asked.shares) s.masses[blockIdx.x * kBins + i] = sh.masses[i];
    if (asked.k != 0) s.counts[blockIdx.x * kBins + i] = sh.counts[i];
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) sample_sums_kernel(const SampleArgs a, const Parts p) {
  __shared__ Shared sh;
  const int tid = threadIdx.x;
  const Row<T> row(a, blockIdx.y, blockIdx.x, p.parts);
  const Space s(p, blockIdx.y);
  const Asked asked(a, blockIdx.y);
  const float top = top_of(s, p.parts);
  if (is_plain(asked, top)) return;
  clear(sh, false);
  const Weights weight(top, asked.heat(), sh.table);
  Zones z{kBins, kBins, -1, kBins, 0, 0, 0, 0};
  if (asked.cuts()) {
    u64 m[kBins / kThreads] = {};
    unsigned c[kBins / kThreads] = {};
#pragma unroll
    for (int j = 0; j < kSampleParts; ++j) {
      if (j >= p.parts) break;
#pragma unroll
      for (int i = 0; i < kBins / kThreads; ++i) {
        if (asked.shares) m[i] += s.masses[j * kBins + i * kThreads + tid];
        if (asked.k != 0) c[i] += s.counts[j * kBins + i * kThreads + tid];
      }
    }
#pragma unroll
    for (int i = 0; i < kBins / kThreads; ++i) {
      sh.masses[i * kThreads + tid] = m[i];
      sh.counts[i * kThreads + tid] = c[i];
    }
    __syncthreads();
    z = zones_of(sh, asked);
  }
  const u64 sum = gather(sh, row, asked, weight, s.maxima[blockIdx.x * kThreads + tid], z);
  if ((tid & 63) == 0) s.sums[blockIdx.x * kWaves + (tid >> 6)] = sum;
  __syncthreads();
  const int n = (int)sh.listed;
  for (int i = tid; i < n && i < kListed; i += kThreads) s.list[blockIdx.x * kListed + i] = sh.list[i];
  if (tid == 0) {
    s.listed[2 * blockIdx.x] = n;
    s.listed[2 * blockIdx.x + 1] = sh.of_k_bin;
    if (blockIdx.x == 0) *s.zones = z;
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) sample_answers_kernel(const SampleArgs a, const Parts p) {
  __shared__ Shared sh;
  const int tid = threadIdx.x, stretches = p.parts * kWaves;
  Row<T> row(a, blockIdx.x, 0, p.parts);
  const Space s(p, blockIdx.x);
  const Asked asked(a, blockIdx.x);
  const float top = top_of(s, p.parts);
  if (is_plain(asked, top)) {
    int part = 0;
    while (s.tops[part] != key_of(top)) ++part;
    row.to_part(part);
    return draw_plain<T>(sh, a, blockIdx.x, row, asked, top);
  }
  clear(sh, false);
  const Weights weight(top, asked.heat(), sh.table);
  if (tid < stretches) sh.sums[tid] = s.sums[tid];
  const Zones z = *s.zones;
  u64 cut = 0;
  if (z.sure < kBins) {
    int listed[kSampleParts], of_k_bin = 0;  // (4096 and more of a part: no list)
    int64_t n = 0;
#pragma unroll
    for (int j = 0; j < kSampleParts; ++j) {
      listed[j] = j < p.parts ? (int)s.listed[2 * j] : 0;
      of_k_bin += j < p.parts ? (int)s.listed[2 * j + 1] : 0;
    }
#pragma unroll
    for (int j = 0; j < kSampleParts; ++j) n += (unsigned)listed[j];
    if (n <= kListed) {
      for (int i = tid; i < n; i += kThreads) {
        int part = 0, at = i;
#pragma unroll
        for (int j = 0; j + 1 < kSampleParts; ++j) {
          const bool behind = part == j && at >= listed[j];
          at -= behind ? listed[j] : 0;
          part += behind ? 1 : 0;
        }
        sh.list[i] = s.list[part * kListed + at];
      }
      __syncthreads();
      cut = cut_of_list<T>(sh, row, asked, weight, z, (int)n, of_k_bin);
    } else {
      cut = cut_without_list<T>(sh, row, asked, weight, z, stretches);
    }
  }
  draw<T>(sh, a, blockIdx.x, row, asked, weight, cut, stretches);
}

template <typename T>
gpusq_status launch_typed(const SampleArgs& a, int64_t rows, void* workspace, hipStream_t s) {
  const int parts = sample_parts(rows, a.V);
  if (parts == 1) {
    sample_rows_kernel<T><<<(unsigned)rows, kThreads, 0, s>>>(a);
    return check_launch();
  }
  const Parts p{(uint8_t*)workspace, parts};
  const dim3 grid((unsigned)parts, (unsigned)rows);
  gpusq_status st;
  sample_tops_kernel<T><<<grid, kThreads, 0, s>>>(a, p);
  if ((st = check_launch()) != GPUSQ_OK) return st;
  sample_histograms_kernel<T><<<grid, kThreads, 0, s>>>(a, p);
  if ((st = check_launch()) != GPUSQ_OK) return st;
  sample_sums_kernel<T><<<grid, kThreads, 0, s>>>(a, p);
  if ((st = check_launch()) != GPUSQ_OK) return st;
  sample_answers_kernel<T><<<(unsigned)rows, kThreads, 0, s>>>(a, p);
  return check_launch();
}

}  // namespace

gpusq_status launch_sample_tokens(const SampleArgs& a, bool f32, int64_t rows, void* workspace, hipStream_t s) {
  return f32 ? launch_typed<float>(a, rows, workspace, s) : launch_typed<_Float16>(a, rows, workspace, s);
}

}  // namespace gpusq
