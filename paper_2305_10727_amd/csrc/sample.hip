// Tokens drawn from logits by temperature, top-k, top-p and min-p, with random numbers that are given.
//
//   w_i = exp((x_i - max x) / T), 0 below 2^-40;  the tokens in the order of their logits, ties by their index, are cut behind the first k, behind the
//   first whose weights reach p of the first k's, and in front of the first whose weight is below min_p;  drawn is the first token, in the
//   vocabulary's order, up to which the kept weights pass u of their sum.
//
// Where two tokens' shares meet is closer to a neighbour's than 32 bits tell apart, so weights are formed in 64 bits and summed as whole numbers, of
// which no order changes the sum.  A token's place in the order is one number, its logit's bits made monotone and its index counted down: a cut is the
// least such number that is kept.
#include "common.h"

namespace gpusq {

namespace {

constexpr int kThreads = 1024, kBins = 2048;
typedef unsigned long long u64;

// The logits' order: greater numbers first; -0 is 0, what is no number is -infinity
__device__ __forceinline__ unsigned key_of(float x) {
  x = x == x ? x + 0.0f : -__builtin_inff();
  const unsigned u = __float_as_uint(x);
  return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(unsigned key) { return __uint_as_float(key >> 31 ? key & 0x7fffffffu : ~key); }
__device__ __forceinline__ u64 place_of(float x, int i) { return (u64)key_of(x) << 32 | (unsigned)~i; }

// Weights as whole numbers of 2^-44.  exp(y) is 2^(j / 64) 2^e (1 + r + r^2 / 2 + r^3 / 6 + r^4 / 24) with |r| at most ln 2 / 128, off by 4e-14 of
// itself: a dozen operations in 64 bits, a third of the library's exp.
struct Weights {
  float top;            // the greatest logit
  double steps;         // 64 / (T ln 2)
  const double* table;  // 2^(j / 64)
  __device__ __forceinline__ double exact(float x) const {
    // (x equal to an infinite greatest one: 1; of -infinity and of what is no number 2^-42)
    const double d = x == top ? 0.0 : (double)x - (double)top, t = fmax(d * steps, -2700.0);
    const double shifted = t + 0x1.8p52, whole = shifted - 0x1.8p52, r = (t - whole) * 0x1.62e42fefa39efp-7;
    const int k = (int)(unsigned)__double_as_longlong(shifted);
    const double c = table[k & 63], p = r * __builtin_fma(r, __builtin_fma(r, __builtin_fma(r, 1.0 / 24, 1.0 / 6), 0.5), 1.0);
    return __longlong_as_double(__double_as_longlong(__builtin_fma(c, p, c)) + ((long long)(k >> 6) << 52));
  }
  static __device__ __forceinline__ u64 whole(double w) {  // 0 below 2^-40
    return w >= 0x1p-40 ? (u64)(__double_as_longlong(w + 256.0) - __double_as_longlong(256.0)) : 0;
  }
  __device__ __forceinline__ u64 operator()(float x) const { return whole(exact(x)); }
};

struct Block {
  u64 part[kThreads / 64];
  template <class Op>
  __device__ __forceinline__ u64 all(u64 v, Op op) {  // of all threads, to all threads
    __syncthreads();
#pragma unroll
    for (int d = 1; d < 64; d *= 2) v = op(v, (u64)__shfl_xor(v, d));
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int i = 1; i < kThreads / 64; ++i) v = op(v, part[i]);
    return v;
  }
  // sum of the threads in front of this one
  __device__ __forceinline__ u64 before(u64 v) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    u64 upto = v;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const u64 o = __shfl_up(upto, d);
      if (lane >= d) upto += o;
    }
    __syncthreads();
    if (lane == 63) part[wave] = upto;
    __syncthreads();
    u64 sum = upto - v;
    for (int i = 0; i < wave; ++i) sum += part[i];
    return sum;
  }
};
__device__ __forceinline__ u64 sum_of(u64 a, u64 b) { return a + b; }
__device__ __forceinline__ u64 max_of(u64 a, u64 b) { return a > b ? a : b; }

// A row of logits by vectors of 16 bytes, wherever it begins: a wavefront has a stretch of the vocabulary, its lanes a vector each at a time.  each(value,
// index) is called of a lane's values one after the other, unrolled.
template <typename T>
struct Row {
  static constexpr int VEC = 16 / (int)sizeof(T), WAVES = kThreads / 64, AHEAD = 4;
  typedef T vec __attribute__((ext_vector_type(VEC)));
  const T* x;
  int V, off, per_wave;  // values in front of the row in its first vector; vectors of a wavefront
  __device__ __forceinline__ Row(const T* row, int V_) : x(row), V(V_), off((int)(((uintptr_t)row & 15) / sizeof(T))) {
    const int vecs = (V + off + VEC - 1) / VEC;
    per_wave = ((vecs + WAVES - 1) / WAVES + 63) & ~63;
  }
  __device__ __forceinline__ vec load(int v) const {
    const int i = v * VEC - off;
    if (i >= 0 && i + VEC <= V) return *(const vec*)(x + i);
    vec r;
#pragma unroll
    for (int e = 0; e < VEC; ++e) r[e] = i + e >= 0 && i + e < V ? x[i + e] : (T)-__builtin_inff();
    return r;
  }
  template <class Each>
  __device__ __forceinline__ void walk(Each each) const {
    const int begin = (threadIdx.x >> 6) * per_wave, end = begin + per_wave, last = (V + off + VEC - 1) / VEC;
    for (int v0 = begin + (threadIdx.x & 63); v0 < end && v0 < last; v0 += 64 * AHEAD) {
      vec r[AHEAD];
#pragma unroll
      for (int j = 0; j < AHEAD; ++j) {
        const int v = v0 + 64 * j;
        if (v < end && v < last) {
          r[j] = load(v);
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
  // the indices that wavefront w has
  __device__ __forceinline__ int first_of(int w) const {
    const int64_t i = (int64_t)w * per_wave * VEC - off;
    return i < 0 ? 0 : i < V ? (int)i : V;
  }
};

// The row's weights meet a histogram of their distance from the greatest logit, in 2048 bins of 28 / 2048 of the temperature: which bin the k-th token
// lies in, and between which two the p-th share ends, is known from it; the tokens of those bins alone are sorted, and decide.  So a row is read three
// times: for its greatest, for the histogram, for the sums and those tokens.  A wavefront sums its own stretch of the vocabulary; the token lies in the
// stretch that passes the random share, which is looked at once more.
constexpr int kListed = 4096;
constexpr float kBinsOfUnit = kBins / 28.0f;  // (2^-40 is 27.73 below)

struct Shared {
  Block block;
  double table[64];
  u64 masses[kBins];
  unsigned counts[kBins];
  u64 list[kListed];
  u64 sums[kThreads / 64], found[2];
  unsigned listed, of_k_bin;
};

// Descending; n tokens, the rest of a power of two zeros
__device__ __forceinline__ void sort_list(u64* list, int n) {
  int size = 64;
  while (size < n) size *= 2;
  for (int i = n + threadIdx.x; i < size; i += kThreads) list[i] = 0;
  for (int span = 2; span <= size; span *= 2)
    for (int step = span / 2; step > 0; step /= 2) {
      __syncthreads();
      for (int i = threadIdx.x; i < size / 2; i += kThreads) {
        const int lo = 2 * i - (i & (step - 1)), hi = lo + step;
        const u64 a = list[lo], b = list[hi];
        if ((a < b) == ((lo & span) == 0)) {
          list[lo] = b;
          list[hi] = a;
        }
      }
    }
  __syncthreads();
}

// By histograms of the places' digits, one after the other, over the whole row: of rows whose bins hold too many tokens to sort (ties).  The least place of the smallest front part of the order from `from` on that has `target` tokens, or so much weight.
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

template <typename T>
__global__ void __launch_bounds__(kThreads) sample_rows_kernel(const SampleArgs a) {
  __shared__ Shared sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const Row<T> row((const T*)a.logits + (int64_t)blockIdx.x * a.row_stride, a.V);
  if (tid < 64) sh.table[tid] = exp2(tid * (1.0 / 64));
  for (int i = tid; i < kBins; i += kThreads) {
    sh.masses[i] = 0;
    sh.counts[i] = 0;
  }
  if (tid == 0) sh.listed = sh.of_k_bin = 0;
  auto store_sums = [&](u64 sum) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) sum += (u64)__shfl_xor(sum, d);
    if (lane == 0) sh.sums[wave] = sum;
    __syncthreads();
  };
  const float temperature = a.temperature != nullptr ? a.temperature[blockIdx.x] : 1.0f;
  const int k_given = a.top_k != nullptr ? a.top_k[blockIdx.x] : 0, k = k_given > 0 && k_given < a.V ? k_given : 0;
  const float p_given = a.top_p != nullptr ? a.top_p[blockIdx.x] : 1.0f, m = a.min_p != nullptr ? a.min_p[blockIdx.x] : 0.0f;
  const bool shares = p_given < 1.0f;
  const double least = m > 1.0f ? 1.0 : m > 0.0f ? (double)m : 0.0, p = p_given > 0.0f ? (double)p_given : 0.0;
  float mine = -__builtin_inff();
  row.walk([&](float x, int) { mine = fmaxf(mine, x); });  // (a NaN is left out)
  const float top = value_of((unsigned)sh.block.all((u64)key_of(mine), max_of));
  if (top == -__builtin_inff() || !(temperature > 0.0f)) {
    u64 first = 0;  // of the greatest, the lowest index (counted down)
    if (mine == top) row.walk([&](float x, int i) { first = x == top && i >= 0 && i < a.V ? max_of(first, (u64)(unsigned)~i) : first; });
    first = sh.block.all(first, max_of);
    if (tid == 0) {
      a.tokens[blockIdx.x] = top == -__builtin_inff() ? -1 : (int)~(unsigned)first;
      a.probs[blockIdx.x] = top == -__builtin_inff() ? 0.0f : 1.0f;
    }
    return;
  }
  const Weights weight{top, 92.332482616893657 / (double)temperature, sh.table};
  const float scale = fminf(kBinsOfUnit / temperature, 3.4e38f);
  auto bin_of = [&](float x) {  // in the logits' order; kBins: without weight
    const float d = x == top ? 0.0f : (top - x) * scale;
    return d < (float)kBins ? (int)d : kBins;
  };
  auto of_weight = [&](float x) {  // with what min_p leaves
    const double w = weight.exact(x);
    return w >= least ? Weights::whole(w) : (u64)0;
  };
  u64 cut = 0;
  bool summed = false;
  if (k != 0 || shares) {
    // Of the greatest logits of the threads the k-th lies in a bin behind or at the row's k-th: behind it nothing is asked.
    int behind = kBins;
    auto first_bin = [&](auto reached) {  // the first for which it is so, kBins: none
      const u64 at = sh.block.all(reached(2 * tid) ? (u64)(kBins - 2 * tid) : reached(2 * tid + 1) ? (u64)(kBins - 2 * tid - 1) : 0, max_of);
      return kBins - (int)at;
    };
    auto cumulate_counts = [&] {
      __syncthreads();
      const unsigned c0 = sh.counts[2 * tid], c1 = sh.counts[2 * tid + 1], before = (unsigned)sh.block.before(c0 + c1);
      sh.counts[2 * tid] = before + c0;
      sh.counts[2 * tid + 1] = before + c0 + c1;
      __syncthreads();
    };
    auto enough = [&](int b) { return sh.counts[b] >= (unsigned)k; };
    if (k != 0 && k <= kThreads) {
      const int b = bin_of(mine);
      if (b < kBins) atomicAdd(&sh.counts[b], 1u);
      cumulate_counts();
      behind = first_bin(enough);
      if (behind < kBins) ++behind;
      sh.counts[2 * tid] = sh.counts[2 * tid + 1] = 0;
      __syncthreads();
    }
    row.walk([&](float x, int) {
      const int b = bin_of(x);
      if (b < behind) {
        if (k != 0) atomicAdd(&sh.counts[b], 1u);
        if (shares) atomicAdd(&sh.masses[b], weight(x));
      }
    });
    cumulate_counts();
    int k_bin = kBins, z0 = kBins, z1 = -1;  // the k-th token's bin; those that the share may end in
    if (k != 0) k_bin = first_bin(enough);
    if (shares) {
      const u64 m0 = sh.masses[2 * tid], m1 = sh.masses[2 * tid + 1], before = sh.block.before(m0 + m1);
      sh.masses[2 * tid] = before + m0;
      sh.masses[2 * tid + 1] = before + m0 + m1;
      __syncthreads();
      // the k tokens' weight lies between what is in front of the k-th's bin and what is up to it
      const u64 most = sh.masses[k_bin < kBins ? k_bin : kBins - 1], fewest = k_bin == kBins ? most : k_bin > 0 ? sh.masses[k_bin - 1] : 0;
      const double t0 = fmax(p * (double)fewest, 1.0), t1 = fmax(p * (double)most, 1.0);  // (a share of nothing: the greatest's bin)
      z0 = first_bin([&](int b) { return (double)sh.masses[b] >= t0; });
      z1 = first_bin([&](int b) { return (double)sh.masses[b] >= t1; });
      z0 = z0 < k_bin ? z0 : k_bin;
      z1 = z1 < k_bin ? z1 : k_bin;
    }
    if (k_bin < kBins || shares) {
      const int sure = z0 < k_bin ? z0 : k_bin;  // tokens of bins in front of this one are kept, of those behind it those of the list alone
      u64 sum = 0;
      row.walk([&](float x, int i) {
        const int b = bin_of(x);
        if (b < sure) {
          sum += of_weight(x);
        } else if (b < kBins && (b == k_bin || (b >= z0 && b <= z1))) {
          if (b == k_bin) atomicAdd(&sh.of_k_bin, 1u);
          const unsigned at = atomicAdd(&sh.listed, 1u);
          if (at < kListed) sh.list[at] = place_of(x, i);
        }
      });
      store_sums(sum);
      const int n = (int)sh.listed;
      summed = n <= kListed;
      if (summed) {
        sort_list(sh.list, n);
        // four tokens a thread, in order
        constexpr int EACH = kListed / kThreads;
        const int i0 = tid * EACH;
        int end = n - 1;  // the last that is kept
        if (k_bin < kBins) end = n - (int)sh.of_k_bin + (k - (int)(k_bin > 0 ? sh.counts[k_bin - 1] : 0)) - 1;
        if (shares) {
          u64 w[EACH], upto = 0, kept = 0;
#pragma unroll
          for (int j = 0; j < EACH; ++j) {
            w[j] = i0 + j <= end ? weight(value_of((unsigned)(sh.list[i0 + j] >> 32))) : 0;
            upto += w[j];
          }
          const u64 before = sh.block.before(upto), listed = sh.block.all(upto, sum_of), front = sure > 0 ? sh.masses[sure - 1] : 0;
          if (k_bin < kBins)  // (with the bins between the share's and the k-th token's, which are not in the list)
            kept = front + listed + (z1 < k_bin && k_bin > 0 ? sh.masses[k_bin - 1] - sh.masses[z1] : 0);
          else
            kept = sh.masses[kBins - 1];
          const double target = p * (double)kept;
          u64 at = 0;
          upto = front + before;
#pragma unroll
          for (int j = 0; j < EACH; ++j) {
            upto += w[j];
            if (at == 0 && i0 + j <= end && (double)upto >= target) at = (u64)(kListed - (i0 + j));
          }
          at = sh.block.all(at, max_of);
          if (at != 0) end = kListed - (int)at;
        }
        cut = sh.list[end];
        // the kept tokens of the list, to the sums of the stretches that they lie in
        for (int i = tid; i <= end; i += kThreads) {
          const u64 place = sh.list[i];
          atomicAdd(&sh.sums[((int)~(unsigned)place + row.off) / (row.per_wave * Row<T>::VEC)], of_weight(value_of((unsigned)(place >> 32))));
        }
      }
    }
    if (!summed) {
      if (k_bin < kBins) cut = cut_by_digits<T>(sh, row, weight, false, (double)k, 0);
      if (shares) {
        u64 sum = 0;
        row.walk([&](float x, int i) { sum += place_of(x, i) >= cut ? weight(x) : 0; });
        cut = max_of(cut, cut_by_digits<T>(sh, row, weight, true, p * (double)sh.block.all(sum, sum_of), cut));
      }
    }
  }
  if (!summed) {
    u64 sum = 0;
    row.walk([&](float x, int i) { sum += bin_of(x) < kBins && place_of(x, i) >= cut ? of_weight(x) : 0; });
    store_sums(sum);
  }
  __syncthreads();
  // the stretch that the random share ends in (of 1 and more the last one with a token, of what is no number the first), ...
  u64 total = 0, before = 0;
  for (int w = 0; w < kThreads / 64; ++w) total += sh.sums[w];
  const double share = (double)a.random[blockIdx.x] * (double)total;
  int at = -1;
  for (int w = 0; w < kThreads / 64; ++w) {
    const u64 s = sh.sums[w];
    if (s == 0) continue;
    if (at >= 0) before += sh.sums[at];
    at = w;
    if (!((double)(before + s) <= share)) break;
  }
  // ... a piece of it for each thread, and the token
  const int begin = row.first_of(at), end = row.first_of(at + 1), each = (end - begin + kThreads - 1) / kThreads;
  const int i0 = begin + tid * each, i1 = i0 + each < end ? i0 + each : end;
  auto kept = [&](int i) {
    const float x = (float)row.x[i];
    return bin_of(x) < kBins && place_of(x, i) >= cut ? of_weight(x) : (u64)0;
  };
  u64 own = 0;
  for (int i = i0; i < i1; ++i) own += kept(i);
  before += sh.block.before(own);
  const bool here = own != 0 && !((double)(before + own) <= share);
  const u64 who = sh.block.all(here ? (u64)(kThreads - tid) : 0, max_of), last = sh.block.all(own != 0 ? (u64)(tid + 1) : 0, max_of);
  if (tid == (who != 0 ? kThreads - (int)who : (int)last - 1)) {
    int token = -1;
    u64 w = 0;
    for (int i = i0; i < i1; ++i) {
      const u64 next = kept(i);
      if (next == 0) continue;
      token = i;
      w = next;
      before += next;
      if (!((double)before <= share)) break;
    }
    a.tokens[blockIdx.x] = token;
    a.probs[blockIdx.x] = (float)((double)w / (double)total);
  }
}

}  // namespace

gpusq_status launch_sample_tokens(const SampleArgs& a, bool f32, int64_t rows, hipStream_t s) {
  if (f32)
    sample_rows_kernel<float><<<(unsigned)rows, kThreads, 0, s>>>(a);
  else
    sample_rows_kernel<_Float16><<<(unsigned)rows, kThreads, 0, s>>>(a);
  return check_launch();
}

}  // namespace gpusq
