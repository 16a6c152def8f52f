// Tokens drawn from logits by temperature, top-k, top-p and min-p, with random numbers that are given.
//
//   w_i = exp((x_i - max x) / T), 0 below 2^-40;  the tokens in the order of their logits, ties by their index, are cut behind the first k, behind the
//   first whose weights reach p of the first k's, and in front of the first whose weight is below min_p;  drawn is the first token, in the
//   vocabulary's order, up to which the kept weights pass u of their sum.
//
// Where two tokens' shares meet is closer to a neighbour's than 32 bits tell apart, so weights are formed in 64 bits and summed as whole numbers, of
// which no order changes the sum.  A token's place in the order is one number, its logit's bits made monotone and its index counted down: every
// cut is a least such number, found digit by digit from histograms of how many tokens, and how much weight, have a digit.
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

// weights as whole numbers of 2^-bits
struct Weights {
  double top, inv, one;
  __device__ __forceinline__ double exact(float x) const {
    if ((double)x == top) return 1.0;
    const double w = exp(((double)x - top) * inv);
    return w >= 0x1p-40 ? w : 0.0;  // (and of a NaN 0)
  }
  __device__ __forceinline__ u64 operator()(float x) const { return (u64)(exact(x) * one + 0.5); }
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

template <typename T>
__global__ void __launch_bounds__(kThreads) sample_rows_kernel(const SampleArgs a) {
  __shared__ Block block;
  __shared__ unsigned counts[kBins];
  __shared__ u64 masses[kBins];
  __shared__ u64 found[4];
  const int row = blockIdx.x, tid = threadIdx.x, V = a.V;
  const T* x = (const T*)a.logits + (int64_t)row * a.row_stride;
  u64 best = 0;
  for (int i = tid; i < V; i += kThreads) best = max_of(best, place_of((float)x[i], i));
  best = block.all(best, max_of);
  const float top = value_of((unsigned)(best >> 32));
  const int first = (int)~(unsigned)best;
  const float temperature = a.temperature != nullptr ? a.temperature[row] : 1.0f;
  if (top == -__builtin_inff() || !(temperature > 0.0f)) {
    if (tid == 0) {
      a.tokens[row] = top == -__builtin_inff() ? -1 : first;
      a.probs[row] = top == -__builtin_inff() ? 0.0f : 1.0f;
    }
    return;
  }
  const Weights weight{(double)top, 1.0 / (double)temperature, a.one};
  // The least place of the smallest front part of the order that has `target` tokens, or so much weight.  (above: what the order has in front of the
  // range that the digits so far leave.)
  auto cut_at = [&](bool by_mass, double target, u64 from) {
    u64 prefix = 0;
    int shift = 64;
    u64 above = 0;
    while (shift > 0) {
      const int digit = shift > 11 ? 11 : shift, low = shift - digit;
      __syncthreads();
      for (int i = tid; i < kBins; i += kThreads) {
        counts[i] = 0;
        masses[i] = 0;
      }
      __syncthreads();
      for (int i = tid; i < V; i += kThreads) {
        const float v = (float)x[i];
        const u64 place = place_of(v, i);
        if (place >= from && (shift == 64 || place >> shift == prefix)) {
          const int bin = (int)(place >> low & ((1u << digit) - 1));
          atomicAdd(&counts[bin], 1u);
          if (by_mass) atomicAdd(&masses[bin], weight(v));
        }
      }
      __syncthreads();
      // two bins a thread, the highest first
      const int hi = kBins - 1 - 2 * tid, lo = hi - 1;
      const u64 m1 = by_mass ? masses[hi] : counts[hi], m0 = by_mass ? masses[lo] : counts[lo];
      const u64 upto = above + block.before(m1 + m0);
      if (tid == 0) found[0] = 0;
      __syncthreads();
      // (the first bin that reaches it; where rounding leaves none, the last one with tokens)
      u64 mine = 0;
      if (counts[hi] != 0 && ((double)(upto + m1) >= target || target < 0)) mine = (u64)(hi + 1);
      else if (counts[lo] != 0 && ((double)(upto + m1 + m0) >= target || target < 0)) mine = (u64)(lo + 1);
      u64 bin = block.all(mine, max_of);
      if (bin == 0) {
        u64 last = 0;
        if (counts[lo] != 0) last = (u64)(kBins - lo);
        else if (counts[hi] != 0) last = (u64)(kBins - hi);
        bin = kBins + 1 - block.all(last, max_of);
      }
      const int chosen = (int)bin - 1;
      if (chosen == hi) found[1] = upto;
      if (chosen == lo) found[1] = upto + m1;
      __syncthreads();
      above = found[1];
      prefix = prefix << digit | (unsigned)chosen;
      shift = low;
      if (counts[chosen] == 1) break;  // (uniform) one token: it is the last one kept
    }
    return prefix << shift;
  };
  u64 cut = 0;
  const int k = a.top_k != nullptr ? a.top_k[row] : 0;
  if (k > 0 && k < V) cut = cut_at(false, (double)k, 0);
  const float p = a.top_p != nullptr ? a.top_p[row] : 1.0f;
  if (p < 1.0f) {
    u64 sum = 0;
    for (int i = tid; i < V; i += kThreads)
      if (place_of((float)x[i], i) >= cut) sum += weight((float)x[i]);
    sum = block.all(sum, sum_of);
    cut = max_of(cut, p > 0.0f ? cut_at(true, (double)p * (double)sum, cut) : best);
  }
  const float m = a.min_p != nullptr ? a.min_p[row] : 0.0f;
  const double least = m > 1.0f ? 1.0 : m > 0.0f ? (double)m : 0.0;
  auto kept = [&](float v, int i) {
    if (place_of(v, i) < cut) return (u64)0;
    const double w = weight.exact(v);
    return w >= least ? (u64)(w * a.one + 0.5) : (u64)0;
  };
  // a stretch of the vocabulary for each thread
  const int each = (V + kThreads - 1) / kThreads, begin = tid * each < V ? tid * each : V, end = begin + each < V ? begin + each : V;
  u64 mine = 0;
  for (int i = begin; i < end; ++i) mine += kept((float)x[i], i);
  const u64 before = block.before(mine), total = block.all(mine, sum_of);
  const double u = (double)a.random[row] * (double)total;
  if (tid == 0) found[0] = 0;
  __syncthreads();
  // the last thread with a kept token answers where u is 1 or more, the first where it is no number
  const bool here = mine != 0 && !((double)(before + mine) <= u);
  const u64 who = block.all(here ? (u64)(kThreads - tid) : 0, max_of), last = block.all(mine != 0 ? (u64)(tid + 1) : 0, max_of);
  if (tid == (who != 0 ? kThreads - (int)who : (int)last - 1)) {
    u64 upto = before, w = 0;
    int token = -1;
    for (int i = begin; i < end; ++i) {
      const u64 next = kept((float)x[i], i);
      if (next == 0) continue;
      token = i;
      w = next;
      upto += next;
      if (!((double)upto <= u)) break;
    }
    a.tokens[row] = token;
    a.probs[row] = (float)((double)w / (double)total);
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
