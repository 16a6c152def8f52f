// What the kernels of attention share: their arguments, the running softmax, the columns and the output of a wavefront.
//
//   o[q] = sum_j exp(s_qj - m_q) v_j / sum_j exp(s_qj - m_q),  s_qj = scale q . k_j,  m_q the largest visible s_qj;  0 where none is visible
//
// One pass over the keys with the running maximum and sum of the softmax; scores never leave the registers.  A wavefront takes 32 keys
// at a time.  The first product is turned over, scores^T = K Q^T, so that a lane of the result has one query (column lane % 16) and the
// keys 4 g .. + 3 (g = lane / 16) of either 16: these are, as they lie, the second operand of output^T = V^T P^T, if V^T's k runs over
// the same keys in the same order.  Nothing crosses lanes between the products.
// Queries of the heads that share a key head are columns side by side: column = token * (heads per key head) + head.
//
// The maximum moves only when a score passes it by 2^8 (kSlack): p = 2^(s - m + 6) then lies in fp16 up to 2^14, and down to 2^-24,
// that is to 2^-30 of the largest where it has not moved.  Most tiles need neither the maximum across lanes nor a rescaled sum.
// The exponent is formed of a score in one fused step from the maximum in log2 units, which is held to less than 1 up to 2^23, so that p stays in fp16 for scores
// up to 2^22.  (Larger ones would need the maximum taken off before they are scaled: 1 to 3 % of a call, for scores that 32 bits hold to a factor of two.)
// P is rounded to fp16 for the matrix instruction (the one rounding between the scores and the output); its sum is that of the rounded
// values, in 32 bits, one matrix instruction with a first operand of ones instead of 8 additions a lane.
#pragma once
#include "attend_plan.h"
#include "kv4.h"

namespace gpusq {

constexpr float kLog2e = 1.4426950408889634f, kShift = 6.0f, kSlack = 8.0f;

struct AttendArgs {
  const _Float16* q;
  _Float16* out;
  int64_t q_batch, q_token, q_head;  // in values
  int64_t o_token;                   // out: [token][heads][D]
  int heads, kv_heads, rep, D, batch, q_len;
  float c, inv_c;  // scale * log2(e) and 1 by it
  // over the cache
  const uint8_t* cache;
  const int32_t *table, *cu_q;
  int max_pages, num_pages, tokens;
  // over fp16 states
  const _Float16 *k, *v;
  int64_t k_batch, k_token, k_head, v_batch, v_token, v_head;
  const uint8_t* mask;
  int kv_len;
  const int32_t* lens;
  // work: column blocks of a (batch, key head), parts of its keys
  int col_blocks, parts, part_tiles;
  float* part_o;   // [part][row][D] sums, [part][row][2] maximum and sum
  float* part_ml;
};

__device__ __forceinline__ h8 join(h2 a, h2 b, h2 c, h2 d) { return h8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]}; }

// What a workgroup works on: part of the keys of a (batch, key head) and a block of its columns.  Blocks of the same keys run on one XCD, whose
// L2 then reads these once: many keys are dealt out over the XCDs in turn (batches are of different lengths), few in equal shares.
struct Work {
  int b, kh, part, block;
  __device__ __forceinline__ bool find(const AttendArgs& a) {
    const int units = a.batch * a.kv_heads * a.parts, xcd = blockIdx.x & 7, local = blockIdx.x >> 3;
    // (divisions take a scalar unit that has none some forty instructions each: none by 1)
    int unit;
    if (attend_in_turn(units)) {
      const int first = a.col_blocks == 1 ? local : local / a.col_blocks;
      block = local - first * a.col_blocks;
      unit = first * 8 + xcd;
      if (unit >= units) return false;
    } else {
      const int total = units * a.col_blocks, per_xcd = (total + 7) >> 3, at = xcd * per_xcd + local;
      if (local >= per_xcd || at >= total) return false;
      unit = a.col_blocks == 1 ? at : at / a.col_blocks;
      block = at - unit * a.col_blocks;
    }
    const int pair = a.parts == 1 ? unit : unit / a.parts;
    part = unit - pair * a.parts;
    b = a.batch == 1 ? 0 : pair / a.kv_heads;
    kh = pair - b * a.kv_heads;
    return true;
  }
  static unsigned workgroups(const AttendArgs& a) { return (unsigned)attend_workgroups((int64_t)a.batch * a.kv_heads * a.parts, a.col_blocks); }
};

// The tokens of a batch's queries (nq that are answered), the keys that it has, those in front of its first query (fewer than none, if it has more
// queries than keys)
template <bool KV4>
struct Span {
  int t0, nq, len, before;
  int64_t q_base;
  __device__ __forceinline__ Span(const AttendArgs& a, int b) : t0(b * a.q_len), nq(a.q_len) {
    if constexpr (KV4) {
      if (a.cu_q != nullptr) {
        t0 = a.cu_q[b];
        const int t1 = a.cu_q[b + 1];
        nq = t0 >= 0 && t1 <= a.tokens && t1 > t0 ? t1 - t0 : 0;
      }
      q_base = (int64_t)t0 * a.q_token;
      const int most = a.max_pages * kPageTokens;
      len = a.lens[b];
      len = len < 0 ? 0 : len < most ? len : most;
      before = len - nq;  // (of all of its queries, also where more of them are there than are answered)
      nq = nq < a.q_len ? nq : a.q_len;
    } else {
      q_base = b * a.q_batch;
      len = a.kv_len;
      if (a.lens != nullptr) {
        const int l = a.lens[b];
        len = l < 0 ? 0 : l < len ? l : len;
      }
    }
  }
  // keys that the query of token `tok` sees
  __device__ __forceinline__ int sees(int tok) const {
    const int limit = KV4 ? before + tok + 1 : len;
    return limit < len ? limit : len;
  }
};

// (One instruction.  A NaN is passed on, which fmaxf would leave out, with another instruction for each operand to see to it: a column with a
// NaN among its scores has no other value.)
__device__ __forceinline__ float max3(float a, float b, float c) { return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c); }

// QT blocks of 16 columns of a wavefront
template <bool KV4, int DP, int QT>
struct Columns {
  static constexpr int J = DP / 32, CH = DP / 16;
  h8 q[QT][J];
  int limit[QT], row[QT];  // keys that this lane's column sees; its row of the output, or -1
  f4 o[QT][CH], l[QT];
  float m[QT], limit_s[QT], off[QT];  // the maxima in log2 units; the scores beyond which they move; what takes them off, and adds the shift

  // block i begins at column first(i)
  template <class First>
  __device__ __forceinline__ void load(const AttendArgs& a, const Span<KV4>& span, int kh, int g, int r, First first) {
#pragma unroll
    for (int i = 0; i < QT; ++i) {
      const int col = first(i) + r, tok = a.rep == 1 ? col : col / a.rep, head = kh * a.rep + (col - tok * a.rep);
      const bool in = col < span.nq * a.rep;
      row[i] = in ? (span.t0 + tok) * a.heads + head : -1;
      limit[i] = span.sees(tok);
      const _Float16* p = a.q + span.q_base + tok * a.q_token + head * a.q_head;
#pragma unroll
      for (int j = 0; j < J; ++j) q[i][j] = in && 32 * j + 8 * g < a.D ? *(const h8*)(p + 32 * j + 8 * g) : h8(0);
    }
    clear();
  }
  // no key seen
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < QT; ++i) {
      m[i] = limit_s[i] = -__builtin_inff();
      off[i] = kShift;
      l[i] = f4(0);
#pragma unroll
      for (int t = 0; t < CH; ++t) o[i][t] = f4(0);
    }
  }

  // Scores^T of 32 keys to p^T, in three steps.  hidden(i, t, e): whether block i's column of this lane does not see key 16 t + 4 g + e
  // (of the first N blocks)
  template <int N, class Hidden>
  __device__ __forceinline__ void hide(f4 (&s)[N][2], Hidden hidden) const {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[i][t][e] = hidden(i, t, e) ? -__builtin_inff() : s[i][t][e];
  }
  // Moves the maxima if a score passes one by kSlack, and rescales the sums.
  template <int N>
  __device__ __forceinline__ void follow(const f4 (&s)[N][2], const AttendArgs& a) {
    float top[N];
    bool moves = false;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      top[i] = max3(max3(s[i][0][0], s[i][0][1], s[i][0][2]), max3(s[i][0][3], s[i][1][0], s[i][1][1]), max3(s[i][1][2], s[i][1][3], s[i][1][3]));
      moves |= top[i] > limit_s[i];
    }
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(moves) != 0, 0)) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        float n = fmaxf(top[i], __shfl_xor(top[i], 16));
        n = fmaxf(n, __shfl_xor(n, 32)) * a.c;
        n = fmaxf(n, m[i]);
        const float f = m[i] == n ? 1.0f : __builtin_amdgcn_exp2f(m[i] - n);  // (-inf by -inf: nothing there to scale)
        m[i] = n;
        limit_s[i] = (n + kSlack) * a.inv_c;
        off[i] = kShift - (n == -__builtin_inff() ? 0.0f : n);
        l[i] *= f;
#pragma unroll
        for (int t = 0; t < CH; ++t) o[i][t] *= f;
      }
    }
  }
  template <int N>
  __device__ __forceinline__ void weights(const f4 (&s)[N][2], float c, h8 (&p)[N]) const {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) p[i][4 * t + e] = (_Float16)__builtin_amdgcn_exp2f(__builtin_fmaf(s[i][t][e], c, off[i]));
  }
  template <int N>
  __device__ __forceinline__ void sum(const h8 (&p)[N]) {
    const _Float16 u = (_Float16)1.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) l[i] = mfma16(h8{u, u, u, u, u, u, u, u}, p[i], l[i]);
  }

  // Lane 16 g + r has channels 16 t + 4 g .. + 3 of its column in o[.][t].  Whole results go out by 8 channels: two blocks of channels' odd and
  // even groups of lanes change places, and four lanes write 64 bytes of a row.
  __device__ __forceinline__ void store(const AttendArgs& a, int part, int g) const {
#pragma unroll
    for (int i = 0; i < QT; ++i) {
      const int64_t at = (int64_t)part * a.tokens * a.heads + row[i];
      if (a.parts > 1) {
        if (row[i] < 0) continue;
        if (g == 0) {
          a.part_ml[2 * at] = m[i];
          a.part_ml[2 * at + 1] = l[i][0];
        }
#pragma unroll
        for (int t = 0; t < CH; ++t)
          if (16 * t + 4 * g < a.D) *(f4*)(a.part_o + at * a.D + 16 * t + 4 * g) = o[i][t];
        continue;
      }
      const float f = l[i][0] == 0.0f ? 0.0f : __builtin_amdgcn_rcpf(l[i][0]);
#pragma unroll
      for (int t = 0; t < CH; t += 2) {
        u4 w;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const f4 x = o[i][t], y = o[i][t + 1];
          const h2 p = {(_Float16)(x[2 * e] * f), (_Float16)(x[2 * e + 1] * f)}, q = {(_Float16)(y[2 * e] * f), (_Float16)(y[2 * e + 1] * f)};
          const auto s = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, p), __builtin_bit_cast(uint32_t, q), false, false);
          w[e] = s[0];
          w[2 + e] = s[1];
        }
        const int c = 16 * (t + (g & 1)) + 8 * (g >> 1);
        if (row[i] >= 0 && c < a.D) *(u4*)(a.out + (int64_t)row[i] * a.D + c) = w;
      }
    }
  }
};

// the kernel for many columns (attend_tiles.hip)
void launch_attend_tiles(bool kv4, AttendArgs a, hipStream_t s);

}  // namespace gpusq
