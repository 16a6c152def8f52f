// Attention of a few or many queries to keys and values of another length: over the paged 4-bit cache (attention_kv4) and over an
// encoder's fp16 states (cross_attention).  One pass over the keys with the running maximum and sum of the softmax; scores never
// leave the registers.
//
//   o[q] = sum_j exp(s_qj - m_q) v_j / sum_j exp(s_qj - m_q),  s_qj = scale q . k_j,  m_q the largest visible s_qj;  0 where none is visible
//
// A wavefront takes 32 keys at a time.  The first product is turned over, scores^T = K Q^T, so that a lane of the result has one query
// (column lane % 16) and the keys 4 g .. + 3 (g = lane / 16) of either 16: these are, as they lie, the second operand of
// output^T = V^T P^T, if V^T's k runs over the same keys in the same order.  Nothing crosses lanes between the products.
// Queries of the heads that share a key head are columns side by side: column = token * (heads per key head) + head.
//
// The maximum moves only when a score passes it by 2^8 (kSlack): p = 2^(s - m + 6) then lies in fp16 up to 2^14, and down to 2^-24,
// that is to 2^-30 of the largest where it has not moved.  Most tiles need neither the maximum across lanes nor a rescaled sum.
// P is rounded to fp16 for the matrix instruction; its sum is of the unrounded 32-bit values.
#include "kv4.h"

namespace gpusq {

namespace {

constexpr float kLog2e = 1.4426950408889634f, kShift = 6.0f, kSlack = 8.0f;

struct AttendArgs {
  const _Float16* q;
  _Float16* out;
  int64_t q_batch, q_token, q_head;  // in values
  int64_t o_token;                   // out: [token][heads][D]
  int heads, kv_heads, rep, D, batch, q_len;
  float c;  // scale * log2(e)
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

template <int N>
__device__ __forceinline__ void load_words(const uint8_t* p, unsigned (&w)[N]) {
  if constexpr (N == 2) {
    const u2 v = *(const u2*)p;
    w[0] = v[0];
    w[1] = v[1];
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const u4 v = *(const u4*)(p + 4 * i);
#pragma unroll
      for (int j = 0; j < 4; ++j) w[i + j] = v[j];
    }
  }
}

// 32 keys of the cache as they lie: codes and scales of keys, of values
template <int DP>
struct Keys4 {
  static constexpr int J = DP / 32;
  unsigned w[2][J];
  h2 s[2][J / 2];
  __device__ __forceinline__ void load(const uint8_t* page, int half, int g, int r) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int key = half * 32 + t * 16 + r;
      load_words<J>(page + key * (DP / 2) + g * J * 4, w[t]);
      unsigned u[J / 2];
      if constexpr (J == 2) u[0] = *(const unsigned*)(page + key_scales_at(DP) + key * J * 2);
      else load_words<J / 2>(page + key_scales_at(DP) + key * J * 2, u);
#pragma unroll
      for (int i = 0; i < J / 2; ++i) s[t][i] = __builtin_bit_cast(h2, u[i]);
    }
  }
};
template <int DP>
struct Values4 {
  static constexpr int CH = DP / 16;
  unsigned w[2][CH / 2];
  h4 s[2];
  __device__ __forceinline__ void load(const uint8_t* page, int half, int g, int r) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int quad = half * 8 + t * 4 + g;
      load_words<CH / 2>(page + value_codes_at(DP) + (quad * 16 + r) * (2 * CH), w[t]);
      s[t] = *(const h4*)(page + value_scales_at(DP) + (r * CH / 32 * kPageTokens + quad * 4) * 2);
    }
  }
};

__device__ __forceinline__ h8 join(h2 a, h2 b, h2 c, h2 d) { return h8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]}; }

constexpr int waves_per_simd(bool kv4, int DP, int QT) { return DP > 128 ? 1 : QT == 1 ? (kv4 || DP == 64 ? 4 : 3) : QT == 2 ? 2 : 1; }

// KV4: over the cache, else fp16 states.  QT: blocks of 16 columns of a wavefront.  WQ x WK wavefronts: WQ have columns of their own, WK
// deal out the tiles of 32 keys and join their sums in LDS.
template <bool KV4, int DP, int QT, int WQ, int WK, bool MASKED>
__global__ void __launch_bounds__(64 * WQ * WK, waves_per_simd(KV4, DP, QT)) attend_kernel(const AttendArgs a) {
  constexpr int J = DP / 32, CH = DP / 16;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, r = lane & 15;
  const int wq = wave / WK, wk = wave % WK;
  // workgroups of one key head run on one XCD, whose L2 then reads its keys and values once
  const int units = a.batch * a.kv_heads, per_unit = a.col_blocks * a.parts;
  const int xcd = blockIdx.x & 7, rest = blockIdx.x >> 3;
  const int unit = rest / per_unit * 8 + xcd;
  if (unit >= units) return;
  const int part = rest % per_unit / a.col_blocks, block = rest % a.col_blocks;
  const int b = unit / a.kv_heads, kh = unit % a.kv_heads;

  int t0 = b * a.q_len, nq = a.q_len, len;
  int64_t q_base;
  if constexpr (KV4) {
    if (a.cu_q != nullptr) {
      t0 = a.cu_q[b];
      const int t1 = a.cu_q[b + 1];
      nq = t0 >= 0 && t1 <= a.tokens && t1 > t0 ? (t1 - t0 < a.q_len ? t1 - t0 : a.q_len) : 0;
    }
    q_base = (int64_t)t0 * a.q_token;
    const int most = a.max_pages * kPageTokens;
    len = a.lens[b];
    len = len < 0 ? 0 : len < most ? len : most;
  } else {
    q_base = b * a.q_batch;
    len = a.kv_len;
    if (a.lens != nullptr) {
      const int l = a.lens[b];
      len = l < 0 ? 0 : l < len ? l : len;
    }
  }
  const int cols = nq * a.rep, col0 = (block * WQ + wq) * 16 * QT;
  if (block * WQ * 16 * QT >= cols) return;  // the whole workgroup

  // queries: column c is token c / rep, head kh * rep + c % rep
  h8 q[QT][J];
  int limit[QT], row[QT];  // keys that the column sees; the row of the output, or -1
  int least = len;         // of the limits of this wavefront's columns (the first column's)
#pragma unroll
  for (int i = 0; i < QT; ++i) {
    const int col = col0 + 16 * i + r, tok = col / a.rep, head = kh * a.rep + (col - tok * a.rep);
    const bool in = col < cols;
    row[i] = in ? (t0 + tok) * a.heads + head : -1;
    limit[i] = len;
    if constexpr (KV4) {
      limit[i] = len - nq + tok + 1;
      limit[i] = limit[i] < len ? limit[i] : len;
    }
    const _Float16* p = a.q + q_base + tok * a.q_token + head * a.q_head;
#pragma unroll
    for (int j = 0; j < J; ++j) q[i][j] = in && 32 * j + 8 * g < a.D ? *(const h8*)(p + 32 * j + 8 * g) : h8(0);
  }
  if constexpr (KV4) {
    const int first = len - nq + col0 / a.rep + 1;
    least = first < len ? first : len;
  }
  int most_seen = len;  // no column of the workgroup sees a key from here on
  if constexpr (KV4) {
    const int last_col = (block + 1) * WQ * 16 * QT < cols ? (block + 1) * WQ * 16 * QT - 1 : cols - 1;
    const int last = len - nq + last_col / a.rep + 1;
    most_seen = last < len ? last : len;
  }
  const int tiles = most_seen > 0 ? (most_seen + 31) >> 5 : 0;
  const int begin = part * a.part_tiles, end = begin + a.part_tiles < tiles ? begin + a.part_tiles : tiles;

  f4 o[QT][CH] = {};
  float m[QT], l[QT];
#pragma unroll
  for (int i = 0; i < QT; ++i) {
    m[i] = -__builtin_inff();
    l[i] = 0.0f;
  }

  // scores^T of a tile to p^T; vis: bit 4 t + e says whether this lane's key 16 t + 4 g + e is there at all
  auto softmax = [&](f4 (&s)[QT][2], int key0, bool check, unsigned vis, h8 (&p)[QT]) {
    if (check) {
#pragma unroll
      for (int i = 0; i < QT; ++i)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (!((vis >> (4 * t + e)) & 1) || key0 + 16 * t + 4 * g + e >= limit[i]) s[i][t][e] = -__builtin_inff();
    }
    float top[QT];
    bool moves = false;
#pragma unroll
    for (int i = 0; i < QT; ++i) {
      top[i] = fmaxf(fmaxf(fmaxf(s[i][0][0], s[i][0][1]), fmaxf(s[i][0][2], s[i][0][3])), fmaxf(fmaxf(s[i][1][0], s[i][1][1]), fmaxf(s[i][1][2], s[i][1][3]))) * a.c;
      moves |= top[i] > m[i] + kSlack;
    }
    if (__builtin_amdgcn_ballot_w64(moves) != 0) {
#pragma unroll
      for (int i = 0; i < QT; ++i) {
        float n = fmaxf(top[i], __shfl_xor(top[i], 16));
        n = fmaxf(n, __shfl_xor(n, 32));
        n = fmaxf(n, m[i]);
        const float f = m[i] == n ? 1.0f : __builtin_amdgcn_exp2f(m[i] - n);  // (-inf by -inf: nothing there to scale)
        m[i] = n;
        l[i] *= f;
#pragma unroll
        for (int t = 0; t < CH; ++t) o[i][t] *= f;
      }
    }
#pragma unroll
    for (int i = 0; i < QT; ++i) {
      const float off = kShift - (m[i] == -__builtin_inff() ? 0.0f : m[i]);
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float v = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i][t][e], a.c, off));
          l[i] += v;
          p[i][4 * t + e] = (_Float16)v;
        }
    }
  };

  if constexpr (KV4) {
    // a wavefront takes whole pages: both halves of one, then the next of its own
    const int32_t* table = a.table + (int64_t)b * a.max_pages;
    auto page_at = [&](int number) { return a.cache + ((int64_t)number * a.kv_heads + kh) * page_bytes(DP); };
    auto after = [&](int tile) { return tile & 1 ? tile + 2 * WK - 1 : tile + 1; };
    auto page_of = [&](int tile, int otherwise) { return tile < end ? table[tile >> 1] : otherwise; };
    Keys4<DP> k;
    Values4<DP> v;
    int tile = begin + 2 * wk;
    // page numbers are read a tile ahead of the keys, keys a product ahead; a number that is no page is read as page 0 and not seen
    int number = page_of(tile, 0), next = page_of(after(tile), 0);
    bool there = (unsigned)number < (unsigned)a.num_pages;
    const uint8_t* page = page_at(there ? number : 0);
    if (tile < end) {
      k.load(page, 0, g, r);
      v.load(page, 0, g, r);
    }
    while (tile < end) {
      const int key0 = tile * 32;
      f4 s[QT][2] = {};
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const h2 sc = {k.s[t][j / 2][j & 1], k.s[t][j / 2][j & 1]};
          h2 c[4];
          codes_to_halves(k.w[t][j], sc, sc * (_Float16)-72.0f, c);
          const h8 ka = join(c[0], c[1], c[2], c[3]);
#pragma unroll
          for (int i = 0; i < QT; ++i) s[i][t] = mfma16(ka, q[i][j], s[i][t]);
        }
      const int ahead = after(tile);
      const bool next_there = (unsigned)next < (unsigned)a.num_pages;
      const uint8_t* next_page = page_at(next_there ? next : 0);
      if (ahead < end) k.load(next_page, ahead & 1, g, r);
      next = page_of(after(ahead), 0);
      const bool check = key0 + 32 > least || !there;
      h8 p[QT];
      softmax(s, key0, check, there ? 0xFFu : 0u, p);
      h4 vs[2] = {v.s[0], v.s[1]};
      if (check) {  // places behind the last token may hold anything: a scale of theirs may be infinite or NaN
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) vs[t][e] = there && key0 + 16 * t + 4 * g + e < len ? vs[t][e] : (_Float16)0.0f;
      }
      h2 sc[4], off[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        sc[i] = h2{vs[i >> 1][2 * (i & 1)], vs[i >> 1][2 * (i & 1) + 1]};
        off[i] = sc[i] * (_Float16)-72.0f;
      }
#pragma unroll
      for (int qd = 0; qd < CH / 4; ++qd) {
        h2 d[4][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) codes_to_halves(v.w[i >> 1][(i & 1) * (CH / 4) + qd], sc[i], off[i], d[i]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const h8 va = join(d[0][e], d[1][e], d[2][e], d[3][e]);
#pragma unroll
          for (int i = 0; i < QT; ++i) o[i][4 * qd + e] = mfma16(va, p[i], o[i][4 * qd + e]);
        }
      }
      if (ahead < end) v.load(next_page, ahead & 1, g, r);
      tile = ahead;
      there = next_there;
    }
  } else {
    const _Float16 *kp = a.k + b * a.k_batch + kh * a.k_head + 8 * g, *vp = a.v + b * a.v_batch + kh * a.v_head + CH * r;
    const uint8_t* mask = MASKED ? a.mask + (int64_t)b * a.kv_len : nullptr;
    constexpr int VW = CH < 8 ? 4 : 8;  // values of one load
    typedef _Float16 hv __attribute__((ext_vector_type(VW)));
    h8 k[2][J];
    hv v[2][4][CH / VW];
    auto load_k = [&](int key0) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int key = key0 + 16 * t + r;
#pragma unroll
        for (int j = 0; j < J; ++j) k[t][j] = key < len && 32 * j + 8 * g < a.D ? *(const h8*)(kp + key * a.k_token + 32 * j) : h8(0);
      }
    };
    auto load_v = [&](int key0) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int key = key0 + 16 * t + 4 * g + e;
#pragma unroll
          for (int h = 0; h < CH / VW; ++h) v[t][e][h] = key < len && CH * r + VW * h < a.D ? *(const hv*)(vp + key * a.v_token + VW * h) : hv(0);
        }
    };
    int tile = begin + wk;
    if (tile < end) {
      load_k(tile * 32);
      load_v(tile * 32);
    }
    for (; tile < end; tile += WK) {
      const int key0 = tile * 32;
      unsigned vis = 0xFFu;
      if constexpr (MASKED) {
        vis = 0;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int key = key0 + 16 * t + 4 * g + e;
            if (key < len && mask[key] != 0) vis |= 1u << (4 * t + e);
          }
      }
      f4 s[QT][2] = {};
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
          for (int i = 0; i < QT; ++i) s[i][t] = mfma16(k[t][j], q[i][j], s[i][t]);
      if (tile + WK < end) load_k((tile + WK) * 32);
      h8 p[QT];
      softmax(s, key0, MASKED || key0 + 32 > len, vis, p);
#pragma unroll
      for (int h = 0; h < CH / VW; ++h)
#pragma unroll
        for (int c = 0; c < VW; ++c) {
          h8 va;
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              va[4 * t + e] = v[t][e][h][c];
              if constexpr (MASKED) va[4 * t + e] = (vis >> (4 * t + e)) & 1 ? va[4 * t + e] : (_Float16)0.0f;  // (0 times infinity)
            }
#pragma unroll
          for (int i = 0; i < QT; ++i) o[i][h * VW + c] = mfma16(va, p[i], o[i][h * VW + c]);
        }
      if (tile + WK < end) load_v((tile + WK) * 32);
    }
  }

  // sums over the lanes that share a column
#pragma unroll
  for (int i = 0; i < QT; ++i) {
    l[i] += __shfl_xor(l[i], 16);
    l[i] += __shfl_xor(l[i], 32);
  }
  if constexpr (WK > 1) {
    __shared__ float ml[WQ][WK][2][16 * QT];
    __shared__ f4 sums[WQ][WK / 2][QT][CH][64];
    if (g == 0) {
#pragma unroll
      for (int i = 0; i < QT; ++i) {
        ml[wq][wk][0][16 * i + r] = m[i];
        ml[wq][wk][1][16 * i + r] = l[i];
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < QT; ++i) {
      float n = ml[wq][0][0][16 * i + r];
#pragma unroll
      for (int w = 1; w < WK; ++w) n = fmaxf(n, ml[wq][w][0][16 * i + r]);
      const float ref = n == -__builtin_inff() ? 0.0f : n;
      float total = 0.0f;
#pragma unroll
      for (int w = 0; w < WK; ++w) total += ml[wq][w][1][16 * i + r] * __builtin_amdgcn_exp2f(ml[wq][w][0][16 * i + r] - ref);
      const float f = __builtin_amdgcn_exp2f(m[i] - ref);
#pragma unroll
      for (int t = 0; t < CH; ++t) o[i][t] *= f;
      m[i] = n;
      l[i] = total;
    }
#pragma unroll
    for (int n = WK / 2; n > 0; n /= 2) {  // the upper half of the wavefronts hands its sums to the lower half
      if (wk >= n && wk < 2 * n) {
#pragma unroll
        for (int i = 0; i < QT; ++i)
#pragma unroll
          for (int t = 0; t < CH; ++t) sums[wq][wk - n][i][t][lane] = o[i][t];
      }
      __syncthreads();
      if (wk < n) {
#pragma unroll
        for (int i = 0; i < QT; ++i)
#pragma unroll
          for (int t = 0; t < CH; ++t) o[i][t] += sums[wq][wk][i][t][lane];
      }
      __syncthreads();
    }
    if (wk != 0) return;
  }
#pragma unroll
  for (int i = 0; i < QT; ++i) {
    if (row[i] < 0) continue;
    if (a.parts > 1) {
      const int64_t at = (int64_t)part * a.tokens * a.heads + row[i];
      if (g == 0) {
        a.part_ml[2 * at] = m[i];
        a.part_ml[2 * at + 1] = l[i];
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int t = 0; t < CH; t += 4)
          if ((4 * g + e) * CH + t < a.D) *(f4*)(a.part_o + at * a.D + (4 * g + e) * CH + t) = f4{o[i][t][e], o[i][t + 1][e], o[i][t + 2][e], o[i][t + 3][e]};
    } else {
      const float f = l[i] == 0.0f ? 0.0f : 1.0f / l[i];
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int t = 0; t < CH; t += 4)
          if ((4 * g + e) * CH + t < a.D)
            *(h4*)(a.out + (int64_t)row[i] * a.D + (4 * g + e) * CH + t) =
                h4{(_Float16)(o[i][t][e] * f), (_Float16)(o[i][t + 1][e] * f), (_Float16)(o[i][t + 2][e] * f), (_Float16)(o[i][t + 3][e] * f)};
    }
  }
}

// Joins the parts of a row: a workgroup for each.  Its threads read the parts' maxima side by side, then take (channels, share of the
// parts) each and add the shares up in LDS.
constexpr int kMostParts = 256;
__global__ void __launch_bounds__(256) join_parts_kernel(const float* __restrict__ part_o, const float* __restrict__ part_ml, _Float16* __restrict__ out, int rows, int D,
                                                          int parts) {
  __shared__ float weight[kMostParts], wave_max[4], wave_sum[4];
  __shared__ f4 sums[256];
  const int row = blockIdx.x, tid = threadIdx.x;
  float m = -__builtin_inff(), l = 0.0f;
  if (tid < parts) {
    const float* p = part_ml + 2 * ((int64_t)tid * rows + row);
    m = p[0];
    l = p[1];
  }
  float top = m;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
  if ((tid & 63) == 0) wave_max[tid >> 6] = top;
  __syncthreads();
  top = fmaxf(fmaxf(wave_max[0], wave_max[1]), fmaxf(wave_max[2], wave_max[3]));
  const float f = m == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(m - top);  // a part without a visible key: its sums may not be there
  weight[tid] = f;
  l *= f;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) l += __shfl_xor(l, d);
  if ((tid & 63) == 0) wave_sum[tid >> 6] = l;
  __syncthreads();
  l = (wave_sum[0] + wave_sum[1]) + (wave_sum[2] + wave_sum[3]);
  const int quads = D / 4, shares = 256 / quads, share = tid / quads, quad = tid - share * quads;
  f4 o = f4(0);
  if (share < shares) {
#pragma unroll 4
    for (int p = share; p < parts; p += shares) {
      const float w = weight[p];
      const f4 v = *(const f4*)(part_o + ((int64_t)p * rows + row) * D + 4 * quad);
      if (w != 0.0f) o += v * w;
    }
  }
  sums[tid] = o;
  __syncthreads();
  if (tid < quads) {
    for (int i = 1; i < shares; ++i) o += sums[i * quads + tid];
    const float r = l == 0.0f ? 0.0f : 1.0f / l;
    *(h4*)(out + (int64_t)row * D + 4 * tid) = h4{(_Float16)(o[0] * r), (_Float16)(o[1] * r), (_Float16)(o[2] * r), (_Float16)(o[3] * r)};
  }
}

template <bool KV4, int DP, int QT, int WQ, int WK>
void launch_shape(AttendArgs a, hipStream_t s) {
  a.col_blocks = (int)ceil_div((int64_t)a.q_len * a.rep, 16 * QT * WQ);
  const unsigned blocks = (unsigned)(ceil_div((int64_t)a.batch * a.kv_heads, 8) * 8 * a.col_blocks * a.parts);
  if constexpr (!KV4) {
    if (a.mask != nullptr) {
      attend_kernel<KV4, DP, QT, WQ, WK, true><<<blocks, 64 * WQ * WK, 0, s>>>(a);
      return;
    }
  }
  attend_kernel<KV4, DP, QT, WQ, WK, false><<<blocks, 64 * WQ * WK, 0, s>>>(a);
}

template <bool KV4, int DP>
void launch_head(const AttendArgs& a, hipStream_t s) {
  const int64_t cols = (int64_t)a.q_len * a.rep;
  constexpr int MOST = DP > 128 ? 2 : 4;
  if (cols <= 16)
    launch_shape<KV4, DP, 1, 1, 8>(a, s);
  else if (cols <= 32)
    launch_shape<KV4, DP, 2, 1, 4>(a, s);
  else if constexpr (KV4)
    launch_shape<KV4, DP, MOST, 1, 4>(a, s);
  else
    launch_shape<KV4, DP, 2, 4, 1>(a, s);
}

}  // namespace

// The keys are cut into parts where the (batch, key head) pairs alone are too few workgroups, of 32 tiles (1024 keys) at least
AttendParts attend_parts(int64_t batch, int64_t q_len, int64_t heads, int64_t kv_heads, int64_t most_keys) {
  const int64_t tiles = ceil_div(most_keys > 0 ? most_keys : 1, 32), cols = q_len * (heads / kv_heads);
  const int64_t groups = batch * kv_heads * ceil_div(cols, 64);
  int64_t parts = ceil_div(256, groups);
  if (parts > ceil_div(tiles, 32)) parts = ceil_div(tiles, 32);
  if (parts > kMostParts) parts = kMostParts;
  AttendParts p;
  p.tiles = (int)(ceil_div(ceil_div(tiles, parts), 2) * 2);
  p.parts = (int)ceil_div(tiles, p.tiles);
  return p;
}

static gpusq_status run(AttendArgs a, bool kv4, const AttendParts& p, void* workspace, hipStream_t s) {
  a.rep = a.heads / a.kv_heads;
  a.parts = p.parts;
  a.part_tiles = p.tiles;
  const int64_t rows = (int64_t)a.tokens * a.heads;
  a.part_o = (float*)workspace;
  a.part_ml = a.part_o + p.parts * rows * a.D;
  const int DP = padded_head(a.D);
  if (kv4)
    DP == 64 ? launch_head<true, 64>(a, s) : DP == 128 ? launch_head<true, 128>(a, s) : launch_head<true, 256>(a, s);
  else
    DP == 64 ? launch_head<false, 64>(a, s) : DP == 128 ? launch_head<false, 128>(a, s) : launch_head<false, 256>(a, s);
  gpusq_status st = check_launch();
  if (st != GPUSQ_OK || p.parts == 1) return st;
  join_parts_kernel<<<(unsigned)rows, 256, 0, s>>>(a.part_o, a.part_ml, a.out, (int)rows, a.D, p.parts);
  return check_launch();
}

gpusq_status launch_attention_kv4(const AttentionKv4& x, hipStream_t s) {
  AttendArgs a{};
  a.q = (const _Float16*)x.q;
  a.out = (_Float16*)x.out;
  a.q_token = x.heads * x.head_dim;
  a.q_head = x.head_dim;
  a.heads = (int)x.heads;
  a.kv_heads = (int)x.kv_heads;
  a.D = (int)x.head_dim;
  a.batch = (int)x.batch;
  a.q_len = (int)x.max_q;
  a.c = x.scale * kLog2e;
  a.cache = (const uint8_t*)x.cache;
  a.table = x.block_table;
  a.cu_q = x.cu_q;
  a.max_pages = (int)x.max_pages;
  a.num_pages = (int)x.num_pages;
  a.tokens = (int)x.tokens;
  a.lens = x.kv_lens;
  return run(a, true, attend_parts(x.batch, x.max_q, x.heads, x.kv_heads, x.max_pages * kPageTokens), x.workspace, s);
}

gpusq_status launch_cross_attention(const CrossAttention& x, hipStream_t s) {
  AttendArgs a{};
  a.q = (const _Float16*)x.q;
  a.k = (const _Float16*)x.k;
  a.v = (const _Float16*)x.v;
  a.out = (_Float16*)x.out;
  a.q_batch = x.q_stride[0];
  a.q_token = x.q_stride[1];
  a.q_head = x.q_stride[2];
  a.k_batch = x.k_stride[0];
  a.k_token = x.k_stride[1];
  a.k_head = x.k_stride[2];
  a.v_batch = x.v_stride[0];
  a.v_token = x.v_stride[1];
  a.v_head = x.v_stride[2];
  a.heads = (int)x.heads;
  a.kv_heads = (int)x.kv_heads;
  a.D = (int)x.head_dim;
  a.batch = (int)x.batch;
  a.q_len = (int)x.q_len;
  a.kv_len = (int)x.kv_len;
  a.tokens = (int)(x.batch * x.q_len);
  a.c = x.scale * kLog2e;
  a.lens = x.kv_lens;
  a.mask = x.key_mask;
  return run(a, false, attend_parts(x.batch, x.q_len, x.heads, x.kv_heads, x.kv_len), x.workspace, s);
}

}  // namespace gpusq
