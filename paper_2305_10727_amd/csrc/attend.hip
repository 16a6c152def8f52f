// Attention of few queries to keys and values of another length: over the paged 4-bit cache (attention_kv4) and over an encoder's fp16
// states (cross_attention).  A workgroup's wavefronts have the same columns and deal out the keys: what bounds such a call is the keys'
// bytes, so they go from memory straight into the registers of the one wavefront that multiplies them.
// Over the cache, one new token, 32 heads of 128 over 8: 131071 tokens (151 MB) in 37 us with the join, 4.0 TB/s; 64 sequences of up to 4096
// (191 MB) 48 us, 4.0 TB/s.  A large copy has 5.0.  One token to the 257 states of an image, 16 heads of 80: 5.7 us, a launch and four trips
// to memory (queries and first keys, second keys, the sums through LDS, the output).
#include "attend.h"

namespace gpusq {

namespace {

// 32 keys of the cache as they lie: codes and scales of keys, of values
template <int DP>
struct Keys4 {
  static constexpr int J = DP / 32;
  typename WordsOf<J>::type w[2];
  typename WordsOf<J / 2>::type s[2];
  __device__ __forceinline__ void load(const uint8_t* page, int half, int g, int r) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int key = half * 32 + t * 16 + r;
      w[t] = load_words<J>(page + key * (DP / 2) + g * J * 4);
      s[t] = load_words<J / 2>(page + key_scales_at(DP) + key * J * 2);
    }
  }
};
template <int DP>
struct Values4 {
  static constexpr int CH = DP / 16;
  typename WordsOf<CH / 2>::type w[2];
  u2 s[2];
  __device__ __forceinline__ void load(const uint8_t* page, int half, int g, int r) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int quad = half * 8 + t * 4 + g;
      w[t] = load_words<CH / 2>(page + value_codes_at(DP) + (quad * 16 + r) * (2 * CH));
      s[t] = load_words<2>(page + value_scales_at(DP) + (r * CH / 32 * kPageTokens + quad * 4) * 2);
    }
  }
};

constexpr int waves_per_simd(bool kv4, int DP, int QT) { return DP > 128 ? 1 : QT == 1 ? (kv4 || DP == 64 ? 4 : 3) : 2; }

// KV4: over the cache, else fp16 states.  QT: blocks of 16 columns, the same ones for each of WK wavefronts, which deal out the keys and join
// their sums in LDS.  MASKED: over the cache a tree of new tokens, whose words are looked at for the last tiles only, those that reach behind the
// history; over states a mask of bytes.
template <bool KV4, int DP, int QT, int WK, bool MASKED>
__global__ void __launch_bounds__(64 * WK, waves_per_simd(KV4, DP, QT)) attend_few_kernel(const AttendArgs a) {
  constexpr int J = DP / 32, CH = DP / 16;
  const int lane = threadIdx.x & 63, wk = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, r = lane & 15;
  Work w;
  if (!w.find(a)) return;
  const Span<KV4> span(a, w.b);
  constexpr bool TREE = KV4 && MASKED;
  const int cols = span.nq * a.rep, col0 = w.block * 16 * QT, len = span.len;
  if (col0 >= cols) return;  // the whole workgroup, like above
  Columns<KV4, DP, QT> x;
  x.load(a, span, w.kh, g, r, [&](int i) { return col0 + 16 * i; });
  const int least = TREE ? span.before : span.sees(col0 / a.rep);  // every column sees the keys in front of it, none those from `most` on
  const int most = TREE ? len : span.sees((col0 + 16 * QT < cols ? col0 + 16 * QT - 1 : cols - 1) / a.rep);
  // the bits of block i's column of this lane, and which row of the output it is: formed where they are used, the loop has no registers to keep them in
  auto words = [&](int i) {
    const int col = col0 + 16 * i + r < cols ? col0 + 16 * i + r : cols - 1;
    return a.tree + (int64_t)(span.t0 + (a.rep == 1 ? col : col / a.rep)) * a.tree_words;
  };
  auto row_of = [&](int i) {
    const int col = col0 + 16 * i + r, tok = a.rep == 1 ? col : col / a.rep;
    return col < cols ? (span.t0 + tok) * a.heads + w.kh * a.rep + (col - tok * a.rep) : -1;
  };
  const int tiles = most > 0 ? (most + 31) >> 5 : 0;
  const int begin = w.part * a.part_tiles, end = begin + a.part_tiles < tiles ? begin + a.part_tiles : tiles;
  // The first keys, values and the queries are waited for together, in front of the loop: left to itself the compiler waits at its top, for
  // whatever order these were requested in, which in later rounds means for the values requested just before.
  auto first_wait = [] { __builtin_amdgcn_s_waitcnt(0x0F70); };  // vmcnt(0)

  if constexpr (KV4) {
    // a wavefront takes whole pages: both halves of one, then the next of its own
    const int32_t* table = a.table + (int64_t)w.b * a.max_pages;
    auto page_at = [&](int number) { return a.cache + ((int64_t)number * a.kv_heads + w.kh) * page_bytes(DP); };
    auto after = [&](int tile) { return tile & 1 ? tile + 2 * WK - 1 : tile + 1; };
    auto page_of = [&](int tile) { return tile < end ? table[tile >> 1] : 0; };
    Keys4<DP> k;
    Values4<DP> v;
    int tile = begin + 2 * wk;
    // Page numbers are read a tile ahead of the keys, keys a product ahead, whether there are more or not: of loads that are left out at the
    // end the compiler makes registers without a value, and has then put 72 times a scale where the scale was.  (Also a branch less.)
    // A number that is no page is read as page 0 and not seen.
    int number = page_of(tile), next = page_of(after(tile));
    bool there = (unsigned)number < (unsigned)a.num_pages;
    const uint8_t* page = page_at(there ? number : 0);
    k.load(page, 0, g, r);  // (without a tile of its own: page 0, not used)
    v.load(page, 0, g, r);
    first_wait();
    while (tile < end) {
      const int key0 = tile * 32;
      f4 s[QT][2] = {};
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const h2 pair = __builtin_bit_cast(h2, (unsigned)k.s[t][j / 2]), sc = {pair[j & 1], pair[j & 1]};
          h2 c[4];
          codes_to_halves(k.w[t][j], sc, sc * (_Float16)-72.0f, c);
          const h8 ka = join(c[0], c[1], c[2], c[3]);
#pragma unroll
          for (int i = 0; i < QT; ++i) s[i][t] = mfma16(ka, x.q[i][j], s[i][t]);
        }
      const int ahead = after(tile);
      const bool next_there = (unsigned)next < (unsigned)a.num_pages;
      const uint8_t* next_page = page_at(next_there ? next : 0);
      k.load(next_page, ahead & 1, g, r);  // (behind the last tile: page 0 once more)
      next = page_of(after(ahead));
      const bool check = key0 + 32 > least || !there;
      h8 p[QT];
      if constexpr (TREE) {
        if (check) {
          unsigned seen[QT];
#pragma unroll
          for (int i = 0; i < QT; ++i) seen[i] = there ? tree_keys(words(i), a.tree_words, least, len, key0) >> (4 * g) : 0u;
          x.hide(s, [&](int i, int t, int e) { return (seen[i] >> (16 * t + e) & 1) == 0; });
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            v.s[t] = scales_in_front(v.s[t], there ? len - (key0 + 16 * t + 4 * g) : 0);
            const unsigned bad = take_out_infinite(v.s[t], CH * r < a.D, g);
#pragma unroll
            for (int i = 0; i < QT; ++i)
#pragma unroll
              for (int e = 0; e < 4; ++e) s[i][t][e] = (seen[i] >> (16 * t) & bad) >> e & 1 ? __builtin_nanf("") : s[i][t][e];
          }
        }
      } else if (check) {
        x.hide(s, [&](int i, int t, int e) { return key0 + 16 * t + 4 * g + e >= (there ? x.limit[i] : 0); });
      }
      x.follow(s, a);
      x.weights(s, a.c, p);
      x.sum(p);
      if (!TREE && check) {
#pragma unroll
        for (int t = 0; t < 2; ++t) v.s[t] = scales_in_front(v.s[t], there ? len - (key0 + 16 * t + 4 * g) : 0);
      }
      h2 sc[4], off[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        sc[i] = __builtin_bit_cast(h2, (unsigned)v.s[i >> 1][i & 1]);
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
          for (int i = 0; i < QT; ++i) x.o[i][4 * qd + e] = mfma16(va, p[i], x.o[i][4 * qd + e]);
        }
      }
      v.load(next_page, ahead & 1, g, r);
      tile = ahead;
      there = next_there;
    }
  } else {
    const _Float16 *kp = a.k + w.b * a.k_batch + w.kh * a.k_head + 8 * g, *vp = a.v + w.b * a.v_batch + w.kh * a.v_head + CH * r;
    const uint8_t* mask = MASKED ? a.mask + (int64_t)w.b * a.kv_len : nullptr;
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
    first_wait();
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
          for (int i = 0; i < QT; ++i) s[i][t] = mfma16(k[t][j], x.q[i][j], s[i][t]);
      if (tile + WK < end) load_k((tile + WK) * 32);
      h8 p[QT];
      if (MASKED || key0 + 32 > len) x.hide(s, [&](int, int t, int e) { return ((vis >> (4 * t + e)) & 1) == 0 || key0 + 16 * t + 4 * g + e >= len; });
      x.follow(s, a);
      x.weights(s, a.c, p);
      x.sum(p);
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
          for (int i = 0; i < QT; ++i) x.o[i][h * VW + c] = mfma16(va, p[i], x.o[i][h * VW + c]);
        }
      if (tile + WK < end) load_v((tile + WK) * 32);
    }
  }

  // Through LDS, of a tree a block of 16 columns at a time (three or four of 8 wavefronts' are more than it holds), else all in one trip (of 17 to 32 columns two
  // would take 1 to 3 % of a call more: 32 heads of 128 over 8, 8 tokens of 256 sequences of 100 31.3 us in one, 32.2 in two; 1000 states 13.1 and 13.4):
  // every wavefront's sums, maxima and sums of weights, then a thread for each (column, four channels).
  // Column c keeps its quad i in place i ^ (c % 16): what lanes write together lies in different banks.
  constexpr int QUADS = DP / 4, TRIP = TREE ? 1 : QT, COLS = 16 * TRIP;
  __shared__ f4 sums[WK][COLS][QUADS];
  __shared__ float ml[WK][2][COLS];
  __shared__ int rows[COLS];
#pragma unroll
  for (int i0 = 0; i0 < QT; i0 += TRIP) {
    if (i0 > 0) {
      if (col0 + 16 * i0 >= cols) break;
      __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < TRIP; ++j) {
      const int i = i0 + j, c = 16 * j + r;
      if (g == 0) {
        ml[wk][0][c] = x.m[i];
        ml[wk][1][c] = x.l[i][0];
        if (wk == 0) rows[c] = TREE ? row_of(i) : x.row[i];
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int t = 0; t < CH; t += 4) sums[wk][c][(((4 * g + e) * CH + t) / 4) ^ r] = f4{x.o[i][t][e], x.o[i][t + 1][e], x.o[i][t + 2][e], x.o[i][t + 3][e]};
    }
    __syncthreads();
    for (int at = threadIdx.x; at < COLS * QUADS; at += 64 * WK) {
      const int col = at / QUADS, quad = at % QUADS, row = rows[col];
      if (row < 0 || 4 * quad >= a.D) continue;
      float top = ml[0][0][col];
#pragma unroll
      for (int k = 1; k < WK; ++k) top = fmaxf(top, ml[k][0][col]);
      const float ref = top == -__builtin_inff() ? 0.0f : top;
      float total = 0.0f;
      f4 y = f4(0);
#pragma unroll
      for (int k = 0; k < WK; ++k) {
        const float f = __builtin_amdgcn_exp2f(ml[k][0][col] - ref);
        total += ml[k][1][col] * f;
        y += sums[k][col][quad ^ (col & 15)] * f;
      }
      if (a.parts > 1) {
        const int64_t place = (int64_t)w.part * a.tokens * a.heads + row;
        if (quad == 0) {
          a.part_ml[2 * place] = top;
          a.part_ml[2 * place + 1] = total;
        }
        *(f4*)(a.part_o + place * a.D + 4 * quad) = y;
      } else {
        const float f = total == 0.0f ? 0.0f : 1.0f / total;
        *(h4*)(a.out + (int64_t)row * a.D + 4 * quad) = h4{(_Float16)(y[0] * f), (_Float16)(y[1] * f), (_Float16)(y[2] * f), (_Float16)(y[3] * f)};
      }
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
  const float f = m == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(m - top);  // a part without a visible key (scores that are no numbers: 0 times its sum is NaN)
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

// Few parts: a thread for four channels of a row.  The maxima are requested side by side, and so are the sums, four parts at a time.
__global__ void __launch_bounds__(256) join_few_parts_kernel(const float* __restrict__ part_o, const float* __restrict__ part_ml, _Float16* __restrict__ out, int64_t rows,
                                                              int D, int parts) {
  const int quads = D / 4, at = threadIdx.x / quads, quad = threadIdx.x - at * quads;
  const int64_t row = (int64_t)blockIdx.x * (256 / quads) + at;
  if (at >= 256 / quads || row >= rows) return;
  typedef float f2 __attribute__((ext_vector_type(2)));
  f2 ml[kFewParts];
#pragma unroll
  for (int p = 0; p < kFewParts; ++p)
    ml[p] = p < parts ? *(const f2*)(part_ml + 2 * (p * rows + row)) : f2{-__builtin_inff(), 0.0f};
  float top = ml[0][0];
#pragma unroll
  for (int p = 1; p < kFewParts; ++p) top = fmaxf(top, ml[p][0]);
  float l = 0.0f;
  f4 o = f4(0);
#pragma unroll
  for (int p0 = 0; p0 < kFewParts; p0 += 4) {
    if (p0 >= parts) break;
    f4 v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = *(const f4*)(part_o + ((p0 + i < parts ? p0 + i : parts - 1) * rows + row) * D + 4 * quad);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f2 x = ml[p0 + i];
      // a part without a visible key (one whose scores are no numbers has no maximum either, but its sum is NaN, and has to be the row's)
      const bool none = x[0] == -__builtin_inff() && x[1] == 0.0f;
      const float f = none ? 0.0f : __builtin_amdgcn_exp2f(x[0] - top);
      l += none ? 0.0f : x[1] * f;
      o += none ? f4(0) : v[i] * f;
    }
  }
  const float r = l == 0.0f ? 0.0f : 1.0f / l;
  *(h4*)(out + row * D + 4 * quad) = h4{(_Float16)(o[0] * r), (_Float16)(o[1] * r), (_Float16)(o[2] * r), (_Float16)(o[3] * r)};
}

template <bool KV4, int DP, int QT, int WK, bool MASKED>
void launch_masked(AttendArgs a, hipStream_t s) {
  a.col_blocks = (int)ceil_div((int64_t)a.q_len * a.rep, 16 * QT);
  attend_few_kernel<KV4, DP, QT, WK, MASKED><<<Work::workgroups(a), 64 * WK, 0, s>>>(a);
}
template <bool KV4, int DP, int QT, int WK>
void launch_shape(const AttendArgs& a, hipStream_t s) {
  if constexpr (!KV4) {
    if (a.mask != nullptr) return launch_masked<KV4, DP, QT, WK, true>(a, s);
  }
  launch_masked<KV4, DP, QT, WK, false>(a, s);
}

template <int DP, int QT>
void launch_tree(const AttendArgs& a, const AttendShape& shape, hipStream_t s) {
  shape.threads == 512 ? launch_masked<true, DP, QT, 8, true>(a, s) : launch_masked<true, DP, QT, 4, true>(a, s);
}

template <bool KV4, int DP>
void launch_head(const AttendArgs& a, hipStream_t s) {
  const AttendShape shape = attend_shape(KV4, DP, (int64_t)a.q_len * a.rep, KV4 || tiles_reach(a.k_token, a.v_token), KV4 && a.tree != nullptr ? (int64_t)a.batch * a.kv_heads : 0);
  if constexpr (KV4) {
    if (a.tree != nullptr && !shape.many) {
      if (shape.columns == 16) return launch_masked<KV4, DP, 1, 8, true>(a, s);
      if constexpr (tree_blocks(DP) >= 3) {
        if (shape.columns == 32) return launch_tree<DP, 2>(a, shape, s);
        if (shape.columns == 48) return launch_tree<DP, 3>(a, shape, s);
      }
      if constexpr (tree_blocks(DP) == 4) launch_tree<DP, 4>(a, shape, s);
      return;
    }
  }
  if (shape.many)
    launch_attend_tiles(KV4, a, s);
  else if (shape.columns == 16)
    launch_shape<KV4, DP, 1, 8>(a, s);
  else if constexpr (DP < 256)
    launch_shape<KV4, DP, 2, 4>(a, s);
}

}  // namespace

// The keys are cut into parts where the (batch, key head, block of columns) are too few workgroups for the device.
// Few columns: 256 workgroups, one a CU (8 key heads, 131071 tokens: 37.4 us; 512 workgroups 38.0, 1024 42.7), with 8 tiles (256 keys) each or
// more: a tile for each wavefront.  (One token, in one piece and in parts: of 32 heads over 8 of 128 after 8000 tokens 10.5 in 32 parts, 12.8 in 8;
// 16 heads of 128 to 1000 states 12.3 and 8.6, of 256 24 and 13.)  What one piece does in 8.5 us stays one, as the second launch and the workspace
// take the host 4: 1024 keys at most, over the cache 128K channels of keys, over states 64K (16 heads of 64, 1000 states: 8.3 and 7.2).
// Many columns: parts of 16 tiles at least.  (Trees of more than 16 columns have registers for one workgroup a CU: 256 of them or a few less, not more.)
AttendParts attend_parts(bool kv4, int64_t batch, int64_t q_len, int64_t heads, int64_t kv_heads, int64_t head_dim, int64_t most_keys, bool tree) {
  const int64_t tiles = ceil_div(most_keys > 0 ? most_keys : 1, 32), cols = q_len * (heads / kv_heads);
  const AttendShape shape = attend_shape(kv4, padded_head((int)head_dim), cols, true, tree ? batch * kv_heads : 0);
  const bool few = !shape.many;
  const int64_t groups = batch * kv_heads * ceil_div(cols, shape.columns);
  int64_t parts = few && (!tree || shape.columns == 16) ? ceil_div(256, groups) : (kv4 ? 256 : 512) / groups;
  const int64_t one = (kv4 ? 4096 : 2048) / padded_head((int)head_dim);
  const int64_t most = !few ? ceil_div(tiles, 16) : tiles <= (one < 32 ? one : 32) ? 1 : ceil_div(tiles, 8);
  parts = parts < 1 ? 1 : parts < most ? parts : most;
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
  if (p.parts <= kFewParts)
    join_few_parts_kernel<<<(unsigned)join_workgroups(rows, a.D, p.parts), 256, 0, s>>>(a.part_o, a.part_ml, a.out, rows, a.D, p.parts);
  else
    join_parts_kernel<<<(unsigned)join_workgroups(rows, a.D, p.parts), 256, 0, s>>>(a.part_o, a.part_ml, a.out, (int)rows, a.D, p.parts);
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
  a.inv_c = 1.0f / a.c;
  a.cache = (const uint8_t*)x.cache;
  a.table = x.block_table;
  a.cu_q = x.cu_q;
  a.tree = x.tree;
  a.tree_words = (int)x.tree_words;
  a.max_pages = (int)x.max_pages;
  a.num_pages = (int)x.num_pages;
  a.tokens = (int)x.tokens;
  a.lens = x.kv_lens;
  return run(a, true, attend_parts(true, x.batch, x.max_q, x.heads, x.kv_heads, x.head_dim, x.max_pages * kPageTokens, x.tree != nullptr), x.workspace, s);
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
  a.inv_c = 1.0f / a.c;
  a.lens = x.kv_lens;
  a.mask = x.key_mask;
  return run(a, false, attend_parts(false, x.batch, x.q_len, x.heads, x.kv_heads, x.head_dim, x.kv_len), x.workspace, s);
}

}  // namespace gpusq
