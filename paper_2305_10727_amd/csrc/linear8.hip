// Linear layers in 8-bit integers with a scale for each token and each channel: Y = act(s_m w_n (q_m . c_n) + b_n), s_m = max|x_m| / 127,
// q_m = clamp(rint(x_m / s_m)).  This file: the codes of the tokens, the kernel for few of them, the choice; linear8_tiles.h: many tokens.
//
// Few tokens are bound by the bytes of the weights, one each; every other choice follows from reading them once, with much in flight:
//   - the weights stay as they are, rows of K bytes: a wavefront reads 64 consecutive bytes of 16 rows with an instruction, and the next 64 with the next;
//   - they are the first operand of the 16 x 16 x 64 instruction, whose rows are channels, and the tokens the second: one to 16 tokens cost the same;
//   - a workgroup's wavefronts share its channels and deal out K; their sums, which are exact, meet in LDS once a tile;
//   - a few of 32768 values in all each workgroup quantises itself, straight into the registers that are multiplied: no launch in front, no codes in memory.
// 9 tokens, 4096 -> 131072 (542 MB): 102 us with the quantiser, weights at 5.3 TB/s, where a large copy has 5.0.  1, 16 and 32 tokens, 5120 -> 13824
// (71 MB; 216 workgroups have four tiles each, 40 CUs none): 20, 23 and 26; 8, 16, 32 and 64, 4096 -> 4096: 12.4, 10.8, 12.9, 16.7; 1, 1024 -> 1024: 5.8.
#include "epilogue.h"
#include "gelu4.h"
#include "linear8_plan.h"

namespace gpusq {

// linear8_tiles.h by the channels of a tile
void launch_linear8_tiles8(const Linear8Args& a, const Tokens8Plan& plan, hipStream_t s);
void launch_linear8_tiles4(const Linear8Args& a, const Tokens8Plan& plan, hipStream_t s);
void launch_linear8_tiles2(const Linear8Args& a, const Tokens8Plan& plan, hipStream_t s);

namespace {

typedef int i4v __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float token_scale(float most) { return most == 0.0f ? 1.0f : __fdiv_rn(most, 127.0f); }

// 16 consecutive values as they are
template <typename T>
struct Raw16 {
  typedef T vec __attribute__((ext_vector_type(16 / sizeof(T))));
  vec v[sizeof(T)];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T); ++i) v[i] = *(const vec*)(p + i * (16 / (int)sizeof(T)));
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T); ++i) v[i] = vec(0);
  }
  __device__ __forceinline__ void values(float (&x)[16]) const {
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = (float)v[e * sizeof(T) / 16][e % (16 / sizeof(T))];
  }
};
// ... in fp32
template <typename T>
__device__ __forceinline__ void load16(const T* p, float (&x)[16]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f4 v = *(const f4*)(p + 4 * i);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[4 * i + e] = v[e];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const h8 v = *(const h8*)(p + 8 * i);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[8 * i + e] = (float)v[e];
    }
  }
}
__device__ __forceinline__ float most_of(const float (&x)[16]) {
  float m = 0.0f;
#pragma unroll
  for (int e = 0; e < 16; ++e) m = fmaxf(m, fabsf(x[e]));
  return m;
}

// ---- codes and scales of many tokens: a workgroup each, a thread 16 values at a time, held between the range and the codes up to K = 8192.
// Behind the row zeros up to the pitch.  (K % 16 == 0.)
template <typename T, int HELD>
__global__ void __launch_bounds__(256) quantize_tokens_kernel(const T* __restrict__ X, int8_t* __restrict__ Q, float* __restrict__ scales, int K, int pitch) {
  __shared__ float part[4];
  const int row = blockIdx.x, tid = threadIdx.x;
  const T* x = X + (int64_t)row * K;
  float v[HELD][16];
  float most = 0.0f;
#pragma unroll
  for (int i = 0; i < HELD; ++i) {
    const int at = (i * 256 + tid) * 16;
    if (at < K) {
      load16(x + at, v[i]);
      most = fmaxf(most, most_of(v[i]));
    }
  }
  for (int at = (HELD * 256 + tid) * 16; at < K; at += 256 * 16) {
    float w[16];
    load16(x + at, w);
    most = fmaxf(most, most_of(w));
  }
  most = wave_max_magnitude(most);
  if ((tid & 63) == 0) part[tid >> 6] = most;
  __syncthreads();
  most = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
  const float s = token_scale(most), r = scale_reciprocal(s);
  if (tid == 0) scales[row] = s;
  int8_t* q = Q + (int64_t)row * pitch;
  auto put = [&](int at, const float (&w)[16]) {
    unsigned c[4];
    quantize_words<16>(w, s, r, c, 127.0f);
    *(u4*)(q + at) = u4{c[0], c[1], c[2], c[3]};
  };
#pragma unroll
  for (int i = 0; i < HELD; ++i) {
    const int at = (i * 256 + tid) * 16;
    if (at < K) put(at, v[i]);
  }
  for (int at = (HELD * 256 + tid) * 16; at < K; at += 256 * 16) {
    float w[16];
    load16(x + at, w);
    put(at, w);
  }
  if (K + 16 * tid < pitch) *(u4*)(q + K + 16 * tid) = u4(0);
}

// ---- few tokens ---------------------------------------------------------------------------------------------------------------------------
// Channels n .. n + 3 of token m, if they are there (N % 4 == 0: inside or outside together)
template <bool F32>
__device__ __forceinline__ void store_channels(const Linear8Args& a, i4v sum, float s, int n, int m) {
  if (n >= a.N || m >= a.M) return;
  const f4 w = *(const f4*)(a.w_scale + n), b = a.epilogue & GPUSQ_EPI_BIAS ? *(const f4*)(a.bias + n) : f4(0);
  f4 y;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = __builtin_fmaf((float)sum[e] * s, w[e], b[e]);
  if (a.epilogue & GPUSQ_EPI_GELU) y = gelu4<F32>(y);
  const int64_t at = (int64_t)m * a.N + n;
  if constexpr (F32)
    *(f4*)((float*)a.Y + at) = y;
  else
    *(h4*)((_Float16*)a.Y + at) = h4{(_Float16)y[0], (_Float16)y[1], (_Float16)y[2], (_Float16)y[3]};
}

// A workgroup takes NT tiles of 16 channels at a time; wavefront w has the steps (chunk NW + w) S .. + S - 1 of 64 k of all of them, so that its tokens
// (MT blocks of 16) stay in registers.  A longer K is taken in chunks of S NW steps, the tiles' sums waiting in LDS.
// T: what the tokens are, fp16 or fp32, quantised here (MT == 1), or the codes that are there (int8_t).
template <typename T, int MT, int NW, int S, int NT, bool CHUNKS, bool F32>
__global__ void __launch_bounds__(64 * NW, NW / 4) linear8_rows_kernel(const Linear8Args a) {
  constexpr bool HERE = sizeof(T) != 1;
  static_assert(!HERE || MT == 1, "a block of tokens");
  extern __shared__ __attribute__((aligned(16))) i4v lds[];  // [2][NW][NT][MT][64], and with chunks [tiles of the workgroup][MT][64]
  __shared__ float scales[16], ranges[HERE ? NW : 1][16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, r = lane & 15;
  const int nt = (a.N + 15) >> 4, steps = (a.K + 63) >> 6, chunks = CHUNKS ? (steps + NW * S - 1) / (NW * S) : 1;
  const int groups = (nt + NT - 1) / NT, m0 = blockIdx.y * 16 * MT;
  i4v* totals = lds + 2 * NW * NT * MT * 64;
  i4v w[NT][S];
  // (a chunk behind the end of a row: the row's last, met by codes of 0; a row behind the last channel: that one, not stored)
  auto load = [&](int chunk, int group) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int n = (group * NT + t) * 16 + r;
      const int8_t* row = a.W + (int64_t)(n < a.N ? n : a.N - 1) * a.K;
#pragma unroll
      for (int i = 0; i < S; ++i) {
        const int k = ((chunk * NW + wave) * S + i) * 64 + 16 * g;
        w[t][i] = *(const i4v*)(row + (k < a.K ? k : a.K - 16));
      }
    }
  };
  // the tokens that are quantised here, in registers from the range to the codes where they fit (asked for in front of the weights, which take longer)
  constexpr bool HELD = HERE && !CHUNKS && S * sizeof(T) <= 12;
  Raw16<T> raw[HELD ? S : 1];
  const T* x = (const T*)a.X + (int64_t)(r < a.M ? r : a.M - 1) * a.K;  // (a column beyond the last token: zeros)
  if constexpr (HELD) {
#pragma unroll
    for (int i = 0; i < S; ++i) {
      const int k = (wave * S + i) * 64 + 16 * g;
      raw[i].zero();
      if (r < a.M && k < a.K) raw[i].load(x + k);
    }
  }
  load(0, blockIdx.x);
  float s_row = 1.0f, rs_row = 1.0f;
  if constexpr (HERE) {  // the tokens' ranges: a lane has token r, 16 values in 64
    float most = 0.0f;
    if constexpr (HELD) {
#pragma unroll
      for (int i = 0; i < S; ++i) {
        float v[16];
        raw[i].values(v);
        most = fmaxf(most, most_of(v));
      }
    } else {
      for (int chunk = 0; chunk < chunks; ++chunk)
#pragma unroll 2
        for (int i = 0; i < S; ++i) {
          const int k = ((chunk * NW + wave) * S + i) * 64 + 16 * g;
          if (r < a.M && k < a.K) {
            float v[16];
            load16(x + k, v);
            most = fmaxf(most, most_of(v));
          }
        }
    }
    most = fmaxf(most, __shfl_xor(most, 16));
    most = fmaxf(most, __shfl_xor(most, 32));
    if (g == 0) ranges[wave][r] = most;
    __syncthreads();
    most = ranges[0][r];
#pragma unroll
    for (int w = 1; w < NW; ++w) most = fmaxf(most, ranges[w][r]);
    s_row = token_scale(most);
    rs_row = scale_reciprocal(s_row);
    if (threadIdx.x < 16) scales[r] = s_row;
    // (what the range was taken of is not kept in 32 bits for the codes: these begin with the values, or with memory, again)
    if constexpr (HELD) {
#pragma unroll
      for (int i = 0; i < S; ++i)
#pragma unroll
        for (int j = 0; j < (int)sizeof(T); ++j) asm volatile("" : "+v"(raw[i].v[j]));
    } else {
      asm volatile("" : "+v"(x));
    }
  }
  int buf = 0, turn = 0;
  for (int chunk = 0; chunk < chunks; ++chunk) {
    i4v b[MT][S];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int i = 0; i < S; ++i) {
        const int k = ((chunk * NW + wave) * S + i) * 64 + 16 * g;
        if constexpr (HERE) {
          float v[16];
          unsigned c[4];
          if constexpr (HELD) {
            raw[i].values(v);
          } else {
            Raw16<T> now;
            now.zero();
            if (r < a.M && k < a.K) now.load(x + k);
            now.values(v);
          }
          quantize_words<16>(v, s_row, rs_row, c, 127.0f);
          b[m][i] = i4v{(int)c[0], (int)c[1], (int)c[2], (int)c[3]};
          if (HELD || (i & 1)) __builtin_amdgcn_sched_barrier(0);  // (one after the other, or two: all of them side by side do not fit the registers)
        } else {
          const int row = m0 + 16 * m + r < a.M ? m0 + 16 * m + r : a.M - 1;  // (columns beyond the last token repeat it and are not stored)
          b[m][i] = k < (int)a.pitch ? *(const i4v*)(a.Xq + (int64_t)row * a.pitch + k) : i4v(0);
        }
      }
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): else the loop waits for the tokens again, and with them for the next tile's weights
    for (int group = blockIdx.x, n = 0; group < groups; group += gridDim.x, ++n) {
      i4v acc[NT][MT];
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          acc[t][m] = i4v(0);
#pragma unroll
          for (int i = 0; i < S; ++i) acc[t][m] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[t][i], b[m][i], acc[t][m], 0, 0, 0);
        }
      // the next weights, into the registers that have just been read
      __builtin_amdgcn_sched_barrier(0);
      const int ahead = group + gridDim.x;
      if constexpr (CHUNKS)
        load(ahead < groups || chunk + 1 == chunks ? chunk : chunk + 1, ahead < groups ? ahead : chunk + 1 == chunks ? group : blockIdx.x);
      else
        load(0, ahead < groups ? ahead : group);  // (behind the last one: that one again)
      __builtin_amdgcn_sched_barrier(0);
      i4v* part = lds + buf * NW * NT * MT * 64;
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int m = 0; m < MT; ++m) part[((wave * NT + t) * MT + m) * 64 + lane] = acc[t][m];
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");  // (the next weights stay in flight)
      // NT MT wavefronts add up, others from turn to turn
      constexpr int JOBS = NT * MT;
      static_assert(JOBS <= NW && NW % JOBS == 0, "a job a wavefront");
      const int job = wave >= turn ? wave - turn : wave - turn + NW;
      if (job < JOBS) {
        i4v y = part[job * 64 + lane];
#pragma unroll 3
        for (int v = 1; v < NW; ++v) y += part[(v * JOBS + job) * 64 + lane];  // (all at once they would take the registers of the weights)
        i4v* total = totals + (n * JOBS + job) * 64 + lane;
        if (CHUNKS && chunk > 0) y += *total;
        if (CHUNKS && chunk + 1 < chunks) {
          *total = y;
        } else {
          const int t = job / MT, m = m0 + 16 * (job % MT) + r;
          store_channels<F32>(a, y, HERE ? scales[r] : a.x_scale[m < a.M ? m : a.M - 1], (group * NT + t) * 16 + 4 * g, m);
        }
      }
      buf ^= 1;
      turn = turn + JOBS < NW ? turn + JOBS : 0;
    }
  }
}

template <typename T, int MT, int S, int NT, bool CHUNKS>
void launch_rows(const Linear8Args& a, hipStream_t s) {
  constexpr int NW = 16;
  // one workgroup a CU, with as many groups of tiles each (and no more sums than LDS holds)
  constexpr int JOBS = NT * MT;
  const int64_t groups = ceil_div(a.N, 16 * NT), each = ceil_div(groups, num_cus()), most = (156 - 2 * NW * JOBS) / JOBS, per = CHUNKS && each > most ? most : each;
  static_assert(!CHUNKS || (156 - 2 * NW * JOBS) / JOBS >= 1, "sums in LDS");
  const size_t lds = (size_t)(2 * NW + (CHUNKS ? per : 0)) * JOBS * 1024;
  const dim3 grid((unsigned)ceil_div(groups, per), (unsigned)ceil_div(a.M, 16 * MT));
  if (a.out_f32)
    linear8_rows_kernel<T, MT, NW, S, NT, CHUNKS, true><<<grid, 64 * NW, lds, s>>>(a);
  else
    linear8_rows_kernel<T, MT, NW, S, NT, CHUNKS, false><<<grid, 64 * NW, lds, s>>>(a);
}
// The fewest steps a wavefront that K needs, up to 64 steps.
template <typename T>
void launch_16(const Linear8Args& a, int steps, hipStream_t s) {
  steps <= 16 ? launch_rows<T, 1, 1, 4, false>(a, s) : steps <= 32 ? launch_rows<T, 1, 2, 2, false>(a, s) : launch_rows<T, 1, 4, 1, false>(a, s);
}
template <typename T>
void launch_quantiser(const Linear8Args& a, hipStream_t s) {
  const T* x = (const T*)a.X;
  if (a.K <= 4096)
    quantize_tokens_kernel<T, 1><<<(unsigned)a.M, 256, 0, s>>>(x, a.Xq, a.x_scale, a.K, (int)a.pitch);
  else
    quantize_tokens_kernel<T, 2><<<(unsigned)a.M, 256, 0, s>>>(x, a.Xq, a.x_scale, a.K, (int)a.pitch);
}

}  // namespace

gpusq_status launch_linear_int8_tokens(const Linear8Args& a, hipStream_t s) {
  const int steps = (int)ceil_div(a.K, 64);
  // Tokens quantised by the product's own workgroups: a launch less, but each of them reads them all (4096 -> 4096: 8 tokens 12.7 us so, 12.4 with the
  // quantiser's launch in front, 16 tokens 18.1 and 12.6), and up to K = 4096 they fit the registers beside the weights.
  if (a.M <= 16 && steps <= 64 && (int64_t)a.M * a.K <= 32768) {
    a.x_f32 ? launch_16<float>(a, steps, s) : launch_16<_Float16>(a, steps, s);
    return check_launch();
  }
  a.x_f32 ? launch_quantiser<float>(a, s) : launch_quantiser<_Float16>(a, s);
  gpusq_status st = check_launch();
  if (st != GPUSQ_OK) return st;
  // Whole rows of weights against tokens in registers, or tiles: with 32 tokens the rows are ahead up to 4096 -> 4096 (12.9 us, tiles 20.0) and level at
  // 5120 -> 13824 (25.5, 24.7).  With 64 of 4096 values they are ahead up to 8192 channels (4096 16.8 and 20.3, 8192 19.6 and 20.7, 8196 21.7 and 20.6, 12288 23.0 and
  // 20.5, 28672 32.9 and 28.0; with 33 tokens to 12288, 20.1 and 20.5), of 2048 and less, where the tiles have fewer steps to make up for idle CUs, up to 12288
  // (64 tokens of 2048: 8192 12.6 and 15.1, 12288 14.9 and 15.2, 14336 16.7 and 15.6; 33 of 1024: 12288 11.3 and 12.4, 14336 12.7 and 12.3).  A workgroup's registers
  // hold 64 tokens of 4096 values.
  if (a.M <= 16)
    steps <= 64 ? launch_16<int8_t>(a, steps, s) : steps <= 96 ? launch_rows<int8_t, 1, 6, 1, false>(a, s) : steps <= 128 ? launch_rows<int8_t, 1, 8, 1, false>(a, s) : launch_rows<int8_t, 1, 8, 1, true>(a, s);
  else if (a.M <= 32)
    steps <= 16   ? launch_rows<int8_t, 2, 1, 2, false>(a, s)
    : steps <= 32 ? launch_rows<int8_t, 2, 2, 1, false>(a, s)
    : steps <= 64 ? launch_rows<int8_t, 2, 4, 1, false>(a, s)
    : steps <= 96 ? launch_rows<int8_t, 2, 6, 1, false>(a, s)
                  : launch_rows<int8_t, 2, 4, 1, true>(a, s);
  else if (a.M <= 64 && steps <= 64 && a.N <= (steps <= 32 ? 12288 : 8192))
    steps <= 32 ? launch_rows<int8_t, 4, 2, 1, false>(a, s) : launch_rows<int8_t, 4, 4, 1, false>(a, s);
  else {
    const Tokens8Plan plan = tokens8_plan(a.M, a.N, a.K, num_cus());
    plan.tn == 8 ? launch_linear8_tiles8(a, plan, s) : plan.tn == 4 ? launch_linear8_tiles4(a, plan, s) : launch_linear8_tiles2(a, plan, s);
  }
  return check_launch();
}

}  // namespace gpusq
