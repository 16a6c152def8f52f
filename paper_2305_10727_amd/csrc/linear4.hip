// Linear layers on 4-bit weights with group scales, for a few activation rows: Y = act(X W^T + b), W[n][k] = code[n][k] scale[n][k / G].
//
// Such a layer is bound by the bytes of its weights, half a byte and 2 / G of one for each; every other choice follows from reading them
// once, in whole lines, with much in flight:
//   - the packed operand is in the order of the registers that multiply it: 16 channels x 128 k are 1 KB, one 16-byte vector a lane,
//     four words of 8 codes for the four 16 x 16 x 32 products of a step;
//   - the weights are the first operand, whose rows are channels, and X the second, whose 16 columns are activation rows: one to 16
//     rows cost the same;
//   - codes are turned into fp16 integers, exact, and the products of a group summed in 32 bits before its scale, in 32 bits too,
//     multiplies the sum: nothing is rounded before the output, whatever the scales;
//   - a workgroup's wavefronts share its channels and deal out the steps of K; their sums meet in LDS once, at the end.
// Replayed from a graph: 5120 -> 13824 with GELU for one row (36.6 MB) 11 us, 3.4 TB/s; 8192 -> 24576 for 13 rows (109 MB) 27 us, 4.0 TB/s, for 50
// rows 60 us; 13824 -> 5120 for one row 13 us; a large copy has 5.0.  1024 -> 1024 for one row: 3.0 us, a launch and three trips to memory.
#include "epilogue.h"
#include "gelu4.h"

namespace gpusq {

namespace {

// ---- codes and scales of fp32 weights: the largest magnitude of each group / 7, as fp16; codes against the scale as it is kept ------------
// One lane has 8 values: a group of 32, 64 or 128 is 4, 8 or 16 lanes.
template <int GROUP>
__global__ void __launch_bounds__(256) quantize_groups_kernel(const float* __restrict__ W, int8_t* __restrict__ codes, _Float16* __restrict__ scales, int64_t vecs) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const bool in = i < vecs;  // (vecs % (GROUP / 8) == 0: a group is inside or outside as a whole)
  float x[8];
  float amax = 0.0f;
  if (in) {
    const f4 a = ((const f4*)W)[2 * i], b = ((const f4*)W)[2 * i + 1];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[j] = a[j];
      x[4 + j] = b[j];
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = 0.0f;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) amax = fmaxf(amax, fabsf(x[j]));  // (a NaN is left out)
#pragma unroll
  for (int d = 1; d < GROUP / 8; d *= 2) amax = fmaxf(amax, __shfl_xor(amax, d));
  _Float16 s16 = (_Float16)fminf(__fdiv_rn(amax, 7.0f), 65504.0f);
  if (s16 == (_Float16)0.0f) s16 = (_Float16)1.0f;
  const float s = (float)s16;
  int q[8];
  quantize_codes<8>(x, s, scale_reciprocal(s), q, 7.0f);
  if (!in) return;
  u2 out;
#pragma unroll
  for (int h = 0; h < 2; ++h)
    out[h] = low_bytes((unsigned)q[4 * h], (unsigned)q[4 * h + 1], (unsigned)q[4 * h + 2], (unsigned)q[4 * h + 3]);
  ((u2*)codes)[i] = out;
  if (i % (GROUP / 8) == 0) scales[i / (GROUP / 8)] = s16;
}

// ---- packing: a thread writes one word (8 codes), or one scale ------------------------------------------------------------------------
__global__ void __launch_bounds__(256) pack_int4_groups_kernel(const int8_t* __restrict__ codes, const _Float16* __restrict__ scales, uint8_t* __restrict__ packed,
                                                                int N, int K, int group, int kt, int64_t words, int64_t scale_places) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < words) {
    const int j = (int)(i & 3), lane = (int)(i >> 2) & 63;
    const int64_t tile = i >> 8;
    const int64_t n = tile / kt * 16 + (lane & 15);
    const int k = (int)(tile % kt) * 128 + 32 * j + 8 * (lane >> 4);
    unsigned w = 0x88888888u;  // zeros beyond the matrix
    if (n < N && k < K) {
      const u2 c = *(const u2*)(codes + n * K + k);
      w = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const unsigned code = (c[e >> 2] >> (8 * (e & 3))) & 0xFFu;
        w |= ((code + 8u) & 15u) << ((e & 1) * 16 + (e >> 1) * 4);
      }
    }
    ((unsigned*)packed)[i] = w;
  }
  if (i < scale_places) {
    const int per = kt * (128 / group);
    const int64_t n = i / 16 / per * 16 + (i & 15);
    const int g = (int)(i / 16 % per);
    _Float16 s = (_Float16)0.0f;
    if (n < N && g < K / group) s = scales[n * (K / group) + g];
    ((_Float16*)(packed + words * 4))[i] = s;
  }
}

// ---- the product ----------------------------------------------------------------------------------------------------------------------
struct Linear4Args {
  const _Float16* X;
  const uint8_t* W;
  const float* bias;
  void* Y;
  int M, N, K, kt, epilogue;
};

// Channels n .. n + 3 of row m, if they are there (N % 4 == 0: they are inside or outside together)
template <bool F32>
__device__ __forceinline__ void store_channels(const Linear4Args& a, f4 y, int n, int m) {
  if (n >= a.N || m >= a.M) return;
  if (a.epilogue & GPUSQ_EPI_BIAS) y += *(const f4*)(a.bias + n);
  if (a.epilogue & GPUSQ_EPI_GELU) y = gelu4<F32>(y);
  const int64_t at = (int64_t)m * a.N + n;
  if constexpr (F32)
    *(f4*)((float*)a.Y + at) = y;
  else
    *(h4*)((_Float16*)a.Y + at) = h4{(_Float16)y[0], (_Float16)y[1], (_Float16)y[2], (_Float16)y[3]};
}

// the last word of a buffer's descriptor: bytes as they are (data format 32, no swizzle); loads behind its end give 0
constexpr int kRawBuffer = 4 << 15;

// A few rows: a workgroup takes one tile of 16 channels after another, each wavefront the same S steps of all of them, so that its rows (MT
// columns of 16) stay in registers.  (A load of 16 bytes a lane takes the first-level cache 16 clocks, whether its lanes ask for the same
// bytes or not: a step's rows cost four times what its weights do.)  A longer K is taken in chunks of S NW steps, the tiles' sums waiting in LDS.
template <int MT, int NW, int S, bool CHUNKS, int GROUP, bool F32>
__global__ void __launch_bounds__(64 * NW, NW / 4) linear_int4_rows_kernel(const Linear4Args a) {
  static_assert(NW * S <= kLinear4Steps, "k behind the end of K");
  constexpr int PER = 128 / GROUP, CH = GROUP / 32;
  extern __shared__ __attribute__((aligned(16))) f4 lds[];  // [2][NW][MT][64], and with chunks [tiles of the workgroup][MT][64]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, r = lane & 15;
  const int nt = (a.N + 15) >> 4, chunks = CHUNKS ? (a.kt + NW * S - 1) / (NW * S) : 1;
  const int m0 = blockIdx.y * 16 * MT;
  f4* totals = lds + 2 * NW * MT * 64;
  struct Weights {
    u4 w[S];
    h4 s[S][PER];
  };
  auto load = [&](int chunk, int tile, Weights& x) {
    const u4* codes = (const u4*)(a.W + (int64_t)tile * a.kt * 1024) + lane;
    // (a step beyond the last: the last one's codes again, with rows of zeros; and with scales of zeros, which is what is loaded behind the end of a
    // buffer: 0 times a scale that is infinite would not be 0)
    const auto scales = __builtin_amdgcn_make_buffer_rsrc((void*)(a.W + (int64_t)nt * a.kt * 1024 + (int64_t)tile * a.kt * PER * 32), 0, (unsigned)a.kt * (PER * 32), kRawBuffer);
    const unsigned scales_at = (unsigned)((chunk * NW + wave) * S) * (PER * 32) + 8 * g;
#pragma unroll
    for (int i = 0; i < S; ++i) {
      const int at = (chunk * NW + wave) * S + i, step = at < a.kt ? at : a.kt - 1;
#pragma unroll
      for (int p = 0; p < PER; ++p) x.s[i][p] = __builtin_bit_cast(h4, __builtin_amdgcn_raw_buffer_load_b64(scales, scales_at + (i * PER + p) * 32, 0, 0));
      x.w[i] = codes[(int64_t)step * 64];
    }
  };
  const _Float16* rows[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int row = m0 + 16 * m + r < a.M ? m0 + 16 * m + r : a.M - 1;  // (columns beyond the last row repeat it and are not stored)
    rows[m] = a.X + (int64_t)row * a.K + 8 * g;
  }
  Weights next;
  load(0, blockIdx.x, next);
  int buf = 0, turn = 0;
  for (int chunk = 0; chunk < chunks; ++chunk) {
    h8 b[MT][S][4];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int i = 0; i < S; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int k = 128 * ((chunk * NW + wave) * S + i) + 32 * j;
          b[m][i][j] = k < a.K ? *(const h8*)(rows[m] + k) : h8(0);
        }
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): else the loop waits for the rows again, and with them for the next tile's weights
    for (int tile = blockIdx.x, n = 0; tile < nt; tile += gridDim.x, ++n) {
      const Weights now = next;
      const int ahead = tile + gridDim.x;
      if constexpr (CHUNKS)
        load(ahead < nt || chunk + 1 == chunks ? chunk : chunk + 1, ahead < nt ? ahead : chunk + 1 == chunks ? tile : blockIdx.x, next);
      else
        load(0, ahead < nt ? ahead : tile, next);  // (behind the last one: that one again)
      f4 acc[MT] = {};
#pragma unroll
      for (int i = 0; i < S; ++i)
#pragma unroll
        for (int p = 0; p < PER; ++p) {
          f4 sum[MT] = {};
#pragma unroll
          for (int c = 0; c < CH; ++c) {
            h2 v[4];
            codes_to_halves(now.w[i][p * CH + c], v);
            const h8 wa = {v[0][0], v[0][1], v[1][0], v[1][1], v[2][0], v[2][1], v[3][0], v[3][1]};
#pragma unroll
            for (int m = 0; m < MT; ++m) sum[m] = mfma16(wa, b[m][i][p * CH + c], sum[m]);
          }
#pragma unroll
          for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[m][e] = __builtin_fmaf(sum[m][e], (float)now.s[i][p][e], acc[m][e]);
        }
      f4* part = lds + buf * NW * MT * 64;
#pragma unroll
      for (int m = 0; m < MT; ++m) part[(wave * MT + m) * 64 + lane] = acc[m];
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");  // (the next weights stay in flight)
      // MT wavefronts add up, others from tile to tile
      const int m = wave >= turn ? wave - turn : wave - turn + NW;
      if (m < MT) {
        f4 y = part[m * 64 + lane];
#pragma unroll
        for (int w = 1; w < NW; ++w) y += part[(w * MT + m) * 64 + lane];
        f4* total = totals + (n * MT + m) * 64 + lane;
        if (CHUNKS && chunk > 0) y += *total;
        if (CHUNKS && chunk + 1 < chunks)
          *total = y;
        else
          store_channels<F32>(a, y, tile * 16 + 4 * g, m0 + 16 * m + r);
      }
      buf ^= 1;
      turn = turn + MT < NW ? turn + MT : 0;
    }
  }
}

template <int MT, int NW, int S, bool CHUNKS>
void launch_rows(const Linear4Args& a, int group, bool f32, hipStream_t s) {
  // one workgroup a CU, with as many tiles each (and no more sums than LDS holds)
  const int64_t nt = ceil_div(a.N, 16), each = ceil_div(nt, num_cus()), most = 160 / MT - 2 * NW, per = CHUNKS && each > most ? most : each;
  const size_t lds = (size_t)(2 * NW + (CHUNKS ? per : 0)) * MT * 1024;
  const dim3 grid((unsigned)ceil_div(nt, per), (unsigned)ceil_div(a.M, 16 * MT));
#define GPUSQ_LINEAR4(G, F) linear_int4_rows_kernel<MT, NW, S, CHUNKS, G, F><<<grid, 64 * NW, lds, s>>>(a)
  if (group == 32)
    f32 ? GPUSQ_LINEAR4(32, true) : GPUSQ_LINEAR4(32, false);
  else if (group == 64)
    f32 ? GPUSQ_LINEAR4(64, true) : GPUSQ_LINEAR4(64, false);
  else
    f32 ? GPUSQ_LINEAR4(128, true) : GPUSQ_LINEAR4(128, false);
#undef GPUSQ_LINEAR4
}

}  // namespace

gpusq_status launch_quantize_groups_int4(const float* W, int group, int8_t* codes, void* scales, int64_t N, int64_t K, hipStream_t s) {
  const int64_t vecs = N * (K / 8);
  const unsigned blocks = (unsigned)ceil_div(vecs, 256);
  if (group == 32)
    quantize_groups_kernel<32><<<blocks, 256, 0, s>>>(W, codes, (_Float16*)scales, vecs);
  else if (group == 64)
    quantize_groups_kernel<64><<<blocks, 256, 0, s>>>(W, codes, (_Float16*)scales, vecs);
  else
    quantize_groups_kernel<128><<<blocks, 256, 0, s>>>(W, codes, (_Float16*)scales, vecs);
  return check_launch();
}

gpusq_status launch_pack_int4_groups(const int8_t* codes, const void* scales, int group, void* packed, int64_t N, int64_t K, hipStream_t s) {
  const int64_t nt = ceil_div(N, 16), kt = ceil_div(K, 128), words = nt * kt * 256, places = nt * kt * (128 / group) * 16;
  pack_int4_groups_kernel<<<(unsigned)ceil_div(words, 256), 256, 0, s>>>(codes, (const _Float16*)scales, (uint8_t*)packed, (int)N, (int)K, group, (int)kt, words, places);
  return check_launch();
}

gpusq_status launch_linear_int4(const void* X, const void* W, int group, const float* bias, void* Y, bool f32, int64_t M, int64_t N, int64_t K, int epilogue,
                                hipStream_t s) {
  const Linear4Args a{(const _Float16*)X, (const uint8_t*)W, bias, Y, (int)M, (int)N, (int)K, (int)ceil_div(K, 128), epilogue};
  // The fewest steps a wavefront that K needs: registers for rows, and wavefronts for as much of the weights in flight as there are
  // (8 wavefronts rather than 16 up to K = 2048: 1024 -> 1024 for one row 2.7 us, 3.4 with 16; 8 with twice the steps are within 2 % of 16 up to
  // K = 5120: 4096 -> 16384 11.3 and 11.1, 5120 -> 13824 10.7 and 10.8).
  if (M <= 16)
    a.kt <= 8    ? launch_rows<1, 8, 1, false>(a, group, f32, s)
    : a.kt <= 16 ? launch_rows<1, 8, 2, false>(a, group, f32, s)
    : a.kt <= 32 ? launch_rows<1, 16, 2, false>(a, group, f32, s)
    : a.kt <= 48 ? launch_rows<1, 16, 3, false>(a, group, f32, s)
    : a.kt <= 64 ? launch_rows<1, 16, 4, false>(a, group, f32, s)
                 : launch_rows<1, 16, 4, true>(a, group, f32, s);
  else if (M <= 32)
    a.kt <= 16   ? launch_rows<2, 16, 1, false>(a, group, f32, s)
    : a.kt <= 32 ? launch_rows<2, 16, 2, false>(a, group, f32, s)
                 : launch_rows<2, 16, 2, true>(a, group, f32, s);
  else
    a.kt <= 16 ? launch_rows<4, 16, 1, false>(a, group, f32, s) : launch_rows<4, 16, 1, true>(a, group, f32, s);
  return check_launch();
}

}  // namespace gpusq
