// Linear layers in 8-bit integers with a scale for each token and each channel: Y = act(s_m w_n (q_m . c_n) + b_n), s_m = max|x_m| / 127,
// q_m = clamp(rint(x_m / s_m)).
#include "epilogue.h"
#include "gelu4.h"

namespace gpusq {

namespace {

typedef int i4v __attribute__((ext_vector_type(4)));

// ---- codes and scale of a token, the code rule of the other quantisers; behind the row zeros up to the pitch -------------------------------
template <typename T>
__global__ void __launch_bounds__(256) quantize_tokens_kernel(const T* __restrict__ X, int8_t* __restrict__ Q, float* __restrict__ scales, int K, int pitch) {
  __shared__ float part[4];
  const int row = blockIdx.x, tid = threadIdx.x;
  const T* x = X + (int64_t)row * K;
  float most = 0.0f;
  for (int i = tid; i < K; i += 256) most = fmaxf(most, fabsf((float)x[i]));
  most = wave_max_magnitude(most);
  if ((tid & 63) == 0) part[tid >> 6] = most;
  __syncthreads();
  most = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
  const float s = most == 0.0f ? 1.0f : __fdiv_rn(most, 127.0f), r = scale_reciprocal(s);
  if (tid == 0) scales[row] = s;
  for (int i = tid; i < pitch; i += 256) Q[(int64_t)row * pitch + i] = i < K ? (int8_t)quantize_code((float)x[i], s, r) : (int8_t)0;
}

// ---- the product: a wavefront has 64 channels of 16 rows ------------------------------------------------------------------------------------
template <bool F32>
__global__ void __launch_bounds__(256) linear8_kernel(const Linear8Args a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, r = lane & 15;
  const int n0 = blockIdx.x * 64, m = (blockIdx.y * 4 + wave) * 16 + r;
  if (m - r >= a.M) return;
  const int8_t* xp = a.Xq + (int64_t)(m < a.M ? m : a.M - 1) * a.pitch + 16 * g;
  const int8_t* wp[4];
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const int n = n0 + 16 * t + r;
    wp[t] = a.W + (int64_t)(n < a.N ? n : a.N - 1) * a.K;
  }
  i4v acc[4] = {};
  for (int k = 0; k < a.K; k += 64) {
    const i4v x = *(const i4v*)(xp + k);
    const int at = k + 16 * g < a.K ? k + 16 * g : 0;  // (behind the row: 0 times any code)
#pragma unroll
    for (int t = 0; t < 4; ++t) acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(*(const i4v*)(wp[t] + at), x, acc[t], 0, 0, 0);
  }
  if (m >= a.M) return;
  const float s = a.x_scale[m];
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const int n = n0 + 16 * t + 4 * g;
    if (n >= a.N) continue;
    const f4 w = *(const f4*)(a.w_scale + n), b = a.epilogue & GPUSQ_EPI_BIAS ? *(const f4*)(a.bias + n) : f4(0);
    f4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = __builtin_fmaf((float)acc[t][e] * s, w[e], b[e]);
    if (a.epilogue & GPUSQ_EPI_GELU) y = gelu4<F32>(y);
    const int64_t at = (int64_t)m * a.N + n;
    if constexpr (F32)
      *(f4*)((float*)a.Y + at) = y;
    else
      *(h4*)((_Float16*)a.Y + at) = h4{(_Float16)y[0], (_Float16)y[1], (_Float16)y[2], (_Float16)y[3]};
  }
}

}  // namespace

gpusq_status launch_linear_int8_tokens(const Linear8Args& a, hipStream_t s) {
  if (a.x_f32)
    quantize_tokens_kernel<float><<<(unsigned)a.M, 256, 0, s>>>((const float*)a.X, a.Xq, a.x_scale, a.K, (int)a.pitch);
  else
    quantize_tokens_kernel<_Float16><<<(unsigned)a.M, 256, 0, s>>>((const _Float16*)a.X, a.Xq, a.x_scale, a.K, (int)a.pitch);
  gpusq_status st = check_launch();
  if (st != GPUSQ_OK) return st;
  const dim3 grid((unsigned)ceil_div(a.N, 64), (unsigned)ceil_div(a.M, 64));
  if (a.out_f32)
    linear8_kernel<true><<<grid, 256, 0, s>>>(a);
  else
    linear8_kernel<false><<<grid, 256, 0, s>>>(a);
  return check_launch();
}

}  // namespace gpusq
