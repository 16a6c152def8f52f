// Norms of queries and keys for each head and the rotation by position, from a packed projection [token][q heads | k heads | v heads], in
// one pass; with a cache the keys and values are quantised to 4 bits and written to their places in the same pass.
//
//   h = x r w,  r = 1 / sqrt(mean(x^2) + eps) over the D channels of a head;  channels a, b of a pair turn to (a c - b s, a s + b c)
//
// Every value is read once and written once, so the pass is bound by memory.  A head's vector is a group of lanes, each with two quads
// of channels: the quads that turn with each other (4 i .. and R / 2 + 4 i .., or 8 i .. + 7 where pairs are neighbours), so that the
// rotation stays inside the lane and both ways of pairing read the same four cosines and sines.  Statistics are in 32 bits, and so is
// everything up to the one rounding of a result (fp16, or the codes of the cache).
#include "kv4.h"

namespace gpusq {

namespace {

struct QkArgs {
  const void* qkv;
  int64_t row_stride;
  const float *q_weight, *k_weight, *cos, *sin;
  const int32_t *positions, *slots;
  _Float16 *q_out, *k_out, *v_out;
  uint8_t* cache;
  int64_t vectors;
  int heads, kv_heads, D, R, table_rows, num_pages, norm, interleaved, per_token;
  float eps;
};

template <typename T>
__device__ __forceinline__ f4 load_quad(const T* p) {
  if constexpr (sizeof(T) == 4) {
    return *(const f4*)p;
  } else {
    const h4 v = *(const h4*)p;
    return f4{(float)v[0], (float)v[1], (float)v[2], (float)v[3]};
  }
}
__device__ __forceinline__ void store_quad(_Float16* p, f4 v) { *(h4*)p = h4{(_Float16)v[0], (_Float16)v[1], (_Float16)v[2], (_Float16)v[3]}; }

// T: type of the projection; L: lanes of a vector (a power of two, 8 L >= D); CACHE: keys and values go into the cache
template <typename T, int L, bool CACHE>
__global__ void __launch_bounds__(256) qk_norm_rope_kernel(const QkArgs a) {
  constexpr int VECS = 256 / L;
  __shared__ unsigned most[CACHE ? VECS : 1][8];  // of the groups of 32 channels, as the bits of non-negative floats
  const int sub = threadIdx.x / L, lane = threadIdx.x % L;
  const int64_t vec = (int64_t)blockIdx.x * VECS + sub;
  const bool in_vec = vec < a.vectors;
  const int64_t t = in_vec ? vec / a.per_token : 0;
  const int h = in_vec ? (int)(vec - t * a.per_token) : 0;
  const bool in = in_vec && 8 * lane < a.D;
  const bool is_q = h < a.heads, is_v = h >= a.heads + a.kv_heads;
  // the two quads
  const bool turns = !is_v && 8 * lane < a.R;
  const int lo = turns && !a.interleaved ? 4 * lane : 8 * lane, hi = turns && !a.interleaved ? a.R / 2 + 4 * lane : 8 * lane + 4;
  f4 x = f4(0), y = f4(0);
  if (in) {
    const T* row = (const T*)a.qkv + t * a.row_stride + (int64_t)h * a.D;
    x = load_quad(row + lo);
    y = load_quad(row + hi);
  }
  if (a.norm) {
    float sum = 0.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e) sum += x[e] * x[e] + y[e] * y[e];
#pragma unroll
    for (int d = 1; d < L; d *= 2) sum += __shfl_xor(sum, d);
    if (!is_v && in) {
      const float r = 1.0f / __fsqrt_rn(sum / (float)a.D + a.eps);
      x *= r;
      y *= r;
      const float* w = is_q ? a.q_weight : a.k_weight;
      if (w != nullptr) {
        x *= *(const f4*)(w + lo);
        y *= *(const f4*)(w + hi);
      }
    }
  }
  if (in && turns) {
    int p = a.positions[t];
    p = p < 0 ? 0 : p < a.table_rows ? p : a.table_rows - 1;  // (a place beyond the table: its end)
    const f4 c = *(const f4*)(a.cos + (int64_t)p * (a.R / 2) + 4 * lane), s = *(const f4*)(a.sin + (int64_t)p * (a.R / 2) + 4 * lane);
    if (a.interleaved) {
      const f4 u = {x[0], x[2], y[0], y[2]}, v = {x[1], x[3], y[1], y[3]};
      const f4 m = u * c - v * s, n = u * s + v * c;
      x = f4{m[0], n[0], m[1], n[1]};
      y = f4{m[2], n[2], m[3], n[3]};
    } else {
      const f4 u = x, v = y;
      x = u * c - v * s;
      y = u * s + v * c;
    }
  }
  if (is_q || !CACHE) {
    if (in) {
      _Float16* out = is_q ? a.q_out + (t * a.heads + h) * a.D : a.k_out + (t * a.kv_heads + (h - a.heads)) * a.D;
      store_quad(out + lo, x);
      store_quad(out + hi, y);
    }
    if constexpr (!CACHE) return;
  }
  if constexpr (CACHE) {
    // (No wavefront leaves before the barriers.  Channels beyond the head are quads of zeros, which the lanes beyond it write: 8 L is what
    // the head is padded to.)
    for (int i = threadIdx.x; i < VECS * 8; i += 256) (&most[0][0])[i] = 0;
    __syncthreads();
    constexpr int DP = 8 * L;
    const bool keeps = in_vec && !is_q;
    if (keeps && in) {
      float mx = 0.0f, my = 0.0f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        mx = fmaxf(mx, fabsf(x[e]));  // (a NaN is left out)
        my = fmaxf(my, fabsf(y[e]));
      }
      atomicMax(&most[sub][lo / 32], __float_as_uint(mx));
      atomicMax(&most[sub][hi / 32], __float_as_uint(my));
    }
    __syncthreads();
    if (!keeps) return;
    const int64_t slot = a.slots[t];
    const bool kept = slot >= 0 && slot < (int64_t)a.num_pages * kPageTokens;
    const int kh = is_v ? h - a.heads - a.kv_heads : h - a.heads;
    uint8_t* page = a.cache + ((slot >> 6) * a.kv_heads + kh) * page_bytes(DP);
    constexpr int J = DP / 32;
    const int tok = (int)(slot & 63);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int d = half ? hi : lo;
      const f4 v = half ? y : x;
      const float s = group_scale(__uint_as_float(most[sub][d / 32]));
      const float xs[4] = {v[0], v[1], v[2], v[3]};
      int q[4];
      quantize_codes<4>(xs, s, scale_reciprocal(s), q, 7.0f);
      if (kept) {
        const unsigned n0 = (unsigned)(q[0] + 8), n1 = (unsigned)(q[1] + 8), n2 = (unsigned)(q[2] + 8), n3 = (unsigned)(q[3] + 8);
        if (is_v) {
          const int n = d / (DP / 16), quarter = d % (DP / 16) / 4;
          const int unit = (((tok >> 2) * 16 + n) * 2 + ((tok >> 1) & 1)) * (DP / 64) * 2 + quarter * 2 + (tok & 1);
          ((uint16_t*)(page + value_codes_at(DP)))[unit] = (uint16_t)(n0 | n1 << 4 | n2 << 8 | n3 << 12);
          if (d % 32 == 0) ((_Float16*)(page + value_scales_at(DP)))[d / 32 * kPageTokens + tok] = (_Float16)s;
        } else {
          uint8_t* word = page + tok * (DP / 2) + (d % 32 / 8 * J + d / 32) * 4 + d % 8 / 4;
          word[0] = (uint8_t)(n0 | n2 << 4);
          word[2] = (uint8_t)(n1 | n3 << 4);
          if (d % 32 == 0) ((_Float16*)(page + key_scales_at(DP)))[tok * J + d / 32] = (_Float16)s;
        }
      }
      _Float16* out = is_v ? a.v_out : a.k_out;
      if (out != nullptr && in) store_quad(out + (t * a.kv_heads + kh) * a.D + d, f4{(float)q[0] * s, (float)q[1] * s, (float)q[2] * s, (float)q[3] * s});
    }
  }
}

template <typename T, int L>
gpusq_status launch_lanes(const QkArgs& a, hipStream_t s) {
  const int64_t blocks = ceil_div(a.vectors, 256 / L);
  if (blocks > INT32_MAX) return GPUSQ_ERR_SHAPE;
  if (a.cache != nullptr)
    qk_norm_rope_kernel<T, L, true><<<(unsigned)blocks, 256, 0, s>>>(a);
  else
    qk_norm_rope_kernel<T, L, false><<<(unsigned)blocks, 256, 0, s>>>(a);
  return check_launch();
}

template <typename T>
gpusq_status launch_typed(const QkArgs& a, hipStream_t s) {
  if (a.D <= 64) return launch_lanes<T, 8>(a, s);
  return a.D <= 128 ? launch_lanes<T, 16>(a, s) : launch_lanes<T, 32>(a, s);
}

}  // namespace

gpusq_status launch_qk_norm_rope(const void* qkv, gpusq_dtype dt, int64_t row_stride, int64_t T, int64_t heads, int64_t kv_heads, int64_t D, int norm,
                                 const float* q_weight, const float* k_weight, float eps, const float* cos, const float* sin, const int32_t* positions,
                                 int64_t table_rows, int64_t R, int interleaved, void* q_out, void* k_out, void* v_out, void* cache, const int32_t* slots,
                                 int64_t num_pages, hipStream_t s) {
  const int per_token = (int)(heads + kv_heads + (cache != nullptr ? kv_heads : 0));
  const QkArgs a{qkv, row_stride, q_weight, k_weight, cos, sin, positions, slots, (_Float16*)q_out, (_Float16*)k_out, (_Float16*)v_out, (uint8_t*)cache,
                 T * per_token, (int)heads, (int)kv_heads, (int)D, (int)R, (int)table_rows, (int)num_pages, norm, interleaved, per_token, eps};
  return dt == GPUSQ_F32 ? launch_typed<float>(a, s) : launch_typed<_Float16>(a, s);
}

}  // namespace gpusq
