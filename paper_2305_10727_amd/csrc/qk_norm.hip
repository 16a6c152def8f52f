// Norms of queries and keys for each head and the rotation by position, from a packed projection [token][q heads | k heads | v heads], in
// one pass; with a cache the keys and values are quantised to 4 bits and written to their places in the same pass.
//
//   h = x r w,  r = 1 / sqrt(mean(x^2) + eps) over the D channels of a head;  channels a, b of a pair turn to (a c - b s, a s + b c)
//
// Every value is read once and written once, so the pass is bound by memory.  A head's vector is a group of lanes, each with two quads
// of channels: the quads that turn with each other (4 i .. and R / 2 + 4 i .., or 8 i .. + 7 where pairs are neighbours), so that the
// rotation stays inside the lane and both ways of pairing read the same four cosines and sines.  Statistics are in 32 bits, and so is
// everything up to the one rounding of a result (fp16, or the codes of the cache).
// Queries and keys of 128 images of 257 tokens, 16 heads of 80: 337 MB in 78 us, 4.3 TB/s where a large copy has 5.0.  509 tokens of 32 + 8 + 8
// heads of 128 into the cache: 6.3 us, 3.5 for one token: a launch and three trips to memory (slots and positions, rows, stores).
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
  int heads, kv_heads, D, R, table_rows, num_pages, norm;
  int vectors, per_token;   // of this launch: below 2^31
  unsigned magic, shift;    // vector / per_token = (vector * magic >> 32) >> shift
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

// T: type of the projection.  INTER: pairs are neighbours (or nothing turns).  CACHE: keys and values go into the cache.  L: lanes of a vector,
// 8, 16 or 32, with CACHE those of the head as it is padded; 0: as many as it needs, a.D / 8, side by side in a wavefront.
template <typename T, int L_, bool INTER, bool CACHE>
__global__ void __launch_bounds__(256) qk_norm_rope_kernel(const QkArgs a) {
  const int L = L_ != 0 ? L_ : a.D / 8, lane = threadIdx.x & 63;
  const int in_wave = L_ != 0 ? lane / L_ : (int)((unsigned)lane * (unsigned)(65536 / L + 1) >> 16), at = lane - in_wave * L;  // (exact: lane < 64, L <= 32)
  const int of_wave = 64 / L, sub = (threadIdx.x >> 6) * of_wave + in_wave;
  __shared__ unsigned most[CACHE ? 256 / (CACHE ? L_ : 1) : 1][8];  // of the groups of 32 channels, as the bits of non-negative floats
  const int vec = blockIdx.x * (4 * of_wave) + sub;
  const bool in_vec = in_wave < of_wave && vec < a.vectors;
  const int token = in_vec ? (int)(__umulhi((unsigned)vec, a.magic) >> a.shift) : 0, h = in_vec ? vec - token * a.per_token : 0;
  const int64_t t = token;
  const bool in = in_vec && 8 * at < a.D;
  const bool is_q = h < a.heads, is_v = CACHE && h >= a.heads + a.kv_heads;
  // the two quads
  const bool turns = !is_v && 8 * at < a.R;
  const int lo = turns && !INTER ? 4 * at : 8 * at, hi = turns && !INTER ? a.R / 2 + 4 * at : 8 * at + 4;
  f4 x = f4(0), y = f4(0), c = f4(0), s = f4(0), wx = f4(1), wy = f4(1);
  if (in) {
    const T* row = (const T*)a.qkv + t * a.row_stride + (int64_t)h * a.D;
    x = load_quad(row + lo);
    y = load_quad(row + (INTER ? lo + 4 : hi));
    if (turns) {
      int p = a.positions[t];
      p = p < 0 ? 0 : p < a.table_rows ? p : a.table_rows - 1;  // (a place beyond the table: its end)
      const int64_t from = (int64_t)p * (a.R / 2) + 4 * at;
      c = *(const f4*)(a.cos + from);
      s = *(const f4*)(a.sin + from);
    }
    const float* w = is_q ? a.q_weight : a.k_weight;
    if (w != nullptr && !is_v) {
      wx = *(const f4*)(w + lo);
      wy = *(const f4*)(w + hi);
    }
  }
  if (a.norm) {
    float sum = 0.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e) sum = __builtin_fmaf(x[e], x[e], __builtin_fmaf(y[e], y[e], sum));
    if constexpr (L_ != 0) {
#pragma unroll
      for (int d = 1; d < L_; d *= 2) sum += __shfl_xor(sum, d);
    } else {  // sums of the lanes from this one on; the first lane's is the vector's
      for (int d = 1; d < L; d *= 2) {
        const float other = __shfl(sum, lane + d);
        sum += at + d < L ? other : 0.0f;
      }
      sum = __shfl(sum, lane - at);
    }
    if (!is_v) {
      const float r = __builtin_amdgcn_rsqf(sum / (float)a.D + a.eps);
      x *= r;
      y *= r;
      x *= wx;
      y *= wy;
    }
  }
  if (in && turns) {
    if (INTER) {
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
      if constexpr (INTER) {
        *(h8*)(out + lo) = h8{(_Float16)x[0], (_Float16)x[1], (_Float16)x[2], (_Float16)x[3], (_Float16)y[0], (_Float16)y[1], (_Float16)y[2], (_Float16)y[3]};
      } else {
        store_quad(out + lo, x);
        store_quad(out + hi, y);
      }
    }
    if constexpr (!CACHE) return;
  }
  if constexpr (CACHE) {
    // (No wavefront leaves before the barriers.  Channels beyond the head are quads of zeros, which the lanes beyond it write: 8 L is what the
    // head is padded to.)
    for (int i = threadIdx.x; i < 256 / L_ * 8; i += 256) (&most[0][0])[i] = 0;
    __syncthreads();
    constexpr int DP = 8 * L_;
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

// vectors of a workgroup: in the cache heads have the lanes of what they are padded to
int64_t vectors_of_workgroup(int64_t D, bool cached) { return 4 * (64 / (cached ? padded_head((int)D) / 8 : D / 8)); }

template <typename T, int L>
void launch_lanes(const QkArgs& a, bool interleaved, hipStream_t s) {
  const unsigned blocks = (unsigned)ceil_div(a.vectors, vectors_of_workgroup(a.D, false));
  if (interleaved || a.R == 0)
    qk_norm_rope_kernel<T, L, true, false><<<blocks, 256, 0, s>>>(a);
  else
    qk_norm_rope_kernel<T, L, false, false><<<blocks, 256, 0, s>>>(a);
}
template <typename T, int L>
void launch_cached(const QkArgs& a, bool interleaved, hipStream_t s) {
  const unsigned blocks = (unsigned)ceil_div(a.vectors, vectors_of_workgroup(a.D, true));
  if (interleaved || a.R == 0)
    qk_norm_rope_kernel<T, L, true, true><<<blocks, 256, 0, s>>>(a);
  else
    qk_norm_rope_kernel<T, L, false, true><<<blocks, 256, 0, s>>>(a);
}
template <typename T>
void launch_typed(const QkArgs& a, bool interleaved, hipStream_t s) {
  if (a.cache != nullptr)
    a.D <= 64 ? launch_cached<T, 8>(a, interleaved, s) : a.D <= 128 ? launch_cached<T, 16>(a, interleaved, s) : launch_cached<T, 32>(a, interleaved, s);
  else if (a.D == 64)
    launch_lanes<T, 8>(a, interleaved, s);
  else if (a.D == 128)
    launch_lanes<T, 16>(a, interleaved, s);
  else
    launch_lanes<T, 0>(a, interleaved, s);
}

}  // namespace

gpusq_status launch_qk_norm_rope(const void* qkv, gpusq_dtype dt, int64_t row_stride, int64_t T, int64_t heads, int64_t kv_heads, int64_t D, int norm,
                                 const float* q_weight, const float* k_weight, float eps, const float* cos, const float* sin, const int32_t* positions,
                                 int64_t table_rows, int64_t R, int interleaved, void* q_out, void* k_out, void* v_out, void* cache, const int32_t* slots,
                                 int64_t num_pages, hipStream_t s) {
  const int64_t per_token = heads + kv_heads + (cache != nullptr ? kv_heads : 0), most = qk_norm_tokens(per_token, vectors_of_workgroup(D, cache != nullptr));
  unsigned bits = 1;  // per_token >= 2
  while ((int64_t)1 << bits < per_token) ++bits;
  const unsigned magic = (unsigned)(((uint64_t)1 << (31 + bits)) / per_token + 1);
  for (int64_t from = 0; from < T; from += most) {
    const int64_t n = T - from < most ? T - from : most;
    const QkArgs a{(const uint8_t*)qkv + from * row_stride * (dt == GPUSQ_F32 ? 4 : 2), row_stride, q_weight, k_weight, cos, sin, positions ? positions + from : nullptr,
                   slots ? slots + from : nullptr, (_Float16*)q_out + from * heads * D, k_out ? (_Float16*)k_out + from * kv_heads * D : nullptr,
                   v_out ? (_Float16*)v_out + from * kv_heads * D : nullptr, (uint8_t*)cache, (int)heads, (int)kv_heads, (int)D, (int)R, (int)table_rows,
                   (int)num_pages, norm, (int)(n * per_token), (int)per_token, magic, bits - 1, eps};
    dt == GPUSQ_F32 ? launch_typed<float>(a, interleaved != 0, s) : launch_typed<_Float16>(a, interleaved != 0, s);
    const gpusq_status st = check_launch();
    if (st != GPUSQ_OK) return st;
  }
  return GPUSQ_OK;
}

}  // namespace gpusq
