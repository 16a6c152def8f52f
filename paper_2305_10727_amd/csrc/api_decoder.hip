// C ABI of the decoder's operators: argument validation, status codes, dispatch to the kernels.  No computation happens here.
#include <math.h>

#include "attend_plan.h"
#include "kv4.h"

using namespace gpusq;

namespace {
constexpr int64_t kMaxElems = (int64_t)1 << 40;

constexpr int64_t kMostPages = INT32_MAX / kPageTokens - 1;  // of a sequence: tokens are counted in 31 bits, a page beyond the last too

bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
bool aligned4(const void* p) { return ((uintptr_t)p & 3u) == 0; }
bool is_size(int64_t n) { return n > 0 && n <= INT32_MAX; }

gpusq_status check_groups(int64_t N, int64_t K, int group) {
  if (!is_size(N) || !is_size(K) || N * K > kMaxElems) return GPUSQ_ERR_SHAPE;
  if (group != 32 && group != 64 && group != 128) return GPUSQ_ERR_UNSUPPORTED;
  return K % group == 0 ? GPUSQ_OK : GPUSQ_ERR_SHAPE;
}

gpusq_status check_heads(int64_t heads, int64_t kv_heads, int64_t D) {
  if (!is_size(heads) || !is_size(kv_heads) || !is_size(D) || heads % kv_heads != 0) return GPUSQ_ERR_SHAPE;
  if (heads > 65536) return GPUSQ_ERR_SHAPE;
  return D % 8 == 0 && D <= 256 ? GPUSQ_OK : GPUSQ_ERR_UNSUPPORTED;
}

// sizes of the attentions, heads checked: products of what passes stay in 64 bits
bool are_kv4_sizes(int64_t tokens, int64_t batch, int64_t max_q, int64_t max_pages, int64_t heads, int64_t D) {
  return is_size(tokens) && is_size(batch) && is_size(max_q) && is_size(max_pages) && max_pages <= kMostPages && tokens * heads <= INT32_MAX &&
         tokens * heads * D <= kMaxElems && max_q <= tokens;
}
bool are_cross_sizes(int64_t batch, int64_t q_len, int64_t kv_len, int64_t heads, int64_t D) {
  return is_size(batch) && is_size(q_len) && is_size(kv_len) && kv_len <= kMostStates && batch * q_len <= INT32_MAX / heads && batch * q_len * heads * D <= kMaxElems;
}

// whether the launches of an attention and of its parts' join count their threads
bool is_launchable(bool kv4, int64_t batch, int64_t q_len, int64_t tokens, int64_t heads, int64_t kv_heads, int64_t D, const AttendParts& p, bool reach) {
  const int64_t cols = q_len * (heads / kv_heads);
  return attend_launchable(batch * kv_heads * p.parts, cols, attend_shape(kv4, padded_head((int)D), cols, reach)) &&
         (p.parts == 1 || launchable(join_workgroups(tokens * heads, D, p.parts), 256));
}

// the scale of the scores: positive; 0 stands for 1 / sqrt(D)
bool score_scale(float given, int64_t D, float* scale) {
  *scale = given == 0.0f ? 1.0f / sqrtf((float)D) : given;
  return *scale > 0.0f && *scale <= 3.4e38f;
}

size_t parts_bytes(const AttendParts& p, int64_t tokens, int64_t heads, int64_t D) {
  return p.parts > 1 ? (size_t)p.parts * tokens * heads * (D + 2) * 4 : 0;
}
}  // namespace

extern "C" {

size_t gpusq_int4_groups_packed_bytes(int64_t N, int64_t K, int group) {
  if (check_groups(N, K, group) != GPUSQ_OK) return 0;
  return (size_t)ceil_div(N, 16) * ceil_div(K, 128) * (1024 + 128 / group * 32);
}

gpusq_status gpusq_quantize_groups_int4(const float* W, int group, int8_t* codes, void* scales, int64_t N, int64_t K, void* stream) {
  if (!W || !codes || !scales) return GPUSQ_ERR_NULL;
  gpusq_status st = check_groups(N, K, group);
  if (st != GPUSQ_OK) return st;
  if (!launchable(ceil_div(N * K, 8 * 256), 256)) return GPUSQ_ERR_SHAPE;
  if (!aligned16(W) || !aligned16(codes) || !aligned16(scales)) return GPUSQ_ERR_ALIGN;
  return launch_quantize_groups_int4(W, group, codes, scales, N, K, (hipStream_t)stream);
}

gpusq_status gpusq_pack_int4_groups(const int8_t* codes, const void* scales, int group, void* packed, int64_t N, int64_t K, void* stream) {
  if (!codes || !scales || !packed) return GPUSQ_ERR_NULL;
  gpusq_status st = check_groups(N, K, group);
  if (st != GPUSQ_OK) return st;
  if (!launchable(ceil_div(N, 16) * ceil_div(K, 128), 256)) return GPUSQ_ERR_SHAPE;
  if (!aligned16(codes) || !aligned16(scales) || !aligned16(packed)) return GPUSQ_ERR_ALIGN;
  return launch_pack_int4_groups(codes, scales, group, packed, N, K, (hipStream_t)stream);
}

gpusq_status gpusq_linear_int4(const void* X, const void* Wpacked, int group, const float* bias, void* Y, gpusq_dtype out_dt, int64_t M, int64_t N, int64_t K,
                               int epilogue, void* stream) {
  if (!X || !Wpacked || !Y || ((epilogue & GPUSQ_EPI_BIAS) && !bias)) return GPUSQ_ERR_NULL;
  gpusq_status st = check_groups(N, K, group);
  if (st != GPUSQ_OK) return st;
  if (!is_size(M) || K > kMostLinear4K || ceil_div(M, 16) > 65535 || M * N > kMaxElems || M * K > kMaxElems) return GPUSQ_ERR_SHAPE;
  if (N % 4 != 0 || (out_dt != GPUSQ_F16 && out_dt != GPUSQ_F32) || (epilogue & ~(GPUSQ_EPI_BIAS | GPUSQ_EPI_GELU))) return GPUSQ_ERR_UNSUPPORTED;
  if (!aligned16(X) || !aligned16(Wpacked) || !aligned16(Y) || (bias && !aligned16(bias))) return GPUSQ_ERR_ALIGN;
  return launch_linear_int4(X, Wpacked, group, bias, Y, out_dt == GPUSQ_F32, M, N, K, epilogue, (hipStream_t)stream);
}

size_t gpusq_kv4_page_bytes(int64_t kv_heads, int64_t head_dim) {
  if (check_heads(kv_heads, kv_heads, head_dim) != GPUSQ_OK) return 0;
  return (size_t)kv_heads * page_bytes(padded_head((int)head_dim));
}

gpusq_status gpusq_qk_norm_rope(const void* qkv, gpusq_dtype dt, int64_t row_stride, int64_t tokens, int64_t heads, int64_t kv_heads, int64_t head_dim, int norm,
                                const float* q_weight, const float* k_weight, float eps, const float* cos, const float* sin, const int32_t* positions,
                                int64_t table_rows, int64_t rot_dim, int interleaved, void* q_out, void* k_out, void* v_out, void* cache,
                                const int32_t* slots, int64_t num_pages, void* stream) {
  if (!qkv || !q_out || (!cache && !k_out) || (cache && !slots)) return GPUSQ_ERR_NULL;
  if (rot_dim != 0 && (!cos || !sin || !positions)) return GPUSQ_ERR_NULL;
  gpusq_status st = check_heads(heads, kv_heads, head_dim);
  if (st != GPUSQ_OK) return st;
  const int64_t width = (heads + 2 * kv_heads) * head_dim;
  if (!is_size(tokens) || row_stride < width || row_stride > INT32_MAX || tokens * row_stride > kMaxElems) return GPUSQ_ERR_SHAPE;
  if (rot_dim < 0 || rot_dim > head_dim || (rot_dim != 0 && !is_size(table_rows)) || (cache && !is_size(num_pages))) return GPUSQ_ERR_SHAPE;
  if (cache && num_pages > INT32_MAX / kPageTokens) return GPUSQ_ERR_SHAPE;  // slots are 32-bit numbers
  if ((dt != GPUSQ_F32 && dt != GPUSQ_F16) || rot_dim % 8 != 0 || row_stride % 8 != 0 || (!cache && v_out)) return GPUSQ_ERR_UNSUPPORTED;
  if (norm && !(eps >= 0.0f)) return GPUSQ_ERR_UNSUPPORTED;
  if (!aligned16(qkv) || !aligned16(q_out) || !aligned16(k_out) || !aligned16(v_out) || !aligned16(cache) || !aligned16(q_weight) || !aligned16(k_weight) ||
      !aligned16(cos) || !aligned16(sin) || !aligned4(positions) || !aligned4(slots))
    return GPUSQ_ERR_ALIGN;
  return launch_qk_norm_rope(qkv, dt, row_stride, tokens, heads, kv_heads, head_dim, norm != 0, q_weight, k_weight, eps, cos, sin, positions, table_rows, rot_dim,
                             interleaved != 0, q_out, k_out, v_out, cache, slots, num_pages, (hipStream_t)stream);
}

size_t gpusq_attention_kv4_workspace_bytes(int64_t tokens, int64_t batch, int64_t max_q, int64_t max_pages, int64_t heads, int64_t kv_heads, int64_t head_dim) {
  if (check_heads(heads, kv_heads, head_dim) != GPUSQ_OK || !are_kv4_sizes(tokens, batch, max_q, max_pages, heads, head_dim)) return 0;
  return parts_bytes(attend_parts(true, batch, max_q, heads, kv_heads, head_dim, max_pages * kPageTokens), tokens, heads, head_dim);
}

gpusq_status gpusq_attention_kv4(const void* q, const void* cache, const int32_t* block_table, const int32_t* kv_lens, const int32_t* cu_q, void* out,
                                 void* workspace, int64_t tokens, int64_t batch, int64_t max_q, int64_t max_pages, int64_t num_pages, int64_t heads,
                                 int64_t kv_heads, int64_t head_dim, float scale, void* stream) {
  if (!q || !cache || !block_table || !kv_lens || !out) return GPUSQ_ERR_NULL;
  gpusq_status st = check_heads(heads, kv_heads, head_dim);
  if (st != GPUSQ_OK) return st;
  if (!are_kv4_sizes(tokens, batch, max_q, max_pages, heads, head_dim) || !is_size(num_pages) || (!cu_q && tokens != batch * max_q)) return GPUSQ_ERR_SHAPE;
  AttentionKv4 x{q, cache, block_table, kv_lens, cu_q, out, workspace, tokens, batch, max_q, max_pages, num_pages, heads, kv_heads, head_dim, 0.0f};
  if (!score_scale(scale, head_dim, &x.scale)) return GPUSQ_ERR_UNSUPPORTED;
  const AttendParts p = attend_parts(true, batch, max_q, heads, kv_heads, head_dim, max_pages * kPageTokens);
  if (!is_launchable(true, batch, max_q, tokens, heads, kv_heads, head_dim, p, true)) return GPUSQ_ERR_SHAPE;
  if (p.parts > 1 && !workspace) return GPUSQ_ERR_NULL;
  if (!aligned16(q) || !aligned16(cache) || !aligned16(out) || !aligned16(workspace) || !aligned4(block_table) || !aligned4(kv_lens) || !aligned4(cu_q))
    return GPUSQ_ERR_ALIGN;
  return launch_attention_kv4(x, (hipStream_t)stream);
}

size_t gpusq_cross_attention_workspace_bytes(int64_t batch, int64_t q_len, int64_t kv_len, int64_t heads, int64_t kv_heads, int64_t head_dim) {
  if (check_heads(heads, kv_heads, head_dim) != GPUSQ_OK || !are_cross_sizes(batch, q_len, kv_len, heads, head_dim)) return 0;
  return parts_bytes(attend_parts(false, batch, q_len, heads, kv_heads, head_dim, kv_len), batch * q_len, heads, head_dim);
}

gpusq_status gpusq_cross_attention(const void* q, const void* k, const void* v, const int32_t* kv_lens, const uint8_t* key_mask, void* out, void* workspace,
                                   int64_t batch, int64_t q_len, int64_t kv_len, int64_t heads, int64_t kv_heads, int64_t head_dim, int64_t q_batch_stride,
                                   int64_t q_stride, int64_t q_head_stride, int64_t k_batch_stride, int64_t k_stride, int64_t k_head_stride,
                                   int64_t v_batch_stride, int64_t v_stride, int64_t v_head_stride, float scale, void* stream) {
  if (!q || !k || !v || !out) return GPUSQ_ERR_NULL;
  gpusq_status st = check_heads(heads, kv_heads, head_dim);
  if (st != GPUSQ_OK) return st;
  if (!are_cross_sizes(batch, q_len, kv_len, heads, head_dim)) return GPUSQ_ERR_SHAPE;
  CrossAttention x{q, k, v, kv_lens, key_mask, out, workspace, batch, q_len, kv_len, heads, kv_heads, head_dim, {q_batch_stride, q_stride, q_head_stride},
                   {k_batch_stride, k_stride, k_head_stride}, {v_batch_stride, v_stride, v_head_stride}, 0.0f};
  for (const int64_t* strides : {x.q_stride, x.k_stride, x.v_stride})
    for (int i = 0; i < 3; ++i) {
      if (strides[i] < 0 || strides[i] > kMaxElems) return GPUSQ_ERR_SHAPE;
      if (strides[i] % 8 != 0) return GPUSQ_ERR_ALIGN;
    }
  if (!score_scale(scale, head_dim, &x.scale)) return GPUSQ_ERR_UNSUPPORTED;
  const AttendParts p = attend_parts(false, batch, q_len, heads, kv_heads, head_dim, kv_len);
  if (!is_launchable(false, batch, q_len, batch * q_len, heads, kv_heads, head_dim, p, tiles_reach(k_stride, v_stride))) return GPUSQ_ERR_SHAPE;
  if (p.parts > 1 && !workspace) return GPUSQ_ERR_NULL;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || !aligned16(workspace) || !aligned4(kv_lens)) return GPUSQ_ERR_ALIGN;
  return launch_cross_attention(x, (hipStream_t)stream);
}

}  // extern "C"
