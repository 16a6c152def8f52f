// C ABI of the decoder's operators: argument validation, status codes, dispatch to the kernels.  No computation happens here.
#include <math.h>

#include <algorithm>

#include "attend_plan.h"
#include "drafts_plan.h"
#include "linear8_plan.h"
#include "sample_plan.h"
#include "kv4.h"

using namespace gpusq;

namespace {
constexpr int64_t kMaxElems = (int64_t)1 << 40;

// sums of products of codes, -128 the least of a weight's, stay in 32 bits
constexpr int64_t kMostTokens8K = INT32_MAX / (127 * 128) / 64 * 64;
// a row's weights, whole numbers up to 2^44, are together below 2^63
constexpr int64_t kMostVocabulary = (int64_t)1 << 18;

constexpr int64_t kMostCaches = 1024;  // of a call that moves tokens in them
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
bool is_launchable(bool kv4, int64_t batch, int64_t q_len, int64_t tokens, int64_t heads, int64_t kv_heads, int64_t D, const AttendParts& p, bool reach, bool tree = false) {
  const int64_t cols = q_len * (heads / kv_heads);
  return attend_launchable(batch * kv_heads * p.parts, cols, attend_shape(kv4, padded_head((int)D), cols, reach, tree ? batch * kv_heads : 0)) &&
         (p.parts == 1 || launchable(join_workgroups(tokens * heads, D, p.parts), 256));
}

// the scale of the scores: positive; 0 stands for 1 / sqrt(D)
bool score_scale(float given, int64_t D, float* scale) {
  *scale = given == 0.0f ? 1.0f / sqrtf((float)D) : given;
  return *scale > 0.0f && *scale <= 3.4e38f;
}

// attention over the cache, causal or of a tree: sizes, workspace and pointers
gpusq_status attend_kv4(AttentionKv4 x, hipStream_t s) {
  if (!x.q || !x.cache || !x.block_table || !x.kv_lens || !x.out) return GPUSQ_ERR_NULL;
  gpusq_status st = check_heads(x.heads, x.kv_heads, x.head_dim);
  if (st != GPUSQ_OK) return st;
  if (!are_kv4_sizes(x.tokens, x.batch, x.max_q, x.max_pages, x.heads, x.head_dim) || !is_size(x.num_pages) || (!x.cu_q && x.tokens != x.batch * x.max_q))
    return GPUSQ_ERR_SHAPE;
  if (!score_scale(x.scale, x.head_dim, &x.scale)) return GPUSQ_ERR_UNSUPPORTED;
  const AttendParts p = attend_parts(true, x.batch, x.max_q, x.heads, x.kv_heads, x.head_dim, x.max_pages * kPageTokens, x.tree != nullptr);
  if (!is_launchable(true, x.batch, x.max_q, x.tokens, x.heads, x.kv_heads, x.head_dim, p, true, x.tree != nullptr)) return GPUSQ_ERR_SHAPE;
  if (p.parts > 1 && !x.workspace) return GPUSQ_ERR_NULL;
  if (!aligned16(x.q) || !aligned16(x.cache) || !aligned16(x.out) || !aligned16(x.workspace) || !aligned4(x.block_table) || !aligned4(x.kv_lens) || !aligned4(x.cu_q))
    return GPUSQ_ERR_ALIGN;
  return launch_attention_kv4(x, s);
}

// the new tokens of sequences, with a tree of at most kMostDrafts each
gpusq_status check_drafts(int64_t tokens, int64_t batch, int64_t max_q, const int32_t* cu_q) {
  if (!is_size(tokens) || !is_size(batch) || !is_size(max_q) || max_q > tokens || (!cu_q && tokens != batch * max_q) || !launchable(batch, 256)) return GPUSQ_ERR_SHAPE;
  return max_q <= kMostDrafts ? GPUSQ_OK : GPUSQ_ERR_UNSUPPORTED;
}

bool are_samples(int64_t rows, int64_t vocabulary) { return is_size(rows) && is_size(vocabulary) && vocabulary <= kMostVocabulary && launchable(rows, kSampleThreads); }

// codes of M tokens of K values in the workspace, rows of whole steps of 64; their scales behind them
bool are_tokens8(int64_t M, int64_t K) { return is_size(M) && is_size(K) && K <= kMostTokens8K && ceil_div(M, 64) <= 65535 && M * K <= kMaxElems; }
size_t tokens8_scales_at(int64_t M, int64_t K) { return (size_t)M * ceil_div(K, 64) * 64; }

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

size_t gpusq_attention_tree_kv4_workspace_bytes(int64_t tokens, int64_t batch, int64_t max_q, int64_t max_pages, int64_t heads, int64_t kv_heads, int64_t head_dim) {
  if (check_heads(heads, kv_heads, head_dim) != GPUSQ_OK || !are_kv4_sizes(tokens, batch, max_q, max_pages, heads, head_dim)) return 0;
  return parts_bytes(attend_parts(true, batch, max_q, heads, kv_heads, head_dim, max_pages * kPageTokens, true), tokens, heads, head_dim);
}

gpusq_status gpusq_attention_kv4(const void* q, const void* cache, const int32_t* block_table, const int32_t* kv_lens, const int32_t* cu_q, void* out,
                                 void* workspace, int64_t tokens, int64_t batch, int64_t max_q, int64_t max_pages, int64_t num_pages, int64_t heads,
                                 int64_t kv_heads, int64_t head_dim, float scale, void* stream) {
  return attend_kv4(AttentionKv4{q, cache, block_table, kv_lens, cu_q, out, workspace, tokens, batch, max_q, max_pages, num_pages, heads, kv_heads, head_dim, scale},
                    (hipStream_t)stream);
}

gpusq_status gpusq_attention_tree_kv4(const void* q, const void* cache, const int32_t* block_table, const int32_t* kv_lens, const int32_t* cu_q,
                                      const int32_t* tree, int64_t tree_words, void* out, void* workspace, int64_t tokens, int64_t batch, int64_t max_q,
                                      int64_t max_pages, int64_t num_pages, int64_t heads, int64_t kv_heads, int64_t head_dim, float scale, void* stream) {
  if (!tree) return GPUSQ_ERR_NULL;
  if (!is_size(max_q) || !is_size(tree_words) || tree_words < ceil_div(max_q, 32) || tokens > INT32_MAX / 2) return GPUSQ_ERR_SHAPE;
  if (!aligned4(tree)) return GPUSQ_ERR_ALIGN;
  return attend_kv4(AttentionKv4{q, cache, block_table, kv_lens, cu_q, out, workspace, tokens, batch, max_q, max_pages, num_pages, heads, kv_heads, head_dim, scale,
                                 tree, tree_words},
                    (hipStream_t)stream);
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

gpusq_status gpusq_draft_tree(const int32_t* parents, const int32_t* kv_lens, const int32_t* cu_q, const int32_t* block_table, int32_t* tree, int32_t* positions,
                              int32_t* slots, int64_t tokens, int64_t batch, int64_t max_q, int64_t max_pages, void* stream) {
  if (!parents || !kv_lens || !tree || (slots && !block_table)) return GPUSQ_ERR_NULL;
  gpusq_status st = check_drafts(tokens, batch, max_q, cu_q);
  if (st != GPUSQ_OK) return st;
  if (slots && (!is_size(max_pages) || max_pages > kMostPages)) return GPUSQ_ERR_SHAPE;
  if (!aligned4(parents) || !aligned4(kv_lens) || !aligned4(cu_q) || !aligned4(block_table) || !aligned4(tree) || !aligned4(positions) || !aligned4(slots))
    return GPUSQ_ERR_ALIGN;
  return launch_draft_tree(DraftArgs{kv_lens, cu_q, (int)tokens, (int)batch, (int)max_q}, parents, block_table, max_pages, tree, ceil_div(max_q, 32), positions, slots,
                           (hipStream_t)stream);
}

gpusq_status gpusq_accept_drafts(const int32_t* drafted, const int32_t* sampled, const int32_t* parents, const int32_t* kv_lens, const int32_t* cu_q,
                                 const int32_t* block_table, void* const* caches, int64_t layers, int32_t* path, int32_t* accepted, int32_t* answers,
                                 int32_t* new_lens, int64_t tokens, int64_t batch, int64_t max_q, int64_t max_pages, int64_t num_pages, int64_t kv_heads,
                                 int64_t head_dim, void* stream) {
  if (!drafted || !sampled || !parents || !kv_lens || !path || !accepted || !answers || !new_lens) return GPUSQ_ERR_NULL;
  if (layers != 0 && (!caches || !block_table)) return GPUSQ_ERR_NULL;
  gpusq_status st = check_drafts(tokens, batch, max_q, cu_q);
  if (st != GPUSQ_OK) return st;
  if (layers < 0 || layers > kMostCaches || batch * max_q > kMaxElems) return GPUSQ_ERR_SHAPE;
  if (layers != 0) {
    st = check_heads(kv_heads, kv_heads, head_dim);
    if (st != GPUSQ_OK) return st;
    if (!is_size(max_pages) || max_pages > kMostPages || !is_size(num_pages) || num_pages > INT32_MAX / kPageTokens || caches_of_launch(batch, kv_heads) < 1)
      return GPUSQ_ERR_SHAPE;
    const uint64_t bytes = (uint64_t)num_pages * kv_heads * page_bytes(padded_head((int)head_dim));
    uintptr_t at[kMostCaches];
    for (int64_t i = 0; i < layers; ++i) {
      if (!caches[i]) return GPUSQ_ERR_NULL;
      if (!aligned16(caches[i])) return GPUSQ_ERR_ALIGN;
      at[i] = (uintptr_t)caches[i];
    }
    // (the same tokens moved twice: of caches of one size that overlap some two are neighbours in the order of their addresses)
    std::sort(at, at + layers);
    for (int64_t i = 1; i < layers; ++i)
      if (at[i] - at[i - 1] < bytes) return GPUSQ_ERR_UNSUPPORTED;
  }
  if (!aligned4(drafted) || !aligned4(sampled) || !aligned4(parents) || !aligned4(kv_lens) || !aligned4(cu_q) || !aligned4(block_table) || !aligned4(path) ||
      !aligned4(accepted) || !aligned4(answers) || !aligned4(new_lens))
    return GPUSQ_ERR_ALIGN;
  return launch_accept_drafts(DraftArgs{kv_lens, cu_q, (int)tokens, (int)batch, (int)max_q}, drafted, sampled, parents, block_table, max_pages, path, accepted, answers,
                              new_lens, caches, layers, num_pages, layers != 0 ? kv_heads : 1, layers != 0 ? head_dim : 64, (hipStream_t)stream);
}

size_t gpusq_linear_int8_tokens_workspace_bytes(int64_t M, int64_t K) {
  if (!are_tokens8(M, K)) return 0;
  return tokens8_scales_at(M, K) + (size_t)ceil_div(M, 4) * 16;
}

gpusq_status gpusq_linear_int8_tokens(const void* X, gpusq_dtype dt, const int8_t* Wq, const float* w_scale, const float* bias, void* Y, gpusq_dtype out_dt,
                                      void* workspace, int64_t M, int64_t N, int64_t K, int epilogue, void* stream) {
  if (!X || !Wq || !w_scale || !Y || !workspace || ((epilogue & GPUSQ_EPI_BIAS) && !bias)) return GPUSQ_ERR_NULL;
  if (!are_tokens8(M, K) || !is_size(N) || N > kMostTokens8N || !tokens8_countable(M, N) || M * N > kMaxElems) return GPUSQ_ERR_SHAPE;
  if (K % 16 != 0 || N % 4 != 0 || (dt != GPUSQ_F16 && dt != GPUSQ_F32) || (out_dt != GPUSQ_F16 && out_dt != GPUSQ_F32) ||
      (epilogue & ~(GPUSQ_EPI_BIAS | GPUSQ_EPI_GELU)))
    return GPUSQ_ERR_UNSUPPORTED;
  if (!aligned16(X) || !aligned16(Wq) || !aligned16(w_scale) || !aligned16(bias) || !aligned16(Y) || !aligned16(workspace)) return GPUSQ_ERR_ALIGN;
  Linear8Args a{X, dt == GPUSQ_F32, Wq, w_scale, bias, Y, out_dt == GPUSQ_F32, epilogue, (int)M, (int)N, (int)K, (int8_t*)workspace,
                (float*)((uint8_t*)workspace + tokens8_scales_at(M, K)), ceil_div(K, 64) * 64};
  return launch_linear_int8_tokens(a, (hipStream_t)stream);
}

size_t gpusq_sample_tokens_workspace_bytes(int64_t rows, int64_t vocabulary) {
  if (!are_samples(rows, vocabulary)) return 0;
  const int parts = sample_parts(rows, vocabulary);
  return parts > 1 ? (size_t)(rows * sample_space(parts).bytes) : 0;
}

gpusq_status gpusq_sample_tokens(const void* logits, gpusq_dtype dt, int64_t row_stride, const float* random, const float* temperature, const int32_t* top_k,
                                 const float* top_p, const float* min_p, int32_t* tokens, float* probs, void* workspace, int64_t rows, int64_t vocabulary,
                                 void* stream) {
  if (!logits || !random || !tokens || !probs) return GPUSQ_ERR_NULL;
  if (!are_samples(rows, vocabulary) || row_stride < vocabulary || row_stride > INT32_MAX || rows * row_stride > kMaxElems) return GPUSQ_ERR_SHAPE;
  if (sample_parts(rows, vocabulary) > 1 && !workspace) return GPUSQ_ERR_NULL;
  if (dt != GPUSQ_F16 && dt != GPUSQ_F32) return GPUSQ_ERR_UNSUPPORTED;
  if (((uintptr_t)logits & (dt == GPUSQ_F32 ? 3u : 1u)) != 0 || !aligned4(random) || !aligned4(temperature) || !aligned4(top_k) || !aligned4(top_p) || !aligned4(min_p) ||
      !aligned4(tokens) || !aligned4(probs) || !aligned16(workspace))
    return GPUSQ_ERR_ALIGN;
  const SampleArgs a{logits, row_stride, random, temperature, top_p, min_p, top_k, tokens, probs, (int)vocabulary};
  return launch_sample_tokens(a, dt == GPUSQ_F32, rows, workspace, (hipStream_t)stream);
}

}  // extern "C"
