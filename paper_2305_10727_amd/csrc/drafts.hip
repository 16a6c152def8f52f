// Trees of drafted tokens: what each token of a step follows, where it stands and where the cache keeps it; and, when the step's answers are
// there, the branch that was drafted as it would have been answered, its tokens moved together in the caches.
//
// A tree has a few dozen nodes and a kept branch a few tokens of a cache: bytes and operations are nothing, so what bounds these calls is a launch
// and the trips to memory that depend on one another, and the choices below are the ones with the fewest of those.  Everything is whole numbers.
// (A tree of 8 nodes 3.9 us, 64 of 61 5.2; a branch of one tree kept and moved in one layer 5.7.)
#include "drafts_plan.h"
#include "kv4.h"

namespace gpusq {

namespace {

// The new tokens of a sequence, as attention counts them: `nodes` of them are answered, `before` places of the cache lie in front of the first
struct Drafts {
  int t0, nodes, before;
  __device__ __forceinline__ Drafts(const DraftArgs& a, int b) : t0(b * a.max_q), nodes(a.max_q) {
    if (a.cu_q != nullptr) {
      t0 = a.cu_q[b];
      const int t1 = a.cu_q[b + 1];
      nodes = t0 >= 0 && t1 <= a.tokens && t1 > t0 ? t1 - t0 : 0;
    }
    const int len = a.kv_lens[b];
    before = (len > 0 ? len : 0) - nodes;
    nodes = nodes < a.max_q ? nodes : a.max_q;
  }
};

// The page of a place of a sequence, or -1
__device__ __forceinline__ int page_of(const int32_t* table, int max_pages, int place) {
  return place >= 0 && (place >> 6) < max_pages ? table[place >> 6] : -1;
}

// ---- what each node follows -------------------------------------------------------------------------------------------------------------
// Chains of parents are followed by doubling: a node's set takes in that of the node it has come to, and goes on from where that one has come to.
// A workgroup for each sequence; sets and pointers go from one half of LDS to the other.
__global__ void __launch_bounds__(256) draft_tree_kernel(const DraftArgs a, const int32_t* __restrict__ parents, const int32_t* __restrict__ table, int max_pages,
                                                         int32_t* __restrict__ tree, int words, int32_t* __restrict__ positions, int32_t* __restrict__ slots) {
  extern __shared__ unsigned lds[];  // [2][max_q][words] sets, [2][max_q] pointers
  const int b = blockIdx.x, tid = threadIdx.x;
  const Drafts d(a, b);
  const int n = d.nodes, cells = n * words, half = a.max_q * words;
  int* const next = (int*)(lds + 2 * half);
  for (int i = tid; i < cells; i += 256) {
    const int node = i / words;
    lds[i] = i - node * words == node >> 5 ? 1u << (node & 31) : 0u;
  }
  for (int i = tid; i < n; i += 256) {
    const int p = parents[d.t0 + i];
    next[i] = p >= 0 && p < i ? p : -1;  // (what is no node in front of it is no parent)
    if (slots != nullptr) {
      const int place = d.before + i, page = page_of(table + (int64_t)b * max_pages, max_pages, place);
      slots[d.t0 + i] = page >= 0 && page < 1 << 25 ? page * kPageTokens + (place & 63) : -1;
    }
  }
  int from = 0;
  for (;;) {
    __syncthreads();
    const unsigned* set = lds + from * half;
    const int* ptr = next + from * a.max_q;
    unsigned* set2 = lds + (from ^ 1) * half;
    int* ptr2 = next + (from ^ 1) * a.max_q;
    int more = 0;
    for (int i = tid; i < cells; i += 256) {
      const int node = i / words, p = ptr[node];
      set2[i] = set[i] | (p >= 0 ? set[p * words + (i - node * words)] : 0u);
    }
    for (int i = tid; i < n; i += 256) {
      const int p = ptr[i], q = p >= 0 ? ptr[p] : -1;
      ptr2[i] = q;
      more |= q >= 0;
    }
    from ^= 1;
    if (!__syncthreads_or(more)) break;
  }
  const unsigned* set = lds + from * half;
  for (int i = tid; i < cells; i += 256) tree[(int64_t)d.t0 * words + i] = (int)set[i];
  if (positions != nullptr)
    for (int i = tid; i < n; i += 256) {
      int depth = -1;
      for (int w = 0; w < words; ++w) depth += __popc(set[i * words + w]);
      positions[d.t0 + i] = d.before + depth;
    }
}

// ---- the kept branch --------------------------------------------------------------------------------------------------------------------
// From node 0 on to the first child whose draft is what was drawn behind its parent.  Every workgroup walks by itself, one wavefront with 64 nodes at
// a time: the first of a sequence's writes the results, the others move some heads' tokens in a layer's cache each.  (16 trees, 24 layers of 4 heads: all of a
// layer's heads in a workgroup 10.2 us, a workgroup a head 13.6.)
__global__ void __launch_bounds__(256) accept_drafts_kernel(const DraftArgs a, const int32_t* __restrict__ drafted, const int32_t* __restrict__ sampled,
                                                            const int32_t* __restrict__ parents, const int32_t* __restrict__ table, int max_pages,
                                                            int32_t* __restrict__ path, int32_t* __restrict__ accepted, int32_t* __restrict__ answers,
                                                            int32_t* __restrict__ new_lens, const CacheList caches, int num_pages, int kv_heads, int heads, int DP) {
  __shared__ int parent[kMostDrafts], draft[kMostDrafts], drawn[kMostDrafts], kept[kMostDrafts], count;
  __shared__ int64_t place[kMostDrafts];  // of the kept node and of where it goes: token of a page, -1 where there is none
  __shared__ int pages[kMostDrafts / kPageTokens + 1];  // of the new tokens
  const int b = blockIdx.x, tid = threadIdx.x;
  const Drafts d(a, b);
  const int n = d.nodes;
  for (int i = tid; i < n; i += 256) {
    parent[i] = parents[d.t0 + i];
    draft[i] = drafted[d.t0 + i];
    drawn[i] = sampled[d.t0 + i];
  }
  const int first_page = d.before >> 6;  // (in front of the sequence: negative, and no page)
  if (blockIdx.y > 0 && tid <= kMostDrafts / kPageTokens) pages[tid] = first_page + tid >= 0 && first_page + tid < max_pages ? table[(int64_t)b * max_pages + first_page + tid] : -1;
  __syncthreads();
  if (tid < 64) {
    int at = 0, len = 0;
    while (n > 0) {
      if (tid == 0) kept[len] = at;
      ++len;
      const int want = drawn[at];
      int child = -1;
      if (want < 0) break;  // (nothing was drawn)
      for (int i0 = (at + 1) & ~63; i0 < n; i0 += 64) {  // (a child is behind its parent, so the walk ends)
        const int i = i0 + tid;
        const uint64_t fits = __builtin_amdgcn_ballot_w64(i > at && i < n && parent[i < n ? i : 0] == at && draft[i < n ? i : 0] == want);
        if (fits != 0) {
          child = i0 + __builtin_ctzll(fits);
          break;
        }
      }
      if (child < 0) break;
      at = child;
    }
    if (tid == 0) count = len;
    if (tid == 0 && blockIdx.y == 0) {
      accepted[b] = len;
      answers[b] = n > 0 ? drawn[at] : -1;
      const int64_t l = (int64_t)d.before + len;
      new_lens[b] = l > 0 ? (int)l : 0;
    }
  }
  __syncthreads();
  const int len = count;
  if (blockIdx.y == 0) {
    for (int i = tid; i < a.max_q; i += 256) path[(int64_t)b * a.max_q + i] = i < len ? kept[i] : -1;
    return;
  }
  const int groups = (kv_heads + heads - 1) / heads, group = blockIdx.y - 1, layer = group / groups, head0 = (group - layer * groups) * heads;
  const int own = kv_heads - head0 < heads ? kv_heads - head0 : heads;
  uint8_t* cache = (uint8_t*)caches.of[layer];
  // (32 bits each: pages and tokens of them, together 31)
  for (int i = tid; i < len; i += 256) {
    auto slot = [&](int at) {
      const int page = at >= 0 ? pages[(at >> 6) - first_page] : -1;
      return page >= 0 && page < num_pages ? page * kPageTokens + (at & 63) : -1;
    };
    const int from = slot(d.before + kept[i]), to = slot(d.before + i);
    place[i] = from < 0 || to < 0 || from == to ? -1 : (int64_t)from << 32 | (unsigned)to;
  }
  __syncthreads();
  // A token of a head is DP / 4 units of key codes, J of key scales, DP / 4 of value codes, J of value scales.
  const int J = DP / 32, quads = DP / 4, per = token_units(DP);
  auto unit_at = [&](int slot, int head, int u) {  // in 16-bit units from the cache's beginning
    const int t = slot & 63;
    const int64_t page = ((int64_t)(slot >> 6) * kv_heads + head) * (page_bytes(DP) / 2);
    if (u < quads) return page + t * quads + u;
    u -= quads;
    if (u < J) return page + key_scales_at(DP) / 2 + t * J + u;
    u -= J;
    if (u < quads) {
      const int CQ = DP / 64, n16 = u / CQ;  // block of channels, quad of it
      return page + value_codes_at(DP) / 2 + (((t >> 2) * 16 + n16) * 2 + (t >> 1 & 1)) * CQ * 2 + (u - n16 * CQ) * 2 + (t & 1);
    }
    u -= quads;
    return page + value_scales_at(DP) / 2 + u * kPageTokens + t;
  };
  uint16_t* units = (uint16_t*)cache;
  // Some tokens at a time, all of them read before any is written; a token moves to the front or stays, so what is written lies in front of what
  // the later ones are read from.
  const int of_token = per * own, chunk = kUnitsOfWorkgroup / of_token;
  for (int i0 = 0; i0 < len; i0 += chunk) {
    const int total = (len - i0 < chunk ? len - i0 : chunk) * of_token;
    constexpr int kUnits = kUnitsOfWorkgroup / 256;
    uint16_t v[kUnits];
    int64_t to[kUnits];
#pragma unroll
    for (int j = 0; j < kUnits; ++j) {
      const int x = tid + 256 * j;
      to[j] = -1;
      v[j] = 0;
      if (x >= total) continue;
      const int i = x / of_token, rest = x - i * of_token, head = rest / per, u = rest - head * per;
      const int64_t p = place[i0 + i];
      if (p >= 0) {
        to[j] = unit_at((int)(unsigned)p, head0 + head, u);
        v[j] = units[unit_at((int)(p >> 32), head0 + head, u)];
      }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kUnits; ++j)
      if (to[j] >= 0) units[to[j]] = v[j];
    __syncthreads();
  }
}

}  // namespace

gpusq_status launch_draft_tree(const DraftArgs& a, const int32_t* parents, const int32_t* table, int64_t max_pages, int32_t* tree, int64_t words, int32_t* positions,
                               int32_t* slots, hipStream_t s) {
  const size_t lds = (size_t)8 * a.max_q * (words + 1);
  draft_tree_kernel<<<(unsigned)a.batch, 256, lds, s>>>(a, parents, table, (int)max_pages, tree, (int)words, positions, slots);
  return check_launch();
}

gpusq_status launch_accept_drafts(const DraftArgs& a, const int32_t* drafted, const int32_t* sampled, const int32_t* parents, const int32_t* table, int64_t max_pages,
                                  int32_t* path, int32_t* accepted, int32_t* answers, int32_t* new_lens, void* const* caches, int64_t layers, int64_t num_pages,
                                  int64_t kv_heads, int64_t D, hipStream_t s) {
  const int DP = padded_head((int)D), heads = heads_of_workgroup(kv_heads, DP);
  const int64_t groups = ceil_div(kv_heads, heads), most = caches_of_launch(a.batch, groups);
  int64_t from = 0;
  do {  // (at least once: the results)
    CacheList list{};
    const int64_t n = layers - from < most ? layers - from : most;
    for (int64_t i = 0; i < n; ++i) list.of[i] = caches[from + i];
    const dim3 grid((unsigned)a.batch, (unsigned)(1 + n * groups));
    accept_drafts_kernel<<<grid, 256, 0, s>>>(a, drafted, sampled, parents, table, (int)max_pages, path, accepted, answers, new_lens, list, (int)num_pages, (int)kv_heads,
                                              heads, DP);
    const gpusq_status st = check_launch();
    if (st != GPUSQ_OK) return st;
    from += most;
  } while (from < layers);
  return GPUSQ_OK;
}

}  // namespace gpusq
