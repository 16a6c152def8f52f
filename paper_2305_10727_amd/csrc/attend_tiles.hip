// Attention of many queries (a prompt's chunk over the cache, an image's tokens to its own or another's states): the kernel whose bound is
// arithmetic.  A workgroup's wavefronts have columns of their own and share the keys: keys and values go through LDS a tile at a time, in rows
// as they lie in memory, with the 16-byte pieces of a row in places that differ from row to row (place()), so that neither the 16 rows of a
// key operand nor the transposed reads of a value operand meet in a bank.  While one buffer is multiplied the others are filled.
// Prompts of 1000 queries, 32 heads of 128 over 8, to up to 2313 states: 124-129 us, 0.9 PFLOP/s, the matrix units busy half of the time; for 34
// matrix instructions (32 keys, 32 columns) there are 16 exponentials and some 70 other vector ones, of which a SIMD does little side by side.
// ViT-B's attention at batch 128: 41 us for 155 MB, 3.7 TB/s where a large copy has 5.0.
//   fp16 states go from memory to LDS directly; the cache's codes become fp16 numbers on the way, once for all the workgroup's columns.
#include "attend.h"
#include "tile_common.h"

#include <type_traits>

namespace gpusq {

namespace {

// Where a row keeps its 16-byte piece c: rows that a wavefront reads together have the same piece in different banks.  (16 rows of 256 bytes
// or 8 pairs of rows of 128.)
template <int DP>
__device__ __forceinline__ int place(int row, int c) {
  return DP == 64 ? c ^ ((row >> 1) & 7) : c ^ (row & 15);
}
template <int DP>
constexpr int kRow = 2 * DP;  // bytes

// Four keys of a value operand: lane 16 g + r reads 8 bytes of row 4 g + r / 4 and gets channel r of the four rows
__device__ __forceinline__ h4 read_transposed(const uint8_t* p) {
  typedef __fp16 t4 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) t4 lds_t4;
  return __builtin_bit_cast(h4, __builtin_amdgcn_ds_read_tr16_b64_v4f16((lds_t4*)p));
}

// ---- fp16 states on their way: memory to LDS, 1 KB a wavefront and instruction -----------------------------------------------------------
// Behind a mask of bytes only the keys that are seen are copied: what the others hold, which may be anything (0 times it would not be 0), does
// not get there, and their rows keep what an earlier tile left or the zeros of the beginning.  The first product begins at 0 or -inf by key.
template <int DP, int KT, int NW, bool MASKED>
struct States {
  static constexpr int PIECES = DP / 8, ROWS = 64 / PIECES;          // pieces of a row, rows of an instruction
  static constexpr int COPIES = KT / (ROWS * NW);                    // instructions of a wavefront, for keys and for values
  static_assert(COPIES > 0 && COPIES * ROWS * NW == KT, "whole instructions");
  const uint8_t *kp, *vp;  // of the next tile to load: tiles are loaded in order
  int64_t k_row, v_row;    // bytes
  uint32_t lds;
  int row[COPIES], piece[COPIES], len, D2;
  const uint8_t* mask;
  uint8_t byte[COPIES];
  float* begin;  // [buffer][key of a tile]
  unsigned seen;  // whether this lane copied of any key
  bool first;    // of a row's lanes

  __device__ __forceinline__ States(const AttendArgs& a, const Work& w, int len_, int wave, int lane, uint8_t* tiles, float* begin_, int first_key)
      : kp((const uint8_t*)(a.k + w.b * a.k_batch + w.kh * a.k_head + first_key * a.k_token)),
        vp((const uint8_t*)(a.v + w.b * a.v_batch + w.kh * a.v_head + first_key * a.v_token)), k_row(2 * a.k_token), v_row(2 * a.v_token),
        lds(lds_address(tiles) + wave * COPIES * 1024), len(len_), D2(2 * a.D),
        mask(MASKED ? a.mask + (int64_t)w.b * a.kv_len : nullptr), begin(begin_), seen(0), first(lane % PIECES == 0) {
#pragma unroll
    for (int i = 0; i < COPIES; ++i) {
      row[i] = (wave * COPIES + i) * ROWS + lane / PIECES;
      piece[i] = 16 * place<DP>(row[i], lane % PIECES);
    }
  }
  // the bytes for load(., key0), a tile before it
  __device__ __forceinline__ void look(int key0) {
#pragma unroll
    for (int i = 0; i < COPIES; ++i) byte[i] = mask[key0 + row[i] < len ? key0 + row[i] : len - 1];
  }
  // Rows from `len` on are its last row once more (finite where that is), pieces beyond the head are left out.
  __device__ __forceinline__ void load(int buf, int key0) {
    const uint8_t *k = kp, *v = vp;
    kp += KT * k_row;
    vp += KT * v_row;
    const int last = len - 1 - key0;
    unsigned sees = ~0u;
    if constexpr (MASKED) {
#pragma unroll
      for (int i = 0; i < COPIES; ++i) sees = row[i] <= last && byte[i] != 0 ? sees : sees & ~(1u << i);
      seen |= sees & ((1u << COPIES) - 1);
      asm volatile("" : "+v"(sees));  // (all of the bytes, before a copy: the compiler, which does not count these, would wait for them as well)
    }
#pragma unroll
    for (int i = 0; i < COPIES; ++i) {
      const unsigned r = row[i] < last ? row[i] : last;
      const uint32_t at = lds + buf * (2 * KT * kRow<DP>) + i * 1024;
      const bool see = !MASKED || (sees >> i & 1) != 0;
      if (MASKED && first) begin[buf * KT + row[i]] = see ? 0.0f : -__builtin_inff();
      if (see && piece[i] < D2) {
        copy16_to_lds(k, r * (unsigned)k_row + piece[i], at);
        copy16_to_lds(v, r * (unsigned)v_row + piece[i], at + KT * kRow<DP>);
      }
    }
  }
};

// ---- the cache's codes on their way -----------------------------------------------------------------------------------------------------
// Each wavefront has 16 tokens' keys (lane 16 g + r pieces 4 j + g of key r) or 16 tokens' values (channels CH r .. of quad g).
template <int DP, int KT, int NW>
struct Codes {
  static_assert(KT / 8 == NW, "16 keys or values a wavefront");
  static constexpr int J = DP / 32, CH = DP / 16;
  static constexpr int SW = J > 4 ? J / 2 : 2;
  typename WordsOf<J>::type w;   // codes, of a key or of a quad of values
  typename WordsOf<SW>::type s;  // scales: J / 2 words of a key, 2 of a quad of values
  const uint8_t* cache;
  const int32_t* table;
  int len, num_pages, kv_heads, kh, part, lane, last_page, number;
  bool values, there;

  // (a page's number is read a tile ahead of its words: first_key's here)
  __device__ __forceinline__ Codes(const AttendArgs& a, const Work& w, int len_, int wave, int lane_, const uint8_t*, const float*, int first_key)
      : cache(a.cache), table(a.table + (int64_t)w.b * a.max_pages), len(len_), num_pages(a.num_pages), kv_heads(a.kv_heads), kh(w.kh), part(wave % (NW / 2)), lane(lane_),
        last_page((len_ - 1) >> 6), number(0), values(wave >= NW / 2), there(false) {
    if (first_key < len_) number = table[first_key >> 6];
  }
  __device__ __forceinline__ void load(int, int key0) {
    there = (unsigned)number < (unsigned)num_pages;  // (a number that is no page is read as page 0, and not seen)
    const uint8_t* page = cache + ((int64_t)(there ? number : 0) * kv_heads + kh) * page_bytes(DP);
    const int after = (key0 + KT) >> 6;
    number = table[after < last_page ? after : last_page];
    const int g = lane >> 4, r = lane & 15, token = (key0 & 63) + part * 16;
    if (!values) {
      w = load_words<J>(page + (token + r) * (DP / 2) + g * J * 4);
      const auto u = load_words<J / 2>(page + key_scales_at(DP) + (token + r) * J * 2);
#pragma unroll
      for (int i = 0; i < SW; ++i) s[i] = i < J / 2 ? u[i] : 0u;
    } else {
      const int quad = (token >> 2) + g;
      w = load_words<J>(page + value_codes_at(DP) + (quad * 16 + r) * (2 * CH));
      u2 u = load_words<2>(page + value_scales_at(DP) + (r * CH / 32 * kPageTokens + quad * 4) * 2);
      if (!there || key0 + KT > len) u = scales_in_front(u, there ? len - (key0 + part * 16 + 4 * g) : 0);
      s[0] = u[0];
      s[1] = u[1];
    }
  }
  __device__ __forceinline__ void write(uint8_t* rows_of_keys, uint8_t* rows_of_values) const {
    const int g = lane >> 4, r = lane & 15;
    if (!values) {
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const h2 pair = __builtin_bit_cast(h2, (unsigned)s[j / 2]), sc = {pair[j & 1], pair[j & 1]};
        h2 c[4];
        codes_to_halves(w[j], sc, sc * (_Float16)-72.0f, c);
        *(h8*)(rows_of_keys + (part * 16 + r) * kRow<DP> + place<DP>(r, 4 * j + g) * 16) = join(c[0], c[1], c[2], c[3]);
      }
      return;
    }
    const h2 s0 = __builtin_bit_cast(h2, (unsigned)s[0]), s1 = __builtin_bit_cast(h2, (unsigned)s[1]), off0 = s0 * (_Float16)-72.0f, off1 = s1 * (_Float16)-72.0f;
    constexpr int Q = CH >= 8 ? 2 : 1;  // quads of channels that are a piece of a row, or its half
#pragma unroll
    for (int q0 = 0; q0 < CH / 4; q0 += Q) {
      h2 c[Q][2][4];  // [quad][tokens 0, 1 and 2, 3][channel]
#pragma unroll
      for (int i = 0; i < Q; ++i) {
        codes_to_halves(w[q0 + i], s0, off0, c[i][0]);
        codes_to_halves(w[CH / 4 + q0 + i], s1, off1, c[i][1]);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int token = 4 * g + e;
        uint8_t* at = rows_of_values + (part * 16 + token) * kRow<DP> + place<DP>(token, (CH * r + 4 * q0) >> 3) * 16;
        const h2(&x)[4] = c[0][e >> 1], (&y)[4] = c[Q - 1][e >> 1];
        if constexpr (Q == 2)
          *(h8*)at = h8{x[0][e & 1], x[1][e & 1], x[2][e & 1], x[3][e & 1], y[0][e & 1], y[1][e & 1], y[2][e & 1], y[3][e & 1]};
        else
          *(h4*)(at + (r & 1) * 8) = h4{x[0][e & 1], x[1][e & 1], x[2][e & 1], x[3][e & 1]};
      }
    }
  }
};

// The cache: 8 wavefronts on tiles of 64 keys, one workgroup a CU, as the codes are unpacked once for all of them (chunks of 300 tokens behind
// 6000, 32 heads of 128 over 8: 87 us; with 4 wavefronts on tiles of 32 and three workgroups a CU 129.  Heads of 64: 63 us, and 70).
// States: tiles of 32, as many workgroups a CU as registers allow.  Heads of 64 need more loads on their way than two buffers hold: four (ViT-B's
// attention, batch 128: 42.8 us with two, 41.5 with four); heads of 128, whose tile takes twice as long to multiply, gain nothing (prompts of 1000
// over 2313 states: 126 us with two, 129 with three).
constexpr int tile_waves_per_simd(bool kv4, int DP, bool masked) { return kv4 || DP == 256 ? 2 : DP == 64 ? 4 : masked ? 2 : 3; }
constexpr int state_buffers(int DP) { return DP == 64 ? 4 : 2; }  // (a mask's bytes come one tile ahead of two buffers)

template <bool KV4, int DP, int QT, int NW, int KT, int NB, bool MASKED>
__global__ void __launch_bounds__(64 * NW, tile_waves_per_simd(KV4, DP, MASKED)) attend_tiles_kernel(const AttendArgs a) {
  static_assert(NB == 2 || (NB == 4 && !KV4), "the waits for copies");
  static_assert(!MASKED || NB == 2, "bytes of one tile");
  static_assert(QT <= 2, "count below QT is 1 or 0");
  static_assert(NB * KT <= kMostAhead, "key0 + NB * KT");
  constexpr int J = DP / 32, CH = DP / 16, NT = 64 * NW, kTile = KT * kRow<DP>;
  __shared__ __attribute__((aligned(16))) uint8_t lds[NB * 2 * kTile];  // [buffer][keys, values]
  __shared__ __attribute__((aligned(16))) float begin[MASKED ? NB * KT + 4 : 4];
  __shared__ int pages[2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, r = lane & 15;
  Work w;
  if (!w.find(a)) return;
  const Span<KV4> span(a, w.b);
  // blocks of 16 columns, dealt out evenly over the workgroups that they need and then over the wavefronts
  const int cols = span.nq * a.rep, col_tiles = (cols + 15) >> 4, groups = (col_tiles + NW * QT - 1) / (NW * QT);
  if (w.block >= groups) return;
  const ColumnShare share = column_share(col_tiles, groups, w.block);
  const int tile0 = share.first, tile1 = share.last;
  const int least = span.sees(16 * (tile0 + wave) / a.rep);
  const int last = 16 * tile1 < cols ? 16 * tile1 - 1 : cols - 1;
  const int most = span.sees(last / a.rep);
  const KeyRange keys = keys_of_part(w.part, a.part_tiles, most);
  const int first_key = keys.begin, end_key = keys.end;
  typedef typename std::conditional<KV4, Codes<DP, KT, NW>, States<DP, KT, NW, MASKED>>::type Stage;
  Stage stage(a, w, span.len, wave, lane, lds, begin, first_key);
  if (!KV4 && (MASKED || a.D < DP)) {  // the pieces beyond the head, and rows that are not copied: zeros, once
    for (int i = threadIdx.x; i < NB * 2 * kTile / 16; i += NT) ((u4*)lds)[i] = u4(0);
    if (MASKED && threadIdx.x == 0) begin[NB * KT] = 0.0f;
    __syncthreads();
  }
  if constexpr (KV4) {
    if (first_key < end_key) stage.load(0, first_key);
  } else {
    if (MASKED && first_key < end_key) stage.look(first_key);
#pragma unroll
    for (int i = 0; i < NB - 1; ++i)
      if (first_key + i * KT < end_key) stage.load(i, first_key + i * KT);
    if (MASKED && first_key + KT < end_key) stage.look(first_key + KT);
  }
  Columns<KV4, DP, QT> x;
  // (block i of a wavefront beyond the workgroup's last: columns that are no columns)
  x.load(a, span, w.kh, g, r, [&](int i) { return tile0 + wave + NW * i < tile1 ? 16 * (tile0 + wave + NW * i) : cols; });
  // The queries are waited for here: their first use is inside the loop, where the compiler, which does not know of the copies to LDS, would
  // wait for all of these as well, in every turn.
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)

  // this lane's key operands and value operands: pieces by their places
  int key_at[J], value_at[CH];
#pragma unroll
  for (int j = 0; j < J; ++j) key_at[j] = r * kRow<DP> + place<DP>(r, 4 * j + g) * 16;
#pragma unroll
  for (int t = 0; t < CH; ++t) {
    const int row = 4 * g + (r >> 2);
    value_at[t] = kTile + row * kRow<DP> + place<DP>(row, 2 * t + ((r & 3) >> 1)) * 16 + (r & 1) * 8;
  }

  auto multiply = [&](auto blocks, int buf, int key0, bool there) {
    constexpr int N = decltype(blocks)::value;
    const uint8_t* tile = lds + buf * 2 * kTile;
#pragma unroll
    for (int half = 0; half < KT / 32; ++half) {
      f4 s[N][2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const f4 begins = MASKED ? *(const f4*)&begin[buf * KT + 32 * half + 16 * t + 4 * g] : f4(0);
#pragma unroll
        for (int i = 0; i < N; ++i) s[i][t] = begins;
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const h8 k = *(const h8*)(tile + key_at[j] + (2 * half + t) * 16 * kRow<DP>);
#pragma unroll
          for (int i = 0; i < N; ++i) s[i][t] = mfma16(k, x.q[i][j], s[i][t]);
        }
      }
      h8 p[N];
      const int at = key0 + 32 * half + 4 * g;
      if (!MASKED && (!there || key0 + 32 * half + 32 > least)) x.hide(s, [&](int i, int t, int e) { return at + 16 * t + e >= (there ? x.limit[i] : 0); });
      x.follow(s, a);
      x.weights(s, a.c, p);
      x.sum(p);
#pragma unroll
      for (int t = 0; t < CH; ++t) {
        const h4 v0 = read_transposed(tile + value_at[t] + 32 * half * kRow<DP>), v1 = read_transposed(tile + value_at[t] + (32 * half + 16) * kRow<DP>);
        const h8 v = __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
        for (int i = 0; i < N; ++i) x.o[i][t] = mfma16(v, p[i], x.o[i][t]);
      }
    }
  };

  // The loop over the tiles for N blocks of columns: wavefronts meet at its barriers, whichever of its copies they are in.
  auto run = [&](auto blocks) {
    int buf = 0;
    if constexpr (KV4) {
      auto put = [&](int to) {
        stage.write(lds + to * 2 * kTile, lds + to * 2 * kTile + kTile);
        if (threadIdx.x == 0) pages[to] = stage.there;
      };
      if (first_key < end_key) {
        put(0);
        if (first_key + KT < end_key) stage.load(0, first_key + KT);
      }
      for (int key0 = first_key; key0 < end_key; key0 += KT) {
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");  // (loads for registers stay in flight)
        // the next tile, whose words have had the time of the one before, goes to LDS first: nobody waits for the writes at the next barrier
        const bool there = pages[buf] != 0;
        if (key0 + KT < end_key) {
          put(buf ^ 1);
          if (key0 + 2 * KT < end_key) stage.load(0, key0 + 2 * KT);
        }
        if constexpr (decltype(blocks)::value > 0) multiply(blocks, buf, key0, there);
        buf ^= 1;
      }
    } else {
      for (int key0 = first_key; key0 < end_key; key0 += KT) {
        // this tile is there (of the wavefront's own copies, which come back in order, only later tiles' are left), and nobody reads the buffer of
        // the one before it
        const int later = (end_key - key0 - 1) / KT;
        if (NB == 4 && later >= 2)
          asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(4 * Stage::COPIES) : "memory");
        else if (NB == 4 && later >= 1)
          asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(2 * Stage::COPIES) : "memory");
        else
          asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (key0 + (NB - 1) * KT < end_key) {
          stage.load(buf == 0 ? NB - 1 : buf - 1, key0 + (NB - 1) * KT);
          if (MASKED && key0 + NB * KT < end_key) stage.look(key0 + NB * KT);
        }
        if constexpr (decltype(blocks)::value > 0) multiply(blocks, buf, key0, true);
        buf = buf + 1 < NB ? buf + 1 : 0;
      }
    }
  };
  // a wavefront whose last block is none leaves it out
  const int count = tile1 - tile0 - wave > 0 ? (tile1 - tile0 - wave + NW - 1) / NW : 0;
  if (count == QT)
    run(std::integral_constant<int, QT>());
  else if (count == 1)
    run(std::integral_constant<int, 1>());
  else
    run(std::integral_constant<int, 0>());
  // Columns that see nothing have nothing, also where a query is no number: -inf, which the scores of hidden keys begin at, and NaN are NaN.
  if constexpr (MASKED) {
    if (stage.seen != 0) begin[NB * KT] = 1.0f;  // (whoever writes it: the same)
    __syncthreads();
    if (begin[NB * KT] == 0.0f) x.clear();
  }
  if (count > 0) x.store(a, w.part, g);
}

template <bool KV4, int DP, int QT, int NW, int KT, int NB>
void launch_shape(AttendArgs a, hipStream_t s) {
  static_assert(16 * QT * NW == tiles_columns(KV4, DP) && 64 * NW == tiles_threads(KV4), "as the host counts workgroups");
  a.col_blocks = (int)ceil_div((int64_t)a.q_len * a.rep, 16 * QT * NW);
  const unsigned blocks = Work::workgroups(a);
  if constexpr (!KV4) {
    if (a.mask != nullptr) {
      attend_tiles_kernel<KV4, DP, QT, NW, KT, 2, true><<<blocks, 64 * NW, 0, s>>>(a);
      return;
    }
  }
  attend_tiles_kernel<KV4, DP, QT, NW, KT, NB, false><<<blocks, 64 * NW, 0, s>>>(a);
}

}  // namespace

void launch_attend_tiles(bool kv4, AttendArgs a, hipStream_t s) {
  const int DP = padded_head(a.D);
  if (kv4)
    DP == 64 ? launch_shape<true, 64, 2, 8, 64, 2>(a, s) : DP == 128 ? launch_shape<true, 128, 2, 8, 64, 2>(a, s) : launch_shape<true, 256, 1, 8, 64, 2>(a, s);
  else
    DP == 64 ? launch_shape<false, 64, 2, 4, 32, state_buffers(64)>(a, s)
    : DP == 128 ? launch_shape<false, 128, 2, 4, 32, state_buffers(128)>(a, s) : launch_shape<false, 256, 1, 4, 32, state_buffers(256)>(a, s);
}

}  // namespace gpusq
