// Linear layers in 8-bit integers with token scales, many rows: tiles of 256 channels x up to 256 rows, one persistent workgroup a CU.
//
// Such a layer is bound by the matrix pipe (2 M N K operations; 3.1 POP/s is what the dense 8-bit instruction sustains on random operands), so the
// choices follow from keeping it fed: 8 wavefronts, 2 along n x 4 along m, each with 128 channels x up to 64 rows in 128 accumulators, so that a
// step of 64 k (32 KB of operands a CU) has 64 matrix instructions a SIMD, 1050 clocks, beside 512 of copies and 420 of LDS reads.  Operands come
// from memory to LDS directly, 3 steps ahead and more, also across tiles; registers are read ahead of the instructions by half a step.
// 2309 tokens, 5120 -> 13824 with GELU (327 GOP): 172 us behind the quantiser's 10, 1.9 POP/s, matrix units 50 % busy; 8192^3 465, 2.37 POP/s; 4096 x
// 8192 -> 8192 241; 1024 x 4096 -> 4096 32; 256 and 512, 5120 -> 13824: 43 and 55.  Between the steps' first and last instructions stands no scalar work
// that could stand elsewhere: a wavefront of two a SIMD issues one instruction in about 5 clocks, of whatever kind.
//
// A block of 16 rows x 64 bytes is 1 KB of LDS, for weights as for activations: row r's 16-byte chunk c at 64 r + 16 (c ^ (r / 4)), so that the 16
// rows that a quarter of a wavefront reads at one k fall into 16 different groups of banks; four lanes fetch a row's 64 bytes.  A tile's blocks of
// weights are in the order in which a lane ends up with 8 consecutive channels of a row (packed_row_to_channel).
// K steps are numbered over a workgroup's whole sequence of tiles; step g lives in stage g % R.  One barrier a step, in front of the last
// instructions of its first half: by then a wavefront has its last read of the step's stage, and its own copies of step g + 1 have landed.  Behind
// it stage g + 1 is whole and is read ahead, and stage g is free for the copies of step g + R.
// K that is no whole number of steps: the rows of codes have zeros behind their end, and the chunks of weights there are the step's first once more.
#pragma once
#include <type_traits>

#include "gelu4.h"
#include "linear8_plan.h"
#include "tile_common.h"

namespace gpusq {

namespace {

// A stage: the tile's blocks of weights, then those of its rows.  A wavefront copies block `wave` and every eighth behind it: kCopies, or one less (the
// waits count them).
template <int TN, int NX>
struct Ring8 {
  static constexpr int kW = 2 * TN, kBlocks = kW + 4 * NX, kStage = kBlocks * 1024, kCopies = (kBlocks + 7) / 8;
  static constexpr int kStages = 148 * 1024 / kStage < 10 ? 148 * 1024 / kStage : 10;
  static_assert(kStages >= 4 && kStages * kStage + 6144 <= 160 * 1024, "LDS");
};

template <int N>
__device__ __forceinline__ void wait_copies() {  // lgkmcnt(0) and vmcnt(N)
  static_assert(N >= 0 && N < 64, "6-bit counter");
  __builtin_amdgcn_s_waitcnt(0x0070 | (N & 15) | ((N >> 4) << 14));
}

// 8 consecutive channels of a row: sums to values.  The order of the operations is the other kernel's, so that a row's result does not depend on
// which one it meets.
template <bool F32, bool GELU>
__device__ __forceinline__ void values8(const v4i& a0, const v4i& a1, float s, const float (&c)[8], const float (&b)[8], f4 (&y)[2]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    y[0][e] = __builtin_fmaf((float)a0[e] * s, c[e], b[e]);
    y[1][e] = __builtin_fmaf((float)a1[e] * s, c[4 + e], b[4 + e]);
  }
  if constexpr (GELU) {
    y[0] = gelu4<F32>(y[0]);
    y[1] = gelu4<F32>(y[1]);
  }
}

// The wavefront's 16 TN channels x 16 MT rows to Y.  Whole lines (see store_line_pair): fp16 pairs two batches of 32 channels, fp32 a batch's halves.
// p: 128 channel scales, 128 biases; rows: the wavefront's token scales.  CHECKED: some of it lies outside Y.
template <bool F32, bool GELU, bool CHECKED, int TN, int NX, int MT>
__device__ __forceinline__ void lines8(const Linear8Args& a, const v4i (&acc)[TN][NX], const float* p, const float* rows, int n_wave, int64_t m_wave, int lane, int mine) {
  asm volatile("" : "+v"(lane));  // (computed here, per tile: nothing lane-dependent is carried across the K loop)
  const int c = lane & 15, q = lane >> 4, up = c >> 3;
  constexpr int OB = F32 ? 4 : 2;
  const int64_t slab_bytes = (int64_t)16 * a.N * OB, half_bytes = (int64_t)8 * a.N * OB;
  global_u8* ywave = uniform_ptr((uint8_t*)a.Y + (m_wave * a.N + n_wave) * OB);
  const uint32_t row_off = (uint32_t)(c & 7) * (uint32_t)a.N * OB;
  auto constants = [&](int g, float (&c8)[8], float (&b8)[8]) {
    const int nl = (g >> 1) * kRowBlock + (g & 1) * 32 + q * 8;
#pragma unroll
    for (int j = 0; j < 8; j += 4) {
      const float4 cc = *(const float4*)(p + nl + j), bb = *(const float4*)(p + 128 + nl + j);
      c8[j] = cc.x; c8[j + 1] = cc.y; c8[j + 2] = cc.z; c8[j + 3] = cc.w;
      b8[j] = bb.x; b8[j + 1] = bb.y; b8[j + 2] = bb.z; b8[j + 3] = bb.w;
    }
  };
  float s[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) s[mt] = rows[16 * mt + c];
  if constexpr (F32) {
#pragma unroll
    for (int g = 0; g < TN / 2; ++g) {
      const int nb = (g >> 1) * kRowBlock + (g & 1) * 32 + q * 8 + up * 4;  // the 4 channels that this lane stores
      const bool n_ok = n_wave + nb < a.N;
      float c8[8], b8[8];
      constants(g, c8, b8);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        if (CHECKED && mt >= mine) break;
        f4 y[2];
        values8<true, GELU>(acc[2 * g][mt], acc[2 * g + 1][mt], s[mt], c8, b8, y);
        const int64_t row = m_wave + mt * 16 + (c & 7);
        store_line_pair(__builtin_bit_cast(ep_v4i, y[0]), __builtin_bit_cast(ep_v4i, y[1]), ywave + mt * slab_bytes, row_off + nb * 4, half_bytes,
                        !CHECKED || (n_ok && row < a.M), !CHECKED || (n_ok && row + 8 < a.M));
      }
    }
  } else {
#pragma unroll
    for (int gp = 0; gp < TN / 4; ++gp) {
      const bool n_ok = n_wave + gp * kRowBlock + up * 32 + q * 8 < a.N;
      float c8[2][8], b8[2][8];
      constants(2 * gp, c8[0], b8[0]);
      constants(2 * gp + 1, c8[1], b8[1]);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        if (CHECKED && mt >= mine) break;
        ep_v4i H[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          f4 y[2];
          values8<false, GELU>(acc[4 * gp + 2 * h][mt], acc[4 * gp + 2 * h + 1][mt], s[mt], c8[h], b8[h], y);
          H[h] = __builtin_bit_cast(ep_v4i, h8{(_Float16)y[0][0], (_Float16)y[0][1], (_Float16)y[0][2], (_Float16)y[0][3], (_Float16)y[1][0], (_Float16)y[1][1],
                                              (_Float16)y[1][2], (_Float16)y[1][3]});
        }
        const int64_t row = m_wave + mt * 16 + (c & 7);
        store_line_pair(H[0], H[1], ywave + mt * slab_bytes, row_off + gp * (kRowBlock * 2) + up * 64 + q * 16, half_bytes, !CHECKED || (n_ok && row < a.M),
                        !CHECKED || (n_ok && row + 8 < a.M));
      }
    }
  }
}

// fp16 output by batches of 32 channels, a lane's 8 channels of a row at a time: of wavefronts with one batch, or where N % 8 == 4 and rows begin at odd
// multiples of 8 bytes (halves then)
template <bool GELU, int TN, int NX>
__device__ __forceinline__ void batches8(const Linear8Args& a, const v4i (&acc)[TN][NX], const float* p, const float* rows, int n_wave, int64_t m_wave, int lane, int mine) {
  asm volatile("" : "+v"(lane));
  const int c = lane & 15, q = lane >> 4;
  const bool whole = (a.N & 7) == 0;
#pragma unroll
  for (int g = 0; g < TN / 2; ++g) {
    const int nl = (g >> 1) * kRowBlock + (g & 1) * 32 + q * 8;
    float c8[8], b8[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      c8[j] = p[nl + j];
      b8[j] = p[128 + nl + j];
    }
#pragma unroll
    for (int mt = 0; mt < NX; ++mt) {
      if (mt >= mine) break;
      const int64_t m = m_wave + 16 * mt + c;
      f4 y[2];
      values8<false, GELU>(acc[2 * g][mt], acc[2 * g + 1][mt], rows[16 * mt + c], c8, b8, y);
      const h8 h = {(_Float16)y[0][0], (_Float16)y[0][1], (_Float16)y[0][2], (_Float16)y[0][3], (_Float16)y[1][0], (_Float16)y[1][1], (_Float16)y[1][2], (_Float16)y[1][3]};
      _Float16* out = (_Float16*)a.Y + m * a.N + n_wave + nl;
      if (m >= a.M || n_wave + nl >= a.N) continue;
      if (whole) {
        *(h8*)out = h;
      } else {
        *(h4*)out = h4{h[0], h[1], h[2], h[3]};
        if (n_wave + nl + 4 < a.N) *(h4*)(out + 4) = h4{h[4], h[5], h[6], h[7]};
      }
    }
  }
}

// NX: slabs of 16 rows that a wavefront has at most
template <int TN, int NX, bool F32, bool GELU>
__global__ void __launch_bounds__(512, 1) linear8_tiles_kernel(const Linear8Args a, const Tokens8Plan plan) {
  typedef Ring8<TN, NX> R;
  constexpr bool LINES = F32 || TN > 2;  // whole lines of fp16 take 64 channels
  constexpr int kStores = (F32 ? TN : TN / 2) * (NX > 1 ? NX - 1 : 1);  // the fewest that a wavefront inside Y issues for a tile in lines
  __shared__ __attribute__((aligned(1024))) uint8_t ring[R::kStages * R::kStage];
  __shared__ __attribute__((aligned(1024))) float prm[2][2][256];     // by parity of the tile and half of its channels: 128 scales, 128 biases
  __shared__ __attribute__((aligned(1024))) float row_scales[2][256];  // by parity of the tile

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wn = wave & 1, wm = wave >> 1;
  const int ksteps = (a.K + 63) >> 6, tail = a.K & 63;  // bytes of a row of weights in its last step, 0: all
  const int place = (int)(blockIdx.x & 7) * plan.grid8 + (int)(blockIdx.x >> 3);
  const int my_items = plan.rounds + (place < plan.last_round ? 1 : 0);
  if (my_items == 0) return;  // the whole workgroup, in front of any barrier
  auto tile_of = [&](int i) { return tokens8_tile(plan, i * 8 * plan.grid8 + place); };
  const bool has_bias = (a.epilogue & GPUSQ_EPI_BIAS) != 0;
  if (!has_bias && wm == 0) {
#pragma unroll
    for (int par = 0; par < 2; ++par) {
      prm[par][wn][128 + lane] = 0.0f;
      prm[par][wn][192 + lane] = 0.0f;
    }
  }
  const uint32_t ring_lds = lds_address(ring), prm_lds = lds_address(prm[0][wn]), rows_lds = lds_address(row_scales[0]);
  // a tile's constants, asked for by the first wavefronts along m (its channels') and the second (its rows')
  auto request_constants = [&](int n0, int64_t m0, int parity) {
    int l = lane;
    asm volatile("" : "+v"(l));
    if (wm == 0) {
      const uint32_t dst = prm_lds + (uint32_t)parity * (uint32_t)sizeof(prm[0]);
#pragma unroll
      for (int i = 0; i < (TN + 3) / 4; ++i) {
        int n = n0 + wn * (16 * TN) + i * 64 + l;
        n = n < a.N ? n : a.N - 1;  // (channels past the end are not stored)
        copy4_to_lds(a.w_scale, (uint32_t)n * 4u, dst + (uint32_t)i * 256u);
        if (has_bias) copy4_to_lds(a.bias, (uint32_t)n * 4u, dst + 512u + (uint32_t)i * 256u);
      }
    } else if (wm == 1) {
      const uint32_t dst = rows_lds + (uint32_t)parity * (uint32_t)sizeof(row_scales[0]) + (uint32_t)wn * 512u;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int64_t m = m0 + wn * 128 + i * 64 + l;
        copy4_to_lds(a.x_scale, (uint32_t)(m < a.M ? m : a.M - 1) * 4u, dst + (uint32_t)i * 256u);
      }
    }
  };
  const uint32_t a_off = (uint32_t)(wn * TN * 1024 + (lane & 15) * 64 + (((lane >> 4) ^ ((lane & 15) >> 2)) * 16));

  // cursor of the copies: the next step to request, as (tile, step); at the end of the sequence it stays on the last step
  // (A copy's block is the wavefront's for the whole launch; its source is a base in scalar registers for a tile and a lane's offset that moves by
  // 64 a step, its place the stage's and the block's: four instructions a copy.)
  int pf_item = 0, pf_ks = 0;
  const uint8_t* pf_base[R::kCopies];
  uint32_t pf_off[R::kCopies];
  auto block_of = [&](int i) { return wave + 8 * i; };
  const bool all_copies = block_of(R::kCopies - 1) < R::kW + 2 * tokens8_units(plan);  // (no block that no tile has)
  auto clip_tail = [&]() {  // chunks of weights behind the end of a row
    if (tail != 0 && pf_ks + 1 == ksteps) {
      int l = lane;
      asm volatile("" : "+v"(l));
      const uint32_t at = (uint32_t)((l & 3) ^ (l >> 4)) * 16u, back = at >= (uint32_t)tail ? at : 0u;
#pragma unroll
      for (int i = 0; i < R::kCopies; ++i) pf_off[i] -= block_of(i) < R::kW ? back : 0u;
    }
  };
  auto seek = [&](int item) {
    pf_item = item;
    pf_ks = 0;
    const Tokens8Tile t = tile_of(item);
    int l = lane;
    asm volatile("" : "+v"(l));
    const int r = l >> 2, c = (l & 3) ^ (l >> 4), n0 = t.n_blk * (32 * TN);
    int64_t last = (int64_t)a.M - 1 - t.m0;
    last = last < 16 * t.slabs - 1 ? last : 16 * t.slabs - 1;  // a lower tile draws no rows that it does not use
#pragma unroll
    for (int i = 0; i < R::kCopies; ++i) {
      const int f = block_of(i);
      pf_base[i] = f < R::kW ? (const uint8_t*)a.W + (int64_t)n0 * a.K : (const uint8_t*)a.Xq + t.m0 * a.pitch;
      if (f < R::kW) {
        int ch = 64 * (f >> 2) + packed_row_to_channel(f & 3, r);
        ch = n0 + ch < a.N ? ch : a.N - 1 - n0;
        pf_off[i] = (uint32_t)ch * (uint32_t)a.K + c * 16;
      } else {
        const int64_t row = 16 * (f - R::kW) + r;
        pf_off[i] = (uint32_t)((row < last ? row : last) * a.pitch + c * 16);
      }
    }
    clip_tail();
  };
  auto advance = [&]() {
    if (pf_ks + 1 < ksteps) {
      ++pf_ks;
#pragma unroll
      for (int i = 0; i < R::kCopies; ++i) pf_off[i] += 64;
      clip_tail();
    } else if (pf_item + 1 < my_items) {
      seek(pf_item + 1);
    }
  };
  auto request_copy = [&](int i, uint32_t stage_lds) {
    if (i == R::kCopies - 1 && !all_copies) return;
    asm volatile("s_add_u32 m0, %0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3" ::"s"(stage_lds), "s"((uint32_t)block_of(i) * 1024u), "v"(pf_off[i]), "s"(pf_base[i])
                 : "memory", "m0", "scc");
  };

  v4i acc[TN][NX], b[NX], av[TN];
  {
    const Tokens8Tile t = tile_of(0);
    request_constants(t.n_blk * (32 * TN), t.m0, 0);
  }
  seek(0);
#pragma nounroll
  for (int g = 0; g < R::kStages; ++g) {
    const uint32_t stage = ring_lds + (uint32_t)g * R::kStage;
#pragma unroll
    for (int i = 0; i < R::kCopies; ++i) request_copy(i, stage);
    advance();
  }
  if (all_copies)  // the constants and step 0
    wait_copies<(R::kStages - 1) * R::kCopies>();
  else
    wait_copies<(R::kStages - 1) * (R::kCopies - 1)>();
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");

  int slot_off = 0;
  bool stores_behind = false;
#pragma nounroll
  for (int item = 0; item < my_items; ++item) {
    const Tokens8Tile t = tile_of(item);
    // this wavefront's slabs: a quarter of the tile's, the first t.slabs % 4 (0 or 2) wavefronts along m one more
    const int quarter = t.slabs >> 2, extra = t.slabs & 3;
    const int mine = quarter + (wm < extra ? 1 : 0), row0 = 16 * (wm * quarter + (wm < extra ? wm : extra));
    int l = lane;
    asm volatile("" : "+v"(l));
    const uint32_t b_off = (uint32_t)(R::kW * 1024 + row0 * 64 + (l & 15) * 64 + (((l >> 4) ^ ((l & 15) >> 2)) * 16));
    const bool more = item + 1 < my_items;
    const Tokens8Tile after = tile_of(more ? item + 1 : item);
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
      for (int j = 0; j < NX; ++j) acc[i][j] = v4i{0, 0, 0, 0};
    auto k_loop = [&](auto tma) {
      constexpr int TMA = decltype(tma)::value, F = TN / 2, H = F * TMA, kBarrierSlot = TMA > 2 && F > 1 ? H - 2 : H;
      constexpr int kBehind = (R::kStages - 2) * R::kCopies, kBehindLess = (R::kStages - 2) * (R::kCopies - 1);
#pragma unroll
      for (int f = 0; f < F; ++f) av[f] = *(const v4i*)(ring + slot_off + a_off + f * 1024);
#pragma unroll
      for (int mt = 0; mt + 1 < TMA; ++mt) b[mt] = *(const v4i*)(ring + slot_off + b_off + mt * 1024);
      // A step.  EDGE: of a tile's first, beside the output of the one before, or its last, from which on the copies are the next tile's.  Between them a
      // step has nothing to decide: a wavefront issues an instruction every five clocks or so, and sixty scalar ones a step took a quarter of its time.
      auto step = [&](auto edge, int ks) {
        constexpr bool EDGE = decltype(edge)::value;
        const int next_off = slot_off + R::kStage == R::kStages * R::kStage ? 0 : slot_off + R::kStage;
        const uint8_t *stage = ring + slot_off, *next = ring + next_off;
        const uint32_t stage_lds = ring_lds + (uint32_t)slot_off;
#pragma unroll
        for (int slot = 0; slot < 2 * H; ++slot) {
          const int mt = slot % H / F, f = slot % F + (slot < H ? 0 : F);
          if (slot == kBarrierSlot) {
            __builtin_amdgcn_sched_barrier(0);
            // (with fewer steps to a tile than stages the constants asked for in the last one's would not be waited for)
            if (EDGE && ksteps < R::kStages)
              wait_copies<0>();
            else if (EDGE && stores_behind && ks < R::kStages - 1)
              all_copies ? wait_copies<kBehind + kStores>() : wait_copies<kBehindLess + kStores>();
            else
              all_copies ? wait_copies<kBehind>() : wait_copies<kBehindLess>();
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            if (EDGE && ks + 1 == ksteps && more) request_constants(after.n_blk * (32 * TN), after.m0, (item + 1) & 1);
          }
          if (slot < H) {
            // (in front of the barrier, all of them)
            auto at = [&](int i) { return slot == (H >= 3 * F ? i : i * (H / F) / 4); };
            if (at(0)) b[TMA - 1] = *(const v4i*)(stage + b_off + (TMA - 1) * 1024);
#pragma unroll
            for (int j = 0; j < F; ++j)
              if (at(1 + j)) av[F + j] = *(const v4i*)(stage + a_off + (F + j) * 1024);
          } else {
            const int s = slot - H;
            if (s < F) av[s] = *(const v4i*)(next + a_off + s * 1024);
            // slab mt is free once its instructions of this half are issued
            if (s >= F && s % F == 0 && s / F - 1 < TMA - 1) b[s / F - 1] = *(const v4i*)(next + b_off + (s / F - 1) * 1024);
#pragma unroll
            for (int i = 0; i < R::kCopies; ++i)
              if (s == i * H / R::kCopies) request_copy(i, stage_lds);
          }
          __builtin_amdgcn_sched_barrier(0);
          acc[f][mt] = __builtin_amdgcn_mfma_i32_16x16x64_i8(av[f], b[mt], acc[f][mt], 0, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (EDGE) {
          advance();
        } else {
#pragma unroll
          for (int i = 0; i < R::kCopies; ++i) pf_off[i] += 64;
        }
        slot_off = next_off;
      };
      const int plain = ksteps - R::kStages - 2;  // up to here the cursor stays in front of the tile's last step
#pragma nounroll
      for (int ks = 0; ks < ksteps; ++ks) {
        if (ks == (stores_behind ? R::kStages - 1 : 0) && ks < plain) {
          pf_ks += plain - ks;
#pragma nounroll
          do step(std::false_type(), ks);
          while (++ks < plain);
        }
        step(std::true_type(), ks);
      }
    };
    if constexpr (NX > 1) {
      if (mine == NX)
        k_loop(std::integral_constant<int, NX>{});
      else
        k_loop(std::integral_constant<int, NX - 1>{});
    } else {
      k_loop(std::integral_constant<int, 1>{});
    }
    const int n_wave = t.n_blk * (32 * TN) + wn * (TN * 16);
    const int64_t m_wave = t.m0 + row0, rows = (int64_t)a.M - m_wave;
    const bool lines = F32 || (LINES && (a.N & 7) == 0), inside = lines && rows >= mine * 16 && a.N - n_wave >= TN * 16;
    const float *p = prm[item & 1][wn], *rs = row_scales[item & 1] + row0;
    if constexpr (LINES) {
      if (inside && mine == NX)
        lines8<F32, GELU, false, TN, NX, NX>(a, acc, p, rs, n_wave, m_wave, lane, NX);
      else if (inside && NX > 1)
        lines8<F32, GELU, false, TN, NX, (NX > 1 ? NX - 1 : 1)>(a, acc, p, rs, n_wave, m_wave, lane, NX - 1);
      else if (lines)
        lines8<F32, GELU, true, TN, NX, NX>(a, acc, p, rs, n_wave, m_wave, lane, mine);
    }
    if constexpr (!F32) {
      if (!lines) batches8<GELU, TN, NX>(a, acc, p, rs, n_wave, m_wave, lane, mine);
    }
    stores_behind = inside && mine > 0 && ksteps >= R::kStages;
  }
  wait_copies<0>();  // those asked for past the end of the sequence land before the LDS is given up
}

template <int TN, int NX>
void launch_nx(const Linear8Args& a, const Tokens8Plan& plan, hipStream_t s) {
  const bool gelu = (a.epilogue & GPUSQ_EPI_GELU) != 0;
  const unsigned grid = (unsigned)plan.grid8 * 8;
  if (a.out_f32)
    gelu ? linear8_tiles_kernel<TN, NX, true, true><<<grid, 512, 0, s>>>(a, plan) : linear8_tiles_kernel<TN, NX, true, false><<<grid, 512, 0, s>>>(a, plan);
  else
    gelu ? linear8_tiles_kernel<TN, NX, false, true><<<grid, 512, 0, s>>>(a, plan) : linear8_tiles_kernel<TN, NX, false, false><<<grid, 512, 0, s>>>(a, plan);
}

}  // namespace

template <int TN>
void launch_linear8_tiles_of(const Linear8Args& a, const Tokens8Plan& plan, hipStream_t s) {
  switch ((tokens8_units(plan) + 1) / 2) {
    case 1: return launch_nx<TN, 1>(a, plan, s);
    case 2: return launch_nx<TN, 2>(a, plan, s);
    case 3: return launch_nx<TN, 3>(a, plan, s);
    default: return launch_nx<TN, 4>(a, plan, s);
  }
}
}  // namespace gpusq
