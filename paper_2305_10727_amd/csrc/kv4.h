// The 4-bit formats of the decoder's operators: codes of 4 bits with a scale for a group of values, in places that the matrix
// instructions' operands are read from as they lie.
#pragma once
#include "common.h"

namespace gpusq {

typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef unsigned u2 __attribute__((ext_vector_type(2)));
typedef unsigned u4 __attribute__((ext_vector_type(4)));

// ---- 4-bit layers ---------------------------------------------------------------------------------------------------------------
// Steps of 128 k that a workgroup takes at once, at most.  All but one of them may lie behind the end of K, and are found to by comparing their k with
// it in 31 bits: so K is kMostLinear4K at most.
constexpr int kLinear4Steps = 64, kMostLinear4K = INT32_MAX - kLinear4Steps * 128;

// ---- the cache ------------------------------------------------------------------------------------------------------------------
// A page holds 64 tokens of one head, DP = the head's channels padded to 64, 128 or 256:
//   key codes     [64 tokens][4 g][DP / 32 j] words: channels 32 j + 8 g + 0..7, the even ones in the lower half of the word.  Lane
//                 16 g + r of a wavefront reads one vector of token r: the rows of the 16 x 16 x 32 instruction's first operand.
//   key scales    [64 tokens][DP / 32 groups] fp16
//   value codes   [16 quads of tokens][16 n][2 pairs][DP / 64][2 tokens] of 16 bits: four channels of one token, channels (DP / 16) n + ...
//                 Lane 16 g + n reads one vector of quad g: both halves of a word are the same channels of two tokens, next to each
//                 other in the sum that the second product takes.
//   value scales  [DP / 32 groups][64 tokens] fp16
// A token touches whole 16-bit places (value codes) and bytes (key codes) only: tokens can be written side by side.
constexpr int kPageTokens = 64, kGroupChannels = 32;
__host__ __device__ constexpr int padded_head(int D) { return D <= 64 ? 64 : D <= 128 ? 128 : 256; }
__host__ __device__ constexpr int page_bytes(int DP) { return 72 * DP; }
__host__ __device__ constexpr int key_scales_at(int DP) { return 32 * DP; }
__host__ __device__ constexpr int value_codes_at(int DP) { return 36 * DP; }
__host__ __device__ constexpr int value_scales_at(int DP) { return 68 * DP; }

// The scale of a group: max|x| / 7 with 7 significant bits, half to even, in 2^-24 .. 896; 1 where that rounds to 0 in fp16.  A code
// has 3 bits besides its sign, so code times scale is an fp16 number: what the cache stands for meets the matrix instructions unrounded.
// (A step that is up to 1/128 longer or shorter, beside codes that are half a step off.)  896: 72 times it is still an fp16 number, see
// codes_to_halves.
__device__ __forceinline__ float group_scale(float amax) {
  unsigned u = __float_as_uint(__fdiv_rn(amax, 7.0f));
  u += 0xFFFFu + ((u >> 17) & 1u);
  const float s = (float)(_Float16)fminf(__uint_as_float(u & 0xFFFE0000u), 896.0f);
  return s == 0.0f ? 1.0f : s;
}

// The eight codes of a word (code + 8 in 4 bits) as products with the scale: pair p is nibble p of the lower half and of the upper one.
// A nibble in bits 4..7 of 0x5400 is 64 + nibble; (64 + nibble) s - 72 s is the exact product, 72 s having 11 significant bits at most.
// 11 instructions for 8 values.
// (One instruction, its constants in registers: with two literal constants the compiler makes two.)
__device__ __forceinline__ unsigned nibbles_at_4(unsigned w) {
  unsigned mask = 0x00f000f0u, base = 0x54005400u, d;
  asm("v_and_or_b32 %0, %1, %2, %3" : "=v"(d) : "v"(w), "s"(mask), "v"(base));
  return d;
}
__device__ __forceinline__ void codes_to_halves(unsigned w, h2 s, h2 m72s, h2 (&out)[4]) {
  out[0] = __builtin_elementwise_fma(__builtin_bit_cast(h2, nibbles_at_4(w << 4)), s, m72s);
  out[1] = __builtin_elementwise_fma(__builtin_bit_cast(h2, nibbles_at_4(w)), s, m72s);
  out[2] = __builtin_elementwise_fma(__builtin_bit_cast(h2, nibbles_at_4(w >> 4)), s, m72s);
  out[3] = __builtin_elementwise_fma(__builtin_bit_cast(h2, nibbles_at_4(w >> 8)), s, m72s);
}
// ... as they are, -8 .. 7
__device__ __forceinline__ void codes_to_halves(unsigned w, h2 (&out)[4]) {
  const h2 m72 = {(_Float16)-72.0f, (_Float16)-72.0f};
  out[0] = __builtin_bit_cast(h2, nibbles_at_4(w << 4)) + m72;
  out[1] = __builtin_bit_cast(h2, nibbles_at_4(w)) + m72;
  out[2] = __builtin_bit_cast(h2, nibbles_at_4(w >> 4)) + m72;
  out[3] = __builtin_bit_cast(h2, nibbles_at_4(w >> 8)) + m72;
}

// N words, in vectors of up to four
template <int N>
struct WordsOf {
  typedef unsigned type __attribute__((ext_vector_type(N)));
};
template <int N>
__device__ __forceinline__ typename WordsOf<N>::type load_words(const uint8_t* p) {
  if constexpr (N == 8) {
    const u4 a = *(const u4*)p, b = *(const u4*)(p + 16);
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  } else if constexpr (N == 1) {
    return *(const unsigned*)p;
  } else {
    return *(const typename WordsOf<N>::type*)p;
  }
}

// Scales of four tokens as two pairs; those of tokens from `left` on are 0 (places behind the last token may hold anything: a scale of
// theirs may be infinite or NaN, and 0 times it too).
__device__ __forceinline__ u2 scales_in_front(u2 s, int left) {
  return u2{s[0] & (left > 1 ? 0xFFFFFFFFu : left > 0 ? 0xFFFFu : 0u), s[1] & (left > 3 ? 0xFFFFFFFFu : left > 2 ? 0xFFFFu : 0u)};
}

// v_mfma_f32_16x16x32_f16: lane 16 g + r has row (column) r and k = 8 g .. + 7 of the operands, column r and rows 4 g .. + 3 of the result
__device__ __forceinline__ f4 mfma16(h8 a, h8 b, f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

}  // namespace gpusq
