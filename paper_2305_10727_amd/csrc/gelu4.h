// GELU of four sums of a lane, shared by the layers whose workgroup has few of them.
#pragma once
#include "kv4.h"

namespace gpusq {

// GELU of four values, x Phi(x) = max(x, 0) - t Phi(-t), t = |x|.  For fp32 output by erfc; for fp16 output Phi(-t) = 2^P(t), P of degree 9
// fitted to log2 Phi(-t) on 0 .. 6.5 (the result within 9e-8 of the exact one, and 2^-18 of it down to 2^-14; held at 9, where t Phi(-t) is 1e-18):
// a tenth of erfc's instructions, which one wavefront has for all of a tile.  (5120 -> 13824 for one row 11.4 us with erfc, 10.8 with this.)
template <bool F32>
__device__ __forceinline__ f4 gelu4(f4 x) {
  constexpr float P[10] = {-0.999999463558197f,    -1.1511276960372925f,    -0.459060937166214f,     -0.05285963416099548f,   0.007497080136090517f,
                           -0.000410962849855423f, -9.486963972449303e-05f, 2.5571362129994668e-05f, -2.5830624963418813e-06f, 1.011514996207552e-07f};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (F32) {
      x[e] = 0.5f * x[e] * erfcf(-0.70710678118654752f * x[e]);
    } else {
      const float t = fabsf(x[e]) > 9.0f ? 9.0f : fabsf(x[e]);  // (a NaN stays)
      float p = P[9];
#pragma unroll
      for (int i = 8; i >= 0; --i) p = __builtin_fmaf(p, t, P[i]);
      x[e] = __builtin_fmaf(-t, __builtin_amdgcn_exp2f(p), x[e] < 0.0f ? 0.0f : x[e]);
    }
  }
  return x;
}

}  // namespace gpusq
