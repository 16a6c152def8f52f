// Reads sizes of products (rows, channels, K), prints how each is cut into tiles on 256 CUs: blocks of 32 channels of a tile, most slabs of 16 rows of a
// wavefront, steps of 64 k, the most tiles of a workgroup.
#include <hip/hip_runtime.h>
#include <stdio.h>

#include "linear8_plan.h"

int main() {
  long long M, N, K;
  while (scanf("%lld %lld %lld", &M, &N, &K) == 3) {
    const gpusq::Tokens8Plan p = gpusq::tokens8_plan(M, N, K, 256);
    printf("%d %d %lld %d\n", p.tn, (gpusq::tokens8_units(p) + 1) / 2, (long long)gpusq::ceil_div(K, 64), p.rounds + (p.last_round > 0));
  }
}
