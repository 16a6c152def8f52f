// Reads trees (padded head, pairs of sequence and key head, columns of a pair), prints whether the kernel for many columns takes them.
#include <hip/hip_runtime.h>
#include <stdio.h>

#include "attend_plan.h"

int main() {
  long long DP, pairs, cols;
  while (scanf("%lld %lld %lld", &DP, &pairs, &cols) == 3) printf("%d\n", (int)gpusq::attend_shape(true, (int)DP, cols, true, pairs).many);
}
