// Sums of losses, for the criteria on arrays of logits.
#pragma once
#include "rows.h"

namespace rnnlm_dev {

// Sum of n losses in 64 bits, in a fixed order, by one workgroup.
static __global__ void __launch_bounds__(1024) sum_losses_kernel(const float *__restrict__ loss, long n, double *__restrict__ out) {
  __shared__ double sh[16];
  double a = 0.0;
  for (long i = threadIdx.x; i < n; i += 1024) a += (double)loss[i];
  a = wave_sum(a);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = a;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < 16; ++i) a += sh[i];
    *out = a;
  }
}

}  // namespace rnnlm_dev
