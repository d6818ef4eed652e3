// What the kernels of the selective state space scan share.
#pragma once

#include "kata_common.cuh"

namespace kata {

// s_t: the step size of a token from its raw entry.
__device__ __forceinline__ float ssm_step_size(const Ssm& a, float dt, int h) {
  if (a.dt_bias != nullptr) dt += a.dt_bias[h];
  // log(1 + e^x); beyond 20 the difference to x is below 2^-28
  return !a.softplus || dt > 20.f ? dt : log1pf(expf(dt));
}

// Place of slot j of a head in the scratch of the token by token kernel.
__host__ __device__ inline size_t ssm_slot(int segments, int bh, int j) { return (size_t)bh * segments + j; }

}  // namespace kata
