// What the kernels of the selective state space scan share.
#pragma once

#include "kata_common.cuh"

namespace kata {

// log(1 + e^x) to a few units in the last place: max(x, 0) + log1p(e^-|x|), log1p(u) = 2 atanh(z) with z = u / (2 + u) <= 1/3, whose
// series in z^2 is cut behind z^17 (2e-9 of itself).
__device__ __forceinline__ float softplus(float x) {
  const float u = expf(-fabsf(x)), z = __fdividef(u, 2.f + u), y = z * z;
  float p = 1.f / 17.f;
  p = fmaf(p, y, 1.f / 15.f);
  p = fmaf(p, y, 1.f / 13.f);
  p = fmaf(p, y, 1.f / 11.f);
  p = fmaf(p, y, 1.f / 9.f);
  p = fmaf(p, y, 1.f / 7.f);
  p = fmaf(p, y, 1.f / 5.f);
  p = fmaf(p, y, 1.f / 3.f);
  p = fmaf(p, y, 1.f);
  return fmaf(2.f * z, p, x > 0.f ? x : (x <= 0.f ? 0.f : x));      // (the last: NaN)
}

// s_t: the step size of a token from its raw entry.
__device__ __forceinline__ float ssm_step_size(const Ssm& a, float dt, int h) {
  if (a.dt_bias != nullptr) dt += a.dt_bias[h];
  return a.softplus ? softplus(dt) : dt;
}

// Place of slot j of a head in the scratch of the token by token kernel.
__host__ __device__ inline size_t ssm_slot(int segments, int bh, int j) { return (size_t)bh * segments + j; }

}  // namespace kata
