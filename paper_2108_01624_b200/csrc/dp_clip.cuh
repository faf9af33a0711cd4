// The factor of a clip by the global norm, shared by the list kernels and the AdamW step.
#pragma once

namespace dpk {

// min(1, max_norm / sqrt(sqsum)), 1 where sqsum = 0.  The sum of squares is fp64 and so is this, rounded once: a norm
// beyond fp32's range still gives the right factor, as far as fp32 holds it (below 2^-126 it loses bits).  An infinite norm
// gives 0, NaN gives NaN (x > 1 is false for it).
__device__ __forceinline__ float clip_factor(double sqsum, double max_norm, float* norm_out = nullptr) {
  const double norm = sqrt(sqsum);
  if (norm_out) *norm_out = (float)norm;
  if (norm == 0.0) return 1.0f;
  const double f = max_norm / norm;
  return f > 1.0 ? 1.0f : (float)f;
}

}  // namespace dpk
