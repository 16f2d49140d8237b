// Declarations of the norm's kernels (rms_norm.hip).
#pragma once

#include "isa_internal.h"

namespace isa {

// What the kernels get of an isa_norm_problem; strides in elements (of y8: bytes).
struct NormArgs {
  const void *x, *residual, *weight;
  void *h, *y;                              // backward: y = dx
  float* rstd;                              // backward: read
  float* scales;
  const void *dy, *dh;
  float* partial;                           // backward: [workgroups][channels], null without a weight's gradient
  long long rows;
  int C, group;
  int w_f32;                                // the weight's type
  float eps;
  // Elements are squared times square_scale, a power of two near 1 / sqrt(C), and mean(h^2) = sum_scale times the sum: it then
  // overflows only where the mean does, and nothing is rounded that would not be without
  float square_scale, sum_scale;
  long long sx, sr, sh, sy, sdy, sdh;
};

bool norm_streams(const NormArgs& a, int dtype, bool eight);  // whether rows go past the caches; looks at the pointers that are set and the sizes
int norm_backward_workgroups(const isa_norm_problem* p);     // rows of `partial`
hipError_t launch_rms_norm(const NormArgs& a, int dtype, bool eight, hipStream_t st);
hipError_t launch_rms_norm_backward(const NormArgs& a, int dtype, int wgs, void* d_weight, hipStream_t st);

}  // namespace isa
