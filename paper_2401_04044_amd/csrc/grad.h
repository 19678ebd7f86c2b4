// Internal: launchers of the gradient kernels (grad.hip).
#pragma once
#include "common.h"

namespace ffsplit {

// dx = [residual +] the gradient of x behind n(x) = x / sqrt(mean(x^2) + eps) whose gradient is dn;
// dx_cast (may be null): the same in the storage type
int launch_rmsnorm_backward(const float* x, const void* dn, int64_t T, int d, float eps, int bf16, const float* residual,
                            float* dx, void* dx_cast, hipStream_t st);
// n elements (a multiple of 8) of an fp32 stream, in bf16 or as they are
int launch_cast(const float* src, int64_t n, int bf16, void* dst, hipStream_t st);

// The tensors of a norm: listed one by one, or the matrices of a stack (tensor i is mats[i % n_mats][i / n_mats],
// `count` elements each; in place).
struct GradSet {
  int n;
  const void* const* src;
  void* const* dst;
  const int64_t* counts;
  const int32_t* dtypes;
  int n_mats;   // 0: listed
  void* const* mats[3];
  int64_t count;
  int f32;
};
size_t grad_norm_ws_bytes(int64_t n_tensors);
int launch_grad_norm(const GradSet& g, float* norm, int32_t* nonfinite, double* ws, hipStream_t st);
int launch_grad_clip(const GradSet& g, const float* norm, float max_norm, hipStream_t st);

}  // namespace ffsplit
