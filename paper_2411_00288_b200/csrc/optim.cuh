// What the calls over many tensors (optim.cu) and their argument checks share.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace ssconv {

struct AdamwParams {
  float lr, beta1, one_minus_beta1, beta2, one_minus_beta2, eps, weight_decay, c1, c2;
};

size_t grad_norm_scratch(int tensors);
cudaError_t launch_grad_norm(const void* const* g, const int64_t* n, const int32_t* type, int tensors, bool inf, float* norm, double* partial,
                             cudaStream_t st);
cudaError_t launch_clip_grads(const void* const* g, void* const* out, const int64_t* n, const int32_t* type, int tensors, const float* norm,
                              float max_norm, cudaStream_t st);
cudaError_t launch_adamw_multi(void* const* theta, const void* const* g, void* const* m, void* const* v, const int64_t* n, const int32_t* type,
                               int tensors, const AdamwParams& a, const float* norm, float max_norm, cudaStream_t st);

}  // namespace ssconv
