// What the residual-and-norm calls (resnorm.cu) and their argument checks share.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "ssconv.h"

namespace ssconv {

constexpr int kResnormMostC = 8192;

struct ResnormTensors {  // of a forward call
  const void *x, *b;
  const float *gate, *post_gamma, *post_beta, *pre_gamma, *pre_beta;
  void *h, *y;
  float* stats;
};
struct ResnormGradients {  // of a backward call, beside its inputs
  const void *dh, *dy;
  void *dx, *db;
  float *dgate, *dpost_gamma, *dpost_beta, *dpre_gamma, *dpre_beta;
};

cudaError_t launch_resnorm(const ssconv_resnorm_t& d, const ResnormTensors& t, cudaStream_t st);
size_t resnorm_scratch(const ssconv_resnorm_t& d);
cudaError_t launch_resnorm_backward(const ssconv_resnorm_t& d, const ResnormTensors& t, const ResnormGradients& g, float* ws, cudaStream_t st);

}  // namespace ssconv
