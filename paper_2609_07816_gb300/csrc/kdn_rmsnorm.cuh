// kdn_rmsnorm.cuh -- internal arguments of the residual RMS norm (kdn_rmsnorm.cu).
#pragma once

#include "kdn_internal.cuh"

namespace kdn {

struct NormArgs {
  long long rows;
  int D, dtype, f8, block;
  float eps;
  const void *x, *res, *w;
  void *y, *h;
  float *rstd, *scales;
  // backward
  const void *hin, *dy, *dh;
  const float *rstd_in;
  void *dx;
  float *dw, *part;
};

int rmsnorm_bwd_blocks(long long rows, int D);
kdn_status_t launch_add_rmsnorm(const NormArgs &a, cudaStream_t s);
kdn_status_t launch_add_rmsnorm_bwd(const NormArgs &a, cudaStream_t s);

}  // namespace kdn
