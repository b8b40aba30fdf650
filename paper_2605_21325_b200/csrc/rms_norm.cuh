// Root-mean-square norm: arguments and launchers (rms_norm_kernel.cu).
#pragma once
#include "common.cuh"

namespace tri_inv {

constexpr int kRmsNormPartials = 592;   // rows of partial sums of dw, at most: the blocks of the gradient's kernel, four for each of 148 SMs

struct RmsNormArgs {
  const void *X, *R, *w;   // R: residual or null
  void *Y, *H;             // H: where X + R goes, or null
  float* scales;           // with an output in 8 bits
  long long rows;
  int n;
  float eps;
};
struct RmsNormBackwardArgs {
  const void *dY, *X, *w, *dH;   // dH: what reaches X past the norm, or null
  void *dX, *dw;
  float* partial;                // [kRmsNormPartials][n]
  long long rows;
  int n;
  float eps;
};
// out: 0 the storage type, 1 e4m3 with a scale for each 128 columns, 2 e4m3 with a scale for the row
cudaError_t launch_rms_norm(const RmsNormArgs& a, int dtype, int out, cudaStream_t stream);
cudaError_t launch_rms_norm_backward(const RmsNormBackwardArgs& a, int dtype, cudaStream_t stream);

}  // namespace tri_inv
