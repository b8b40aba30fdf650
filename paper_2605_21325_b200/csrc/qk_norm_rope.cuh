// Norm of each query and key head with the position rotation: arguments and launchers (qk_norm_rope_kernel.cu).
#pragma once
#include "common.cuh"

namespace tri_inv {

constexpr int kHeadsMaxDim = 256;        // features of a head, at most
constexpr int kHeadsPartials = 592;      // rows of partial sums of the weights' gradients, at most: the blocks of the gradient's kernel

// Queries or keys
struct HeadsSide {
  const void *x, *w, *dy;                // w: null for ones; dy: gradient only
  void *y, *dx, *dw;
  long long ld_x, ld_dy, ld_y, ld_dx;    // values from one token to the next
  int H;
};
struct HeadsArgs {
  HeadsSide side[2];
  const float* inv_freq;                 // [r]
  const int32_t* positions;              // [tokens] or null: a token's place among T
  float* partial;                        // gradient: [kHeadsPartials][d]
  long long tokens;
  int T, d, r, interleaved;
  int units;                             // pairs of vectors of a head (set by the launcher)
  float eps;
};
cudaError_t launch_qk_norm_rope(const HeadsArgs& a, int dtype, cudaStream_t stream);
cudaError_t launch_qk_norm_rope_backward(const HeadsArgs& a, int dtype, cudaStream_t stream);

}  // namespace tri_inv
