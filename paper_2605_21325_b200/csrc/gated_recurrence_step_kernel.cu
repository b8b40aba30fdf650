// Gated linear recurrence: one token for each of B rows, on states that lie in the slots of a cache.
//     h <- a h + u,   y = h          (h of slot slots[b], updated in place)
// A thread has two neighbouring channels of a row.  What bounds it: for many rows the bytes (256 x 4096 bf16, inputs in the L2 cache, 5 us a call, which is its host side), for few the latency of the slot, one load and one store (1.6 us on the device).
// A slot that an earlier row of the call has, or one past the cache, is an error of the caller's that only the device can see: the row's output is zero, its state is left alone and the
// status word says TRI_INV_ERR_INVALID_ARG.
#include "gated_recurrence.cuh"

namespace tri_inv {
namespace {

constexpr int kThreads = 128;

template <class T, int MODE>
__global__ void __launch_bounds__(kThreads) gated_recurrence_step_kernel(const __grid_constant__ RecStepArgs a) {
  const int tid = threadIdx.x, blocks = (a.D + 2 * kThreads - 1) / (2 * kThreads), row = blockIdx.x / blocks, c = ((blockIdx.x - row * blocks) * kThreads + tid) * 2;
  wait_for_predecessor();
  const int slot = a.slots ? a.slots[row] : row;
  bool use = slot >= 0 && slot < a.n_slots;
  float* h = a.h + (long long)(use ? slot : 0) * a.D;
  const Pair x = RecLane<T>::widen(rec_load((const T*)a.x + row * a.ld_x, c, a.D, rec_access<T>(a.x, a.ld_x)));
  const Pair g = RecLane<T>::widen(rec_load((const T*)a.g + row * a.ld_g, c, a.D, rec_access<T>(a.g, a.ld_g)));
  const int h_access = rec_access<float>(a.h, a.D);
  Pair s = use ? RecLane<float>::widen(rec_load(h, c, a.D, h_access)) : twice(0.f);
  bool again = false;
  if (a.slots && use)
    for (int b = tid; b < row; b += kThreads) again = again || a.slots[b] == slot;
  if (__syncthreads_or(again) || slot >= a.n_slots) {
    use = false;
    if (tid == 0) atomicMax(a.status, (int)TRI_INV_ERR_INVALID_ARG);
  }
  Pair am, m;
  rec_factors<MODE>(g, am, m);
  s = use ? rec_step(am, s, rec_input<MODE>(m, x)) : twice(0.f);
  if (use) rec_store(h, c, a.D, h_access, s);
  rec_store((T*)a.y + row * a.ld_y, c, a.D, rec_access<T>(a.y, a.ld_y), s);
}

template <class T, int MODE>
cudaError_t launch_one(const RecStepArgs& a, cudaStream_t stream) {
  constexpr int per = 2 * kThreads;
  const long long grid = (long long)a.B * (((long long)a.D + per - 1) / per);
  if (grid > 0x7fffffffLL) return cudaErrorInvalidValue;
  const cudaError_t e = launch_early(gated_recurrence_step_kernel<T, MODE>, dim3((unsigned)grid), kThreads, 0, stream, a);
  return e == cudaSuccess ? launched() : e;
}
template <class T>
cudaError_t launch_type(const RecStepArgs& a, cudaStream_t stream) {
  return a.mode == kRecDecay ? launch_one<T, kRecDecay>(a, stream) : a.mode == kRecNormed ? launch_one<T, kRecNormed>(a, stream) : launch_one<T, kRecGate>(a, stream);
}

}  // namespace

cudaError_t launch_gated_recurrence_step(const RecStepArgs& a, int dtype, cudaStream_t stream) {
  return dtype == TRI_INV_F32 ? launch_type<float>(a, stream) : launch_type<__nv_bfloat16>(a, stream);
}

}  // namespace tri_inv
