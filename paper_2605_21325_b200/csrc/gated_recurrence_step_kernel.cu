// Gated linear recurrence: one token for each of B rows, on states that lie in the slots of a cache.
//     h <- a h + u,   y = h          (h of slot slots[b], updated in place)
// A thread has two neighbouring channels of a row (one in fp32).
// A slot that an earlier row of the call has, or one past the cache, is an error of the caller's that only the device can see: the row's output is zero, its state is left alone and the
// status word says TRI_INV_ERR_INVALID_ARG.
#include "gated_recurrence.cuh"

namespace tri_inv {
namespace {

constexpr int kThreads = 128;

template <class T, int MODE>
__global__ void __launch_bounds__(kThreads) gated_recurrence_step_kernel(const __grid_constant__ RecStepArgs a) {
  constexpr int N = RecLane<T>::N;
  const int tid = threadIdx.x, blocks = (a.D + kThreads * N - 1) / (kThreads * N), row = blockIdx.x / blocks, c = ((blockIdx.x - row * blocks) * kThreads + tid) * N;
  const T *X = (const T*)a.x + row * a.ld_x, *G = (const T*)a.g + row * a.ld_g;
  T* Y = (T*)a.y + row * a.ld_y;
  wait_for_predecessor();
  const int slot = a.slots ? a.slots[row] : row;
  bool use = slot >= 0 && slot < a.n_slots;
  float* h = a.h + (long long)(use ? slot : 0) * a.D;
  float x[N], g[N], s[N];
  RecLane<T>::widen(x, rec_load(X, c, a.D, rec_access<T>(a.x, a.ld_x) != kRecSingle));
  RecLane<T>::widen(g, rec_load(G, c, a.D, rec_access<T>(a.g, a.ld_g) != kRecSingle));
#pragma unroll
  for (int j = 0; j < N; ++j) s[j] = use && c + j < a.D ? h[c + j] : 0.f;
  bool twice = false;
  if (a.slots && use)
    for (int b = tid; b < row; b += kThreads) twice = twice || a.slots[b] == slot;
  if (__syncthreads_or(twice) || slot >= a.n_slots) {
    use = false;
    if (tid == 0) atomicMax(a.status, (int)TRI_INV_ERR_INVALID_ARG);
  }
#pragma unroll
  for (int j = 0; j < N; ++j) {
    float am, m, over;
    rec_factors<MODE>(g[j], am, m, over);
    s[j] = use ? rec_step(am, s[j], m * x[j]) : 0.f;
    if (use && c + j < a.D) h[c + j] = s[j];
  }
  rec_store(Y, c, a.D, rec_access<T>(a.y, a.ld_y) != kRecSingle, s);
}

template <class T, int MODE>
cudaError_t launch_one(const RecStepArgs& a, cudaStream_t stream) {
  constexpr int per = kThreads * RecLane<T>::N;
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
