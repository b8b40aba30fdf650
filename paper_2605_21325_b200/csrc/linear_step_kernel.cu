// Linear attention with a decay for each head: one token for each of B rows, on states that lie in the slots of a cache.
//     S <- lambda S + k v^T,     o = scale S^T q          (S of slot slots[b], updated in place)
//
// One CTA per (row, head, 4 LANES value columns): a lane has four columns, a group of LANES lanes a run of features, so that the state streams
// through registers once, in rows of 16 LANES bytes, all of a thread's loads in flight before the first is used.  What bounds it: the bytes of
// the state, read once and written once; with few rows the latency of one load, one exchange and one store.  256 rows x 32 heads of 128 x 128 (9 of them padding): 163 us, 6.4 TB/s, 0.98 of a copy's rate; 8 rows x 16
// heads 4.2 us on the device.
// A slot that an earlier row of the call has, or one past the cache, is an error of the caller's that only the device can see: the row's output is zero,
// its state is left alone and the status word says TRI_INV_ERR_INVALID_ARG.
#include "linear_attention.cuh"

namespace tri_inv {
namespace {

constexpr int kThreadsStep = 256;

template <int LANES, int R>   // R: features of a thread, at most
__global__ void __launch_bounds__(kThreadsStep) linear_step_kernel(const __grid_constant__ LinStepArgs a) {
  constexpr int GROUPS = kThreadsStep / LANES;
  __shared__ float sk[GROUPS * R], sq[GROUPS * R];
  __shared__ float4 part[kThreadsStep / 32][LANES];
  const int tid = threadIdx.x, lane = tid % LANES, group = tid / LANES;
  const int blocks = (a.d_v + 4 * LANES - 1) / (4 * LANES);
  int x = blockIdx.x;
  const int c = (x % blocks) * 4 * LANES + 4 * lane; x /= blocks;
  const int h = x % a.H, row = x / a.H;
  const size_t at = (size_t)row * a.H + h;
  wait_for_predecessor();
  const int slot = a.slots ? a.slots[row] : row;
  const bool in = c < a.d_v;
  bool use = slot >= 0 && slot < a.n_slots;
  float4* S = reinterpret_cast<float4*>(a.S + ((size_t)(use ? slot : 0) * a.H + h) * a.d_k * a.d_v);
  const int ld = a.d_v / 4, rows = a.d_k / GROUPS + (group < a.d_k % GROUPS ? 1 : 0);   // the group's features: group, group + GROUPS, ...
  float4 s[R];
#pragma unroll
  for (int r = 0; r < R; ++r)
    if (use && in && r < rows) s[r] = S[(size_t)(group + r * GROUPS) * ld + c / 4];
  for (int d = tid; d < a.d_k; d += kThreadsStep) {
    sk[d] = load_kv(a.k, a.bf16 ? TRI_INV_BF16 : TRI_INV_F32, at * a.d_k + d);
    sq[d] = load_kv(a.q, a.bf16 ? TRI_INV_BF16 : TRI_INV_F32, at * a.d_k + d);
  }
  float v[4] = {0.f, 0.f, 0.f, 0.f};
  if (in)
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = load_kv(a.v, a.bf16 ? TRI_INV_BF16 : TRI_INV_F32, at * a.d_v + c + i);
  bool twice = false;
  if (a.slots)
    for (int b = tid; b < row; b += kThreadsStep) twice = twice || a.slots[b] == slot;
  const float lambda = expf(a.log_decay[h]);
  const bool bad = __syncthreads_or(twice && use) || slot >= a.n_slots;
  if (bad) {
    use = false;
    if (tid == 0) atomicMax(a.status, (int)TRI_INV_ERR_INVALID_ARG);
  }
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  if (use && in) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (r < rows) {
        const float k = sk[group + r * GROUPS], q = sq[group + r * GROUPS];
        s[r].x = fmaf(k, v[0], lambda * s[r].x); s[r].y = fmaf(k, v[1], lambda * s[r].y);
        s[r].z = fmaf(k, v[2], lambda * s[r].z); s[r].w = fmaf(k, v[3], lambda * s[r].w);
        o.x = fmaf(q, s[r].x, o.x); o.y = fmaf(q, s[r].y, o.y); o.z = fmaf(q, s[r].z, o.z); o.w = fmaf(q, s[r].w, o.w);
        S[(size_t)(group + r * GROUPS) * ld + c / 4] = s[r];
      }
    }
  }
#pragma unroll
  for (int m = LANES; m < 32; m <<= 1) {
    o.x += __shfl_xor_sync(0xffffffffu, o.x, m); o.y += __shfl_xor_sync(0xffffffffu, o.y, m);
    o.z += __shfl_xor_sync(0xffffffffu, o.z, m); o.w += __shfl_xor_sync(0xffffffffu, o.w, m);
  }
  if ((tid & 31) < LANES) part[tid >> 5][lane] = o;
  __syncthreads();
  if (tid < 4 * LANES) {
    const int col = (c - 4 * lane) + tid;
    if (col < a.d_v) {
      float y = 0.f;
#pragma unroll
      for (int w = 0; w < kThreadsStep / 32; ++w) y += reinterpret_cast<const float*>(part[w])[tid];
      y *= a.scale;
      if (a.bf16) ((__nv_bfloat16*)a.o)[at * a.d_v + col] = __float2bfloat16_rn(y);
      else ((float*)a.o)[at * a.d_v + col] = y;
    }
  }
}

template <int LANES, int R>
cudaError_t launch_one(const LinStepArgs& a, cudaStream_t stream) {
  const long long grid = (long long)a.B * a.H * ((a.d_v + 4 * LANES - 1) / (4 * LANES));
  if (grid > 0x7fffffffLL) return cudaErrorInvalidValue;
  const cudaError_t e = launch_early(linear_step_kernel<LANES, R>, dim3((unsigned)grid), kThreadsStep, 0, stream, a);
  return e == cudaSuccess ? launched() : e;
}

}  // namespace

cudaError_t launch_linear_step(const LinStepArgs& a, cudaStream_t stream) {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return cudaErrorUnknown;
  const long long pairs = (long long)a.B * a.H;
  if (pairs * ((a.d_v + 127) / 128) < 2 * sms) return a.d_k <= 128 ? launch_one<8, 4>(a, stream) : launch_one<8, 8>(a, stream);
  if (a.d_v % 128 != 0 || a.d_k > 128) return a.d_k <= 128 ? launch_one<16, 8>(a, stream) : launch_one<16, 16>(a, stream);
  return launch_one<32, 16>(a, stream);
}

}  // namespace tri_inv
