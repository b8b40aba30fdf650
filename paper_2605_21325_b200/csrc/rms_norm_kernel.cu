// Root-mean-square norm over rows of n values, with the residual's addition in front and an output in 8 bits behind, and its gradient.
//     h = x + r,    y = h w / sqrt(mean h^2 + eps)
//     y in the storage type, or per group of columns: scale = max |y| / 448 (1 where that is 0), y / scale rounded to e4m3
//     u = dy w,     dx = rstd (u - h rstd^2 mean(u h)) + dh,     dw = sum over rows of dy h rstd                rstd = 1 / sqrt(mean h^2 + eps)
// Sums, h (before it is stored), y (before it is rounded) and dw's sums over rows are fp32.
//
// A row is held in the registers of TPR threads, NV vectors of 16 bytes each: every value is read once and written once, which bounds the large calls; a
// call of a few rows is the latency of one load, one exchange and one store, and takes more threads a row.  Rows that are not whole vectors, or are too
// long, take a kernel that reads them twice.
#include <algorithm>

#include "common.cuh"
#include "rms_norm.cuh"

namespace tri_inv {
namespace {

constexpr int kGroup = 128;         // columns that share a scale
constexpr float kMaxE4m3 = 448.f;

__device__ __forceinline__ float up(float x) { return x; }
__device__ __forceinline__ float up(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

// 16 bytes of values
template <class T> struct Vec;
template <> struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void load(float (&v)[4], const float* p) {
    const float4 x = *reinterpret_cast<const float4*>(p);
    v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
  }
  static __device__ __forceinline__ void store(float* p, const float (&v)[4]) { *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]); }
};
template <> struct Vec<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void load(float (&v)[8], const __nv_bfloat16* p) {
    const uint4 x = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
  }
  static __device__ __forceinline__ void store(__nv_bfloat16* p, const float (&v)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 x = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&x);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  }
};
__device__ __forceinline__ uint32_t pack_e4m3(float lo, float hi) {   // two codes, rounded to nearest even
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}

// The sum (or maximum) of a row over its TPR threads; the block's rows each have sync-free shuffles (TPR = 32) or shared words of their own.
template <int TPR, int K, bool MAX = false>
__device__ __forceinline__ void row_reduce(float (&x)[K], float (*words)[32], int tid) {
#pragma unroll
  for (int m = 16; m >= 1; m >>= 1)
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const float o = __shfl_xor_sync(0xffffffffu, x[k], m);
      x[k] = MAX ? fmaxf(x[k], o) : x[k] + o;
    }
  if constexpr (TPR > 32) {
    constexpr int W = TPR / 32;
    const int warp = tid >> 5, lane = tid & 31, first = warp / W * W;
    __syncthreads();      // the words' last readers are through
    if (lane == 0)
#pragma unroll
      for (int k = 0; k < K; ++k) words[k][warp] = x[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float s = words[k][first];
#pragma unroll
      for (int i = 1; i < W; ++i) s = MAX ? fmaxf(s, words[k][first + i]) : s + words[k][first + i];
      x[k] = s;
    }
  }
}

// OUT: 0 the storage type, 1 e4m3 with a scale for each group of 128 columns, 2 e4m3 with a scale for the row
template <class T, int TPR, int NV, int OUT>
__global__ void __launch_bounds__(TPR > 256 ? TPR : 256) rms_norm_kernel(const __grid_constant__ RmsNormArgs a) {
  constexpr int N = Vec<T>::N, THREADS = TPR > 256 ? TPR : 256, ROWS = THREADS / TPR;
  __shared__ float words[1][32];
  const int tid = threadIdx.x, t = tid % TPR;
  const long long row = (long long)blockIdx.x * ROWS + tid / TPR;
  const bool real = row < a.rows;
  const size_t base = (size_t)(real ? row : 0) * a.n;
  const T *X = (const T*)a.X, *R = (const T*)a.R, *Wt = (const T*)a.w;
  wait_for_predecessor();
  float h[NV][N], w[NV][N], sum[1] = {0.f};
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (t + i * TPR) * N;
#pragma unroll
    for (int j = 0; j < N; ++j) h[i][j] = w[i][j] = 0.f;
    if (real && c < a.n) Vec<T>::load(h[i], X + base + c);
  }
  if (R) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (t + i * TPR) * N;
      float r[N];
      if (real && c < a.n) {
        Vec<T>::load(r, R + base + c);
#pragma unroll
        for (int j = 0; j < N; ++j) h[i][j] += r[j];
      }
    }
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (t + i * TPR) * N;
    if (real && c < a.n) {
      Vec<T>::load(w[i], Wt + c);
      if (a.H) Vec<T>::store((T*)a.H + base + c, h[i]);
    }
#pragma unroll
    for (int j = 0; j < N; ++j) sum[0] = fmaf(h[i][j], h[i][j], sum[0]);
  }
  row_reduce<TPR>(sum, words, tid);
  const float rstd = rsqrtf(sum[0] / (float)a.n + a.eps);
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < N; ++j) h[i][j] *= rstd * w[i][j];
  if constexpr (OUT == 0) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (t + i * TPR) * N;
      if (real && c < a.n) Vec<T>::store((T*)a.Y + base + c, h[i]);
    }
  } else {
    float top[1] = {0.f};
    float scale[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float m = 0.f;
#pragma unroll
      for (int j = 0; j < N; ++j) m = fmaxf(m, fabsf(h[i][j]));
      if constexpr (OUT == 1) {   // N columns a lane: 128 / N neighbouring lanes hold a group
#pragma unroll
        for (int x = kGroup / N / 2; x >= 1; x >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
        scale[i] = m > 0.f ? m / kMaxE4m3 : 1.f;
        const int c = (t + i * TPR) * N;
        if (real && c < a.n && c % kGroup == 0) a.scales[(size_t)row * ((a.n + kGroup - 1) / kGroup) + c / kGroup] = scale[i];
      } else {
        top[0] = fmaxf(top[0], m);
      }
    }
    if constexpr (OUT == 2) {
      row_reduce<TPR, 1, true>(top, words, tid);
      const float s = top[0] > 0.f ? top[0] / kMaxE4m3 : 1.f;
#pragma unroll
      for (int i = 0; i < NV; ++i) scale[i] = s;
      if (real && t == 0) a.scales[row] = s;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (t + i * TPR) * N;
      if (real && c < a.n) {
        uint32_t code[N / 4];
#pragma unroll
        for (int j = 0; j < N; j += 4)
          code[j / 4] = pack_e4m3(h[i][j] / scale[i], h[i][j + 1] / scale[i]) | pack_e4m3(h[i][j + 2] / scale[i], h[i][j + 3] / scale[i]) << 16;
        uint8_t* y = (uint8_t*)a.Y + base + c;
        if constexpr (N == 8) *reinterpret_cast<uint2*>(y) = make_uint2(code[0], code[1]);
        else *reinterpret_cast<uint32_t*>(y) = code[0];
      }
    }
  }
}

// Any n, any alignment: one block a row, which it reads twice (and a third time for a row's scale).
template <class T, int OUT>
__global__ void __launch_bounds__(256) rms_norm_any_kernel(const __grid_constant__ RmsNormArgs a) {
  __shared__ float words[1][32];
  const int tid = threadIdx.x;
  const size_t base = (size_t)blockIdx.x * a.n;
  const T *X = (const T*)a.X + base, *R = a.R ? (const T*)a.R + base : nullptr, *Wt = (const T*)a.w;
  // H may be X or R: every value is read for the last time before its place in H is written, in the last pass
  auto h_at = [&](int c) { return R ? up(X[c]) + up(R[c]) : up(X[c]); };
  float sum[1] = {0.f};
  for (int c = tid; c < a.n; c += 256) { const float h = h_at(c); sum[0] = fmaf(h, h, sum[0]); }
  row_reduce<256>(sum, words, tid);
  const float rstd = rsqrtf(sum[0] / (float)a.n + a.eps);
  auto y_at = [&](float h, int c) { return h * (rstd * up(Wt[c])); };
  float row_scale = 1.f;
  if constexpr (OUT == 2) {
    float top[1] = {0.f};
    for (int c = tid; c < a.n; c += 256) top[0] = fmaxf(top[0], fabsf(y_at(h_at(c), c)));
    row_reduce<256, 1, true>(top, words, tid);
    row_scale = top[0] > 0.f ? top[0] / kMaxE4m3 : 1.f;
    if (tid == 0) a.scales[blockIdx.x] = row_scale;
  }
  const int n_groups = (a.n + kGroup - 1) / kGroup;
  for (int gr = tid >> 5; gr < n_groups; gr += 8) {   // a warp per group of columns
    float h[4], y[4], m = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = gr * kGroup + 32 * i + (tid & 31);
      h[i] = c < a.n ? h_at(c) : 0.f;
      y[i] = c < a.n ? y_at(h[i], c) : 0.f;
      m = fmaxf(m, fabsf(y[i]));
    }
    float scale = row_scale;
    if constexpr (OUT == 1) {
#pragma unroll
      for (int x = 16; x >= 1; x >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
      scale = m > 0.f ? m / kMaxE4m3 : 1.f;
      if ((tid & 31) == 0) a.scales[(size_t)blockIdx.x * n_groups + gr] = scale;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = gr * kGroup + 32 * i + (tid & 31);
      if (c < a.n) {
        if constexpr (OUT == 0) put((T*)a.Y + base + c, y[i]);
        else ((uint8_t*)a.Y)[base + c] = (uint8_t)pack_e4m3(y[i] / scale, 0.f);
        if (a.H) put((T*)a.H + base + c, h[i]);
      }
    }
  }
}

// The gradient: a block takes every gridDim.x-th group of rows; a thread has the same columns in all of them and sums their dw in registers.
template <class T, int TPR, int NV>
__global__ void __launch_bounds__(TPR > 256 ? TPR : 256) rms_norm_backward_kernel(const __grid_constant__ RmsNormBackwardArgs a) {
  constexpr int N = Vec<T>::N, THREADS = TPR > 256 ? TPR : 256, ROWS = THREADS / TPR;
  __shared__ float words[2][32];
  const int tid = threadIdx.x, t = tid % TPR, sub = tid / TPR;
  const T *X = (const T*)a.X, *DY = (const T*)a.dY, *DH = (const T*)a.dH, *Wt = (const T*)a.w;
  wait_for_predecessor();
  float w[NV][N], dw[NV][N];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (t + i * TPR) * N;
#pragma unroll
    for (int j = 0; j < N; ++j) w[i][j] = dw[i][j] = 0.f;
    if (c < a.n) Vec<T>::load(w[i], Wt + c);
  }
  const long long steps = (a.rows + ROWS - 1) / ROWS;
  for (long long step = blockIdx.x; step < steps; step += gridDim.x) {   // the block's threads stay together: the reductions meet all of them
    const long long row = step * ROWS + sub;
    const bool real = row < a.rows;
    const size_t base = (size_t)(real ? row : 0) * a.n;
    float h[NV][N], u[NV][N], sum[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (t + i * TPR) * N;
#pragma unroll
      for (int j = 0; j < N; ++j) h[i][j] = u[i][j] = 0.f;
      if (real && c < a.n) { Vec<T>::load(h[i], X + base + c); Vec<T>::load(u[i], DY + base + c); }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        sum[0] = fmaf(h[i][j], h[i][j], sum[0]);
        sum[1] = fmaf(u[i][j] * w[i][j], h[i][j], sum[1]);
      }
    row_reduce<TPR>(sum, words, tid);
    const float rstd = rsqrtf(sum[0] / (float)a.n + a.eps), back = rstd * rstd * (sum[1] / (float)a.n);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (t + i * TPR) * N;
      if (real && c < a.n) {
        float dx[N];
        if (DH) Vec<T>::load(dx, DH + base + c);
#pragma unroll
        for (int j = 0; j < N; ++j) {
          dw[i][j] = fmaf(u[i][j], h[i][j] * rstd, dw[i][j]);
          const float g = rstd * (u[i][j] * w[i][j] - h[i][j] * back);
          dx[j] = DH ? dx[j] + g : g;
        }
        Vec<T>::store((T*)a.dX + base + c, dx);
      }
    }
  }
  // one row of partial sums for each of the block's rows side by side: ROWS * gridDim.x in all
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (t + i * TPR) * N;
    if (c < a.n) {
      float* p = a.partial + ((size_t)blockIdx.x * ROWS + sub) * a.n + c;
#pragma unroll
      for (int j = 0; j < N; j += 4) *reinterpret_cast<float4*>(p + j) = make_float4(dw[i][j], dw[i][j + 1], dw[i][j + 2], dw[i][j + 3]);
    }
  }
}
template <class T>
__global__ void __launch_bounds__(256) rms_norm_backward_any_kernel(const __grid_constant__ RmsNormBackwardArgs a) {
  __shared__ float words[2][32];
  const int tid = threadIdx.x;
  const T* Wt = (const T*)a.w;
  float* p = a.partial + (size_t)blockIdx.x * a.n;
  for (int c = tid; c < a.n; c += 256) p[c] = 0.f;
  for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const size_t base = (size_t)row * a.n;
    const T *X = (const T*)a.X + base, *DY = (const T*)a.dY + base, *DH = a.dH ? (const T*)a.dH + base : nullptr;
    float sum[2] = {0.f, 0.f};
    for (int c = tid; c < a.n; c += 256) {
      const float h = up(X[c]);
      sum[0] = fmaf(h, h, sum[0]);
      sum[1] = fmaf(up(DY[c]) * up(Wt[c]), h, sum[1]);
    }
    row_reduce<256>(sum, words, tid);
    const float rstd = rsqrtf(sum[0] / (float)a.n + a.eps), back = rstd * rstd * (sum[1] / (float)a.n);
    for (int c = tid; c < a.n; c += 256) {
      const float h = up(X[c]), dy = up(DY[c]);
      p[c] = fmaf(dy, h * rstd, p[c]);   // the thread's own columns
      const float g = rstd * (dy * up(Wt[c]) - h * back);
      put((T*)a.dX + base + c, DH ? up(DH[c]) + g : g);
    }
  }
}
// dw = the sum of the partial rows, in their order: 32 columns and 8 runs of rows a block
template <class T>
__global__ void __launch_bounds__(256) rms_norm_dw_kernel(const float* partial, T* dw, int n, int rows) {
  __shared__ float part[8][33];
  const int lane = threadIdx.x & 31, run = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  wait_for_predecessor();
  float s[4] = {0.f, 0.f, 0.f, 0.f};
  if (c < n) {
    int r = run;
    for (; r + 24 < rows; r += 32)
#pragma unroll
      for (int q = 0; q < 4; ++q) s[q] += partial[(size_t)(r + 8 * q) * n + c];
    for (; r < rows; r += 8) s[0] += partial[(size_t)r * n + c];
  }
  part[run][lane] = (s[0] + s[1]) + (s[2] + s[3]);
  __syncthreads();
  if (run == 0 && c < n) {
    float y = 0.f;
#pragma unroll
    for (int q = 0; q < 8; ++q) y += part[q][lane];
    put(dw + c, y);
  }
}

// Threads a row and vectors a thread for rows of `vecs` vectors: 0 threads where the register kernels do not take the row.
struct RowShape { int tpr, nv; };
RowShape row_shape(int vecs, long long rows, int sms) {
  if (vecs > 2048) return {0, 0};
  // few rows: as many threads as the row has vectors, up to 256
  const bool few = rows <= 2 * sms;
  if (vecs <= 32) return {32, 1};
  if (vecs <= (few ? 32 : 64)) return {32, 2};
  if (vecs <= 128) return few ? RowShape{128, 1} : RowShape{32, 4};
  if (vecs <= 256) return few ? RowShape{256, 1} : RowShape{128, 2};
  if (vecs <= 512) return few ? RowShape{256, 2} : RowShape{128, 4};
  if (vecs <= 1024) return {256, 4};
  return {512, 4};
}
bool aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

template <class T, int OUT>
cudaError_t launch_forward(const RmsNormArgs& a, int sms, cudaStream_t stream) {
  const bool whole = a.n % Vec<T>::N == 0 && aligned(a.X) && aligned(a.R) && aligned(a.w) && aligned(a.Y) && aligned(a.H);
  const RowShape f = whole ? row_shape(a.n / Vec<T>::N, a.rows, sms) : RowShape{0, 0};
  auto go = [&](auto kernel, int tpr) {
    const int threads = std::max(tpr, 256), rows = threads / tpr;
    const long long grid = (a.rows + rows - 1) / rows;
    if (grid > 0x7fffffffLL) return cudaErrorInvalidValue;
    return launch_early(kernel, dim3((unsigned)grid), threads, 0, stream, a);
  };
  cudaError_t e;
  if (f.tpr == 32) e = f.nv == 1 ? go(rms_norm_kernel<T, 32, 1, OUT>, 32) : f.nv == 2 ? go(rms_norm_kernel<T, 32, 2, OUT>, 32) : go(rms_norm_kernel<T, 32, 4, OUT>, 32);
  else if (f.tpr == 128) e = f.nv == 1 ? go(rms_norm_kernel<T, 128, 1, OUT>, 128) : f.nv == 2 ? go(rms_norm_kernel<T, 128, 2, OUT>, 128) : go(rms_norm_kernel<T, 128, 4, OUT>, 128);
  else if (f.tpr == 256) e = f.nv == 1 ? go(rms_norm_kernel<T, 256, 1, OUT>, 256) : f.nv == 2 ? go(rms_norm_kernel<T, 256, 2, OUT>, 256) : go(rms_norm_kernel<T, 256, 4, OUT>, 256);
  else if (f.tpr == 512) e = go(rms_norm_kernel<T, 512, 4, OUT>, 512);
  else {
    if (a.rows > 0x7fffffffLL) return cudaErrorInvalidValue;
    rms_norm_any_kernel<T, OUT><<<(unsigned)a.rows, 256, 0, stream>>>(a);
    return launched();
  }
  return e == cudaSuccess ? launched() : e;
}

template <class T>
cudaError_t launch_backward(const RmsNormBackwardArgs& a, int sms, cudaStream_t stream) {
  const bool whole = a.n % Vec<T>::N == 0 && aligned(a.X) && aligned(a.dY) && aligned(a.w) && aligned(a.dH) && aligned(a.dX);
  const RowShape f = whole ? row_shape(a.n / Vec<T>::N, a.rows, sms) : RowShape{0, 0};
  int partial_rows = 0;
  auto go = [&](auto kernel, int tpr) {
    const int threads = std::max(tpr, 256), rows = threads / tpr;
    const int grid = (int)std::min<long long>((a.rows + rows - 1) / rows, (long long)kRmsNormPartials / rows);
    partial_rows = grid * rows;
    return launch_early(kernel, dim3(grid), threads, 0, stream, a);
  };
  cudaError_t e = cudaSuccess;
  if (a.rows == 0) ;   // the sum of no rows
  else if (f.tpr == 32) e = f.nv == 1 ? go(rms_norm_backward_kernel<T, 32, 1>, 32) : f.nv == 2 ? go(rms_norm_backward_kernel<T, 32, 2>, 32) : go(rms_norm_backward_kernel<T, 32, 4>, 32);
  else if (f.tpr == 128) e = f.nv == 1 ? go(rms_norm_backward_kernel<T, 128, 1>, 128) : f.nv == 2 ? go(rms_norm_backward_kernel<T, 128, 2>, 128) : go(rms_norm_backward_kernel<T, 128, 4>, 128);
  else if (f.tpr == 256) e = f.nv == 1 ? go(rms_norm_backward_kernel<T, 256, 1>, 256) : f.nv == 2 ? go(rms_norm_backward_kernel<T, 256, 2>, 256) : go(rms_norm_backward_kernel<T, 256, 4>, 256);
  else if (f.tpr == 512) e = go(rms_norm_backward_kernel<T, 512, 4>, 512);
  else {
    partial_rows = (int)std::min<long long>(a.rows, kRmsNormPartials);
    rms_norm_backward_any_kernel<T><<<partial_rows, 256, 0, stream>>>(a);
    e = cudaGetLastError();
  }
  if (e != cudaSuccess || (a.rows > 0 && (e = launched()) != cudaSuccess)) return e;
  e = launch_early(rms_norm_dw_kernel<T>, dim3((a.n + 31) / 32), 256, 0, stream, (const float*)a.partial, (T*)a.dw, a.n, partial_rows);
  return e == cudaSuccess ? launched() : e;
}

}  // namespace

cudaError_t launch_rms_norm(const RmsNormArgs& a, int dtype, int out, cudaStream_t stream) {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return cudaErrorUnknown;
  if (dtype == TRI_INV_F32)
    return out == 0 ? launch_forward<float, 0>(a, sms, stream) : out == 1 ? launch_forward<float, 1>(a, sms, stream) : launch_forward<float, 2>(a, sms, stream);
  return out == 0 ? launch_forward<__nv_bfloat16, 0>(a, sms, stream) : out == 1 ? launch_forward<__nv_bfloat16, 1>(a, sms, stream) : launch_forward<__nv_bfloat16, 2>(a, sms, stream);
}

cudaError_t launch_rms_norm_backward(const RmsNormBackwardArgs& a, int dtype, cudaStream_t stream) {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return cudaErrorUnknown;
  return dtype == TRI_INV_F32 ? launch_backward<float>(a, sms, stream) : launch_backward<__nv_bfloat16>(a, sms, stream);
}

}  // namespace tri_inv
