// Root-mean-square norm over rows of n values, with the residual's addition in front and an output in 8 bits behind, and its gradient.
//     h = x + r,    y = h w / sqrt(mean h^2 + eps)
//     y in the storage type, or per group of columns: scale = max |y| / 448 (1 where that is 0), y (1 / scale) rounded to e4m3
//     u = dy w,     dx = rstd (u - h rstd^2 mean(u h)) + dh,     dw = sum over rows of dy h rstd                rstd = 1 / sqrt(mean h^2 + eps)
// Sums, h (before it is stored), y (before it is rounded) and dw's sums over rows are fp32.
//
// A row is held in the registers of TPR threads, NV vectors of 16 bytes each: every value is read once and written once, which bounds the large calls; a
// call of a few rows is the latency of one load, one exchange and one store, and takes more threads a row.  Rows that are not whole vectors, or not aligned to them, are held value by
// value (16384 x 2047 bf16 with residual 58 us, 41 with 2048; their gradient 75 and 54); long ones take a kernel that reads them twice.
// Measured, calls in a captured graph, three input sets in turn: 16384 x 4096 bf16 with residual to e4m3 77 us rested, 80 after 0.3 s of them, 0.90 of a copy's rate; 8 x 2048 2.1 us (6 with the call);
// the gradient of 16384 x 2048 bf16 with dH 54 us, 4.9 TB/s (its blocks pause at two barriers a row and end with 592 partial rows of dw, which the second launch sums), of 40000 x 128 fp32 13 us (11 on one input
// set, which the L2 cache holds).
#include <algorithm>

#include "common.cuh"
#include "rms_norm.cuh"

namespace tri_inv {
namespace {

constexpr int kGroup = 128;         // columns that share a scale
constexpr float kMaxE4m3 = 448.f;
// The scale of a group whose largest value is m: a normal number, so that its reciprocal is finite
__device__ __forceinline__ float scale_of(float m) { return m > 0.f ? fmaxf(m / kMaxE4m3, 1.17549435e-38f) : 1.f; }

__device__ __forceinline__ float up(float x) { return x; }
__device__ __forceinline__ float up(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

// N values that a thread loads at once: 16 bytes, or a single one
template <class T, int N> struct Vec;
template <> struct Vec<float, 4> {
  using Raw = uint4;
  static __device__ __forceinline__ uint4 load(const float* p) { return *reinterpret_cast<const uint4*>(p); }
  static __device__ __forceinline__ void widen(float (&v)[4], const uint4& x) {
    v[0] = __uint_as_float(x.x); v[1] = __uint_as_float(x.y); v[2] = __uint_as_float(x.z); v[3] = __uint_as_float(x.w);
  }
  static __device__ __forceinline__ void store(float* p, const float (&v)[4]) { *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]); }
};
template <> struct Vec<__nv_bfloat16, 8> {
  using Raw = uint4;
  static __device__ __forceinline__ uint4 load(const __nv_bfloat16* p) { return *reinterpret_cast<const uint4*>(p); }
  static __device__ __forceinline__ void widen(float (&v)[8], const uint4& x) {
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
template <> struct Vec<float, 1> {
  using Raw = uint32_t;
  static __device__ __forceinline__ uint32_t load(const float* p) { return *reinterpret_cast<const uint32_t*>(p); }
  static __device__ __forceinline__ void widen(float (&v)[1], uint32_t x) { v[0] = __uint_as_float(x); }
  static __device__ __forceinline__ void store(float* p, const float (&v)[1]) { *p = v[0]; }
};
template <> struct Vec<__nv_bfloat16, 1> {
  using Raw = uint32_t;   // (as 16 bits, two to a register, each load waited for the one before it: 389 us for 8000 x 7001)
  static __device__ __forceinline__ uint32_t load(const __nv_bfloat16* p) { return *reinterpret_cast<const uint16_t*>(p); }
  static __device__ __forceinline__ void widen(float (&v)[1], uint32_t x) { v[0] = __uint_as_float(x << 16); }
  static __device__ __forceinline__ void store(__nv_bfloat16* p, const float (&v)[1]) { *p = __float2bfloat16_rn(v[0]); }
};
template <class T> constexpr int kWide = 16 / sizeof(T);
// The first column of a thread's i-th vector.  Wide: the row's threads side by side.  Single values: a warp takes whole groups of 128 columns, four values a lane, so that a group's
// scale is a warp's own affair.
template <int N, int TPR>
__device__ __forceinline__ int column(int t, int i) {
  if constexpr (N > 1) return (t + i * TPR) * N;
  else return ((i >> 2) * (TPR / 32) + (t >> 5)) * kGroup + (i & 3) * 32 + (t & 31);
}
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
template <class T, int N, int TPR, int NV, int OUT>
__global__ void __launch_bounds__(TPR > 256 ? TPR : 256, N == 1 && NV == 16 ? 2 : 0) rms_norm_kernel(const __grid_constant__ RmsNormArgs a) {
  using V = Vec<T, N>;
  constexpr int THREADS = TPR > 256 ? TPR : 256, ROWS = THREADS / TPR;
  __shared__ float words[1][32];
  const int tid = threadIdx.x, t = tid % TPR;
  const long long row = (long long)blockIdx.x * ROWS + tid / TPR;
  const bool real = row < a.rows;
  const size_t base = (size_t)(real ? row : 0) * a.n;
  const T *X = (const T*)a.X, *R = (const T*)a.R, *Wt = (const T*)a.w;
  wait_for_predecessor();
  typename V::Raw raw[NV], res[NV], wr[NV];   // everything is requested before anything is used
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = column<N, TPR>(t, i);
    raw[i] = res[i] = wr[i] = typename V::Raw{};
    if (real && c < a.n) {
      raw[i] = V::load(X + base + c);
      if (R) res[i] = V::load(R + base + c);
    }
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = column<N, TPR>(t, i);
    if (real && c < a.n) wr[i] = V::load(Wt + c);
  }
  float h[NV][N], sum[1] = {0.f};
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = column<N, TPR>(t, i);
    V::widen(h[i], raw[i]);
    if (R) {
      float r[N];
      V::widen(r, res[i]);
#pragma unroll
      for (int j = 0; j < N; ++j) h[i][j] += r[j];
    }
    if (a.H && real && c < a.n) V::store((T*)a.H + base + c, h[i]);
#pragma unroll
    for (int j = 0; j < N; ++j) sum[0] = fmaf(h[i][j], h[i][j], sum[0]);
  }
  row_reduce<TPR>(sum, words, tid);
  const float rstd = rsqrtf(sum[0] / (float)a.n + a.eps);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    float w[N];
    V::widen(w, wr[i]);
#pragma unroll
    for (int j = 0; j < N; ++j) h[i][j] *= rstd * w[j];
  }
  if constexpr (OUT == 0) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = column<N, TPR>(t, i);
      if (real && c < a.n) V::store((T*)a.Y + base + c, h[i]);
    }
  } else {
    float top[1] = {0.f};
    float scale[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float m = 0.f;
#pragma unroll
      for (int j = 0; j < N; ++j) m = fmaxf(m, fabsf(h[i][j]));
      if constexpr (OUT == 1 && N == 1) {   // four of a lane's values and a warp hold a group
        top[0] = i & 3 ? fmaxf(top[0], m) : m;
        if ((i & 3) == 3) {
          m = top[0];
#pragma unroll
          for (int x = 16; x >= 1; x >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
          scale[i] = scale[i - 1] = scale[i - 2] = scale[i - 3] = scale_of(m);
          const int c = column<N, TPR>(t, i - 3);
          if (real && c < a.n && c % kGroup == 0) a.scales[(size_t)row * ((a.n + kGroup - 1) / kGroup) + c / kGroup] = scale[i];
        }
      } else if constexpr (OUT == 1) {   // N columns a lane: 128 / N neighbouring lanes hold a group
#pragma unroll
        for (int x = kGroup / N / 2; x >= 1; x >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
        scale[i] = scale_of(m);
        const int c = column<N, TPR>(t, i);
        if (real && c < a.n && c % kGroup == 0) a.scales[(size_t)row * ((a.n + kGroup - 1) / kGroup) + c / kGroup] = scale[i];
      } else {
        top[0] = fmaxf(top[0], m);
      }
    }
    if constexpr (OUT == 2) {
      row_reduce<TPR, 1, true>(top, words, tid);
      const float s = scale_of(top[0]);
#pragma unroll
      for (int i = 0; i < NV; ++i) scale[i] = s;
      if (real && t == 0) a.scales[row] = s;
    }
    uint8_t* Y = (uint8_t*)a.Y + base;
    if constexpr (N == 1) {
#pragma unroll
      for (int i = 0; i < NV; i += 4) {   // a group's
        const float up = 1.f / scale[i];
        const uint32_t code = pack_e4m3(h[i][0] * up, h[i + 1][0] * up) | pack_e4m3(h[i + 2][0] * up, h[i + 3][0] * up) << 16;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int c = column<N, TPR>(t, i + q);
          if (real && c < a.n) Y[c] = (uint8_t)(code >> 8 * q);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = column<N, TPR>(t, i);
        if (real && c < a.n) {
          const float up = 1.f / scale[i];   // (a division for every value took as long as all the rest)
          uint32_t code[N / 4];
#pragma unroll
          for (int j = 0; j < N; j += 4)
            code[j / 4] = pack_e4m3(h[i][j] * up, h[i][j + 1] * up) | pack_e4m3(h[i][j + 2] * up, h[i][j + 3] * up) << 16;
          if constexpr (N == 8) *reinterpret_cast<uint2*>(Y + c) = make_uint2(code[0], code[1]);
          else *reinterpret_cast<uint32_t*>(Y + c) = code[0];
        }
      }
    }
  }
}

// Rows that the registers do not take: one block a row, which it reads twice (and a third time for a row's scale).
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
    row_scale = scale_of(top[0]);
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
      scale = scale_of(m);
      if ((tid & 31) == 0) a.scales[(size_t)blockIdx.x * n_groups + gr] = scale;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = gr * kGroup + 32 * i + (tid & 31);
      if (c < a.n) {
        if constexpr (OUT == 0) put((T*)a.Y + base + c, y[i]);
        else ((uint8_t*)a.Y)[base + c] = (uint8_t)pack_e4m3(y[i] * (1.f / scale), 0.f);
        if (a.H) put((T*)a.H + base + c, h[i]);
      }
    }
  }
}

// The gradient: a block takes every gridDim.x-th group of rows; a thread has the same columns in all of them and sums their dw in registers.  The
// next rows are requested before these are worked on; rows side by side join their sums in shared memory, so that a block leaves one row of them.
constexpr int backward_blocks(int n, int tpr, int nv) {   // blocks an SM
  return n > 1 ? (nv == 1 ? (tpr > 256 ? 2 : 4) : 1) : nv <= 4 ? 4 : tpr <= 256 ? 2 : 1;
}
template <class T, int N, int TPR, int NV>
__global__ void __launch_bounds__(TPR > 256 ? TPR : 256, backward_blocks(N, TPR, NV)) rms_norm_backward_kernel(const __grid_constant__ RmsNormBackwardArgs a) {
  using V = Vec<T, N>;
  constexpr bool AHEAD = NV <= (N > 1 ? 2 : 8);   // longer rows leave no registers for the next one
  constexpr int THREADS = TPR > 256 ? TPR : 256, ROWS = THREADS / TPR;
  __shared__ float words[2][32];
  __shared__ __align__(16) float joined[ROWS > 1 ? (ROWS - 1) * TPR * NV * N : 4];
  const int tid = threadIdx.x, t = tid % TPR, sub = tid / TPR;
  const T *X = (const T*)a.X, *DY = (const T*)a.dY, *DH = (const T*)a.dH, *Wt = (const T*)a.w;
  wait_for_predecessor();
  const typename V::Raw zero{};
  typename V::Raw wr[NV];
  float dw[NV][N];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = column<N, TPR>(t, i);
    wr[i] = c < a.n ? V::load(Wt + c) : zero;
#pragma unroll
    for (int j = 0; j < N; ++j) dw[i][j] = 0.f;
  }
  const long long steps = (a.rows + ROWS - 1) / ROWS;
  typename V::Raw xn[NV], dn[NV], pn[NV];
  auto request = [&](long long step) {
    const long long row = step * ROWS + sub;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = column<N, TPR>(t, i);
      const bool in = row < a.rows && c < a.n;
      const size_t at = (size_t)(in ? row : 0) * a.n + c;
      xn[i] = in ? V::load(X + at) : zero;
      dn[i] = in ? V::load(DY + at) : zero;
      pn[i] = in && DH ? V::load(DH + at) : zero;
    }
  };
  if (AHEAD) request(blockIdx.x);
  for (long long step = blockIdx.x; step < steps; step += gridDim.x) {   // the block's threads stay together: the reductions meet all of them
    const long long row = step * ROWS + sub;
    typename V::Raw xr[NV], dr[NV], pr[NV];
    if (!AHEAD) request(step);
#pragma unroll
    for (int i = 0; i < NV; ++i) { xr[i] = xn[i]; dr[i] = dn[i]; pr[i] = pn[i]; }
    // (dX may be dY, X or dH: the next rows are not this block's present ones, and no other block's)
    if (AHEAD && step + gridDim.x < steps) request(step + gridDim.x);
    float sum[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float h[N], u[N], w[N];
      V::widen(h, xr[i]);
      V::widen(u, dr[i]);
      V::widen(w, wr[i]);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        sum[0] = fmaf(h[j], h[j], sum[0]);
        sum[1] = fmaf(u[j] * w[j], h[j], sum[1]);
      }
    }
    row_reduce<TPR>(sum, words, tid);
    // (a row behind the last one adds nothing to dw: without eps its zeros would meet 1 / sqrt(0))
    const float rstd = row < a.rows ? rsqrtf(sum[0] / (float)a.n + a.eps) : 0.f, back = rstd * rstd * (sum[1] / (float)a.n);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = column<N, TPR>(t, i);
      float h[N], u[N], w[N], dx[N];
      V::widen(h, xr[i]);
      V::widen(u, dr[i]);
      V::widen(w, wr[i]);
      V::widen(dx, pr[i]);   // zero without dH
#pragma unroll
      for (int j = 0; j < N; ++j) {
        dw[i][j] = fmaf(u[j], h[j] * rstd, dw[i][j]);
        dx[j] += rstd * (u[j] * w[j] - h[j] * back);
      }
      if (row < a.rows && c < a.n) V::store((T*)a.dX + (size_t)row * a.n + c, dx);
    }
  }
  if constexpr (ROWS > 1) {
    if (sub > 0)
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        if constexpr (N == 1) joined[((sub - 1) * NV + i) * TPR + t] = dw[i][0];
        else
#pragma unroll
          for (int j = 0; j < N; j += 4)
            *reinterpret_cast<float4*>(joined + ((sub - 1) * NV * N + i * N + j) * TPR + 4 * t) = make_float4(dw[i][j], dw[i][j + 1], dw[i][j + 2], dw[i][j + 3]);
      }
    __syncthreads();
    if (sub > 0) return;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int s = 0; s < ROWS - 1; ++s) {
        if constexpr (N == 1) dw[i][0] += joined[(s * NV + i) * TPR + t];
        else
#pragma unroll
          for (int j = 0; j < N; j += 4) {
            const float4 x = *reinterpret_cast<const float4*>(joined + (s * NV * N + i * N + j) * TPR + 4 * t);
            dw[i][j] += x.x; dw[i][j + 1] += x.y; dw[i][j + 2] += x.z; dw[i][j + 3] += x.w;
          }
      }
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = column<N, TPR>(t, i);
    if (c < a.n) {
      float* p = a.partial + (size_t)blockIdx.x * a.n + c;
      if constexpr (N == 1) *p = dw[i][0];
      else
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
// dw = the sum of the partial rows, in an order that the sizes alone fix: 32 columns and 32 runs of rows a block
template <class T>
__global__ void __launch_bounds__(1024) rms_norm_dw_kernel(const float* partial, T* dw, int n, int rows) {
  __shared__ float part[32][33];
  const int lane = threadIdx.x & 31, run = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  wait_for_predecessor();
  constexpr int PER = (kRmsNormPartials + 31) / 32;
  float v[PER], s = 0.f;   // all of a thread's loads at once: one latency
#pragma unroll
  for (int q = 0; q < PER; ++q) v[q] = c < n && run + 32 * q < rows ? partial[(size_t)(run + 32 * q) * n + c] : 0.f;
#pragma unroll
  for (int q = 0; q < PER; ++q) s += v[q];
  part[run][lane] = s;
  __syncthreads();
  float y = part[lane][run];   // a warp a column
#pragma unroll
  for (int m = 16; m >= 1; m >>= 1) y += __shfl_xor_sync(0xffffffffu, y, m);
  if (lane == 0 && blockIdx.x * 32 + run < n) put(dw + blockIdx.x * 32 + run, y);
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
// The gradient holds three rows twice and a row of sums: one vector a thread while the row allows it  (16384 x 2048 in bf16: 256 threads of one vector 52 us, 128 of two 68).
RowShape backward_shape(int vecs) {
  if (vecs <= 32) return {32, 1};
  if (vecs <= 64) return {64, 1};
  if (vecs <= 128) return {128, 1};
  if (vecs <= 256) return {256, 1};
  if (vecs <= 512) return {512, 1};
  if (vecs <= 1024) return {512, 2};
  return vecs <= 2048 ? RowShape{512, 4} : RowShape{0, 0};
}
// Rows of single values, forward and gradient: a warp holds whole groups of 128 columns.  Longer rows take the kernels that read them twice: 8000 x 7001 in bf16 with 16 values a
// thread 219 us, 141 by those (fp32 133, 195), its gradient 350 with 1024 threads, 400 (fp32 228, 486); 8000 x 4001 71 and 101.
template <class T>
RowShape narrow_shape(int n) {
  if (n <= 128) return {32, 4};
  if (n <= 256) return {32, 8};
  if (n <= 512) return {64, 8};
  if (n <= 1024) return {128, 8};
  if (n <= 2048) return {256, 8};
  if (n <= 4096) return {512, 8};
  return n <= 8192 && sizeof(T) == 4 ? RowShape{512, 16} : RowShape{0, 0};
}
bool aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

template <class T, int OUT>
cudaError_t launch_forward(const RmsNormArgs& a, int sms, cudaStream_t stream) {
  constexpr int W = kWide<T>;
  const bool whole = a.n % W == 0 && aligned(a.X) && aligned(a.R) && aligned(a.w) && aligned(a.Y) && aligned(a.H);
  const RowShape f = whole ? row_shape(a.n / W, a.rows, sms) : narrow_shape<T>(a.n);
  auto go = [&](auto kernel, int tpr) {
    const int threads = std::max(tpr, 256), rows = threads / tpr;
    const long long grid = (a.rows + rows - 1) / rows;
    if (grid > 0x7fffffffLL) return cudaErrorInvalidValue;
    return launch_early(kernel, dim3((unsigned)grid), threads, 0, stream, a);
  };
  cudaError_t e;
  if (!whole && f.tpr) {
    if (f.tpr == 32) e = f.nv == 4 ? go(rms_norm_kernel<T, 1, 32, 4, OUT>, 32) : go(rms_norm_kernel<T, 1, 32, 8, OUT>, 32);
    else if (f.tpr == 64) e = go(rms_norm_kernel<T, 1, 64, 8, OUT>, 64);
    else if (f.tpr == 128) e = go(rms_norm_kernel<T, 1, 128, 8, OUT>, 128);
    else if (f.tpr == 256) e = go(rms_norm_kernel<T, 1, 256, 8, OUT>, 256);
    else if (f.nv == 8) e = go(rms_norm_kernel<T, 1, 512, 8, OUT>, 512);
    else e = go(rms_norm_kernel<float, 1, 512, 16, OUT>, 512);
  }
  else if (f.tpr == 32) e = f.nv == 1 ? go(rms_norm_kernel<T, W, 32, 1, OUT>, 32) : f.nv == 2 ? go(rms_norm_kernel<T, W, 32, 2, OUT>, 32) : go(rms_norm_kernel<T, W, 32, 4, OUT>, 32);
  else if (f.tpr == 128) e = f.nv == 1 ? go(rms_norm_kernel<T, W, 128, 1, OUT>, 128) : f.nv == 2 ? go(rms_norm_kernel<T, W, 128, 2, OUT>, 128) : go(rms_norm_kernel<T, W, 128, 4, OUT>, 128);
  else if (f.tpr == 256) e = f.nv == 1 ? go(rms_norm_kernel<T, W, 256, 1, OUT>, 256) : f.nv == 2 ? go(rms_norm_kernel<T, W, 256, 2, OUT>, 256) : go(rms_norm_kernel<T, W, 256, 4, OUT>, 256);
  else if (f.tpr == 512) e = go(rms_norm_kernel<T, W, 512, 4, OUT>, 512);
  else {
    if (a.rows > 0x7fffffffLL) return cudaErrorInvalidValue;
    rms_norm_any_kernel<T, OUT><<<(unsigned)a.rows, 256, 0, stream>>>(a);
    return launched();
  }
  return e == cudaSuccess ? launched() : e;
}

template <class T>
cudaError_t launch_backward(const RmsNormBackwardArgs& a, int sms, cudaStream_t stream) {
  constexpr int W = kWide<T>;
  const bool whole = a.n % W == 0 && aligned(a.X) && aligned(a.dY) && aligned(a.w) && aligned(a.dH) && aligned(a.dX);
  const RowShape f = whole ? backward_shape(a.n / W) : narrow_shape<T>(a.n);
  int partial_rows = 0;
  auto go = [&](auto kernel, int tpr) {
    const int threads = std::max(tpr, 256), rows = threads / tpr;
    const int grid = (int)std::min<long long>((a.rows + rows - 1) / rows, kRmsNormPartials);
    partial_rows = grid;
    return launch_early(kernel, dim3(grid), threads, 0, stream, a);
  };
  cudaError_t e = cudaSuccess;
  if (a.rows == 0) ;   // the sum of no rows
  else if (!whole && f.tpr) {
    if (f.tpr == 32) e = f.nv == 4 ? go(rms_norm_backward_kernel<T, 1, 32, 4>, 32) : go(rms_norm_backward_kernel<T, 1, 32, 8>, 32);
    else if (f.tpr == 64) e = go(rms_norm_backward_kernel<T, 1, 64, 8>, 64);
    else if (f.tpr == 128) e = go(rms_norm_backward_kernel<T, 1, 128, 8>, 128);
    else if (f.tpr == 256) e = go(rms_norm_backward_kernel<T, 1, 256, 8>, 256);
    else if (f.nv == 8) e = go(rms_norm_backward_kernel<T, 1, 512, 8>, 512);
    else e = go(rms_norm_backward_kernel<float, 1, 512, 16>, 512);
  }
  else if (f.tpr == 32) e = go(rms_norm_backward_kernel<T, W, 32, 1>, 32);
  else if (f.tpr == 64) e = go(rms_norm_backward_kernel<T, W, 64, 1>, 64);
  else if (f.tpr == 128) e = go(rms_norm_backward_kernel<T, W, 128, 1>, 128);
  else if (f.tpr == 256) e = go(rms_norm_backward_kernel<T, W, 256, 1>, 256);
  else if (f.tpr == 512) e = f.nv == 1 ? go(rms_norm_backward_kernel<T, W, 512, 1>, 512) : f.nv == 2 ? go(rms_norm_backward_kernel<T, W, 512, 2>, 512) : go(rms_norm_backward_kernel<T, W, 512, 4>, 512);
  else {
    partial_rows = (int)std::min<long long>(a.rows, kRmsNormPartials);
    rms_norm_backward_any_kernel<T><<<partial_rows, 256, 0, stream>>>(a);
    e = cudaGetLastError();
  }
  if (e != cudaSuccess || (a.rows > 0 && (e = launched()) != cudaSuccess)) return e;
  e = launch_early(rms_norm_dw_kernel<T>, dim3((a.n + 31) / 32), 1024, 0, stream, (const float*)a.partial, (T*)a.dw, a.n, partial_rows);
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
