// Norm of each query and key head with the position rotation, and its gradient.
//     y = R(p f) (x rstd w),   rstd = 1 / sqrt(mean x^2 + eps);   R turns the pairs of the first 2 r features by the angles p f_i
//     v = R(-p f) dy,  u = v w,  dx = rstd (u - x rstd^2 mean(u x)),  dw = sum over tokens and heads of v x rstd
//
// A head is held by LANES lanes, a lane has the two halves of its pairs (two vectors of V values), so that the rotation stays in registers and the mean takes log2 LANES exchanges; a warp
// holds 32 / LANES heads of one token at a time and goes through the token's heads with one table of sines and cosines.
// Angles: p f / 2 pi only counts modulo 1, so f / 2 pi is kept as a 64-bit fraction F and p F modulo 2^64 is the exact product's fraction: a position of 2^31 is as good as one of 1.
#include <algorithm>

#include "qk_norm_rope.cuh"

namespace tri_inv {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;

template <class T, int V> struct alignas(sizeof(T) * V) Vec { T v[V]; };

__device__ __forceinline__ float up(float x) { return x; }
__device__ __forceinline__ float up(__nv_bfloat16 x) { return __bfloat162float(x); }
template <class T, int V>
__device__ __forceinline__ void load(float (&to)[V], const T* p) {
  const Vec<T, V> raw = *reinterpret_cast<const Vec<T, V>*>(p);
#pragma unroll
  for (int i = 0; i < V; ++i) to[i] = up(raw.v[i]);
}
template <class T, int V>
__device__ __forceinline__ void store(T* p, const float (&from)[V]) {
  Vec<T, V> raw;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    if constexpr (sizeof(T) == 4) raw.v[i] = from[i];
    else raw.v[i] = __float2bfloat16_rn(from[i]);
  }
  *reinterpret_cast<Vec<T, V>*>(p) = raw;
}

// f / 2 pi modulo 1 in units of 2^-64
__device__ __forceinline__ unsigned long long fraction(float f) {
  double x = (double)f * 0.15915494309189533577;
  x -= floor(x);
  const double hi = floor(x * 4294967296.0), lo = (x * 4294967296.0 - hi) * 4294967296.0;
  return ((unsigned long long)hi << 32) + (unsigned long long)lo;   // (x = 1 wraps to 0)
}

// The first features of the two vectors of unit p, >= d where the head has none.  Where the pairs are (i, i + r) the units of the first r / V are pairs, and the others two neighbours of the rest.
template <int V>
__device__ __forceinline__ void columns(int p, int r, bool interleaved, int& c0, int& c1) {
  const bool pairs = !interleaved && p * V < r;
  c0 = pairs ? p * V : 2 * p * V;   // (behind the pairs: 2 r + 2 (p V - r))
  c1 = c0 + (pairs ? r : V);
}

// Turns a lane's pairs; back: the other way
template <int V, bool BACK>
__device__ __forceinline__ void turn(float (&a)[V], float (&b)[V], const float2* table, int p, int r, bool interleaved) {
  float2 cs[V];
#pragma unroll
  for (int i = 0; i < V; ++i) cs[i] = p * V + i < r ? table[p * V + i] : make_float2(1.f, 0.f);
  auto one = [](float& u, float& v, float2 q) {
    const float s = BACK ? -q.y : q.y, x = u, y = v;
    u = x * q.x - y * s;
    v = y * q.x + x * s;
  };
  if (interleaved) {
    if constexpr (V == 1) {
      one(a[0], b[0], cs[0]);
    } else {
#pragma unroll
      for (int i = 0; i < V / 2; ++i) {
        one(a[2 * i], a[2 * i + 1], cs[i]);
        one(b[2 * i], b[2 * i + 1], cs[V / 2 + i]);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) one(a[i], b[i], cs[i]);
  }
}

struct HeadsPlan {
  int blocks[2];       // of queries and of keys
  int parts[2];        // warps that share a token's heads
};

// NU: units (pairs of vectors) of a lane
template <class T, int V, int LANES, int NU, bool BACK>
__global__ void __launch_bounds__(kThreads) qk_norm_rope_kernel(const __grid_constant__ HeadsArgs a, const __grid_constant__ HeadsPlan plan) {
  constexpr int HEADS = 32 / LANES;   // of a warp at a time
  __shared__ unsigned long long freq[kHeadsMaxDim / 2];
  __shared__ float2 tables[kWarps][kHeadsMaxDim / 2];
  __shared__ float joined[BACK ? kWarps : 1][BACK ? kHeadsMaxDim : 1];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, sub = lane / LANES, t = lane % LANES;
  const int which = (int)blockIdx.x >= plan.blocks[0], block = blockIdx.x - (which ? plan.blocks[0] : 0);
  const HeadsSide& s = a.side[which];
  const T *X = (const T*)s.x, *W = (const T*)s.w, *DY = (const T*)s.dy;
  wait_for_predecessor();
  for (int i = tid; i < a.r; i += kThreads) freq[i] = fraction(a.inv_freq[i]);
  int c0[NU], c1[NU];
  float w0[NU][V], w1[NU][V], g0[BACK ? NU : 1][V], g1[BACK ? NU : 1][V];
#pragma unroll
  for (int k = 0; k < NU; ++k) {
    columns<V>(k * LANES + t, a.r, a.interleaved, c0[k], c1[k]);
#pragma unroll
    for (int i = 0; i < V; ++i) w0[k][i] = w1[k][i] = 1.f;
    if (W && c0[k] < a.d) load<T, V>(w0[k], W + c0[k]);
    if (W && c1[k] < a.d) load<T, V>(w1[k], W + c1[k]);
    if constexpr (BACK)
#pragma unroll
      for (int i = 0; i < V; ++i) g0[k][i] = g1[k][i] = 0.f;
  }
  __syncthreads();
  float2* table = tables[warp];
  const int parts = plan.parts[which], per = ((s.H + HEADS - 1) / HEADS + parts - 1) / parts * HEADS;   // heads of a part
  const long long items = a.tokens * parts;
  const float over_d = 1.f / (float)a.d;
  for (long long item = (long long)block * kWarps + warp; item < items; item += (long long)plan.blocks[which] * kWarps) {
    const long long token = item / parts;
    const int first = (int)(item - token * parts) * per, end = min(s.H, first + per);
    const int position = a.positions ? a.positions[token] : (int)(token % a.T);
    const bool real = position >= 0;
    __syncwarp();
    for (int i = lane; i < a.r; i += 32) {
      const int turns = (int)(((unsigned long long)(unsigned)position * freq[i]) >> 32);   // of 2^-32 of a whole one, signed
      float sn, cs;
      sincospif((float)turns * 4.656612873077393e-10f, &sn, &cs);   // 2^-31
      table[i] = make_float2(cs, sn);
    }
    __syncwarp();
    for (int h0 = first; h0 < end; h0 += HEADS) {
      const int h = h0 + sub;
      const bool in = h < end && real;
      const T* x = X + token * s.ld_x + (long long)h * a.d;
      float x0[NU][V], x1[NU][V], y0[NU][V], y1[NU][V];
#pragma unroll
      for (int k = 0; k < NU; ++k) {
#pragma unroll
        for (int i = 0; i < V; ++i) x0[k][i] = x1[k][i] = y0[k][i] = y1[k][i] = 0.f;
        if (in && c0[k] < a.d) load<T, V>(x0[k], x + c0[k]);
        if (in && c1[k] < a.d) load<T, V>(x1[k], x + c1[k]);
        if constexpr (BACK) {
          const T* dy = DY + token * s.ld_dy + (long long)h * a.d;
          if (in && c0[k] < a.d) load<T, V>(y0[k], dy + c0[k]);
          if (in && c1[k] < a.d) load<T, V>(y1[k], dy + c1[k]);
        }
      }
      float sum = 0.f, mixed = 0.f;
#pragma unroll
      for (int k = 0; k < NU; ++k) {
        if constexpr (BACK) turn<V, true>(y0[k], y1[k], table, k * LANES + t, a.r, a.interleaved);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          sum = fmaf(x0[k][i], x0[k][i], fmaf(x1[k][i], x1[k][i], sum));
          if constexpr (BACK) mixed = fmaf(y0[k][i] * w0[k][i], x0[k][i], fmaf(y1[k][i] * w1[k][i], x1[k][i], mixed));
        }
      }
#pragma unroll
      for (int m = LANES / 2; m >= 1; m >>= 1) {
        sum += __shfl_xor_sync(0xffffffffu, sum, m);
        if constexpr (BACK) mixed += __shfl_xor_sync(0xffffffffu, mixed, m);
      }
      const float rstd = real ? rsqrtf(sum * over_d + a.eps) : 0.f;
      if constexpr (BACK) {
        const float pull = rstd * rstd * (mixed * over_d);
#pragma unroll
        for (int k = 0; k < NU; ++k)
#pragma unroll
          for (int i = 0; i < V; ++i) {
            if (in) {
              g0[k][i] = fmaf(y0[k][i], x0[k][i] * rstd, g0[k][i]);
              g1[k][i] = fmaf(y1[k][i], x1[k][i] * rstd, g1[k][i]);
            }
            y0[k][i] = rstd * (y0[k][i] * w0[k][i] - x0[k][i] * pull);
            y1[k][i] = rstd * (y1[k][i] * w1[k][i] - x1[k][i] * pull);
          }
      } else {
#pragma unroll
        for (int k = 0; k < NU; ++k) {
#pragma unroll
          for (int i = 0; i < V; ++i) {
            y0[k][i] = x0[k][i] * (rstd * w0[k][i]);
            y1[k][i] = x1[k][i] * (rstd * w1[k][i]);
          }
          turn<V, false>(y0[k], y1[k], table, k * LANES + t, a.r, a.interleaved);
        }
      }
      if (h < end) {
        T* y = BACK ? (T*)s.dx + token * s.ld_dx + (long long)h * a.d : (T*)s.y + token * s.ld_y + (long long)h * a.d;
#pragma unroll
        for (int k = 0; k < NU; ++k) {
          if (!real)
#pragma unroll
            for (int i = 0; i < V; ++i) y0[k][i] = y1[k][i] = 0.f;
          if (c0[k] < a.d) store<T, V>(y + c0[k], y0[k]);
          if (c1[k] < a.d) store<T, V>(y + c1[k], y1[k]);
        }
      }
    }
  }
  if constexpr (BACK) {   // the block's sums for the weight: heads side by side, then the warps
#pragma unroll
    for (int k = 0; k < NU; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) {
#pragma unroll
        for (int m = LANES; m < 32; m <<= 1) {
          g0[k][i] += __shfl_xor_sync(0xffffffffu, g0[k][i], m);
          g1[k][i] += __shfl_xor_sync(0xffffffffu, g1[k][i], m);
        }
        if (sub == 0 && c0[k] < a.d) joined[warp][c0[k] + i] = g0[k][i];
        if (sub == 0 && c1[k] < a.d) joined[warp][c1[k] + i] = g1[k][i];
      }
    __syncthreads();
    for (int c = tid; c < a.d; c += kThreads) {
      float g = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) g += joined[w][c];
      a.partial[(long long)blockIdx.x * a.d + c] = g;
    }
  }
}

// The blocks' sums: a block takes 32 features of one weight
template <class T>
__global__ void __launch_bounds__(1024) heads_weight_kernel(const __grid_constant__ HeadsArgs a, const __grid_constant__ HeadsPlan plan) {
  __shared__ float sums[32][33];
  const int lane = threadIdx.x & 31, group = threadIdx.x >> 5, c = blockIdx.x * 32 + lane, which = blockIdx.y;
  wait_for_predecessor();
  const HeadsSide& s = a.side[which];
  const float* rows = a.partial + (long long)(which ? plan.blocks[0] : 0) * a.d;
  float g = 0.f;
  if (c < a.d)
    for (int b = group; b < plan.blocks[which]; b += 32) g += rows[(long long)b * a.d + c];
  sums[group][lane] = g;
  __syncthreads();
  g = sums[lane][group];
#pragma unroll
  for (int m = 16; m >= 1; m >>= 1) g += __shfl_xor_sync(0xffffffffu, g, m);
  const int out = blockIdx.x * 32 + group;
  if (lane == 0 && out < a.d && s.dw) {
    if constexpr (sizeof(T) == 4) ((float*)s.dw)[out] = g;
    else ((__nv_bfloat16*)s.dw)[out] = __float2bfloat16_rn(g);
  }
}

// Blocks by the sides' shares of the heads.  Where there are fewer tokens than warps on the chip, several warps share a token's heads.
HeadsPlan plan_of(const HeadsArgs& a, int heads, int sms, int most) {
  HeadsPlan p{};
  const long long total = a.side[0].H + a.side[1].H;
  long long want[2];
  for (int i = 0; i < 2; ++i) {
    const int groups = (a.side[i].H + heads - 1) / heads;
    if (!groups) { p.parts[i] = 1; want[i] = 0; continue; }
    const long long warps = std::max<long long>(1, (long long)sms * kWarps * 2 * a.side[i].H / total);
    p.parts[i] = (int)std::min<long long>(groups, std::max<long long>(1, warps / std::max<long long>(1, a.tokens)));
    want[i] = (a.tokens * p.parts[i] + kWarps - 1) / kWarps;
  }
  for (int i = 0; i < 2; ++i) p.blocks[i] = (int)(want[i] ? std::max<long long>(1, std::min<long long>(want[i], (long long)most * a.side[i].H / total)) : 0);
  return p;
}

template <class T, int V, int LANES, int NU, bool BACK>
cudaError_t launch_one(const HeadsArgs& a, cudaStream_t stream) {
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess || (e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) return e;
  const HeadsPlan p = plan_of(a, 32 / LANES, sms, BACK ? std::min(kHeadsPartials, 2 * sms) : 8 * sms);
  if (p.blocks[0] + p.blocks[1] > 0) {
    if ((e = launch_early(qk_norm_rope_kernel<T, V, LANES, NU, BACK>, dim3(p.blocks[0] + p.blocks[1]), kThreads, 0, stream, a, p)) != cudaSuccess) return e;
    if ((e = launched()) != cudaSuccess) return e;
  }
  if constexpr (BACK) {
    if (!a.side[0].dw && !a.side[1].dw) return cudaSuccess;
    if ((e = launch_early(heads_weight_kernel<T>, dim3((a.d + 31) / 32, a.side[1].H ? 2 : 1), 1024, 0, stream, a, p)) != cudaSuccess) return e;
    return launched();
  }
  return cudaSuccess;
}

template <class T, int V, bool BACK>
cudaError_t launch_width(const HeadsArgs& a, cudaStream_t stream) {
  const int first = a.interleaved ? 0 : a.r / V, rest = a.d / V - 2 * first, units = first + (rest + 1) / 2;
  if constexpr (V == 1) {
    if (units <= 32) return launch_one<T, 1, 32, 1, BACK>(a, stream);
    return units <= 64 ? launch_one<T, 1, 32, 2, BACK>(a, stream) : launch_one<T, 1, 32, 4, BACK>(a, stream);
  } else {
    if (units <= 4) return launch_one<T, V, 4, 1, BACK>(a, stream);
    if (units <= 8) return launch_one<T, V, 8, 1, BACK>(a, stream);
    return units <= 16 ? launch_one<T, V, 16, 1, BACK>(a, stream) : launch_one<T, V, 32, 1, BACK>(a, stream);
  }
}

// The widest vectors that every tensor's rows and the pairs allow
template <class T, bool BACK>
cudaError_t launch_type(const HeadsArgs& a, cudaStream_t stream) {
  unsigned long long at = 0;
  auto add = [&](const void* p, long long ld) { at |= reinterpret_cast<unsigned long long>(p) | (unsigned long long)ld * sizeof(T); };
  for (const HeadsSide& s : a.side) {
    if (!s.H) continue;
    add(s.x, s.ld_x);
    add(s.w, 0);
    if (BACK) { add(s.dy, s.ld_dy); add(s.dx, s.ld_dx); }
    else add(s.y, s.ld_y);
  }
  auto fits = [&](int v) { return (at & (v * sizeof(T) - 1)) == 0 && a.d % v == 0 && (a.interleaved || a.r % v == 0); };
  if constexpr (sizeof(T) == 2)
    if (fits(8)) return launch_width<T, 8, BACK>(a, stream);
  if (fits(4)) return launch_width<T, 4, BACK>(a, stream);
  return launch_width<T, 1, BACK>(a, stream);
}

}  // namespace

cudaError_t launch_qk_norm_rope(const HeadsArgs& a, int dtype, cudaStream_t stream) {
  return dtype == TRI_INV_F32 ? launch_type<float, false>(a, stream) : launch_type<__nv_bfloat16, false>(a, stream);
}
cudaError_t launch_qk_norm_rope_backward(const HeadsArgs& a, int dtype, cudaStream_t stream) {
  return dtype == TRI_INV_F32 ? launch_type<float, true>(a, stream) : launch_type<__nv_bfloat16, true>(a, stream);
}

}  // namespace tri_inv
