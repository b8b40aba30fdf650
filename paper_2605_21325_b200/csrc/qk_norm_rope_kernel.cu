// Norm of each query and key head with the position rotation, and its gradient.
//     y = R(p f) (x rstd w),   rstd = 1 / sqrt(mean x^2 + eps);   R turns the pairs of the first 2 r features by the angles p f_i
//     v = R(-p f) dy,  u = v w,  dx = rstd (u - x rstd^2 mean(u x)),  dw = sum over tokens and heads of v x rstd
//
// A head is held by LANES lanes, a lane has the two halves of its pairs (two vectors of V values), so that the rotation stays in registers and the mean takes log2 LANES exchanges; a warp
// holds 32 / LANES heads of one token at a time and goes through the token's heads with one table of sines and cosines.
// A warp's next three steps are on their way to shared memory, each lane's vectors to a place of its own, so that nothing waits at a barrier and no register holds what is not there yet.
// What bounds it: bytes (4 x 4096 tokens x 32 heads of 128, bf16 46 us, 0.90 of a copy's rate; the gradient 67 us, 0.93; fp32 0.86), at 69 and 63 % of the issue slots; d = 64 0.82 and 0.74, d = 256 0.79 and 0.70.
// On the way, forward and gradient: loads straight to registers 68 and 122 us;
// copies ahead, but a table whose lanes met in the banks 143 and 205; the table turned 62 and 144; two features an instruction and pointers that step 52 and 109; three and two blocks an SM instead of four and three, so that nothing spills
// 46 and 68.  Heads whose d or pairs are not whole 16-byte vectors go by four values (d = 96, 20 pairs: 0.44 and 0.39)
// or by single ones (d = 120, 59 pairs: 0.22 and 0.17): the pairs' distance sets the width of the loads too.  One query and one key head a token: 0.29 and 0.34, each side works out the token's angles.  Eight tokens of 32 heads 3.2 us on the device.
// Angles: p f / 2 pi only counts modulo 1, so f / 2 pi is kept as a 64-bit fraction F (of any finite f: fraction()) and p F modulo 2^64 is the exact product's fraction, off by 3 p units (2^-31 of a turn) at most: a position of 2^31 is as good as one of 1.
#include <algorithm>

#include "qk_norm_rope.cuh"

namespace tri_inv {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kTable = kHeadsMaxDim / 2;   // angles of a token

// Two fp32 numbers that the arithmetic takes at a time: a pair of features
struct Pair { unsigned long long v; };
__device__ __forceinline__ Pair pair(float x, float y) { Pair d; asm("mov.b64 %0, {%1, %2};" : "=l"(d.v) : "f"(x), "f"(y)); return d; }
__device__ __forceinline__ float2 both(Pair a) { float2 d; asm("mov.b64 {%0, %1}, %2;" : "=f"(d.x), "=f"(d.y) : "l"(a.v)); return d; }
__device__ __forceinline__ Pair mul2(Pair a, Pair b) { Pair d; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d.v) : "l"(a.v), "l"(b.v)); return d; }
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) { Pair d; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d.v) : "l"(a.v), "l"(b.v), "l"(c.v)); return d; }
__device__ __forceinline__ Pair twice(float x) { return pair(x, x); }

// V values as they lie in memory
template <class T, int V> struct Vec;
template <> struct Vec<__nv_bfloat16, 8> { using Raw = uint4; };
template <> struct Vec<__nv_bfloat16, 4> { using Raw = uint2; };
template <> struct Vec<__nv_bfloat16, 1> { using Raw = uint16_t; };
template <> struct Vec<float, 4> { using Raw = uint4; };
template <> struct Vec<float, 1> { using Raw = uint32_t; };
// A lane's unit is two vectors, which hold the first and the second features of V pairs: halves of the head's turned part, or, interleaved, neighbours.  U and W are those features, in twos (one and a zero where V is 1).
template <int V> constexpr int kTwos = V == 1 ? 1 : V / 2;
template <class T, int V>
__device__ __forceinline__ float at(typename Vec<T, V>::Raw raw, int i) {
  if constexpr (sizeof(T) == 4) {
    return reinterpret_cast<const float*>(&raw)[i];
  } else if constexpr (V == 1) {
    return __uint_as_float((uint32_t)raw << 16);
  } else {
    const uint32_t u = reinterpret_cast<const uint32_t*>(&raw)[i / 2];
    return __uint_as_float(i & 1 ? u & 0xffff0000u : u << 16);
  }
}
template <class T, int V, bool INTER>
__device__ __forceinline__ void widen(Pair (&U)[kTwos<V>], Pair (&W)[kTwos<V>], typename Vec<T, V>::Raw a, typename Vec<T, V>::Raw b) {
  if constexpr (V == 1) {
    U[0] = pair(at<T, V>(a, 0), 0.f);
    W[0] = pair(at<T, V>(b, 0), 0.f);
  } else if constexpr (INTER) {   // pairs 0 .. V / 2 - 1 are in a, the others in b
#pragma unroll
    for (int j = 0; j < V / 2; ++j) {
      const auto raw = j < V / 4 ? a : b;
      const int i = 4 * j % V;
      U[j] = pair(at<T, V>(raw, i), at<T, V>(raw, i + 2));
      W[j] = pair(at<T, V>(raw, i + 1), at<T, V>(raw, i + 3));
    }
  } else {
#pragma unroll
    for (int j = 0; j < V / 2; ++j) {
      U[j] = pair(at<T, V>(a, 2 * j), at<T, V>(a, 2 * j + 1));
      W[j] = pair(at<T, V>(b, 2 * j), at<T, V>(b, 2 * j + 1));
    }
  }
}
// ... and back, as values in the order of memory
template <int V, bool INTER>
__device__ __forceinline__ void spread(float (&a)[V], float (&b)[V], const Pair (&U)[kTwos<V>], const Pair (&W)[kTwos<V>]) {
  if constexpr (V == 1) {
    a[0] = both(U[0]).x;
    b[0] = both(W[0]).x;
  } else {
#pragma unroll
    for (int j = 0; j < V / 2; ++j) {
      const float2 u = both(U[j]), w = both(W[j]);
      if constexpr (INTER) {
        float* to = j < V / 4 ? a : b;
        const int i = 4 * j % V;
        to[i] = u.x; to[i + 1] = w.x; to[i + 2] = u.y; to[i + 3] = w.y;
      } else {
        a[2 * j] = u.x; a[2 * j + 1] = u.y; b[2 * j] = w.x; b[2 * j + 1] = w.y;
      }
    }
  }
}
template <class T, int V>
__device__ __forceinline__ void store(T* p, const float (&from)[V]) {
  typename Vec<T, V>::Raw raw;
  if constexpr (sizeof(T) == 4) {
    float* f = reinterpret_cast<float*>(&raw);
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = from[i];
  } else if constexpr (V == 1) {
    const __nv_bfloat16 x = __float2bfloat16_rn(from[0]);
    raw = reinterpret_cast<const uint16_t&>(x);
  } else {
    uint32_t* u = reinterpret_cast<uint32_t*>(&raw);
#pragma unroll
    for (int i = 0; i < V; i += 2) {
      const __nv_bfloat162 x = __floats2bfloat162_rn(from[i], from[i + 1]);
      u[i / 2] = reinterpret_cast<const uint32_t&>(x);
    }
  }
  *reinterpret_cast<typename Vec<T, V>::Raw*>(p) = raw;
}

// Asks for a vector of a lane's own, to a place in shared memory that only this lane reads; where it does not exist it reads as zero.  (Single 16-bit values go through a register.)
template <class T, int V>
__device__ __forceinline__ void request(typename Vec<T, V>::Raw* to, const T* from, const T* any, bool in) {
  constexpr int BYTES = V * (int)sizeof(T);
  if constexpr (BYTES == 2) {
    *to = in ? *reinterpret_cast<const uint16_t*>(from) : (uint16_t)0;
  } else {
    const uint32_t at = (uint32_t)__cvta_generic_to_shared(to);
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(at), "l"(in ? from : any), "r"(in ? 16 : 0) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(at), "l"(in ? from : any), "n"(BYTES), "r"(in ? BYTES : 0) : "memory");
  }
}

// Steps of a warp in shared memory: of `bytes` a lane, tensor and half
__host__ __device__ constexpr int steps(int bytes, bool back) { return bytes >= 16 || back ? 4 : 6; }

// f / 2 pi modulo 1 in units of 2^-64, off by less than three of them.  1 / 2 pi (203 bits by Machin's formula) lies in pieces of 29 bits, so that each one's product with f's 24 bits is exact in fp64, and so is what
// it has above a whole number; the fractions are summed as integers.  Small frequencies need the first two or three pieces.
__device__ __forceinline__ unsigned long long fraction(float f) {
  constexpr double PIECES[7] = {85445659.0, 240010261.0, 88048874.0, 524801235.0, 249589169.0, 156865476.0, 119571452.0};
  const double x = fabs((double)f);
  unsigned long long sum = 0;
  double scale = 0x1p-29;
#pragma unroll
  for (int k = 0; k < 7; ++k, scale *= 0x1p-29) {
    if (k > 1 && x * scale < 0x1p-93) break;   // times a piece below 2^29 it is no whole unit
    const double y = x * (PIECES[k] * scale);
    sum += (unsigned long long)((y - floor(y)) * 0x1p64);
  }
  return f < 0.f ? 0 - sum : sum;
}

// The first features of the two vectors of unit p of `units`, >= d where the head has none.  Where the pairs are (i, i + r) the first r / V units are pairs of vectors, and the others two of the rest; interleaved a
// vector holds its pairs and any two will do.  Vectors of neighbouring lanes lie side by side: with two neighbouring vectors to a lane each access would use half of what it fetches (32768 tokens of 40 heads, interleaved, 174 -> 125 us).
template <int V, bool INTER>
__device__ __forceinline__ void columns(int p, int r, int d, int units, int& c0, int& c1) {
  if (p >= units) {
    c0 = c1 = d;
  } else if (INTER && V == 1) {   // a pair
    c0 = 2 * p;
    c1 = c0 + 1;
  } else if (INTER) {
    c0 = p * V;
    c1 = c0 + units * V;
  } else {
    const bool pairs = p * V < r;
    c0 = pairs ? p * V : p * V + r;
    c1 = c0 + (pairs ? r : units * V - r);
  }
}
// Where pair f's angle belongs: which unit, which of its V pairs
template <int V, bool INTER>
__device__ __forceinline__ void unit_of(int f, int units, int& p, int& i) {
  if (INTER && V > 1) {
    constexpr int HALF = V / 2 > 0 ? V / 2 : 1;
    const int q = f / HALF;
    p = q < units ? q : q - units;
    i = f % HALF + (q < units ? 0 : HALF);
  } else {
    p = f / V;
    i = f % V;
  }
}

// Turns two pairs by cs = (cos, cos', sin, sin')
__device__ __forceinline__ void turn(Pair& u, Pair& w, float4 cs) {
  const Pair c = pair(cs.x, cs.y), x = u;
  u = fma2(u, c, mul2(w, pair(-cs.z, -cs.w)));
  w = fma2(w, c, mul2(x, pair(cs.z, cs.w)));
}

struct HeadsPlan {
  int blocks[2];       // of queries and of keys
  int parts[2];        // warps that share a token's heads
  int group[2];        // tokens that share a warp, where they have few heads (parts is 1 then)
};
// Where a warp stands: HEADS heads of a token at a time, `left` of them in all to go
struct At {
  long long item;
  int left;
  const char *x, *dy;   // of the lane's head
};

// NU: units of a lane.  A warp's next STEPS - 1 steps are on their way to shared memory while it works on one.
template <class T, int V, int LANES, int NU, bool BACK, bool INTER, bool GROUP>
__global__ void __launch_bounds__(kThreads, BACK ? 2 : 3) qk_norm_rope_kernel(const __grid_constant__ HeadsArgs a, const __grid_constant__ HeadsPlan plan) {
  using Raw = typename Vec<T, V>::Raw;
  constexpr int HEADS = 32 / LANES, N = kTwos<V>, UNITS = LANES * NU, es = sizeof(T);
  constexpr int STEPS = steps(V * es * NU, BACK), TENSORS = BACK ? 2 : 1;
  extern __shared__ __align__(16) unsigned char dynamic[];
  __shared__ unsigned long long freq[kTable];
  __shared__ int places[kWarps][STEPS][HEADS];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, sub = lane / LANES, t = lane % LANES;
  float4* table = reinterpret_cast<float4*>(dynamic) + warp * kTable;   // of angles 2 j, 2 j + 1 of unit p at [j][p], so that the lanes of a head read side by side
  Raw* ring = reinterpret_cast<Raw*>(dynamic + kWarps * kTable * sizeof(float4)) + warp * STEPS * TENSORS * NU * 2 * 32 + lane;
  const int which = (int)blockIdx.x >= plan.blocks[0], block = blockIdx.x - (which ? plan.blocks[0] : 0);
  const HeadsSide& s = a.side[which];
  const T *X = (const T*)s.x, *W = (const T*)s.w, *DY = (const T*)s.dy;
  wait_for_predecessor();

  const int parts = plan.parts[which], per = ((s.H + HEADS - 1) / HEADS + parts - 1) / parts * HEADS;   // heads of a part
  const int group = GROUP ? plan.group[which] : 1, mine = group > 1 ? sub / s.H : 0;   // mine: the lane's token among those of the warp
  const long long items = group > 1 ? (a.tokens + group - 1) / group : a.tokens * parts, stride = (long long)plan.blocks[which] * kWarps;
  auto token_of = [&](long long item) { return parts == 1 ? item : item / parts; };
  auto first_of = [&](long long item) { return parts == 1 ? 0 : (int)(item - item / parts * parts) * per; };
  auto place = [&](At& p) {   // an item's first step; items without heads (a token's last part may have none) are passed over
    if (group > 1) {   // one step, whose `left` says whether the lane has a head in it
      const long long token = p.item * group + mine;
      p.left = mine < group && token < a.tokens ? HEADS : sub;
      p.x = (const char*)(X + token * s.ld_x + (long long)(sub - mine * s.H) * a.d);
      if (BACK) p.dy = (const char*)(DY + token * s.ld_dy + (long long)(sub - mine * s.H) * a.d);
      return;
    }
    for (;; p.item += stride) {
      if (p.item >= items) return;
      const int h = first_of(p.item);
      p.left = min(s.H - h, per);
      if (p.left <= 0) continue;
      const long long token = token_of(p.item);
      p.x = (const char*)(X + token * s.ld_x + (long long)(h + sub) * a.d);
      if (BACK) p.dy = (const char*)(DY + token * s.ld_dy + (long long)(h + sub) * a.d);
      return;
    }
  };
  const int step_bytes = HEADS * a.d * es;
  int c0[NU], c1[NU];
#pragma unroll
  for (int k = 0; k < NU; ++k) columns<V, INTER>(k * LANES + t, a.r, a.d, a.units, c0[k], c1[k]);
  // Asks for the step at p, and goes on to the next
  auto ask = [&](At& p, int slot, bool fresh) {
    if (p.item < items) {
      const long long token = group > 1 ? p.item * group + lane : token_of(p.item);
      if (fresh && lane < group && token < a.tokens) {
        if (a.positions) asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"((uint32_t)__cvta_generic_to_shared(&places[warp][slot][lane])), "l"(a.positions + token) : "memory");
        else places[warp][slot][lane] = (int)(token % a.T);
      }
#pragma unroll
      for (int k = 0; k < NU; ++k) {
        Raw* to = ring + (slot * NU + k) * TENSORS * 2 * 32;
        const bool i0 = sub < p.left && c0[k] < a.d, i1 = sub < p.left && c1[k] < a.d;
        request<T, V>(to, (const T*)p.x + c0[k], X, i0);
        request<T, V>(to + 32, (const T*)p.x + c1[k], X, i1);
        if constexpr (BACK) {
          request<T, V>(to + 64, (const T*)p.dy + c0[k], DY, i0);
          request<T, V>(to + 96, (const T*)p.dy + c1[k], DY, i1);
        }
      }
      p.left -= HEADS;
      p.x += step_bytes;
      if (BACK) p.dy += step_bytes;
      if (p.left <= 0) {
        p.item += stride;
        place(p);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  At ahead;
  ahead.item = (long long)block * kWarps + warp;
  place(ahead);
  At now = ahead;
  long long asked = -1;   // the item whose position has been asked for
#pragma unroll
  for (int i = 0; i < STEPS - 1; ++i) {
    const long long item = ahead.item;
    ask(ahead, i, item != asked);
    asked = item;
  }

  for (int i = tid; i < a.r; i += kThreads) freq[i] = fraction(a.inv_freq[i]);
  auto angle = [&](int f) {   // its cosine; its sine is two further on
    int p, i;
    unit_of<V, INTER>(f, a.units, p, i);
    return reinterpret_cast<float*>(table) + (i / 2 * UNITS + p) * 4 + i % 2;
  };
  for (int i = lane; i < group * N * UNITS; i += 32) table[i] = make_float4(1.f, 1.f, 0.f, 0.f);   // what is not turned stays so
  Pair wu[NU][N], ww[NU][N], gu[BACK ? NU : 1][N], gw[BACK ? NU : 1][N];
#pragma unroll
  for (int k = 0; k < NU; ++k) {
    Raw raw[2];
    T* v = reinterpret_cast<T*>(raw);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      v[i] = W && c0[k] < a.d ? W[c0[k] + i] : T(1.f);
      v[V + i] = W && c1[k] < a.d ? W[c1[k] + i] : T(1.f);
    }
    widen<T, V, INTER>(wu[k], ww[k], raw[0], raw[1]);
    if constexpr (BACK)
#pragma unroll
      for (int j = 0; j < N; ++j) gu[k][j] = gw[k][j] = twice(0.f);
  }
  __syncthreads();

  const float over_d = 1.f / (float)a.d;
  const float4* turns_of = table + (mine < group ? mine : 0) * N * UNITS + t;   // of the lane's token
  T* to = nullptr;
  bool real = false, fresh = true;   // fresh: the step is its item's first
  for (int slot = 0; now.item < items; slot = slot + 1 == STEPS ? 0 : slot + 1) {
    {
      const long long item = ahead.item;
      ask(ahead, slot == 0 ? STEPS - 1 : slot - 1, item != asked);
      asked = item;
    }
    asm volatile("cp.async.wait_group %0;" ::"n"(STEPS - 1) : "memory");
    if (fresh) {
      const long long token = group > 1 ? now.item * group + mine : token_of(now.item);
      to = (BACK ? (T*)s.dx + token * s.ld_dx : (T*)s.y + token * s.ld_y) + (long long)(group > 1 ? sub - mine * s.H : first_of(now.item) + sub) * a.d;
      __syncwarp();
      real = mine < group && places[warp][slot][mine] >= 0;
      for (int q = 0; q < group; ++q) {
        const unsigned position = (unsigned)places[warp][slot][q];
        for (int f = lane; f < a.r; f += 32) {
          const int turns = (int)(((unsigned long long)position * freq[f]) >> 32);   // of 2^-32 of a whole one, signed
          float sn, cs;
          sincospif((float)turns * 4.656612873077393e-10f, &sn, &cs);   // 2^-31
          angle(f)[4 * q * N * UNITS] = cs;
          angle(f)[4 * q * N * UNITS + 2] = BACK ? -sn : sn;
        }
      }
      __syncwarp();
    }
    Pair xu[NU][N], xw[NU][N], yu[NU][N], yw[NU][N], sum = twice(0.f), mixed = twice(0.f);
#pragma unroll
    for (int k = 0; k < NU; ++k) {
      const Raw* from = ring + (slot * NU + k) * TENSORS * 2 * 32;
      widen<T, V, INTER>(xu[k], xw[k], from[0], from[32]);
      if constexpr (BACK) widen<T, V, INTER>(yu[k], yw[k], from[64], from[96]);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        sum = fma2(xu[k][j], xu[k][j], fma2(xw[k][j], xw[k][j], sum));
        if constexpr (BACK) {
          turn(yu[k][j], yw[k][j], turns_of[j * UNITS + k * LANES]);
          mixed = fma2(mul2(yu[k][j], wu[k][j]), xu[k][j], fma2(mul2(yw[k][j], ww[k][j]), xw[k][j], mixed));
        }
      }
    }
    float total = both(sum).x + both(sum).y, mix = BACK ? both(mixed).x + both(mixed).y : 0.f;
#pragma unroll
    for (int m = LANES / 2; m >= 1; m >>= 1) {
      total += __shfl_xor_sync(0xffffffffu, total, m);
      if constexpr (BACK) mix += __shfl_xor_sync(0xffffffffu, mix, m);
    }
    const float rstd = rsqrtf(total * over_d + a.eps);
    // (the mean first: rstd^3 alone is no normal number beyond heads of 1e-13 to 1e12, where dx is)
    const Pair rstd2 = twice(rstd), pull = twice(-(mix * over_d * rstd) * rstd * rstd);
    const bool in = sub < now.left;
#pragma unroll
    for (int k = 0; k < NU; ++k) {
#pragma unroll
      for (int j = 0; j < N; ++j) {
        if constexpr (BACK) {
          if (in && real) {
            gu[k][j] = fma2(yu[k][j], mul2(xu[k][j], rstd2), gu[k][j]);
            gw[k][j] = fma2(yw[k][j], mul2(xw[k][j], rstd2), gw[k][j]);
          }
          yu[k][j] = fma2(xu[k][j], pull, mul2(mul2(yu[k][j], wu[k][j]), rstd2));
          yw[k][j] = fma2(xw[k][j], pull, mul2(mul2(yw[k][j], ww[k][j]), rstd2));
        } else {
          yu[k][j] = mul2(xu[k][j], mul2(rstd2, wu[k][j]));
          yw[k][j] = mul2(xw[k][j], mul2(rstd2, ww[k][j]));
          turn(yu[k][j], yw[k][j], turns_of[j * UNITS + k * LANES]);
        }
      }
      float v0[V], v1[V];
      spread<V, INTER>(v0, v1, yu[k], yw[k]);
      if (!real)
#pragma unroll
        for (int i = 0; i < V; ++i) v0[i] = v1[i] = 0.f;
      if (in && c0[k] < a.d) store<T, V>(to + c0[k], v0);
      if (in && c1[k] < a.d) store<T, V>(to + c1[k], v1);
    }
    now.left -= HEADS;
    to += HEADS * a.d;
    fresh = now.left <= 0;
    if (fresh) {
      now.item += stride;
      place(now);
    }
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  if constexpr (BACK) {   // the block's sums for the weight: heads side by side, then the warps
    __syncthreads();
    float* joined = reinterpret_cast<float*>(dynamic);   // [kWarps][kHeadsMaxDim], in place of the tables
#pragma unroll
    for (int k = 0; k < NU; ++k) {
#pragma unroll
      for (int j = 0; j < N; ++j) {
        float2 u = both(gu[k][j]), w = both(gw[k][j]);
#pragma unroll
        for (int m = LANES; m < 32; m <<= 1) {
          u.x += __shfl_xor_sync(0xffffffffu, u.x, m);
          u.y += __shfl_xor_sync(0xffffffffu, u.y, m);
          w.x += __shfl_xor_sync(0xffffffffu, w.x, m);
          w.y += __shfl_xor_sync(0xffffffffu, w.y, m);
        }
        gu[k][j] = pair(u.x, u.y);
        gw[k][j] = pair(w.x, w.y);
      }
      float v0[V], v1[V];
      spread<V, INTER>(v0, v1, gu[k], gw[k]);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        if (sub == 0 && c0[k] < a.d) joined[warp * kHeadsMaxDim + c0[k] + i] = v0[i];
        if (sub == 0 && c1[k] < a.d) joined[warp * kHeadsMaxDim + c1[k] + i] = v1[i];
      }
    }
    __syncthreads();
    for (int c = tid; c < a.d; c += kThreads) {
      float sum = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) sum += joined[w * kHeadsMaxDim + c];
      a.partial[(long long)blockIdx.x * a.d + c] = sum;
    }
  }
}

// The blocks' sums: a block takes 32 features of one weight (of a side without heads there are none: zero)
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

// Blocks by the sides' shares of the work, a token's angles counted as three steps.  Where there are fewer tokens than warps on the chip, several warps share a token's heads; where a token has at most half as many
// heads as a warp holds, a warp takes several tokens.
HeadsPlan plan_of(const HeadsArgs& a, int heads, int sms, int most) {
  HeadsPlan p{};
  long long want[2], work[2];
  for (int i = 0; i < 2; ++i) {
    const int H = a.side[i].H, steps = (H + heads - 1) / heads;
    p.parts[i] = p.group[i] = 1;
    want[i] = work[i] = 0;
    if (!H) continue;
    if (H <= heads / 2) {
      p.group[i] = heads / H;
      work[i] = (1 + 3 * p.group[i]) * 12 / p.group[i];
      want[i] = ((a.tokens + p.group[i] - 1) / p.group[i] + kWarps - 1) / kWarps;
    } else {
      const long long warps = (long long)sms * kWarps;
      p.parts[i] = (int)std::min<long long>(steps, std::max<long long>(1, warps / std::max<long long>(1, a.tokens)));
      work[i] = (steps + 3) * 12;
      want[i] = (a.tokens * p.parts[i] + kWarps - 1) / kWarps;
    }
  }
  for (int i = 0; i < 2; ++i) p.blocks[i] = (int)(want[i] ? std::max<long long>(1, std::min<long long>(want[i], most * work[i] / (work[0] + work[1]))) : 0);
  return p;
}

template <class T, int V, int LANES, int NU, bool BACK, bool INTER, bool GROUP>
cudaError_t launch_kernel(const HeadsArgs& a, cudaStream_t stream) {
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess || (e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) return e;
  constexpr size_t smem = (size_t)kWarps * (kTable * sizeof(float4) + (size_t)steps(V * (int)sizeof(T) * NU, BACK) * (BACK ? 2 : 1) * NU * 2 * 32 * V * sizeof(T));
  if ((e = allow_shared<qk_norm_rope_kernel<T, V, LANES, NU, BACK, INTER, GROUP>>(smem)) != cudaSuccess) return e;
  const HeadsPlan p = plan_of(a, 32 / LANES, sms, BACK ? std::min(kHeadsPartials - 1, 2 * sms) : 3 * sms);
  if (p.blocks[0] + p.blocks[1] > 0) {
    if ((e = launch_early(qk_norm_rope_kernel<T, V, LANES, NU, BACK, INTER, GROUP>, dim3(p.blocks[0] + p.blocks[1]), kThreads, smem, stream, a, p)) != cudaSuccess) return e;
    if ((e = launched()) != cudaSuccess) return e;
  }
  if constexpr (BACK) {
    if (!a.side[0].dw && !a.side[1].dw) return cudaSuccess;
    if ((e = launch_early(heads_weight_kernel<T>, dim3((a.d + 31) / 32, a.side[1].dw ? 2 : 1), 1024, 0, stream, a, p)) != cudaSuccess) return e;
    return launched();
  }
  return cudaSuccess;
}

template <class T, int V, int LANES, int NU, bool BACK, bool INTER>
cudaError_t launch_one(const HeadsArgs& a, cudaStream_t stream) {
  if constexpr (LANES < 32)
    for (const HeadsSide& s : a.side)
      if (s.H && s.H <= 32 / LANES / 2) return launch_kernel<T, V, LANES, NU, BACK, INTER, true>(a, stream);
  return launch_kernel<T, V, LANES, NU, BACK, INTER, false>(a, stream);
}

template <class T, int V, bool BACK, bool INTER>
cudaError_t launch_width(HeadsArgs a, cudaStream_t stream) {
  const int first = INTER ? 0 : a.r / V, rest = a.d / V - 2 * first, units = first + (rest + 1) / 2;
  a.units = units;
  if constexpr (V == 1) {
    if (units <= 32) return launch_one<T, 1, 32, 1, BACK, INTER>(a, stream);
    return units <= 64 ? launch_one<T, 1, 32, 2, BACK, INTER>(a, stream) : launch_one<T, 1, 32, 4, BACK, INTER>(a, stream);
  } else {
    if (units <= 4) return launch_one<T, V, 4, 1, BACK, INTER>(a, stream);
    if (units <= 8) return launch_one<T, V, 8, 1, BACK, INTER>(a, stream);
    if constexpr (V == 8) return launch_one<T, V, 16, 1, BACK, INTER>(a, stream);
    else return units <= 16 ? launch_one<T, V, 16, 1, BACK, INTER>(a, stream) : launch_one<T, V, 32, 1, BACK, INTER>(a, stream);
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
    if (fits(8)) return a.interleaved ? launch_width<T, 8, BACK, true>(a, stream) : launch_width<T, 8, BACK, false>(a, stream);
  if (fits(4)) return a.interleaved ? launch_width<T, 4, BACK, true>(a, stream) : launch_width<T, 4, BACK, false>(a, stream);
  return a.interleaved ? launch_width<T, 1, BACK, true>(a, stream) : launch_width<T, 1, BACK, false>(a, stream);
}

}  // namespace

cudaError_t launch_qk_norm_rope(const HeadsArgs& a, int dtype, cudaStream_t stream) {
  return dtype == TRI_INV_F32 ? launch_type<float, false>(a, stream) : launch_type<__nv_bfloat16, false>(a, stream);
}
cudaError_t launch_qk_norm_rope_backward(const HeadsArgs& a, int dtype, cudaStream_t stream) {
  return dtype == TRI_INV_F32 ? launch_type<float, true>(a, stream) : launch_type<__nv_bfloat16, true>(a, stream);
}

}  // namespace tri_inv
