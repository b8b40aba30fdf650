// Gated linear recurrence: the gradient's walk, from the last tile to the first.
#include <algorithm>

#include "gated_recurrence.cuh"

namespace tri_inv {
namespace {

constexpr int kWarps = 8, kTok = kRecTile / kWarps, kThreads = 32 * kWarps;
constexpr int kStageBytes = 3 * kRecTile * kRecRow;
constexpr size_t kSmem = 2 * (size_t)kStageBytes;

template <class T, int MODE, bool WORDS>
__global__ void __launch_bounds__(kThreads, 3) gated_recurrence_backward_kernel(const __grid_constant__ RecArgs a) {
  constexpr int N = RecLane<T>::N, CH = kRecRow / (int)sizeof(T);
  extern __shared__ __align__(128) unsigned char stages[];
  __shared__ __align__(16) float2 part[kWarps][CH];   // (P, H) of each warp's tokens
  __shared__ __align__(8) float back[kWarps][CH];     // what reaches the token in front of them, where nothing reaches them from behind
  __shared__ __align__(8) float entry[CH];            // what reaches the tile from behind
  __shared__ int drawn;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const T *X = (const T*)a.x, *G = (const T*)a.g, *DY = (const T*)a.dy;
  const int items = a.n_segs * a.cols;
  const int x_access = rec_access<T>(X, a.ld_x), g_access = rec_access<T>(G, a.ld_g), dy_access = rec_access<T>(DY, a.ld_dy);
  const bool dx_pairs = rec_access<T>(a.dx, a.ld_dx) != kRecSingle, dg_pairs = rec_access<T>(a.dg, a.ld_dg) != kRecSingle;
  const unsigned long long limit = a.wait_limit_ns ? a.wait_limit_ns : 2000000000ull;
  wait_for_predecessor();

  auto request = [&](const RecAt& t, int stage) {
    if (t.item < items) {
      const int first = warp * kTok, rows = t.n() - first;
      unsigned char* at = stages + stage * kStageBytes + first * kRecRow;
      rec_request<T, kTok>(at, X, a.ld_x, t.tok0() + first, rows, t.col * CH, a.D, x_access);
      rec_request<T, kTok>(at + kRecTile * kRecRow, G, a.ld_g, t.tok0() + first, rows, t.col * CH, a.D, g_access);
      rec_request<T, kTok>(at + 2 * kRecTile * kRecRow, DY, a.ld_dy, t.tok0() + first, rows, t.col * CH, a.D, dy_access);
    }
    rec_commit();
  };
  int ahead = 0;
  if (WORDS) {
    if (tid == 0) drawn = (int)atomicAdd(a.ticket, 2u);
    __syncthreads();
    ahead = drawn + 1;
  }
  RecAt now = rec_decode<WORDS>(a, WORDS ? ahead - 1 : (int)blockIdx.x, true);
  request(now, 0);
  float carried = 0.f;
  for (int stage = 0; now.item < items; stage ^= 1) {
    const RecAt next = rec_next<WORDS>(a, now, ahead, true);
    request(next, stage ^ 1);
    int ticket = 0;
    if (WORDS && tid == 0) ticket = (int)atomicAdd(a.ticket, 1u);
    const int n = now.n(), c0 = now.col * CH, left = n - warp * kTok;
    const long long slot = rec_slot(now.begin, now.seq) + now.index;
    float h[N];   // the state in front of the tile
    {
      const float* from = now.index > 0 ? a.carries + (slot - 1) * a.D : a.h0 ? a.h0 + (long long)now.seq * a.D : nullptr;
#pragma unroll
      for (int j = 0; j < N; ++j) h[j] = from && c0 + lane * N + j < a.D ? from[c0 + lane * N + j] : 0.f;
    }
    rec_wait<1>();
    __syncwarp();
    const unsigned char* sx = stages + stage * kStageBytes + warp * kTok * kRecRow + 4 * lane;
    auto read = [&](float (&v)[N], int tensor, int t) { RecLane<T>::widen(v, *reinterpret_cast<const uint32_t*>(sx + (tensor * kRecTile + t) * kRecRow)); };
    float av[kTok][N], mv[kTok][N], wv[kTok][N], P[N], H[N], C[N];
#pragma unroll
    for (int j = 0; j < N; ++j) { P[j] = 1.f; H[j] = 0.f; C[j] = 0.f; }
#pragma unroll
    for (int t = 0; t < kTok; ++t) {
      float x[N], g[N], over;
      read(x, 0, t);
      read(g, 1, t);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        rec_factors<MODE>(g[j], av[t][j], mv[t][j], over);
        if (t >= left) { av[t][j] = 1.f; mv[t][j] = 0.f; }
        wv[t][j] = MODE == kRecNormed ? av[t][j] * over * x[j] : x[j];   // beside the state: what w takes from it
        P[j] *= av[t][j];
        H[j] = rec_step(av[t][j], H[j], mv[t][j] * x[j]);
      }
    }
#pragma unroll
    for (int t = kTok - 1; t >= 0; --t) {
      float dy[N];
      read(dy, 2, t);
#pragma unroll
      for (int j = 0; j < N; ++j) C[j] = av[t][j] == 0.f ? 0.f : av[t][j] * (C[j] + dy[j]);
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
      part[warp][lane * N + j] = make_float2(P[j], H[j]);
      back[warp][lane * N + j] = C[j];
    }
    __syncthreads();
    float q_back = 0.f;
    if (tid < CH) {   // a channel of the tile: its word goes out first
      float TP = 1.f, TC = 0.f;
#pragma unroll
      for (int w = kWarps - 1; w >= 0; --w) {
        const float p = part[w][tid].x;
        TP *= p;
        TC = rec_step(p, TC, back[w][tid]);
      }
      const int c = c0 + tid;
      const bool first = now.index == 0, last = now.index + 1 == now.tiles;
      unsigned long long* word = WORDS ? a.words + slot * a.D + c : nullptr;
      if (c < a.D) {
        if (last) q_back = a.dh ? a.dh[(long long)now.seq * a.D + c] : 0.f;
        else if (!WORDS) q_back = carried;
        else {
          if (!first) rec_post(word, TP, TC);
          q_back = rec_look_back(word + a.D, -(long long)a.D, now.tiles - 1 - now.index, limit, a.status);
        }
        carried = rec_step(TP, q_back, TC);
        if (first) { if (a.dh0) a.dh0[(long long)now.seq * a.D + c] = carried; }
        else if (WORDS) rec_post(word, 0.f, carried);
      }
      entry[tid] = q_back;
    }
    // the state in front of the warp's tokens, and what reaches it from the warps behind it
#pragma unroll
    for (int j = 0; j < N; ++j) { P[j] = 1.f; C[j] = 0.f; }
    for (int w = 0; w < warp; ++w)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float2 q = part[w][lane * N + j];
        h[j] = rec_step(q.x, h[j], q.y);
      }
    for (int w = kWarps - 1; w > warp; --w)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float p = part[w][lane * N + j].x;
        P[j] *= p;
        C[j] = rec_step(p, C[j], back[w][lane * N + j]);
      }
#pragma unroll
    for (int t = 0; t < kTok; ++t) {
      float x[N];
      read(x, 0, t);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float av_ = av[t][j];
        float w;
        if constexpr (MODE == kRecDecay) w = av_ * h[j];
        else if constexpr (MODE == kRecNormed) w = av_ * (h[j] - wv[t][j]);
        else w = (h[j] - x[j]) * (av_ * mv[t][j]);
        wv[t][j] = av_ == 0.f ? 0.f : w;
        h[j] = rec_step(av_, h[j], mv[t][j] * x[j]);
      }
    }
    if (WORDS && tid == 0) drawn = ticket;
    __syncthreads();
    if (WORDS) ahead = drawn;
#pragma unroll
    for (int j = 0; j < N; ++j) C[j] = rec_step(P[j], entry[lane * N + j], C[j]);
    T* dx_row = (T*)a.dx + (now.tok0() + warp * kTok) * a.ld_dx;
    T* dg_row = (T*)a.dg + (now.tok0() + warp * kTok) * a.ld_dg;
#pragma unroll
    for (int t = kTok - 1; t >= 0; --t) {
      float dy[N], dx[N], dg[N];
      read(dy, 2, t);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float e = C[j] + dy[j];
        dx[j] = mv[t][j] * e;
        dg[j] = wv[t][j] * e;
        C[j] = av[t][j] == 0.f ? 0.f : av[t][j] * e;
      }
      if (t < left) {
        rec_store(dx_row + t * a.ld_dx, c0 + lane * N, a.D, dx_pairs, dx);
        rec_store(dg_row + t * a.ld_dg, c0 + lane * N, a.D, dg_pairs, dg);
      }
    }
    now = next;
    __syncwarp();
  }
  rec_wait<0>();
}

template <class T, int MODE, bool WORDS>
cudaError_t launch_one(const RecArgs& a, cudaStream_t stream) {
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess || (e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) return e;
  if ((e = allow_shared<gated_recurrence_backward_kernel<T, MODE, WORDS>>(kSmem)) != cudaSuccess) return e;
  const long long items = (long long)a.n_segs * a.cols;
  if ((e = launch_early(gated_recurrence_backward_kernel<T, MODE, WORDS>, dim3((unsigned)std::min<long long>(items, 3ll * sms)), kThreads, kSmem, stream, a)) != cudaSuccess) return e;
  return launched();
}
template <class T>
cudaError_t launch_type(const RecArgs& a, cudaStream_t stream) {
  const bool w = a.words != nullptr;
  switch (a.mode) {
    case kRecDecay: return w ? launch_one<T, kRecDecay, true>(a, stream) : launch_one<T, kRecDecay, false>(a, stream);
    case kRecNormed: return w ? launch_one<T, kRecNormed, true>(a, stream) : launch_one<T, kRecNormed, false>(a, stream);
    default: return w ? launch_one<T, kRecGate, true>(a, stream) : launch_one<T, kRecGate, false>(a, stream);
  }
}

}  // namespace

cudaError_t launch_gated_recurrence_backward(const RecArgs& a, int dtype, cudaStream_t stream) {
  return dtype == TRI_INV_F32 ? launch_type<float>(a, stream) : launch_type<__nv_bfloat16>(a, stream);
}

}  // namespace tri_inv
