// Gated linear recurrence: the gradient's walk, from the last tile to the first.
//
// As the forward walk, with what tokens pass on in the place of the state: the words join (P, C) from behind.  The states are formed again in fp32 from the one carried into the tile, so that the forward call's outputs, rounded to
// their type, play no part, and dY, X and G are all that is read (10 bytes a value in bf16; with the outputs kept it would be 12).  x and dy stay in shared memory for the second pass; the weights w are formed for eight tokens at a
// time, the last first, from the state in front of them.
// What bounds it: no unit is full.  49 instructions a value (normed) take 0.56 of the issue slots at the occupancy that a and m of sixteen tokens leave, 128 registers and three blocks an SM, where the normed and gate forms spill 116
// to 168 bytes a thread; the largest stalls are the barrier, instructions that wait for one another, and shared and local memory.  bf16: 1 x 32768 x 4096 decay 257 us, 0.81 of a copy's rate; 64 x 1024 x 2048 gate 261, 0.80;
// 4 x 4096 x 2560 normed 101, 0.65; fp32 (eight tokens, three blocks, which is what shared memory holds) 0.88 to 0.91.  Eight tokens in bf16: 290 (gate); four blocks, which spill more, 285 (decay).
// Rows at odd places: 4 x 2048 x 2047 gate, bf16 132 us (42 with 2048).
#include <algorithm>

#include "gated_recurrence.cuh"

namespace tri_inv {
namespace {

// Blocks an SM: in bf16 128 registers a thread, in fp32 what shared memory holds
constexpr int kBlocks = 3;

// w: what multiplies e in dg, from the state in front of the token.  SAFE: where m may be zero
template <int MODE, bool SAFE>
__device__ __forceinline__ Pair weight(Pair a, Pair m, Pair h, Pair x) {
  const Pair minus = twice(-1.f);
  if constexpr (MODE == kRecDecay) {
    return mul2(a, h);
  } else if constexpr (MODE == kRecNormed) {
    const float2 f = both(m);
    const Pair over = SAFE ? pair(f.x > 0.f ? rec_reciprocal(f.x) : 0.f, f.y > 0.f ? rec_reciprocal(f.y) : 0.f) : pair(rec_reciprocal(f.x), rec_reciprocal(f.y));
    return mul2(a, fma2(mul2(mul2(a, over), x), minus, h));
  } else {
    return mul2(fma2(x, minus, h), mul2(a, m));
  }
}
__device__ __forceinline__ Pair none_where_zero(Pair a, Pair v) {
  const float2 x = both(a), y = both(v);
  return pair(x.x == 0.f ? 0.f : y.x, x.y == 0.f ? 0.f : y.y);
}

// ANY: some input cannot be moved 16 bytes at a time
template <class T, int MODE, bool WORDS, bool ANY>
__global__ void __launch_bounds__(kRecThreads, kBlocks) gated_recurrence_backward_kernel(const __grid_constant__ RecArgs a) {
  constexpr int kTok = rec_back_tok(sizeof(T)), kPart = 8;   // tokens of a lane; those that are finished at a time
  using Shape = RecShape<T, kTok>;
  using Lane = RecLane<T>;
  using Raw = typename Lane::Raw;
  constexpr int CH = kRecChannels, TILE = Shape::TILE, ROW = Shape::ROW, es = sizeof(T);
  extern __shared__ __align__(128) unsigned char stages[];
  __shared__ __align__(16) float2 part[2][kRecWarps][CH];   // (P, H) of each warp's tokens
  __shared__ __align__(8) float back[2][kRecWarps][CH];     // C: what they pass on where nothing reaches them from behind
  __shared__ __align__(8) float2 total[2][CH];              // (P, C) of a tile
  __shared__ __align__(16) float2 entry[2][CH];             // the state in front of a tile, and what reaches it from behind
  __shared__ RecAt ring[kRecRing];
  __shared__ __align__(4) unsigned char rest[ANY ? 2 : 1][3][kRecWarps][ANY && es == 2 ? 4 * Shape::WARP_TOK : 4];   // of rows at odd places (RecShape)
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int items = a.items;
  RecFeed<WORDS, TILE, 5, true> feed{a, {(int)(a.ld_x * es), (int)(a.ld_g * es), (int)(a.ld_dy * es), (int)(a.ld_dx * es), (int)(a.ld_dg * es)}, es};
  wait_for_predecessor();
  if (tid == 32 * kRecWarps) feed.begin(ring);
  __syncthreads();

  if (warp == kRecWarps) {   // a lane for each channel
    if (lane == 0)
      for (int i = 1; i < 3; ++i) { feed.ask(); feed.give(&ring[i]); }
    __syncthreads();
    const unsigned long long limit = a.wait_limit_ns ? a.wait_limit_ns : 2000000000ull;
    float carried = 0.f;
    for (int i = 0;; ++i) {
      const RecAt& t = ring[i & (kRecRing - 1)];
      if (t.item >= items) break;
      if (lane == 0) feed.ask();
      const int c = t.c0 + lane, behind = t.tiles - 1 - t.index;
      const bool in = c < a.D, first = t.index == 0, last = behind == 0;
      const long long at = rec_at(t.slot, a.D, c), state = rec_at(t.seq, a.D, c);
      float h = 0.f, e = 0.f;
      if (in) {
        if (!first) h = a.carries[rec_at(rec_slot(t.begin, t.seq, kRecCarry) + (long long)t.index * (TILE / kRecCarry) - 1, a.D, c)];
        else if (a.h0) h = a.h0[state];
        if (last) e = a.dh ? a.dh[state] : 0.f;
        else e = WORDS ? rec_look_back(a.words + at + a.D, -(long long)a.D, behind, limit, a.status) : carried;
      }
      entry[i & 1][lane] = make_float2(h, e);
      rec_meet<kRecEntry, kRecThreads>();
      const float2 map = total[i & 1][lane];
      const float s = rec_step(map.x, e, map.y);
      carried = s;
      if (in) {
        if (first) {
          if (a.dh0) {
            if (WORDS && !last && a.dh0 == a.dh) rec_await(a.words + at + (long long)behind * a.D, limit, a.status);
            a.dh0[state] = s;
          }
        } else if (WORDS) rec_post(a.words + at, 0.f, s);
      }
      if (lane == 0) feed.give(&ring[(i + 3) & (kRecRing - 1)]);
      __syncwarp();
    }
    return;
  }

  const T *X = (const T*)a.x, *G = (const T*)a.g, *DY = (const T*)a.dy;
  const int x_access = ANY ? rec_access<T>(X, a.ld_x) : (int)kRecWide, g_access = ANY ? rec_access<T>(G, a.ld_g) : (int)kRecWide, dy_access = ANY ? rec_access<T>(DY, a.ld_dy) : (int)kRecWide;
  const int dx_access = rec_access<T>(a.dx, a.ld_dx), dg_access = rec_access<T>(a.dg, a.ld_dg), most = es == 4 ? kRecEights : kRecFours;
  const bool plain = dx_access <= most && dg_access <= most;   // plain: whole lanes can be written
  const bool odd = x_access == kRecSingle || g_access == kRecSingle || dy_access == kRecSingle;
  const int first = warp * Shape::WARP_TOK;
  const char *x_from = (const char*)X + Shape::copy_from(a.ld_x, first), *g_from = (const char*)G + Shape::copy_from(a.ld_g, first), *dy_from = (const char*)DY + Shape::copy_from(a.ld_dy, first);
  const uint32_t warp_smem = (uint32_t)__cvta_generic_to_shared(stages) + warp * Shape::WARP_BYTES;
  auto request = [&](const RecAt& t, int stage) {
    if (t.item < items) {
      const uint32_t to = warp_smem + stage * 3 * Shape::TENSOR;
      if (!ANY && t.whole) {
        Shape::request_whole(to, x_from + t.at[0], a.ld_x);
        Shape::request_whole(to + Shape::TENSOR, g_from + t.at[1], a.ld_g);
        Shape::request_whole(to + 2 * Shape::TENSOR, dy_from + t.at[2], a.ld_dy);
      } else if (ANY && t.whole) {
        auto space = [&](int tensor) { return (uint32_t)__cvta_generic_to_shared(rest[ANY ? stage : 0][tensor][warp]); };
        Shape::request_any(to, space(0), a, X, t, 0, a.ld_x, first, x_access);
        Shape::request_any(to + Shape::TENSOR, space(1), a, G, t, 1, a.ld_g, first, g_access);
        Shape::request_any(to + 2 * Shape::TENSOR, space(2), a, DY, t, 2, a.ld_dy, first, dy_access);
      } else {
        Shape::request(to, X, a.ld_x, t.tok0 + first, t.n - first, t.c0, a.D, x_access);
        Shape::request(to + Shape::TENSOR, G, a.ld_g, t.tok0 + first, t.n - first, t.c0, a.D, g_access);
        Shape::request(to + 2 * Shape::TENSOR, DY, a.ld_dy, t.tok0 + first, t.n - first, t.c0, a.D, dy_access);
      }
    }
    rec_commit();
  };
  request(ring[0], 0);
  __syncthreads();
  for (int i = 0;; ++i) {
    const RecAt& t = ring[i & (kRecRing - 1)];
    if (t.item >= items) break;
    request(ring[(i + 1) & (kRecRing - 1)], (i + 1) & 1);
    rec_wait<1>();
    __syncwarp();
    if (ANY && odd) {
      unsigned char* rows = stages + (i & 1) * 3 * Shape::TENSOR + warp * Shape::WARP_BYTES;
      Shape::settle_any(rows, rest[ANY ? i & 1 : 0][0][warp], a, X, t, 0, a.ld_x, first, x_access);
      Shape::settle_any(rows + Shape::TENSOR, rest[ANY ? i & 1 : 0][1][warp], a, G, t, 1, a.ld_g, first, g_access);
      Shape::settle_any(rows + 2 * Shape::TENSOR, rest[ANY ? i & 1 : 0][2][warp], a, DY, t, 2, a.ld_dy, first, dy_access);
      __syncwarp();
    }
    const unsigned char* sx = stages + (i & 1) * 3 * Shape::TENSOR + warp * Shape::WARP_BYTES + Shape::place();
    auto read = [&](int tensor, int k) { return Lane::widen(*reinterpret_cast<const Raw*>(sx + tensor * Shape::TENSOR + k * ROW)); };
    Pair av[kTok], mv[kTok];   // (mv is not used where it is 1)
#pragma unroll
    for (int k = 0; k < kTok; ++k) rec_factors<MODE>(read(1, k), av[k], mv[k]);
    const int at = first + Shape::group() * kTok, left = t.n - at;   // of the lane's tokens
    if (!t.whole) {
#pragma unroll
      for (int k = 0; k < kTok; ++k)
        if (k >= left) av[k] = mv[k] = twice(1.f);   // (x and dy read as zero there)
    }
    Pair P = twice(1.f), H = twice(0.f), C = twice(0.f), half_P, half_H;   // half: of the first half of the tokens
#pragma unroll
    for (int k = 0; k < kTok; ++k) {
      if (k == kTok / 2) { half_P = P; half_H = H; }
      P = mul2(P, av[k]);
      H = fma2(av[k], H, rec_input<MODE>(mv[k], read(0, k)));
      C = mul2(av[kTok - 1 - k], add2(C, read(2, kTok - 1 - k)));
    }
    const bool resets = __any_sync(0xffffffffu, any_zero(P));
    bool no_input = false;   // some m is zero
    if constexpr (MODE == kRecNormed) {
      float2 least = both(mv[0]);
#pragma unroll
      for (int k = 1; k < kTok; ++k) { const float2 f = both(mv[k]); least = make_float2(fminf(least.x, f.x), fminf(least.y, f.y)); }
      no_input = __any_sync(0xffffffffu, fminf(least.x, least.y) == 0.f);
    }
    if (resets) {
      float2 least = make_float2(1.f, 1.f);
#pragma unroll
      for (int k = 0; k < kTok; ++k) {
        const float2 f = both(av[k]);
        least = make_float2(fminf(least.x, f.x), fminf(least.y, f.y));   // (passes over what is no number)
        if (k == kTok / 2 - 1) half_P = none_where_zero(pair(least.x, least.y), half_P);
      }
      P = none_where_zero(pair(least.x, least.y), P);
      H = C = twice(0.f);
#pragma unroll
      for (int k = 0; k < kTok; ++k) {
        if (k == kTok / 2) half_H = H;
        H = rec_step(av[k], H, rec_input<MODE>(mv[k], read(0, k)));
        C = none_where_zero(av[kTok - 1 - k], mul2(av[kTok - 1 - k], add2(C, read(2, kTok - 1 - k))));
      }
    }
    const Pair other_P = rec_other(P), other_H = rec_other(H), other_C = rec_other(C);   // the second group's tokens come behind the first one's
    const bool second = lane >= Shape::LANES;
    const float2 pp = both(rec_product(P, other_P)), hh = both(rec_step(other_P, H, other_H)), cc = both(rec_step(P, other_C, C));
    if (!second) {
      *reinterpret_cast<float4*>(&part[i & 1][warp][Shape::channel()]) = make_float4(pp.x, hh.x, pp.y, hh.y);
      *reinterpret_cast<float2*>(&back[i & 1][warp][Shape::channel()]) = cc;
    }
    rec_meet<kRecMaps, 32 * kRecWarps>();
    if (warp == 0) {   // the tile's map; as a word for those in front of it
      float TP = 1.f, TC = 0.f;
#pragma unroll
      for (int w = kRecWarps - 1; w >= 0; --w) {
        const float p = part[i & 1][w][lane].x;
        TP = rec_product(TP, p);
        TC = rec_step(p, TC, back[i & 1][w][lane]);
      }
      total[i & 1][lane] = make_float2(TP, TC);
      if (WORDS && t.index > 0 && t.index + 1 < t.tiles && t.c0 + lane < a.D) rec_post(a.words + rec_at(t.slot, a.D, t.c0 + lane), TP, TC);
    }
    rec_meet<kRecEntry, kRecThreads>();
    const float4 e0 = *reinterpret_cast<const float4*>(&entry[i & 1][Shape::channel()]);
    Pair h = pair(e0.x, e0.z);
    C = pair(e0.y, e0.w);
    for (int w = 0; w < warp; ++w) {
      const float4 q = *reinterpret_cast<const float4*>(&part[i & 1][w][Shape::channel()]);
      h = rec_step(pair(q.x, q.z), h, pair(q.y, q.w));
    }
    for (int w = kRecWarps - 1; w > warp; --w) {
      const float4 q = *reinterpret_cast<const float4*>(&part[i & 1][w][Shape::channel()]);
      const float2 s = *reinterpret_cast<const float2*>(&back[i & 1][w][Shape::channel()]);
      C = rec_step(pair(q.x, q.z), C, pair(s.x, s.y));
    }
    if (second) h = rec_step(other_P, h, other_H);
    else C = rec_step(other_P, C, other_C);
    // The last part first: what multiplies e, in order, then e from behind
    const Pair h_half = rec_step(half_P, h, half_H);
    if (t.whole && plain && !resets && !no_input) {
      char *dx_row = (char*)a.dx + t.at[3] + (at * a.ld_dx + Shape::channel()) * es, *dg_row = (char*)a.dg + t.at[4] + (at * a.ld_dg + Shape::channel()) * es;
      const uint32_t dx_step = (uint32_t)a.ld_dx * es, dg_step = (uint32_t)a.ld_dg * es;
#pragma unroll
      for (int k0 = kTok - kPart; k0 >= 0; k0 -= kPart) {
        Pair wv[kPart], s = k0 ? h_half : h;
#pragma unroll
        for (int j = 0; j < kPart; ++j) {
          const Pair x = read(0, k0 + j);
          wv[j] = weight<MODE, false>(av[k0 + j], mv[k0 + j], s, x);
          s = fma2(av[k0 + j], s, rec_input<MODE>(mv[k0 + j], x));
        }
#pragma unroll
        for (int j = kPart - 1; j >= 0; --j) {
          const int k = k0 + j;
          const Pair e = add2(C, read(2, k));
          *reinterpret_cast<Raw*>(dx_row + (unsigned long long)dx_step * k) = Lane::pack(rec_input<MODE>(mv[k], e));
          *reinterpret_cast<Raw*>(dg_row + (unsigned long long)dg_step * k) = Lane::pack(mul2(wv[j], e));
          C = mul2(av[k], e);
        }
      }
    } else {
      const int c = t.c0 + Shape::channel();
      T *dx_row = (T*)a.dx + (long long)(t.tok0 + at) * a.ld_dx, *dg_row = (T*)a.dg + (long long)(t.tok0 + at) * a.ld_dg;
#pragma unroll
      for (int k0 = kTok - kPart; k0 >= 0; k0 -= kPart) {
        Pair wv[kPart], s = k0 ? h_half : h;
#pragma unroll
        for (int j = 0; j < kPart; ++j) {
          const Pair x = read(0, k0 + j);
          wv[j] = none_where_zero(av[k0 + j], weight<MODE, true>(av[k0 + j], mv[k0 + j], s, x));
          s = rec_step(av[k0 + j], s, rec_input<MODE>(mv[k0 + j], x));
        }
#pragma unroll
        for (int j = kPart - 1; j >= 0; --j) {
          const int k = k0 + j;
          const Pair e = add2(C, read(2, k));
          if (k < left) {
            rec_store(dx_row + k * a.ld_dx, c, a.D, dx_access, rec_input<MODE>(mv[k], e));
            rec_store(dg_row + k * a.ld_dg, c, a.D, dg_access, mul2(wv[j], e));
          }
          C = none_where_zero(av[k], mul2(av[k], e));
        }
      }
    }
    __syncwarp();
  }
  rec_wait<0>();
}

template <class T, int MODE, bool WORDS, bool ANY>
cudaError_t launch_one(const RecArgs& a, cudaStream_t stream) {
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess || (e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) return e;
  constexpr size_t smem = 6 * (size_t)RecShape<T, rec_back_tok(sizeof(T))>::TENSOR;
  static_assert(rec_fit(kBlocks, smem, 8 * 1024), "a grid of blocks that are not all resident");
  if ((e = allow_shared<gated_recurrence_backward_kernel<T, MODE, WORDS, ANY>>(smem)) != cudaSuccess) return e;
  const long long items = a.items;
  if ((e = launch_early(gated_recurrence_backward_kernel<T, MODE, WORDS, ANY>, dim3((unsigned)std::min<long long>(items, (long long)kBlocks * sms)), kRecThreads, smem, stream, a)) != cudaSuccess) return e;
  return launched();
}
template <class T, int MODE>
cudaError_t launch_mode(const RecArgs& a, cudaStream_t stream) {
  const bool any = rec_access<T>(a.x, a.ld_x) != kRecWide || rec_access<T>(a.g, a.ld_g) != kRecWide || rec_access<T>(a.dy, a.ld_dy) != kRecWide;
  if (a.words) return any ? launch_one<T, MODE, true, true>(a, stream) : launch_one<T, MODE, true, false>(a, stream);
  return any ? launch_one<T, MODE, false, true>(a, stream) : launch_one<T, MODE, false, false>(a, stream);
}
template <class T>
cudaError_t launch_type(const RecArgs& a, cudaStream_t stream) {
  return a.mode == kRecDecay ? launch_mode<T, kRecDecay>(a, stream) : a.mode == kRecNormed ? launch_mode<T, kRecNormed>(a, stream) : launch_mode<T, kRecGate>(a, stream);
}

}  // namespace

cudaError_t launch_gated_recurrence_backward(const RecArgs& a, int dtype, cudaStream_t stream) {
  return dtype == TRI_INV_F32 ? launch_type<float>(a, stream) : launch_type<__nv_bfloat16>(a, stream);
}

}  // namespace tri_inv
