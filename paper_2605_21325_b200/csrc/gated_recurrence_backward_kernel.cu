// Gated linear recurrence: the gradient's walk, from the last tile to the first.
#include <algorithm>

#include "gated_recurrence.cuh"

namespace tri_inv {
namespace {

constexpr int kTok = kRecBackTok, kStages = 3;
template <int MODE> constexpr int kBlocks = MODE == kRecDecay ? 4 : 3;   // an SM's, by the registers that a lane's tokens take
// What a warp's tokens of a tile make of x, from what the first pass over them left: a, m
template <int MODE> struct Factors { Pair a[kTok], m[kTok]; };
template <> struct Factors<kRecDecay> { Pair a[kTok]; };
// and the maps of its lane groups: (fP, fH) of those in front of the lane's, (bP, bC) of those behind it
template <int MODE> struct Held : Factors<MODE> { Pair fP, fH, bP, bC; };

// w: what multiplies e in dg, from the state in front of the token
template <int MODE>
__device__ __forceinline__ Pair weight(Pair a, Pair m, Pair h, Pair x) {
  const Pair minus = twice(-1.f);
  if constexpr (MODE == kRecDecay) {
    return mul2(a, h);
  } else if constexpr (MODE == kRecNormed) {
    const float2 f = both(m);
    const Pair over = pair(f.x > 0.f ? rec_reciprocal(f.x) : 0.f, f.y > 0.f ? rec_reciprocal(f.y) : 0.f);
    return mul2(a, fma2(mul2(mul2(a, over), x), minus, h));
  } else {
    return mul2(fma2(x, minus, h), mul2(a, m));
  }
}
__device__ __forceinline__ Pair none_where_zero(Pair a, Pair v) {
  const float2 x = both(a), y = both(v);
  return pair(x.x == 0.f ? 0.f : y.x, x.y == 0.f ? 0.f : y.y);
}

template <class T, int MODE, bool WORDS>
__global__ void __launch_bounds__(kRecThreads, kBlocks<MODE>) gated_recurrence_backward_kernel(const __grid_constant__ RecArgs a) {
  using Shape = RecShape<T, kTok>;
  constexpr int CH = Shape::CHANNELS, TILE = Shape::TILE, ROW = Shape::ROW;
  extern __shared__ __align__(128) unsigned char stages[];
  __shared__ __align__(16) float2 part[2][kRecWarps][CH];   // (P, H) of each warp's tokens; then (P, C) of all tokens of the tile behind them
  __shared__ __align__(8) float side[2][kRecWarps][CH];     // C: what each warp's tokens pass on, where nothing reaches them from behind; then the state in front of them
  __shared__ __align__(8) float entry[2][CH];            // what reaches a tile from behind
  __shared__ RecAt ring[kRecRing];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int items = a.n_segs * a.cols;
  constexpr int es = sizeof(T);
  RecFeed<WORDS, TILE, 5, true> feed{a, {a.ld_x * es, a.ld_g * es, a.ld_dy * es, a.ld_dx * es, a.ld_dg * es}, es};
  wait_for_predecessor();
  if (tid == 32 * kRecWarps) feed.begin(ring, 4);
  __syncthreads();

  if (warp >= kRecWarps) {   // a channel
    const int ch = tid - 32 * kRecWarps;
    const unsigned long long limit = a.wait_limit_ns ? a.wait_limit_ns : 2000000000ull;
    float carried = 0.f;
    for (int i = 0;; ++i) {
      const RecAt& t = ring[i & (kRecRing - 1)];
      if (t.item >= items) break;
      if (ch == 0) feed.ask();
      const int c = t.c0 + ch, behind = t.tiles - 1 - t.index;
      const bool in = c < a.D, first = t.index == 0, last = behind == 0;
      const long long at = t.slot * a.D + c, state = (long long)t.seq * a.D + c;
      float h = !in ? 0.f : !first ? a.carries[(rec_slot(t.begin, t.seq, kRecCarry) + (long long)t.index * (TILE / kRecCarry) - 1) * a.D + c] : a.h0 ? a.h0[state] : 0.f;   // the state in front of the tile
      float e = last && in && a.dh ? a.dh[state] : 0.f;
      rec_meet(kRecMaps + (i & 1), kRecThreads);
      float P = 1.f, C = 0.f, kept[kRecWarps];
#pragma unroll
      for (int w = 0; w < kRecWarps; ++w) {
        const float2 q = part[i & 1][w][ch];
        kept[w] = h;
        h = rec_step(q.x, h, q.y);
      }
#pragma unroll
      for (int w = kRecWarps - 1; w >= 0; --w) {
        const float p = part[i & 1][w][ch].x, c_own = side[i & 1][w][ch];
        part[i & 1][w][ch] = make_float2(P, C);
        side[i & 1][w][ch] = kept[w];
        P *= p;
        C = rec_step(p, C, c_own);
      }
      if (in) {
        if (WORDS && !last) {
          if (!first) rec_post(a.words + at, P, C);
          e = rec_look_back(a.words + at + a.D, -(long long)a.D, behind, limit, a.status);
        } else if (!last) {
          e = carried;
        }
        carried = rec_step(P, e, C);
        if (first) {
          if (a.dh0) a.dh0[state] = carried;
        } else if (WORDS) {
          rec_post(a.words + at, 0.f, carried);
        }
      }
      entry[i & 1][ch] = e;
      if (ch == 0) feed.give(&ring[(i + 4) & (kRecRing - 1)]);
      rec_arrive(kRecEntry + (i & 1), kRecThreads);
    }
    return;
  }

  using Lane = RecLane<T>;
  using Raw = typename Lane::Raw;
  const T *X = (const T*)a.x, *G = (const T*)a.g, *DY = (const T*)a.dy;
  const int x_access = rec_access<T>(X, a.ld_x), g_access = rec_access<T>(G, a.ld_g), dy_access = rec_access<T>(DY, a.ld_dy);
  const int dx_access = rec_access<T>(a.dx, a.ld_dx), dg_access = rec_access<T>(a.dg, a.ld_dg), most = es == 4 ? kRecWide : kRecFours;
  const bool wide = x_access == kRecWide && g_access == kRecWide && dy_access == kRecWide, plain = dx_access <= most && dg_access <= most;   // plain: whole lanes can be written
  const int first = warp * Shape::WARP_TOK;
  const char *x_from = (const char*)X + Shape::copy_from(a.ld_x, first), *g_from = (const char*)G + Shape::copy_from(a.ld_g, first), *dy_from = (const char*)DY + Shape::copy_from(a.ld_dy, first);
  const uint32_t warp_smem = (uint32_t)__cvta_generic_to_shared(stages) + warp * Shape::WARP_BYTES;
  auto request = [&](const RecAt& t, int stage) {
    if (t.item < items) {
      const uint32_t to = warp_smem + stage * 3 * Shape::TENSOR;
      if (t.whole && wide) {
        Shape::request_whole(to, x_from + t.at[0], a.ld_x);
        Shape::request_whole(to + Shape::TENSOR, g_from + t.at[1], a.ld_g);
        Shape::request_whole(to + 2 * Shape::TENSOR, dy_from + t.at[2], a.ld_dy);
      } else {
        Shape::request(to, X, a.ld_x, t.tok0 + first, t.n - first, t.c0, a.D, x_access);
        Shape::request(to + Shape::TENSOR, G, a.ld_g, t.tok0 + first, t.n - first, t.c0, a.D, g_access);
        Shape::request(to + 2 * Shape::TENSOR, DY, a.ld_dy, t.tok0 + first, t.n - first, t.c0, a.D, dy_access);
      }
    }
    rec_commit();
  };
  request(ring[0], 0);
  // Round i: the maps of tile i, and the output of tile i - 1, whose entry the channels' threads have found out meanwhile.  A tile's rows stay for both.
  Held<MODE> even, odd;
  bool resets = false;
  int stage = 0, stage_before = 2;
  auto round = [&](int i, Held<MODE>& now, const Held<MODE>& before) -> bool {
    const int stage_next = 3 - stage - stage_before;
    request(ring[(i + 1) & (kRecRing - 1)], stage_next);
    const bool has_now = ring[i & (kRecRing - 1)].item < items;
    const int place = warp * Shape::WARP_BYTES + Shape::place();
    bool now_resets = false;
    if (has_now) {
      rec_wait<1>();
      __syncwarp();
      const unsigned char* sx = stages + stage * 3 * Shape::TENSOR + place;
      auto read = [&](int tensor, int k) { return Lane::widen(*reinterpret_cast<const Raw*>(sx + tensor * Shape::TENSOR + k * ROW)); };
      const int left = ring[i & (kRecRing - 1)].n - first - Shape::group() * kTok;   // of the lane's tokens
      Pair P = twice(1.f), H = twice(0.f), C = twice(0.f);
#pragma unroll
      for (int k = 0; k < kTok; ++k) {
        Pair m;
        rec_factors<MODE>(read(1, k), now.a[k], m);
        if constexpr (MODE != kRecDecay) now.m[k] = m;
      }
      if (!ring[i & (kRecRing - 1)].whole) {
#pragma unroll
        for (int k = 0; k < kTok; ++k)
          if (k >= left) {
            now.a[k] = twice(1.f);
            if constexpr (MODE != kRecDecay) now.m[k] = twice(0.f);
          }
      }
      auto input = [&](int k) {
        if constexpr (MODE == kRecDecay) return read(0, k);
        else return mul2(now.m[k], read(0, k));
      };
#pragma unroll
      for (int k = 0; k < kTok; ++k) {
        P = mul2(P, now.a[k]);
        H = fma2(now.a[k], H, input(k));
        C = mul2(now.a[kTok - 1 - k], add2(C, read(2, kTok - 1 - k)));
      }
      now_resets = __any_sync(0xffffffffu, any_zero(P));
      if (now_resets) {
        H = C = twice(0.f);
#pragma unroll
        for (int k = 0; k < kTok; ++k) {
          H = rec_step(now.a[k], H, input(k));
          C = none_where_zero(now.a[kTok - 1 - k], mul2(now.a[kTok - 1 - k], add2(C, read(2, kTok - 1 - k))));
        }
      }
      Pair same = P;
      rec_join_groups<true>(same, C, now.bP, now.bC);
      rec_join_groups<false>(P, H, now.fP, now.fH);
      const float2 pp = both(P), hh = both(H), cc = both(C);
      if (lane < Shape::LANES) {
        *reinterpret_cast<float4*>(&part[i & 1][warp][Shape::channel()]) = make_float4(pp.x, hh.x, pp.y, hh.y);
        *reinterpret_cast<float2*>(&side[i & 1][warp][Shape::channel()]) = cc;
      }
      rec_arrive(kRecMaps + (i & 1), kRecThreads);
    }
    if (i > 0) {
      const unsigned char* sx = stages + stage_before * 3 * Shape::TENSOR + place;
      auto read = [&](int tensor, int k) { return Lane::widen(*reinterpret_cast<const Raw*>(sx + tensor * Shape::TENSOR + k * ROW)); };
      rec_meet(kRecEntry + ((i - 1) & 1), kRecThreads);
      const RecAt& p = ring[(i - 1) & (kRecRing - 1)];
      const float4 q = *reinterpret_cast<const float4*>(&part[(i - 1) & 1][warp][Shape::channel()]);
      const float2 s = *reinterpret_cast<const float2*>(&side[(i - 1) & 1][warp][Shape::channel()]), e0 = *reinterpret_cast<const float2*>(&entry[(i - 1) & 1][Shape::channel()]);
      Pair h = pair(s.x, s.y), C = rec_step(pair(q.x, q.z), pair(e0.x, e0.y), pair(q.y, q.w)), w[kTok];
      h = rec_step(before.fP, h, before.fH);
      C = rec_step(before.bP, C, before.bC);
      auto m_of = [&](int k) {
        if constexpr (MODE == kRecDecay) return twice(1.f);
        else return before.m[k];
      };
      if (p.whole && plain && !resets) {
#pragma unroll
        for (int k = 0; k < kTok; ++k) {
          const Pair x = read(0, k);
          w[k] = weight<MODE>(before.a[k], m_of(k), h, x);
          h = fma2(before.a[k], h, rec_input<MODE>(m_of(k), x));
        }
        char *dx_row = (char*)a.dx + p.at[3] + ((first + Shape::group() * kTok) * a.ld_dx + Shape::channel()) * es, *dg_row = (char*)a.dg + p.at[4] + ((first + Shape::group() * kTok) * a.ld_dg + Shape::channel()) * es;
        const uint32_t dx_step = (uint32_t)a.ld_dx * es, dg_step = (uint32_t)a.ld_dg * es;
#pragma unroll
        for (int k = kTok - 1; k >= 0; --k) {
          const Pair e = add2(C, read(2, k));
          *reinterpret_cast<Raw*>(dx_row + (unsigned long long)dx_step * k) = Lane::pack(rec_input<MODE>(m_of(k), e));
          *reinterpret_cast<Raw*>(dg_row + (unsigned long long)dg_step * k) = Lane::pack(mul2(w[k], e));
          C = mul2(before.a[k], e);
        }
      } else {
        const int at = first + Shape::group() * kTok, left = p.n - at, c = p.c0 + Shape::channel();
        T* dx_row = (T*)a.dx + (p.tok0 + at) * a.ld_dx;
        T* dg_row = (T*)a.dg + (p.tok0 + at) * a.ld_dg;
#pragma unroll
        for (int k = 0; k < kTok; ++k) {
          const Pair x = read(0, k);
          w[k] = none_where_zero(before.a[k], weight<MODE>(before.a[k], m_of(k), h, x));
          h = rec_step(before.a[k], h, rec_input<MODE>(m_of(k), x));
        }
#pragma unroll
        for (int k = kTok - 1; k >= 0; --k) {
          const Pair e = add2(C, read(2, k));
          if (k < left) {
            rec_store(dx_row + k * a.ld_dx, c, a.D, dx_access, rec_input<MODE>(m_of(k), e));
            rec_store(dg_row + k * a.ld_dg, c, a.D, dg_access, mul2(w[k], e));
          }
          C = none_where_zero(before.a[k], mul2(before.a[k], e));
        }
      }
    }
    resets = now_resets;
    stage_before = stage;
    stage = stage_next;
    __syncwarp();
    return has_now;
  };
  for (int i = 0;; i += 2) {
    if (!round(i, even, odd)) break;
    if (!round(i + 1, odd, even)) break;
  }
  rec_wait<0>();
}

template <class T, int MODE, bool WORDS>
cudaError_t launch_one(const RecArgs& a, cudaStream_t stream) {
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess || (e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) return e;
  constexpr size_t smem = (size_t)kStages * 3 * RecShape<T, kTok>::TENSOR;
  if ((e = allow_shared<gated_recurrence_backward_kernel<T, MODE, WORDS>>(smem)) != cudaSuccess) return e;
  const long long items = (long long)a.n_segs * a.cols;
  if ((e = launch_early(gated_recurrence_backward_kernel<T, MODE, WORDS>, dim3((unsigned)std::min<long long>(items, (long long)kBlocks<MODE> * sms)), kRecThreads, smem, stream, a)) != cudaSuccess) return e;
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
