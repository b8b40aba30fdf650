// Gated linear recurrence: the forward walk, and what both walks find in their workspace.
//
// One pass: every value is read once, by asynchronous copies one tile ahead, and every output written once.  A block of five warps takes a tile of 128 tokens and 32 channels.  Four warps hold 32 tokens each in
// registers (two lane groups of 16 tokens, two channels a lane), as a and u, form their maps and meet; the fifth, a lane for each channel, meanwhile looks for what enters the tile in the words of the tiles in front of it;
// then the four write h.  Long sequences are spread over the chip that way: a tile's own map is there for the tiles behind it as soon as it has been read.
// What bounds it: with all channels of a large batch bytes (64 x 1024 tokens x 2048 channels, gate, bf16 148 us, 0.84 of a copy's rate; fp32 263, 0.95).  Otherwise (1 x 32768 x 4096 decay 170, 0.74; 4 x 4096 x 2560 normed
// 58, 0.67) neither bytes nor instructions fill: 26 (decay) to 31 (normed) instructions a value take 0.55 to 0.62 of the issue slots, and the largest stall, 2.4 to 3.4 cycles an issued instruction, is the barrier where the warps
// of tokens wait for what enters their tile, with the next one read already.  a and u of 16 tokens and two channels are 64 registers, which leaves four blocks an SM (fp32 three, by shared memory: a grid of four, whose
// last blocks start when others end, took 27.4 us instead of 21.2 for 37 x 100 tokens x 2048, gate).  Long walks over few channels wait for one another (1 x 65536 x 256 43 us, 0.37; 1 x 16384 x 1024 normed 40, 0.39).
// Why this shape, in us (1 x 32768 x 4096 decay | 4 x 4096 x 2560 normed | 64 x 1024 x 2048 gate; 125 | 39 | 125 of memory time): 64 x 64 tiles, every warp waiting for the entry 497 | 143; channels' threads
// aside and the next tile read meanwhile 231 | 90; 128 x 64 tiles of sixteen tokens a lane, places worked out once a tile 184 | 79 (eight tokens 30 % more instructions: the fixed cost of a warp's tile, about
// 200 instructions, is shared by half as many values); four warps and 32 channels, which leaves (in bf16) four blocks whose waits overlap 164 | 60 | 167; the entry looked for ahead of the maps 151 | 52 | 140; carried states
// joined in order, for equal bits, 159 | 53 | 146; decays near 1 without bias 168 | 57 | 147; decays that are not numbers forgotten as states are 170 | 58 | 148.  16 or 64 channels a tile were slower, as were three or five blocks.
// Rows at odd places (4 x 2048 x 2047 gate, bf16 59 us; 25 with 2048) come as the aligned words that hold them, put in order in shared memory; by single loads 102.
#include <algorithm>

#include "gated_recurrence.cuh"

namespace tri_inv {
namespace {

constexpr int kTok = kRecTok;   // tokens of a lane
// Blocks an SM: four leave 96 registers a thread; fp32 has shared memory for three
__host__ __device__ constexpr int blocks(int bytes) { return bytes == 2 ? 4 : 3; }
// ANY: some input cannot be moved 16 bytes at a time
template <class T, int MODE, bool WORDS, bool ANY>
__global__ void __launch_bounds__(kRecThreads, blocks(sizeof(T))) gated_recurrence_kernel(const __grid_constant__ RecArgs a) {
  using Shape = RecShape<T, kTok>;
  using Lane = RecLane<T>;
  using Raw = typename Lane::Raw;
  constexpr int CH = kRecChannels, TILE = Shape::TILE, ROW = Shape::ROW, es = sizeof(T);
  extern __shared__ __align__(128) unsigned char stages[];
  __shared__ __align__(16) float2 part[2][kRecWarps][CH];   // (P, H) of each warp's tokens
  __shared__ __align__(8) float2 total[2][CH];              // ... of the tile
  __shared__ __align__(8) float entry[2][CH];               // what enters a tile
  __shared__ RecAt ring[kRecRing];
  __shared__ __align__(4) unsigned char rest[ANY ? 2 : 1][2][kRecWarps][ANY && es == 2 ? 4 * Shape::WARP_TOK : 4];   // of rows at odd places (RecShape)
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int items = a.items;
  RecFeed<WORDS, TILE, 3, false> feed{a, {(int)(a.ld_x * es), (int)(a.ld_g * es), (int)(a.ld_y * es)}, es};
  wait_for_predecessor();
  if (tid == 32 * kRecWarps) feed.begin(ring);
  __syncthreads();

  if (warp == kRecWarps) {   // a lane for each channel: finds out what enters a tile while the other warps read it
    if (lane == 0)
      for (int i = 1; i < 3; ++i) { feed.ask(); feed.give(&ring[i]); }
    __syncthreads();
    const unsigned long long limit = a.wait_limit_ns ? a.wait_limit_ns : 2000000000ull;
    float carried = 0.f;   // without words: what leaves the tile before
    for (int i = 0;; ++i) {
      const RecAt& t = ring[i & (kRecRing - 1)];
      if (t.item >= items) break;
      if (lane == 0) feed.ask();
      const int c = t.c0 + lane, index = t.index;
      const bool in = c < a.D, first = index == 0, last = index + 1 == t.tiles;
      const long long at = rec_at(t.slot, a.D, c);
      float h = 0.f;
      if (in) {
        if (first) h = a.h0 ? a.h0[rec_at(t.seq, a.D, c)] : 0.f;
        else h = WORDS ? rec_look_back(a.words + at - a.D, a.D, index, limit, a.status) : carried;
      }
      entry[i & 1][lane] = h;
      rec_meet<kRecEntry, kRecThreads>();
      const float2 map = total[i & 1][lane];
      const float s = rec_step(map.x, h, map.y);
      if (a.carries && in) {   // those that a further token of the sequence follows; a tile's last one by its map, as its word says
        float* to = a.carries + rec_at(rec_slot(t.begin, t.seq, kRecCarry) + (long long)index * (TILE / kRecCarry), a.D, c);
        const int left = t.len - index * TILE;
        float m = h;
#pragma unroll
        for (int n = Shape::WARP_TOK; n < TILE; n += Shape::WARP_TOK) {
          const float2 q = part[i & 1][n / Shape::WARP_TOK - 1][lane];
          m = rec_step(q.x, m, q.y);
          if (n % kRecCarry == 0 && n < left) to[(long long)(n / kRecCarry - 1) * a.D] = m;
        }
        if (TILE < left) to[(long long)(TILE / kRecCarry - 1) * a.D] = s;
      }
      carried = s;
      if (in) {
        if (last) {
          if (a.h_out) {
            if (WORDS && !first && a.h_out == a.h0) rec_await(a.words + at - (long long)index * a.D, limit, a.status);
            a.h_out[rec_at(t.seq, a.D, c)] = s;
          }
        } else if (WORDS && !(a.test_stall && t.item == 0)) rec_post(a.words + at, 0.f, s);
      }
      if (lane == 0) feed.give(&ring[(i + 3) & (kRecRing - 1)]);
      __syncwarp();
    }
    return;
  }

  const T *X = (const T*)a.x, *G = (const T*)a.g;
  T* Y = (T*)a.y;
  const int x_access = ANY ? rec_access<T>(X, a.ld_x) : (int)kRecWide, g_access = ANY ? rec_access<T>(G, a.ld_g) : (int)kRecWide, y_access = rec_access<T>(Y, a.ld_y);
  const bool plain = y_access <= (es == 4 ? kRecEights : kRecFours);   // whole lanes can be written
  const bool odd = x_access == kRecSingle || g_access == kRecSingle;
  const int first = warp * Shape::WARP_TOK;   // of the warp's tokens
  const char *x_from = (const char*)X + Shape::copy_from(a.ld_x, first), *g_from = (const char*)G + Shape::copy_from(a.ld_g, first);
  const uint32_t warp_smem = (uint32_t)__cvta_generic_to_shared(stages) + warp * Shape::WARP_BYTES;
  // A warp asks for the rows that it alone reads, so that no barrier stands between a copy and its use.
  auto request = [&](const RecAt& t, int stage) {
    if (t.item < items) {
      const uint32_t to = warp_smem + stage * 2 * Shape::TENSOR;
      if (!ANY && t.whole) {
        Shape::request_whole(to, x_from + t.at[0], a.ld_x);
        Shape::request_whole(to + Shape::TENSOR, g_from + t.at[1], a.ld_g);
      } else if (ANY && t.whole) {
        Shape::request_any(to, (uint32_t)__cvta_generic_to_shared(rest[ANY ? stage : 0][0][warp]), a, X, t, 0, a.ld_x, first, x_access);
        Shape::request_any(to + Shape::TENSOR, (uint32_t)__cvta_generic_to_shared(rest[ANY ? stage : 0][1][warp]), a, G, t, 1, a.ld_g, first, g_access);
      } else {
        Shape::request(to, X, a.ld_x, t.tok0 + first, t.n - first, t.c0, a.D, x_access);
        Shape::request(to + Shape::TENSOR, G, a.ld_g, t.tok0 + first, t.n - first, t.c0, a.D, g_access);
      }
    }
    rec_commit();
  };
  request(ring[0], 0);
  __syncthreads();   // the next tiles are known
  for (int i = 0;; ++i) {
    const RecAt& t = ring[i & (kRecRing - 1)];
    if (t.item >= items) break;
    request(ring[(i + 1) & (kRecRing - 1)], (i + 1) & 1);
    rec_wait<1>();
    __syncwarp();
    if (ANY && odd) {
      unsigned char* rows = stages + (i & 1) * 2 * Shape::TENSOR + warp * Shape::WARP_BYTES;
      Shape::settle_any(rows, rest[ANY ? i & 1 : 0][0][warp], a, X, t, 0, a.ld_x, first, x_access);
      Shape::settle_any(rows + Shape::TENSOR, rest[ANY ? i & 1 : 0][1][warp], a, G, t, 1, a.ld_g, first, g_access);
      __syncwarp();
    }
    const unsigned char* sx = stages + (i & 1) * 2 * Shape::TENSOR + warp * Shape::WARP_BYTES + Shape::place();
    Pair av[kTok], uv[kTok];
#pragma unroll
    for (int k = 0; k < kTok; ++k) {
      const Pair x = Lane::widen(*reinterpret_cast<const Raw*>(sx + k * ROW)), g = Lane::widen(*reinterpret_cast<const Raw*>(sx + Shape::TENSOR + k * ROW));
      Pair m;
      rec_factors<MODE>(g, av[k], m);
      uv[k] = rec_input<MODE>(m, x);
    }
    const int left = t.n - first - Shape::group() * kTok;   // of the lane's tokens
    if (!t.whole) {
#pragma unroll
      for (int k = 0; k < kTok; ++k)
        if (k >= left) { av[k] = twice(1.f); uv[k] = twice(0.f); }
    }
    Pair P = av[0], H = uv[0];
#pragma unroll
    for (int k = 1; k < kTok; ++k) {
      P = mul2(P, av[k]);
      H = fma2(av[k], H, uv[k]);
    }
    const bool resets = __any_sync(0xffffffffu, any_zero(P));   // some decay of the warp's tokens is zero
    if (resets) {
      P = twice(1.f);
      H = twice(0.f);
#pragma unroll
      for (int k = 0; k < kTok; ++k) {
        P = rec_product(P, av[k]);
        H = rec_step(av[k], H, uv[k]);
      }
    }
    const Pair other_P = rec_other(P), other_H = rec_other(H);   // the second group's tokens come behind the first one's
    const bool second = lane >= Shape::LANES;
    const float2 pp = both(rec_product(P, other_P)), hh = both(rec_step(other_P, H, other_H));
    if (!second) *reinterpret_cast<float4*>(&part[i & 1][warp][Shape::channel()]) = make_float4(pp.x, hh.x, pp.y, hh.y);
    rec_meet<kRecMaps, 32 * kRecWarps>();
    if (warp == kRecWarps - 1) {   // the tile's map; as a word for those behind it
      float TP = 1.f, TH = 0.f;
#pragma unroll
      for (int w = 0; w < kRecWarps; ++w) {
        const float2 q = part[i & 1][w][lane];
        TP = rec_product(TP, q.x);
        TH = rec_step(q.x, TH, q.y);
      }
      total[i & 1][lane] = make_float2(TP, TH);
      if (WORDS && t.index > 0 && t.index + 1 < t.tiles && t.c0 + lane < a.D) rec_post(a.words + rec_at(t.slot, a.D, t.c0 + lane), TP, TH);
    }
    P = twice(1.f);
    H = twice(0.f);
    for (int w = 0; w < warp; ++w) {   // the tile's tokens in front of the warp's
      const float4 q = *reinterpret_cast<const float4*>(&part[i & 1][w][Shape::channel()]);
      H = rec_step(pair(q.x, q.z), H, pair(q.y, q.w));
      P = rec_product(P, pair(q.x, q.z));
    }
    rec_meet<kRecEntry, kRecThreads>();
    if (Y) {
      const float2 e = *reinterpret_cast<const float2*>(&entry[i & 1][Shape::channel()]);
      Pair h = rec_step(P, pair(e.x, e.y), H);
      if (second) h = rec_step(other_P, h, other_H);
      if (t.whole && plain && !resets) {
        char* row = (char*)Y + t.at[2] + ((first + Shape::group() * kTok) * a.ld_y + Shape::channel()) * es;
        const uint32_t step = (uint32_t)a.ld_y * es;
#pragma unroll
        for (int k = 0; k < kTok; ++k) {
          h = fma2(av[k], h, uv[k]);
          *reinterpret_cast<Raw*>(row + (unsigned long long)step * k) = Lane::pack(h);
        }
      } else if (t.whole && !resets) {   // by single values
        T* row = Y + (long long)(t.tok0 + first + Shape::group() * kTok) * a.ld_y + t.c0 + Shape::channel();
#pragma unroll
        for (int k = 0; k < kTok; ++k) {
          h = fma2(av[k], h, uv[k]);
          rec_store(row, 0, 2, kRecSingle, h);
          row += a.ld_y;
        }
      } else {
        T* row = Y + (long long)(t.tok0 + first + Shape::group() * kTok) * a.ld_y;
#pragma unroll
        for (int k = 0; k < kTok; ++k) {
          h = rec_step(av[k], h, uv[k]);
          if (k < left) rec_store(row + k * a.ld_y, t.c0 + Shape::channel(), a.D, y_access, h);
        }
      }
    }
    __syncwarp();
  }
  rec_wait<0>();
}

constexpr int kSeqsPerSetup = 320;
struct SeqRange { int32_t tok0, n, seq; };
struct SetupArgs {
  RecSetup walk[2];        // table: where these sequences' entries begin; n_words: to clear, 0 for neither words nor ticket
  int n_walks, n_seqs;
};
template <int SEQS>
struct SeqBatch { SeqRange seq[SEQS]; };   // the longest first
__host__ __device__ __forceinline__ int tiles_of(int n, int tile) { return n > 0 && tile ? (int)(((unsigned)n + tile - 1) / tile) : 1; }
// The tickets, the words, and up to 320 sequences' entries of the tables, a warp per sequence.  Tiles lie in turn, every sequence's first, then every second, so that the tile in front of a tile is
// as far ahead of it as there are sequences left.
template <int SEQS>
__global__ void __launch_bounds__(256) rec_setup_kernel(const __grid_constant__ SetupArgs b, const __grid_constant__ SeqBatch<SEQS> batch) {
  __shared__ SeqRange seq[SEQS];
  let_successor_start();
  if constexpr (SEQS > 1)
    for (int q = threadIdx.x; q < b.n_seqs; q += 256) seq[q] = batch.seq[q];
  __syncthreads();
  wait_for_predecessor();
  for (int i = 0; i < b.n_walks; ++i) {
    const RecSetup& w = b.walk[i];
    if (w.n_words) {
      const bool one = blockIdx.x == 0 && threadIdx.x == 0;
      if (one) *w.ticket = 0;
      const long long pairs = w.n_words / 2, stride = (long long)gridDim.x * 256;
      const uint4 none = make_uint4(~0u, ~0u, ~0u, ~0u);
      for (long long j = blockIdx.x * 256ll + threadIdx.x; j < pairs; j += stride) reinterpret_cast<uint4*>(w.words)[j] = none;
      if (one && (w.n_words & 1)) w.words[w.n_words - 1] = ~0ull;
    }
    if constexpr (SEQS > 1) {
      const int lane = threadIdx.x & 31;
      for (int s = blockIdx.x * 8 + (threadIdx.x >> 5); s < b.n_seqs; s += gridDim.x * 8) {
        RecTile e{seq[s].tok0, seq[s].n, seq[s].seq, 0, tiles_of(seq[s].n, w.tile)};
        for (int k = lane; k < e.tiles; k += 32) {
          long long at = s;   // among the k-th tiles: the sequences before this one are as long at least
          if (k > 0)
            for (int q = 0; q < b.n_seqs; ++q) at += min(tiles_of(seq[q].n, w.tile), k);
          e.index = k;
          w.table[at] = e;
        }
      }
    }
  }
}

template <class T, int MODE, bool WORDS, bool ANY>
cudaError_t launch_one(const RecArgs& a, cudaStream_t stream) {
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess || (e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) return e;
  constexpr size_t smem = 4 * (size_t)RecShape<T, kTok>::TENSOR;   // two tiles of two tensors
  static_assert(rec_fit(blocks(sizeof(T)), smem, 6 * 1024), "a grid of blocks that are not all resident");
  if ((e = allow_shared<gated_recurrence_kernel<T, MODE, WORDS, ANY>>(smem)) != cudaSuccess) return e;
  const long long items = a.items;
  if ((e = launch_early(gated_recurrence_kernel<T, MODE, WORDS, ANY>, dim3((unsigned)std::min<long long>(items, (long long)blocks(sizeof(T)) * sms)), kRecThreads, smem, stream, a)) != cudaSuccess) return e;
  return launched();
}
template <class T, int MODE>
cudaError_t launch_mode(const RecArgs& a, cudaStream_t stream) {
  const bool any = rec_access<T>(a.x, a.ld_x) != kRecWide || rec_access<T>(a.g, a.ld_g) != kRecWide;
  if (a.words) return any ? launch_one<T, MODE, true, true>(a, stream) : launch_one<T, MODE, true, false>(a, stream);
  return any ? launch_one<T, MODE, false, true>(a, stream) : launch_one<T, MODE, false, false>(a, stream);
}
template <class T>
cudaError_t launch_type(const RecArgs& a, cudaStream_t stream) {
  return a.mode == kRecDecay ? launch_mode<T, kRecDecay>(a, stream) : a.mode == kRecNormed ? launch_mode<T, kRecNormed>(a, stream) : launch_mode<T, kRecGate>(a, stream);
}

}  // namespace

cudaError_t launch_gated_recurrence(const RecArgs& a, int dtype, cudaStream_t stream) {
  return dtype == TRI_INV_F32 ? launch_type<float>(a, stream) : launch_type<__nv_bfloat16>(a, stream);
}

cudaError_t launch_rec_setup(const RecSetup* walks, int n_walks, const int32_t* cu, int n_seqs, cudaStream_t stream) {
  SetupArgs b{};
  b.n_walks = n_walks;
  long long words = 0;
  for (int i = 0; i < n_walks; ++i) {
    b.walk[i] = walks[i];
    words += walks[i].n_words;
  }
  auto grid = [&]() { return dim3((unsigned)std::max<long long>(1, std::min<long long>(std::max<long long>((b.n_seqs + 7) / 8, (words / 2 + 1023) / 1024), 592))); };
  if (!cu) return words ? launch_early(rec_setup_kernel<1>, grid(), 256, 0, stream, b, SeqBatch<1>{}) : cudaSuccess;
  SeqBatch<kSeqsPerSetup> batch;
  for (int s0 = 0; s0 < n_seqs; s0 += kSeqsPerSetup) {
    b.n_seqs = std::min(kSeqsPerSetup, n_seqs - s0);
    for (int q = 0; q < b.n_seqs; ++q) batch.seq[q] = SeqRange{cu[s0 + q], cu[s0 + q + 1] - cu[s0 + q], s0 + q};
    std::sort(batch.seq, batch.seq + b.n_seqs, [](const SeqRange& x, const SeqRange& y) { return x.n != y.n ? x.n > y.n : x.seq < y.seq; });
    const cudaError_t e = launch_early(rec_setup_kernel<kSeqsPerSetup>, grid(), 256, 0, stream, b, batch);
    if (e != cudaSuccess) return e;
    words = 0;
    for (int i = 0; i < n_walks; ++i) {
      for (int q = 0; q < b.n_seqs; ++q) b.walk[i].table += tiles_of(batch.seq[q].n, b.walk[i].tile);
      b.walk[i].n_words = 0;
    }
  }
  return cudaSuccess;
}

}  // namespace tri_inv
