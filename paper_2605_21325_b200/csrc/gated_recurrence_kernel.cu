// Gated linear recurrence: the forward walk, and what both walks find in their workspace.
#include <algorithm>

#include "gated_recurrence.cuh"

namespace tri_inv {
namespace {

constexpr int kWarps = 8, kTok = kRecTile / kWarps, kThreads = 32 * kWarps;
constexpr int kStageBytes = 2 * kRecTile * kRecRow;
constexpr size_t kSmem = 2 * (size_t)kStageBytes;

template <class T, int MODE, bool WORDS>
__global__ void __launch_bounds__(kThreads, 4) gated_recurrence_kernel(const __grid_constant__ RecArgs a) {
  constexpr int N = RecLane<T>::N, CH = kRecRow / (int)sizeof(T);
  extern __shared__ __align__(128) unsigned char stages[];
  __shared__ __align__(16) float2 part[kWarps][CH];   // (P, H) of each warp's tokens
  __shared__ __align__(8) float entry[CH];            // what enters the tile
  __shared__ int drawn;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const T *X = (const T*)a.x, *G = (const T*)a.g;
  T* Y = (T*)a.y;
  const int items = a.n_segs * a.cols;
  const int x_access = rec_access<T>(X, a.ld_x), g_access = rec_access<T>(G, a.ld_g);
  const bool y_pairs = rec_access<T>(Y, a.ld_y) != kRecSingle;
  const unsigned long long limit = a.wait_limit_ns ? a.wait_limit_ns : 2000000000ull;
  wait_for_predecessor();

  // A warp asks for the rows that it alone reads, so that no barrier stands between a copy and its use.
  auto request = [&](const RecAt& t, int stage) {
    if (t.item < items) {
      const int first = warp * kTok, rows = t.n() - first;
      unsigned char* at = stages + stage * kStageBytes + first * kRecRow;
      rec_request<T, kTok>(at, X, a.ld_x, t.tok0() + first, rows, t.col * CH, a.D, x_access);
      rec_request<T, kTok>(at + kRecTile * kRecRow, G, a.ld_g, t.tok0() + first, rows, t.col * CH, a.D, g_access);
    }
    rec_commit();
  };
  // Items: with words drawn from the ticket, one ahead, so that the tiles in front of a tile are done or in the hands of blocks that run; else by a fixed stride.
  int ahead = 0;
  if (WORDS) {
    if (tid == 0) drawn = (int)atomicAdd(a.ticket, 2u);
    __syncthreads();
    ahead = drawn + 1;
  }
  RecAt now = rec_decode<WORDS>(a, WORDS ? ahead - 1 : (int)blockIdx.x, false);
  request(now, 0);
  float carried = 0.f;   // without words: what leaves the last tile, channel tid
  for (int stage = 0; now.item < items; stage ^= 1) {
    const RecAt next = rec_next<WORDS>(a, now, ahead, false);
    request(next, stage ^ 1);
    int ticket = 0;
    if (WORDS && tid == 0) ticket = (int)atomicAdd(a.ticket, 1u);
    rec_wait<1>();
    __syncwarp();
    const int n = now.n(), c0 = now.col * CH, left = n - warp * kTok;
    const unsigned char* sx = stages + stage * kStageBytes + warp * kTok * kRecRow + 4 * lane;
    float av[kTok][N], uv[kTok][N], P[N], H[N];
#pragma unroll
    for (int j = 0; j < N; ++j) { P[j] = 1.f; H[j] = 0.f; }
#pragma unroll
    for (int t = 0; t < kTok; ++t) {
      float x[N], g[N];
      RecLane<T>::widen(x, *reinterpret_cast<const uint32_t*>(sx + t * kRecRow));
      RecLane<T>::widen(g, *reinterpret_cast<const uint32_t*>(sx + (kRecTile + t) * kRecRow));
#pragma unroll
      for (int j = 0; j < N; ++j) {
        float m, over;
        rec_factors<MODE>(g[j], av[t][j], m, over);
        uv[t][j] = m * x[j];
        if (t >= left) { av[t][j] = 1.f; uv[t][j] = 0.f; }
        P[j] *= av[t][j];
        H[j] = rec_step(av[t][j], H[j], uv[t][j]);
      }
    }
#pragma unroll
    for (int j = 0; j < N; ++j) part[warp][lane * N + j] = make_float2(P[j], H[j]);
    __syncthreads();
    // what the warps before this one make of the tile's entry
#pragma unroll
    for (int j = 0; j < N; ++j) { P[j] = 1.f; H[j] = 0.f; }
    for (int w = 0; w < warp; ++w)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float2 q = part[w][lane * N + j];
        P[j] *= q.x;
        H[j] = rec_step(q.x, H[j], q.y);
      }
    if (tid < CH) {   // a channel of the tile
      float TP = 1.f, TH = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float2 q = part[w][tid];
        TP *= q.x;
        TH = rec_step(q.x, TH, q.y);
      }
      const int c = c0 + tid;
      const bool in = c < a.D, first = now.index == 0, last = now.index + 1 == now.tiles;
      const long long slot = rec_slot(now.begin, now.seq) + now.index;
      unsigned long long* word = WORDS ? a.words + slot * a.D + c : nullptr;
      const bool stalled = a.test_stall && now.item == 0;
      float h = 0.f;
      if (in) {
        if (first) h = a.h0 ? a.h0[(long long)now.seq * a.D + c] : 0.f;
        else if (!WORDS) h = carried;
        else {
          if (!last) rec_post(word, TP, TH);
          h = rec_look_back(word - a.D, a.D, now.index, limit, a.status);
        }
        carried = rec_step(TP, h, TH);
        if (last) { if (a.h_out) a.h_out[(long long)now.seq * a.D + c] = carried; }
        else {
          if (WORDS && !stalled) rec_post(word, 0.f, carried);
          if (a.carries) a.carries[slot * a.D + c] = carried;
        }
      }
      entry[tid] = h;
    }
    if (WORDS && tid == 0) drawn = ticket;
    __syncthreads();
    if (WORDS) ahead = drawn;
    if (Y) {
      float h[N];
#pragma unroll
      for (int j = 0; j < N; ++j) h[j] = rec_step(P[j], entry[lane * N + j], H[j]);
      T* row = Y + (now.tok0() + warp * kTok) * a.ld_y;
#pragma unroll
      for (int t = 0; t < kTok; ++t) {
#pragma unroll
        for (int j = 0; j < N; ++j) h[j] = rec_step(av[t][j], h[j], uv[t][j]);
        if (t < left) rec_store(row + t * a.ld_y, c0 + lane * N, a.D, y_pairs, h);
      }
    }
    now = next;
    __syncwarp();
  }
  rec_wait<0>();
}

constexpr int kSeqsPerSetup = 320;
struct SeqRange { int32_t tok0, n, seq; };
struct SetupArgs {
  unsigned int* ticket;
  unsigned long long* words;
  RecTile* table;          // where these sequences' entries begin
  long long n_words;       // to clear; 0: neither words nor ticket
  int n_seqs, by_tile;
};
template <int SEQS>
struct SeqBatch { SeqRange seq[SEQS]; };   // the longest first
__host__ __device__ __forceinline__ int tiles_of(int n) { return n > 0 ? (int)(((unsigned)n + kRecTile - 1) / kRecTile) : 1; }
// The ticket, the words, and up to 320 sequences' entries of the table, a warp per sequence.  Tiles lie in turn, every sequence's first, then every second, so that the tile in front of a tile is
// as far ahead of it as there are sequences left.
template <int SEQS>
__global__ void __launch_bounds__(256) rec_setup_kernel(const __grid_constant__ SetupArgs b, const __grid_constant__ SeqBatch<SEQS> batch) {
  __shared__ int tiles[SEQS];
  let_successor_start();
  if constexpr (SEQS > 1)
    for (int q = threadIdx.x; q < b.n_seqs; q += 256) tiles[q] = tiles_of(batch.seq[q].n);
  __syncthreads();
  wait_for_predecessor();
  if (b.n_words) {
    const bool one = blockIdx.x == 0 && threadIdx.x == 0;
    if (one) *b.ticket = 0;
    const long long pairs = b.n_words / 2, stride = (long long)gridDim.x * 256;
    const uint4 none = make_uint4(~0u, ~0u, ~0u, ~0u);
    for (long long i = blockIdx.x * 256ll + threadIdx.x; i < pairs; i += stride) reinterpret_cast<uint4*>(b.words)[i] = none;
    if (one && (b.n_words & 1)) b.words[b.n_words - 1] = ~0ull;
  }
  if constexpr (SEQS > 1) {
    const int lane = threadIdx.x & 31;
    for (int s = blockIdx.x * 8 + (threadIdx.x >> 5); s < b.n_seqs; s += gridDim.x * 8) {
      const SeqRange r = batch.seq[s];
      RecTile e{r.tok0, r.n, r.seq, 0, tiles[s]};
      if (!b.by_tile) {
        if (lane == 0) b.table[s] = e;
        continue;
      }
      for (int k = lane; k < e.tiles; k += 32) {
        long long at = s;   // among the k-th tiles: the sequences before this one are as long at least
        for (int q = 0; q < b.n_seqs; ++q) at += min(tiles[q], k);
        e.index = k;
        b.table[at] = e;
      }
    }
  }
}

template <class T, int MODE, bool WORDS>
cudaError_t launch_one(const RecArgs& a, cudaStream_t stream) {
  static int sms[64] = {0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  int n = sms[dev];
  if (!n) {
    if ((e = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) return e;
    sms[dev] = n;
  }
  if ((e = allow_shared<gated_recurrence_kernel<T, MODE, WORDS>>(kSmem)) != cudaSuccess) return e;
  const long long items = (long long)a.n_segs * a.cols;
  if ((e = launch_early(gated_recurrence_kernel<T, MODE, WORDS>, dim3((unsigned)std::min<long long>(items, 4ll * n)), kThreads, kSmem, stream, a)) != cudaSuccess) return e;
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

cudaError_t launch_gated_recurrence(const RecArgs& a, int dtype, cudaStream_t stream) {
  return dtype == TRI_INV_F32 ? launch_type<float>(a, stream) : launch_type<__nv_bfloat16>(a, stream);
}

cudaError_t launch_rec_setup(unsigned int* ticket, unsigned long long* words, long long n_words, RecTile* table, const int32_t* cu, int n_seqs, cudaStream_t stream) {
  SetupArgs b{ticket, words, table, words ? n_words : 0, 0, words != nullptr};
  auto grid = [&]() { return dim3((unsigned)std::max<long long>(1, std::min<long long>(std::max<long long>((b.n_seqs + 7) / 8, (b.n_words / 2 + 1023) / 1024), 592))); };
  if (!cu) return b.n_words ? launch_early(rec_setup_kernel<1>, grid(), 256, 0, stream, b, SeqBatch<1>{}) : cudaSuccess;
  SeqBatch<kSeqsPerSetup> batch;
  for (int s0 = 0; s0 < n_seqs; s0 += kSeqsPerSetup) {
    long long entries = 0;
    b.n_seqs = std::min(kSeqsPerSetup, n_seqs - s0);
    for (int q = 0; q < b.n_seqs; ++q) {
      batch.seq[q] = SeqRange{cu[s0 + q], cu[s0 + q + 1] - cu[s0 + q], s0 + q};
      entries += words ? tiles_of(batch.seq[q].n) : 1;
    }
    std::sort(batch.seq, batch.seq + b.n_seqs, [](const SeqRange& x, const SeqRange& y) { return x.n != y.n ? x.n > y.n : x.seq < y.seq; });
    const cudaError_t e = launch_early(rec_setup_kernel<kSeqsPerSetup>, grid(), 256, 0, stream, b, batch);
    if (e != cudaSuccess) return e;
    b.table += entries;
    b.n_words = 0;
  }
  return cudaSuccess;
}

}  // namespace tri_inv
