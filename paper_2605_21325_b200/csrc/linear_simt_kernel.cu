// Linear attention with a decay for each head, on the CUDA cores: every shape and storage type, fp32 arithmetic throughout.
//
// One CTA walks one (segment, head, slice of 64 value columns) tile after tile of 64 tokens (the walk's formulas: linear_attention.cuh); value
// columns of the state never mix.  q, k, v, P and the state's slice lie in shared memory; each of the four products is made of
// thread tiles of 4 x 4 (the state: 4 x 4 for every 64 features), rows read as float4 along the summed index, so that a thread reads 8 x 16 bytes for 64 FMAs.
// What bounds it: shared memory's data path (a thread's 8 reads take about as long as its 64 FMAs) and, with few blocks, the latency of a tile's steps.  fp32 tiles arrive by
// asynchronous copies, q, k and v at once, the next tile's while this one's output is stored.  The state's increment is formed only where another tile or the caller takes the state, so that a sequence cut into
// single tiles costs no more products than an uncut one: one in the pass for the states, which keeps them in registers, three in the other.  Three blocks an SM at d_k <= 64 (80 registers a thread and a
// few spills; with two, fp32 2 x 2048 x 8 heads of 64 64 us forward and 162 backward, 66 and 154 so, five packed sequences 57 and 47), two at 128.
// Measured, fp32, calls in a captured graph: 16 x 64 tokens x 8 heads of 128 30 us, 0.37 of the FMAs' rate (the work with a state); 1 x 4096 x 8 of 128 186 (loads through registers and always all four
// products: 252); 4 x 4096 x 16 of 128 1322, 0.22 of that rate; the gradient of five sequences of up to 1000 tokens x 4 heads of 64 50 (87).  bf16, 4 x 4096 x 16 of 256: 6451 us, 12 TFLOP/s.  (512 threads with tiles of 4 x 2: 16 x 64 x 8 of 128 in 52 us, 45 with these before the copies.)
#include <algorithm>
#include <type_traits>

#include "linear_attention.cuh"

namespace tri_inv {
namespace {

constexpr int L = kLinTile, SL = 64, kThreadsLin = 256;
constexpr int kFew = 16;   // a tile of at most this many tokens: a sixteenth of P, a quarter of the other rows

struct alignas(8) Half4 { __nv_bfloat162 a, b; };
template <class T>
__device__ __forceinline__ float4 load4(const T* p) {
  if constexpr (sizeof(T) == 4) {
    return *reinterpret_cast<const float4*>(p);
  } else {
    const Half4 x = *reinterpret_cast<const Half4*>(p);
    const float2 a = __bfloat1622float2(x.a), b = __bfloat1622float2(x.b);
    return make_float4(a.x, a.y, b.x, b.y);
  }
}
template <class T>
__device__ __forceinline__ void store4(T* p, float4 x) {
  if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(p) = x;
  else *reinterpret_cast<Half4*>(p) = Half4{__floats2bfloat162_rn(x.x, x.y), __floats2bfloat162_rn(x.z, x.w)};
}
__device__ __forceinline__ float4 lds4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ void fma4(float (&d)[4], float a, float4 b) {
  d[0] = fmaf(a, b.x, d[0]); d[1] = fmaf(a, b.y, d[1]); d[2] = fmaf(a, b.z, d[2]); d[3] = fmaf(a, b.w, d[3]);
}

// 16 bytes to shared memory, zeros where there is nothing to read
__device__ __forceinline__ void fetch16(float* dst, const float* src, bool valid) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src), "r"(valid ? 16 : 0) : "memory");
}

// MK: groups of 64 features.  WHOLE: outputs; otherwise the pass that only wants states (LinArgs::state_only).
template <class T, int MK, bool WHOLE>
__global__ void __launch_bounds__(kThreadsLin, MK == 4 ? 1 : MK == 2 ? 2 : 3) linear_simt_kernel(const __grid_constant__ LinArgs a, int max_slices) {
  extern __shared__ __align__(16) float sm[];
  constexpr bool F32 = sizeof(T) == 4;
  int x = blockIdx.x;
  const int slice = x % max_slices; x /= max_slices;
  const int h = x % a.H; x /= a.H;
  const int s = x % a.n_segs, wi = x / a.n_segs;
  const LinWalk& w = a.walk[wi];
  const int c0 = slice * SL;
  wait_for_predecessor();
  if (c0 >= w.d_v) return;
  // Rows without padding, so that two blocks of d_k = 128 fit an SM.  Only k is read by rows that differ between lanes: its pieces of 16 bytes change places within 128 bytes by the
  // row (piece ^ row & 7), or, where rows are not whole 128 bytes, rows are padded by one.
  const int dk = w.d_k, ldk = dk % 32 ? dk + 4 : dk, swz = dk % 32 ? 0 : 7;
  float *sk = sm, *sv = sk + L * max(ldk, SL), *pw = sv + L * SL, *wt = pw + L + 4, *sq = wt + L, *sS = sq + L * dk;   // pw: lambda^0 .. lambda^64; wt: the factors of a tile's tokens in the increment
  float* sp = sk;   // P lies where k was: k's other reader, the state's increment, comes first
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, warp = tid >> 5, lane = tid & 31;
  const LinSeg g = lin_segment(a, s);
  float* s_out = lin_exit_state(a, w, wi, s, g, h);
  if (!WHOLE && !s_out) return;
  const T *Q = (const T*)w.q, *K = (const T*)w.k, *V = (const T*)w.v;
  T* O = (T*)w.out;
  const int n_tiles = (g.n + L - 1) / L, b = w.back;
  const size_t row_k = (size_t)a.H * dk, row_v = (size_t)a.H * w.d_v;
  auto tile_at = [&](int it) { return b ? n_tiles - 1 - it : it; };
  auto rows_at = [&](int it) { return min(L, g.n - tile_at(it) * L); };
  // A tile's rows of n features to shared memory, a warp a row, 4 features a lane (fp32: asynchronously)
  auto fetch_rows = [&](const T* src, size_t row, float* dst, int ld, int turn, int rows) {
#pragma unroll 4
    for (int i = warp; i < (rows <= kFew ? kFew : L); i += kThreadsLin / 32) {
#pragma unroll
      for (int m = 0; m < (MK + 1) / 2; ++m) {
        const int d = 4 * (lane + 32 * m);
        if (d < dk) {
          float* to = dst + i * ld + (d ^ (i & turn) << 2);
          if constexpr (F32) fetch16(to, src + (i < rows ? i * row : 0) + d, i < rows);
          else *reinterpret_cast<float4*>(to) = i < rows ? load4(src + i * row + d) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
      }
    }
  };
  auto request = [&](int it) {
    const int rows = rows_at(it);
    const size_t at = (size_t)(g.tok0 + tile_at(it) * L) * a.H + h;
    fetch_rows(K + at * dk, row_k, sk, ldk, swz, rows);
    const T* Vt = V + at * w.d_v + c0;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int i = ty + 16 * r, c = 4 * tx;
      const bool in = i < rows && c0 + c < w.d_v;
      if constexpr (F32) fetch16(sv + i * SL + c, Vt + (in ? i * row_v + c : 0), in);
      else *reinterpret_cast<float4*>(sv + i * SL + c) = in ? load4(Vt + i * row_v + c) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    if constexpr (WHOLE) fetch_rows(Q + at * dk, row_k, sq, dk, 0, rows);
    if constexpr (F32) asm volatile("cp.async.commit_group;" ::: "memory");
  };
  if (n_tiles > 0) request(0);
  const float l2 = lin_log2_decay(a, h);
  if (tid <= L) pw[tid] = exp2f(l2 * tid);
  __syncthreads();
  float state[WHOLE ? 1 : MK][4][4] = {};   // in the pass that only wants it: from zero, in registers
  bool fresh = false;   // the state is still zero: not in shared memory yet, and no part of the first tile's outputs
  if constexpr (WHOLE) {
    bool turned;
    const float* s_in = lin_entry_state(a, w, wi, s, g, h, &turned);
    fresh = !s_in;
    if (fresh) {
    } else if (!turned) {
#pragma unroll 4
      for (int e = tid; e < dk * (SL / 4); e += kThreadsLin) {
        const int d = e / (SL / 4), c = 4 * (e % (SL / 4));
        *reinterpret_cast<float4*>(sS + d * SL + c) = c0 + c < w.d_v ? lds4(s_in + (size_t)d * w.d_v + c0 + c) : make_float4(0.f, 0.f, 0.f, 0.f);
      }
    } else {
      // a warp: 8 columns x 16 features, so that its stores meet in fours on a bank (a column x 32 features: all 32)
      for (int e = warp; e < SL / 8 * ((dk + 15) / 16); e += kThreadsLin / 32) {
        const int c = 8 * (e % (SL / 8)) + (lane & 7), d = 16 * (e / (SL / 8)) + 4 * (lane >> 3);
        if (d < dk) {
          const float4 y = c0 + c < w.d_v ? lds4(s_in + (size_t)(c0 + c) * dk + d) : make_float4(0.f, 0.f, 0.f, 0.f);
          sS[d * SL + c] = y.x; sS[(d + 1) * SL + c] = y.y; sS[(d + 2) * SL + c] = y.z; sS[(d + 3) * SL + c] = y.w;
        }
      }
    }
  }
  for (int it = 0; it < n_tiles; ++it) {
    const int tok0 = g.tok0 + tile_at(it) * L, rows = rows_at(it);
    if (tid < L) wt[tid] = tid < rows ? w.k_factor * pw[b ? tid + 1 : rows - 1 - tid] : 0.f;
    if constexpr (F32) asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();
    // the state's increment, features 64 m + 4 ty .. and columns 4 tx ..: where another tile or the caller takes the state
    const bool passes = it + 1 < n_tiles || s_out;
    float ds[MK][4][4] = {};
    if (passes) {
      for (int j0 = 0; j0 < rows; j0 += 4) {   // (rows of k and v behind the last are zeros, and so are their factors)
        const float4 w4 = lds4(wt + j0);
        const float wj[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int j = j0 + i;
          float4 vv = lds4(sv + j * SL + 4 * tx);
          vv.x *= wj[i]; vv.y *= wj[i]; vv.z *= wj[i]; vv.w *= wj[i];
#pragma unroll
          for (int m = 0; m < MK; ++m) {
            const int d = 64 * m + 4 * ty;
            if (d < dk) {
              const float4 kk = lds4(sk + j * ldk + (d ^ (j & swz) << 2));
              fma4(ds[m][0], kk.x, vv); fma4(ds[m][1], kk.y, vv); fma4(ds[m][2], kk.z, vv); fma4(ds[m][3], kk.w, vv);
            }
          }
        }
      }
    }
    const LinFade fade = lin_fade(l2, rows);   // S <- lambda^rows S + the increment
    if constexpr (WHOLE) {
      // R: 16 R of the tile's rows are in use
      auto outputs = [&](auto rows_in_use) {
        constexpr int R = decltype(rows_in_use)::value;
        {   // P, rows ty + 16 r, columns tx + 16 m
          float acc[R][R] = {};
          const int turn = (tx & swz) << 2;
#pragma unroll 2
          for (int d = 0; d < dk; d += 4) {
            float4 kk[R];
#pragma unroll
            for (int m = 0; m < R; ++m) kk[m] = lds4(sk + (tx + 16 * m) * ldk + (d ^ turn));
#pragma unroll
            for (int r = 0; r < R; ++r) {
              const float4 qq = lds4(sq + (ty + 16 * r) * dk + d);
#pragma unroll
              for (int m = 0; m < R; ++m) acc[r][m] = fmaf(qq.x, kk[m].x, acc[r][m]);
#pragma unroll
              for (int m = 0; m < R; ++m) acc[r][m] = fmaf(qq.y, kk[m].y, acc[r][m]);
#pragma unroll
              for (int m = 0; m < R; ++m) acc[r][m] = fmaf(qq.z, kk[m].z, acc[r][m]);
#pragma unroll
              for (int m = 0; m < R; ++m) acc[r][m] = fmaf(qq.w, kk[m].w, acc[r][m]);
            }
          }
          __syncthreads();   // k has been read
#pragma unroll
          for (int r = 0; r < R; ++r)
#pragma unroll
            for (int m = 0; m < R; ++m) {
              const int i = ty + 16 * r, j = tx + 16 * m, gap = b ? j - i : i - j;
              sp[i * SL + j] = gap >= 0 ? acc[r][m] * (w.k_factor * pw[gap]) : 0.f;
            }
        }
        __syncthreads();
        float acc[R][4] = {};   // rows ty + 16 r, columns 4 tx ..
        if (!fresh) {
#pragma unroll 2
          for (int d = 0; d < dk; d += 4) {
            float4 ss[4];
#pragma unroll
            for (int m = 0; m < 4; ++m) ss[m] = lds4(sS + (d + m) * SL + 4 * tx);
#pragma unroll
            for (int r = 0; r < R; ++r) {
              const float4 qq = lds4(sq + (ty + 16 * r) * dk + d);
              fma4(acc[r], qq.x, ss[0]); fma4(acc[r], qq.y, ss[1]); fma4(acc[r], qq.z, ss[2]); fma4(acc[r], qq.w, ss[3]);
            }
          }
#pragma unroll
          for (int r = 0; r < R; ++r) {
            const int i = ty + 16 * r, p = b ? rows - 1 - i : i;
            const float f = i < rows ? pw[p + 1 - b] : 0.f;
#pragma unroll
            for (int m = 0; m < 4; ++m) acc[r][m] *= f;
          }
        }
#pragma unroll 2
        for (int j = 0; j < 16 * R; j += 4) {
          float4 vv[4];
#pragma unroll
          for (int m = 0; m < 4; ++m) vv[m] = lds4(sv + (j + m) * SL + 4 * tx);
#pragma unroll
          for (int r = 0; r < R; ++r) {
            const float4 pp = lds4(sp + (ty + 16 * r) * SL + j);
            fma4(acc[r], pp.x, vv[0]); fma4(acc[r], pp.y, vv[1]); fma4(acc[r], pp.z, vv[2]); fma4(acc[r], pp.w, vv[3]);
          }
        }
        __syncthreads();   // every reader of the tile and of the entering state is through
        if (it + 1 < n_tiles) request(it + 1);
        T* Ot = O + ((size_t)tok0 * a.H + h) * w.d_v + c0 + 4 * tx;
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const int i = ty + 16 * r;
          if (i < rows && c0 + 4 * tx < w.d_v)
            store4(Ot + i * row_v, make_float4(w.out_factor * acc[r][0], w.out_factor * acc[r][1], w.out_factor * acc[r][2], w.out_factor * acc[r][3]));
        }
      };
      if (rows <= kFew) outputs(std::integral_constant<int, 1>{});
      else outputs(std::integral_constant<int, L / 16>{});
      if (passes) {
#pragma unroll
        for (int m = 0; m < MK; ++m)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int d = 64 * m + 4 * ty + r;
            if (d < dk) {
              float4 y = fresh ? make_float4(0.f, 0.f, 0.f, 0.f) : lds4(sS + d * SL + 4 * tx);
              y.x = fmaf(y.x, fade.less, fade.keep * y.x) + ds[m][r][0]; y.y = fmaf(y.y, fade.less, fade.keep * y.y) + ds[m][r][1];
              y.z = fmaf(y.z, fade.less, fade.keep * y.z) + ds[m][r][2]; y.w = fmaf(y.w, fade.less, fade.keep * y.w) + ds[m][r][3];
              *reinterpret_cast<float4*>(sS + d * SL + 4 * tx) = y;
            }
          }
        fresh = false;
      }
    } else {
      __syncthreads();   // the tile has been read
      if (it + 1 < n_tiles) request(it + 1);
#pragma unroll
      for (int m = 0; m < MK; ++m)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int c = 0; c < 4; ++c) state[m][r][c] = fmaf(state[m][r][c], fade.less, fade.keep * state[m][r][c]) + ds[m][r][c];
    }
  }
  if (s_out) {
    if constexpr (WHOLE) {
      __syncthreads();
#pragma unroll 4
      for (int e = tid; e < dk * (SL / 4); e += kThreadsLin) {
        const int d = e / (SL / 4), c = 4 * (e % (SL / 4));
        if (c0 + c < w.d_v) *reinterpret_cast<float4*>(s_out + (size_t)d * w.d_v + c0 + c) = fresh ? make_float4(0.f, 0.f, 0.f, 0.f) : lds4(sS + d * SL + c);
      }
    } else if (c0 + 4 * tx < w.d_v) {
#pragma unroll
      for (int m = 0; m < MK; ++m)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (64 * m + 4 * ty + r < dk)
            *reinterpret_cast<float4*>(s_out + (size_t)(64 * m + 4 * ty + r) * w.d_v + c0 + 4 * tx) = make_float4(state[m][r][0], state[m][r][1], state[m][r][2], state[m][r][3]);
    }
  }
}

template <class T, int MK, bool WHOLE>
cudaError_t launch_form(const LinArgs& a, int max_dk, int max_dv, cudaStream_t stream) {
  int max_ldk = SL;
  for (int i = 0; i < a.n_walks; ++i) max_ldk = std::max(max_ldk, a.walk[i].d_k % 32 ? a.walk[i].d_k + 4 : a.walk[i].d_k);
  size_t words = (size_t)L * max_ldk + (size_t)L * SL + 2 * L + 4;
  if (WHOLE) words += (size_t)(L + SL) * max_dk;
  const size_t smem = words * sizeof(float);
  const cudaError_t e = allow_shared<linear_simt_kernel<T, MK, WHOLE>>(smem);
  if (e != cudaSuccess) return e;
  const int slices = (max_dv + SL - 1) / SL;
  const long long grid = (long long)slices * a.H * a.n_segs * a.n_walks;
  if (grid > 0x7fffffffLL) return cudaErrorInvalidValue;
  const cudaError_t l = launch_early(linear_simt_kernel<T, MK, WHOLE>, dim3((unsigned)grid), kThreadsLin, smem, stream, a, slices);
  return l == cudaSuccess ? launched() : l;
}
template <class T, int MK>
cudaError_t launch_one(const LinArgs& a, int max_dk, int max_dv, cudaStream_t stream) {
  return a.state_only ? launch_form<T, MK, false>(a, max_dk, max_dv, stream) : launch_form<T, MK, true>(a, max_dk, max_dv, stream);
}

// One block for 256 elements of the states of one (walk, sequence, head): element by element along the sequence's segments.
__global__ void __launch_bounds__(256) linear_join_kernel(const __grid_constant__ LinArgs a, int parts) {
  wait_for_predecessor();
  int x = blockIdx.x;
  const int part = x % parts; x /= parts;
  const int h = x % a.H; x /= a.H;
  const int q = x % a.n_seqs, wi = x / a.n_seqs;
  const LinWalk& w = a.walk[wi];
  const int s0 = a.table ? a.first[q] : q * a.segs_per_seq;   // the sequence's segments follow one another
  const int n = a.table ? (q + 1 < a.n_seqs ? a.first[q + 1] : a.n_segs) - s0 : a.segs_per_seq;
  const int size = w.d_k * w.d_v, e = part * 256 + threadIdx.x;
  if (n == 1 || e >= size) return;   // nothing to join in one segment
  const int seq = lin_segment(a, s0).seq;
  const float l2 = lin_log2_decay(a, h);
  const float* s_in = w.s_in ? w.s_in + ((size_t)seq * a.H + h) * size : nullptr;
  float S = s_in ? s_in[w.s_turned ? (e % w.d_v) * w.d_k + e / w.d_v : e] : 0.f;
  float* at = a.seg_state + ((size_t)wi * a.n_segs * a.H + h) * size + e;
  for (int i0 = 0; i0 < n; i0 += 8) {   // eight segments' states and lengths on their way at once
    float own[8], keep[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const int i = i0 + q, s = s0 + (w.back ? n - 1 - i : i);
      own[q] = i + 1 < n ? at[(size_t)s * a.H * size] : 0.f;
      keep[q] = i < n ? exp2f(l2 * lin_segment(a, s).n) : 0.f;
    }
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const int i = i0 + q, s = s0 + (w.back ? n - 1 - i : i);
      if (i < n) at[(size_t)s * a.H * size] = S;
      S = fmaf(S, keep[q], own[q]);
    }
  }
}

constexpr int kSeqsPerTable = 320;
struct SeqRange { int32_t tok0, n, seq; };
struct TableBatch {
  SeqRange seq[kSeqsPerTable];
  int32_t n_seqs, first_seq, first_seg, seg_tokens;
};
// A warp per sequence, as in the chunk table (chunk_table.cu): its lanes sum the segments of the sequences before it.
__global__ void __launch_bounds__(256) linear_table_kernel(LinSeg* tab, int32_t* first, const __grid_constant__ TableBatch b) {
  __shared__ SeqRange seq[kSeqsPerTable];
  const int lane = threadIdx.x & 31, s = blockIdx.x * 8 + (threadIdx.x >> 5);
  for (int q = threadIdx.x; q < b.n_seqs; q += 256) seq[q] = b.seq[q];
  __syncthreads();
  let_successor_start();
  wait_for_predecessor();
  if (s >= b.n_seqs) return;
  auto segs = [&](int q) { return max(1, (int)(((unsigned)seq[q].n + (unsigned)b.seg_tokens - 1u) / (unsigned)b.seg_tokens)); };   // (the sum may pass 2^31 - 1)
  int before = 0;
  for (int q = lane; q < s; q += 32) before += segs(q);
#pragma unroll
  for (int m = 16; m >= 1; m >>= 1) before += __shfl_xor_sync(0xffffffffu, before, m);
  const int n = segs(s);
  if (lane == 0) first[b.first_seq + s] = b.first_seg + before;
  for (int i = lane; i < n; i += 32) {
    const int at = i * b.seg_tokens;
    tab[b.first_seg + before + i] = LinSeg{seq[s].tok0 + at, min(b.seg_tokens, seq[s].n - at), seq[s].seq, (i == 0 ? 1 : 0) | (i == n - 1 ? 2 : 0)};
  }
}

}  // namespace

cudaError_t launch_linear_simt(const LinArgs& a, int kv_dtype, cudaStream_t stream) {
  int dk = 0, dv = 0;
  for (int i = 0; i < a.n_walks; ++i) { dk = std::max(dk, a.walk[i].d_k); dv = std::max(dv, a.walk[i].d_v); }
  const bool f32 = kv_dtype == TRI_INV_F32;
  if (dk <= 64) return f32 ? launch_one<float, 1>(a, dk, dv, stream) : launch_one<__nv_bfloat16, 1>(a, dk, dv, stream);
  if (dk <= 128) return f32 ? launch_one<float, 2>(a, dk, dv, stream) : launch_one<__nv_bfloat16, 2>(a, dk, dv, stream);
  return f32 ? launch_one<float, 4>(a, dk, dv, stream) : launch_one<__nv_bfloat16, 4>(a, dk, dv, stream);
}

cudaError_t launch_linear_join(const LinArgs& a, cudaStream_t stream) {
  const int parts = (a.walk[0].d_k * a.walk[0].d_v + 255) / 256;
  const long long grid = (long long)parts * a.H * a.n_seqs * a.n_walks;
  if (grid > 0x7fffffffLL) return cudaErrorInvalidValue;
  const cudaError_t e = launch_early(linear_join_kernel, dim3((unsigned)grid), 256, 0, stream, a, parts);
  return e == cudaSuccess ? launched() : e;
}

cudaError_t launch_linear_table(LinSeg* dev_tab, int32_t* dev_first, int seg_tokens, const tri_inv_desc* d, cudaStream_t stream) {
  TableBatch b;
  b.seg_tokens = seg_tokens;
  b.first_seg = 0;
  for (int s0 = 0; s0 < d->n_seqs; s0 += kSeqsPerTable) {
    b.n_seqs = std::min(kSeqsPerTable, d->n_seqs - s0);
    b.first_seq = s0;
    for (int q = 0; q < b.n_seqs; ++q) b.seq[q] = SeqRange{d->cu_seqlens[s0 + q], d->cu_seqlens[s0 + q + 1] - d->cu_seqlens[s0 + q], s0 + q};
    // the longest first, so that blocks, and the items of a persistent block, end about together
    std::sort(b.seq, b.seq + b.n_seqs, [](const SeqRange& x, const SeqRange& y) { return x.n != y.n ? x.n > y.n : x.seq < y.seq; });
    const cudaError_t e = launch_early(linear_table_kernel, dim3((b.n_seqs + 7) / 8), 256, 0, stream, dev_tab, dev_first, b);
    if (e != cudaSuccess) return e;
    for (int q = 0; q < b.n_seqs; ++q) b.first_seg += (int)std::max(1ll, ((long long)b.seq[q].n + seg_tokens - 1) / seg_tokens);
  }
  return cudaSuccess;
}

}  // namespace tri_inv
