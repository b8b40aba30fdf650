// Gated linear recurrence: what its files share.
//
// Per sequence and channel   h_t = a_t h_{t-1} + u_t,   with a and u from what the projections give (x, g) by the mode:
//     decay   a = exp g,        u = x
//     normed  a = exp g,        u = sqrt(1 - a^2) x      (0 x where g >= 0)
//     gate    a = 1/(1+e^-g),   u = (1 - a) x
// and its gradient, with c_t what reaches token t - 1 from token t (c behind the last token: dh, the gradient of the final state):
//     e_t = dy_t + c_{t+1},   c_t = a_t e_t,   dx_t = m_t e_t (m: what multiplies x in u),   dh0 = c_0,
//     dg_t = e_t w_t,   w_t = a_t h_{t-1} (decay),   a_t h_{t-1} - a_t^2 / m_t x_t (normed),   (h_{t-1} - x_t) a_t (1 - a_t) (gate)
//
// Both are walks over tiles of kRecTile tokens of kRecRow bytes of channels.  A tile is an affine map of what enters it, (P, H): h -> P h + H,
// and so is a run of tiles; the tokens of a warp, the warps of a tile and the tiles of a sequence join by the same rule.
#pragma once
#include "common.cuh"

namespace tri_inv {

constexpr int kRecTile = 64;      // tokens of a tile
constexpr int kRecRow = 128;      // bytes of its channels: 64 in bf16, 32 in fp32

// An entry of the table of packed sequences: a tile, or a whole sequence (index 0)
struct RecTile {
  int32_t tok0, n, seq;     // the SEQUENCE's first token, its length and number
  int32_t index, tiles;     // the tile, of how many
};

// Where a tile's words and carried state lie: sequences of any length leave no two tiles at one place.
__host__ __device__ __forceinline__ long long rec_slot(long long tok0, int seq) { return tok0 / kRecTile + seq; }

struct RecArgs {
  const void *x, *g, *dy;          // dy: gradient only
  void *y, *dx, *dg;               // y: null where only the carried states are wanted
  long long ld_x, ld_g, ld_dy, ld_y, ld_dx, ld_dg;   // values from one token to the next
  const float* h0;                 // [n_seqs, D] or null
  float* h_out;                    // [n_seqs, D] or null
  float* carries;                  // [slots, D]: the state behind each tile; written by the forward walk (or null), read by the gradient
  const float* dh;                 // gradient: [n_seqs, D] or null
  float* dh0;                      // [n_seqs, D] or null
  unsigned long long* words;       // [slots, D] (P, H) of each tile, or (0, what leaves it); all ones: not there yet.  Null: whole sequences are walked
  unsigned int* ticket;            // next item, with words
  const RecTile* table;            // packed sequences: tiles (with words) or whole sequences; null: dense
  int n_segs;                      // entries of the table, or tiles (whole sequences) of the dense form
  int n_seqs, T, D, cols;          // cols: column tiles
  int mode;
  int* status;
  unsigned long long wait_limit_ns;   // 0: two seconds
  int test_stall;                  // self-test: the first tile of the first sequence's first columns leaves no word
};

cudaError_t launch_gated_recurrence(const RecArgs& a, int dtype, cudaStream_t stream);
cudaError_t launch_gated_recurrence_backward(const RecArgs& a, int dtype, cudaStream_t stream);
// What the walks find in their workspace: the ticket (zero), the words (all ones; null: none, the table then holds whole sequences) and the table of packed sequences
// from the host offsets `cu` (null: dense, no table).
cudaError_t launch_rec_setup(unsigned int* ticket, unsigned long long* words, long long n_words, RecTile* table, const int32_t* cu, int n_seqs, cudaStream_t stream);

struct RecStepArgs {
  const void *x, *g;
  void* y;
  long long ld_x, ld_g, ld_y;
  float* h;                        // [n_slots, D]
  const int32_t* slots;            // [B] or null: row b has slot b
  int B, D, n_slots, mode;
  int* status;
};
cudaError_t launch_gated_recurrence_step(const RecStepArgs& a, int dtype, cudaStream_t stream);

#ifdef __CUDACC__
// ---- device side

enum : int { kRecDecay = TRI_INV_REC_DECAY, kRecNormed = TRI_INV_REC_NORMED, kRecGate = TRI_INV_REC_GATE };

// A channel pair (bf16) or a channel (fp32) of a lane
template <class T> struct RecLane;
template <> struct RecLane<__nv_bfloat16> {
  static constexpr int N = 2;
  static __device__ __forceinline__ void widen(float (&v)[2], uint32_t raw) { v[0] = __uint_as_float(raw << 16); v[1] = __uint_as_float(raw & 0xffff0000u); }
  static __device__ __forceinline__ uint32_t pack(const float (&v)[2]) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(v[0], v[1]);
    return reinterpret_cast<const uint32_t&>(p);
  }
};
template <> struct RecLane<float> {
  static constexpr int N = 1;
  static __device__ __forceinline__ void widen(float (&v)[1], uint32_t raw) { v[0] = __uint_as_float(raw); }
  static __device__ __forceinline__ uint32_t pack(const float (&v)[1]) { return __float_as_uint(v[0]); }
};

// 1 - e^g for g in [-1/4, 0], from the series of (e^g - 1) / g to the seventh power: the first term left out is 1/8! g^7 < 2^-29 of the sum
__device__ __forceinline__ float rec_fall(float g) {
  float s = 1.f / 5040.f;
  s = fmaf(s, g, 1.f / 720.f);
  s = fmaf(s, g, 1.f / 120.f);
  s = fmaf(s, g, 1.f / 24.f);
  s = fmaf(s, g, 1.f / 6.f);
  s = fmaf(s, g, 0.5f);
  s = fmaf(s, g, 1.f);
  return -g * s;
}

// a, m (what multiplies x) and, for the gradient of the normed form, 1 / m.  Near 1, a is formed as 1 minus what it lacks, so that its error is a rounding's and has no
// preferred side: a state sums a's errors over as many tokens as it remembers.
template <int MODE>
__device__ __forceinline__ void rec_factors(float g, float& a, float& m, float& over_m) {
  if constexpr (MODE == kRecDecay) {
    a = expf(g);
    m = 1.f;
    over_m = 1.f;
  } else if constexpr (MODE == kRecNormed) {
    const float e = expf(g);
    const bool near = g > -0.25f && g <= 0.f;
    const float q = near ? rec_fall(g) : 1.f - e;
    a = near ? 1.f - q : e;
    const float s = q * (1.f + a);
    over_m = s > 0.f ? rsqrtf(s) : s <= 0.f ? 0.f : s;   // (a NaN stays one)
    m = s * over_m;
  } else {
    const float e = expf(-fabsf(g)), r = __fdividef(1.f, 1.f + e), s = e * r;   // s: the smaller of a and 1 - a
    a = g >= 0.f ? 1.f - s : s;
    m = g >= 0.f ? s : r;
    if (g != g) a = m = g;
    over_m = 1.f;
  }
}

// One token, or one map behind another.  Where a is zero nothing of what came before is left, not even what is not finite.
__device__ __forceinline__ float rec_step(float a, float h, float u) { return a == 0.f ? u : fmaf(a, h, u); }

// 4 bytes of a row at channel c: what lies past `width` channels reads as zero.  pairs: 4-byte accesses are aligned.
template <class T>
__device__ __forceinline__ uint32_t rec_load(const T* row, int c, int width, bool pairs) {
  if constexpr (sizeof(T) == 4) {
    return c < width ? __float_as_uint(row[c]) : 0u;
  } else {
    if (pairs && c + 1 < width) return *reinterpret_cast<const uint32_t*>(row + c);
    const uint16_t* p = reinterpret_cast<const uint16_t*>(row);
    const uint32_t lo = c < width ? p[c] : 0u, hi = c + 1 < width ? p[c + 1] : 0u;
    return lo | hi << 16;
  }
}
template <class T>
__device__ __forceinline__ void rec_store(T* row, int c, int width, bool pairs, const float (&v)[RecLane<T>::N]) {
  if constexpr (sizeof(T) == 4) {
    if (c < width) row[c] = v[0];
  } else {
    const uint32_t raw = RecLane<T>::pack(v);
    if (pairs && c + 1 < width) {
      *reinterpret_cast<uint32_t*>(row + c) = raw;
    } else {
      uint16_t* p = reinterpret_cast<uint16_t*>(row);
      if (c < width) p[c] = (uint16_t)raw;
      if (c + 1 < width) p[c + 1] = (uint16_t)(raw >> 16);
    }
  }
}

__device__ __forceinline__ void rec_copy(uint32_t to, const void* from, int bytes16) {   // 16 bytes, of which those past bytes16 are zero
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes16) : "memory");
}
__device__ __forceinline__ void rec_copy4(uint32_t to, const void* from, int bytes4) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to), "l"(from), "r"(bytes4) : "memory");
}
__device__ __forceinline__ void rec_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void rec_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// How a tensor's rows are moved: 16 bytes (everything aligned to them), 4 bytes, or value by value (bf16 at odd places)
enum : int { kRecWide = 0, kRecPairs = 1, kRecSingle = 2 };
template <class T>
__device__ __forceinline__ int rec_access(const void* p, long long ld) {
  const unsigned long long at = reinterpret_cast<unsigned long long>(p) | (unsigned long long)ld * sizeof(T);
  return (at & 15) == 0 ? kRecWide : (at & 3) == 0 ? kRecPairs : kRecSingle;
}

// Asks for a warp's ROWS rows of a tile: rows row0 .. of which `rows` exist, columns c0 .. of `width`; smem: the warp's rows of kRecRow bytes.
template <class T, int ROWS>
__device__ __forceinline__ void rec_request(unsigned char* smem, const T* base, long long ld, long long row0, int rows, int c0, int width, int access) {
  const int lane = threadIdx.x & 31;
  const int left = (width - c0) * (int)sizeof(T);   // bytes of a row from the tile's first column on
  const uint32_t to = (uint32_t)__cvta_generic_to_shared(smem);
  if (access == kRecWide) {
#pragma unroll
    for (int i = 0; i < (ROWS + 3) / 4; ++i) {
      const int r = 4 * i + (lane >> 3), at = 16 * (lane & 7);
      const int bytes = r < rows && r < ROWS ? min(16, max(0, left - at)) : 0;
      const T* from = bytes ? base + (row0 + r) * ld + c0 + at / (int)sizeof(T) : base;
      if (ROWS % 4 == 0 || r < ROWS) rec_copy(to + r * kRecRow + at, from, bytes);
    }
  } else if (access == kRecPairs && (sizeof(T) == 4 || (left & 3) == 0 || left >= kRecRow)) {
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const int bytes = r < rows && 4 * lane < left ? 4 : 0;
      const T* from = bytes ? base + (row0 + r) * ld + c0 + 4 * lane / (int)sizeof(T) : base;
      rec_copy4(to + r * kRecRow + 4 * lane, from, bytes);
    }
  } else {
    uint32_t raw[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) raw[r] = r < rows ? rec_load(base + (row0 + r) * ld, c0 + 4 * lane / (int)sizeof(T), width, access != kRecSingle) : 0u;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) *reinterpret_cast<uint32_t*>(smem + r * kRecRow + 4 * lane) = raw[r];
  }
}

__device__ __forceinline__ unsigned long long rec_peek(const unsigned long long* p) {
  unsigned long long v;
  asm volatile("ld.relaxed.gpu.global.b64 %0, [%1];" : "=l"(v) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ void rec_post(unsigned long long* p, float P, float H) {   // (P, H), never all ones: a NaN of that pattern is left as another
  uint32_t hi = __float_as_uint(H);
  if (hi == 0xffffffffu) hi = 0x7fffffffu;
  const unsigned long long v = (unsigned long long)hi << 32 | __float_as_uint(P);
  asm volatile("st.relaxed.gpu.global.b64 [%0], %1;" ::"l"(p), "l"(v) : "memory");
}
__device__ __forceinline__ unsigned long long rec_now() {
  unsigned long long t;
  asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
  return t;
}

// What enters a tile, from the words of the `count` tiles in front of it in its sequence (words of one channel, `step` from one to the one before): their maps join
// from the nearest on until one forgets what came before (P = 0; a tile that knows what leaves it says so with P = 0, the first one always does).  A word
// that is missing for the time limit raises the status word, and the NaN that is returned then goes on with this tile's own word, so that no later tile waits as long.
__device__ __forceinline__ float rec_look_back(const unsigned long long* word, long long step, int count, unsigned long long limit, int* status) {
  constexpr int AT_ONCE = 4;
  constexpr unsigned long long NONE = ~0ull;
  float P = 1.f, H = 0.f;
  unsigned long long begin = 0;
  unsigned int polls = 0;
  while (count > 0) {
    unsigned long long v[AT_ONCE];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) v[i] = i < count ? rec_peek(word - i * step) : NONE;
    int got = 0;
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      if (got == i && v[i] != NONE) {
        const float p = __uint_as_float((uint32_t)v[i]), h = __uint_as_float((uint32_t)(v[i] >> 32));
        H = fmaf(P, h, H);   // (P is not zero here)
        if (p == 0.f) return H;
        P *= p;
        if (P == 0.f) return H;
        ++got;
      }
    }
    word -= got * step;
    count -= got;
    if (got == 0 && (++polls & 127) == 0) {
      const unsigned long long now = rec_now();
      if (begin == 0) begin = now;
      else if (now - begin > limit) {
        atomicMax(status, (int)TRI_INV_ERR_DEVICE_TIMEOUT);
        return __uint_as_float(0x7fc00000u);
      }
    }
  }
  return H;
}

// Where a block stands: a tile of an item, which is a tile (with words) or a whole sequence
struct RecAt {
  int item;            // >= the number of items: none left
  int seq, col;
  int begin, len;      // the sequence's
  int index, tiles;    // the tile, of how many
  __device__ __forceinline__ long long tok0() const { return (long long)begin + (long long)index * kRecTile; }
  __device__ __forceinline__ int n() const { return min(kRecTile, len - index * kRecTile); }
};
template <bool WORDS>
__device__ __forceinline__ RecAt rec_decode(const RecArgs& a, int item, bool back) {
  RecAt t{};
  t.item = item;
  if (item >= a.n_segs * a.cols) return t;
  const int r0 = item / a.cols, r = back && WORDS ? a.n_segs - 1 - r0 : r0;
  t.col = item - r0 * a.cols;
  if (a.table) {
    const RecTile s = a.table[r];
    t.begin = s.tok0; t.len = s.n; t.seq = s.seq; t.index = s.index; t.tiles = s.tiles;
  } else {
    t.index = WORDS ? r / a.n_seqs : 0;   // the sequences' tiles in turn: the one in front of a tile is n_seqs (times the columns) items ahead of it
    t.tiles = max(1, (int)(((unsigned)a.T + kRecTile - 1) / kRecTile));
    t.seq = WORDS ? r - t.index * a.n_seqs : r;
    t.begin = t.seq * a.T;
    t.len = a.T;
  }
  if (!WORDS && back) t.index = t.tiles - 1;
  return t;
}
// The tile after `t` in its sequence's walk (backwards: in front of it), or the first of the next item
template <bool WORDS>
__device__ __forceinline__ RecAt rec_next(const RecArgs& a, const RecAt& t, int drawn, bool back) {
  if (WORDS) return rec_decode<true>(a, drawn, back);
  if (back ? t.index > 0 : t.index + 1 < t.tiles) {
    RecAt s = t;
    s.index += back ? -1 : 1;
    return s;
  }
  return rec_decode<false>(a, t.item + gridDim.x, back);
}
#endif

}  // namespace tri_inv
