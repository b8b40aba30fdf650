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
// Both are walks over tiles of some tokens and channels.  A tile is an affine map of what enters it, (P, H): h -> P h + H,
// and so is a run of tiles; the tokens of a warp, the warps of a tile and the tiles of a sequence join by the same rule.
#pragma once
#include "common.cuh"

namespace tri_inv {

constexpr int kRecCarry = TRI_INV_REC_TILE;   // tokens from one carried state to the next
constexpr int kRecWarps = 4;     // warps of tokens of a block
constexpr int kRecGroups = 2;    // lane groups of a warp, each with tokens of its own (RecShape)
constexpr int kRecTok = 16;                                                                 // tokens of a lane
// ... in the gradient: sixteen of fp32 would leave shared memory for two blocks an SM
__host__ __device__ constexpr int rec_back_tok(int bytes) { return bytes == 2 ? 16 : 8; }
constexpr int kRecThreads = 32 * kRecWarps + 32;                                            // and a thread for each channel that joins them
constexpr int kRecTile = kRecWarps * kRecGroups * kRecTok, kRecChannels = 64 / kRecGroups;   // of a tile
__host__ __device__ constexpr int rec_back_tile(int bytes) { return kRecWarps * kRecGroups * rec_back_tok(bytes); }

// Whether so many blocks of a walk are resident on an SM together: of its 228 KB of shared memory a block takes 1 KB besides its own.
__host__ __device__ constexpr bool rec_fit(int blocks, size_t dynamic_bytes, size_t static_bytes) { return blocks * (dynamic_bytes + static_bytes + 1024) <= 228 * 1024; }

// n / d for n < 2^30 as (n m) >> (30 + L), 2^L >= d, m = ceil(2^(30 + L) / d): what m d has above 2^(30 + L) is below d <= 2^L, and n times it below 2^(30 + L), so that the quotient's floor is exact.
struct RecDivide {
  uint32_t m;
  int shift;
};
inline RecDivide rec_divide_by(int d) {
  int L = 0;
  while ((1ll << L) < d) ++L;
  return RecDivide{(uint32_t)(((1ull << (30 + L)) + (unsigned)d - 1) / (unsigned)d), 30 + L};
}
__host__ __device__ __forceinline__ int rec_quotient(int n, RecDivide by) { return (int)(((unsigned long long)(unsigned)n * by.m) >> by.shift); }

// An entry of the table of packed sequences: a tile, or a whole sequence (index 0)
struct RecTile {
  int32_t tok0, n, seq;     // the SEQUENCE's first token, its length and number
  int32_t index, tiles;     // the tile, of how many
};

// Where the words of a sequence's tiles, and its carried states, begin: sequences of any length leave no two tiles at one place.
__host__ __device__ __forceinline__ long long rec_slot(long long tok0, int seq, int tile) { return tok0 / tile + seq; }
// Channel c of row `row` of an array of D values a row, as the words, the carried states and the states are: a row's number times D may pass 2^31.
__host__ __device__ __forceinline__ long long rec_at(long long row, int D, int c) { return row * D + c; }

struct RecArgs {
  const void *x, *g, *dy;          // dy: gradient only
  void *y, *dx, *dg;               // y: null where only the carried states are wanted
  long long ld_x, ld_g, ld_dy, ld_y, ld_dx, ld_dg;   // values from one token to the next
  const float* h0;                 // [n_seqs, D] or null
  float* h_out;                    // [n_seqs, D] or null
  float* carries;                  // [slots of kRecCarry, D]: the states carried on; written by the forward walk (or null), read by the gradient
  const float* dh;                 // gradient: [n_seqs, D] or null
  float* dh0;                      // [n_seqs, D] or null
  unsigned long long* words;       // [slots, D] (P, H) of each tile, or (0, what leaves it); all ones: not there yet.  Null: whole sequences are walked
  unsigned int* ticket;            // next item, with words
  const RecTile* table;            // packed sequences: tiles (with words) or whole sequences; null: dense
  int n_segs;                      // entries of the table, or tiles (whole sequences) of the dense form
  int n_seqs, T, D, cols;          // cols: column tiles
  RecDivide by_cols, by_seqs;
  int items;                       // n_segs * cols
  int mode;
  int* status;
  unsigned long long wait_limit_ns;   // 0: two seconds
  int test_stall;                  // self-test: the first tile of the first sequence's first columns leaves no word
};

cudaError_t launch_gated_recurrence(const RecArgs& a, int dtype, cudaStream_t stream);
cudaError_t launch_gated_recurrence_backward(const RecArgs& a, int dtype, cudaStream_t stream);
// What a walk finds in its workspace: the ticket (zero) and the words (all ones), null where whole sequences are walked, and the table of packed sequences, null for dense ones.
struct RecSetup {
  unsigned int* ticket;
  unsigned long long* words;
  RecTile* table;
  long long n_words;
  int tile;                        // tokens of an entry; 0: whole sequences
};
// Sets up one walk or two from the host offsets `cu` (null: dense).
cudaError_t launch_rec_setup(const RecSetup* walks, int n_walks, const int32_t* cu, int n_seqs, cudaStream_t stream);

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

// Two fp32 numbers, a lane's two channels, that the arithmetic takes at a time
struct Pair { unsigned long long v; };
__device__ __forceinline__ Pair pair(float x, float y) { Pair d; asm("mov.b64 %0, {%1, %2};" : "=l"(d.v) : "f"(x), "f"(y)); return d; }
__device__ __forceinline__ float2 both(Pair a) { float2 d; asm("mov.b64 {%0, %1}, %2;" : "=f"(d.x), "=f"(d.y) : "l"(a.v)); return d; }
__device__ __forceinline__ Pair mul2(Pair a, Pair b) { Pair d; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d.v) : "l"(a.v), "l"(b.v)); return d; }
__device__ __forceinline__ Pair add2(Pair a, Pair b) { Pair d; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d.v) : "l"(a.v), "l"(b.v)); return d; }
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) { Pair d; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d.v) : "l"(a.v), "l"(b.v), "l"(c.v)); return d; }
__device__ __forceinline__ Pair twice(float x) { return pair(x, x); }

// A lane's two channels as they lie in a row
template <class T> struct RecLane;
template <> struct RecLane<__nv_bfloat16> {
  using Raw = uint32_t;
  static __device__ __forceinline__ Pair widen(Raw r) { return pair(__uint_as_float(r << 16), __uint_as_float(r & 0xffff0000u)); }
  static __device__ __forceinline__ Raw pack(Pair v) {
    const float2 f = both(v);
    const __nv_bfloat162 p = __floats2bfloat162_rn(f.x, f.y);
    return reinterpret_cast<const uint32_t&>(p);
  }
};
template <> struct RecLane<float> {
  using Raw = uint2;
  static __device__ __forceinline__ Pair widen(Raw r) { return pair(__uint_as_float(r.x), __uint_as_float(r.y)); }
  static __device__ __forceinline__ Raw pack(Pair v) {
    const float2 f = both(v);
    return make_uint2(__float_as_uint(f.x), __float_as_uint(f.y));
  }
};

// e^g as 2^(g log2 e), off by the power's own error, 2^-22.5, and by that of the rounded product, |g| 2^-24, which is what a rounding of g itself would change.  Results below 2^-126 are 0 (squared, below 2^-149).
__device__ __forceinline__ float rec_power(float t) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(t)); return y; }
template <int HALF = 0>   // of g / 2
__device__ __forceinline__ Pair rec_exp(Pair g) {
  const float2 t = both(mul2(g, twice(HALF ? 0.72134752044448170f : 1.44269504088896341f)));
  return pair(rec_power(t.x), rec_power(t.y));
}
__device__ __forceinline__ float rec_reciprocal(float x) { float y; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ float rec_at_least_zero(float x) { float y; asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(y) : "f"(x)); return y; }   // what is not a number stays so
__device__ __forceinline__ float rec_root(float x) { float y; asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }

// a and m (what multiplies x).  A state sums a's errors over as many tokens as it remembers, so near 1 they may have no preferred side: decay and normed take a = 1 - q, q = 1 - e^g = -2 sinh(g / 2) e^{g / 2}, for |g| <= 1/4 (the
// first term left out of sinh(x) / x is x^6 / 7!, x = g / 2: 2^-30), which is off by a rounding, and e^{g / 2} squared elsewhere; gate forms the smaller one of a and 1 - a and takes it from 1.  Measured over
// g = -0.02 .. -0.004, mean (mean of the size) of a's error in 2^-24: 0.00 (0.25); a power of two alone -0.43 (0.54), expf -0.08 (0.42).  normed: 1 - a^2 = q (1 + a), which does not cancel.
template <int MODE>
__device__ __forceinline__ void rec_factors(Pair gp, Pair& a, Pair& m) {
  const float2 g = both(gp);
  const Pair one = twice(1.f), minus = twice(-1.f);
  if constexpr (MODE == kRecDecay || MODE == kRecNormed) {
    const Pair e = rec_exp<1>(gp), y = mul2(gp, gp), poly = fma2(fma2(y, twice(1.f / 1920.f), twice(1.f / 24.f)), y, one), fall = mul2(mul2(gp, e), poly);   // fall: a - 1
    const float2 near = both(add2(fall, one)), far = both(mul2(e, e));
    const bool nx = fabsf(g.x) <= 0.25f, ny = fabsf(g.y) <= 0.25f;
    a = pair(nx ? near.x : far.x, ny ? near.y : far.y);
    if constexpr (MODE == kRecNormed) {
      const float2 n = both(fma2(fall, a, fall)), f = both(fma2(a, a, minus));   // a^2 - 1
      m = pair(rec_root(rec_at_least_zero(-(nx ? n.x : f.x))), rec_root(rec_at_least_zero(-(ny ? n.y : f.y))));
    } else {
      m = one;
    }
  } else {
    const Pair e = rec_exp(pair(-fabsf(g.x), -fabsf(g.y)));
    const float2 d = both(add2(e, one));
    const Pair rp = pair(rec_reciprocal(d.x), rec_reciprocal(d.y)), sp = mul2(e, rp), bp = fma2(sp, minus, one);   // s: the smaller of a and 1 - a
    const float2 r = both(rp), s = both(sp), b = both(bp);
    a = pair(g.x >= 0.f ? b.x : s.x, g.y >= 0.f ? b.y : s.y);
    m = pair(g.x >= 0.f ? s.x : r.x, g.y >= 0.f ? s.y : r.y);
  }
}
template <int MODE>
__device__ __forceinline__ Pair rec_input(Pair m, Pair x) {   // u
  if constexpr (MODE == kRecDecay) return x;
  else return mul2(m, x);
}

// One token, or one map behind another.  Where a is zero nothing of what came before is left, not even what is not finite.
__device__ __forceinline__ float rec_step(float a, float h, float u) { return a == 0.f ? u : fmaf(a, h, u); }
__device__ __forceinline__ Pair rec_step(Pair a, Pair h, Pair u) {
  const float2 x = both(a), y = both(h), z = both(u);
  return pair(rec_step(x.x, y.x, z.x), rec_step(x.y, y.y, z.y));
}
// The product of two maps' decays: zero where either is, whatever the other.  A decay that is not a number (or the product of an infinite one and zero) is forgotten like any state.
__device__ __forceinline__ float rec_product(float a, float b) { return a == 0.f || b == 0.f ? 0.f : a * b; }
__device__ __forceinline__ Pair rec_product(Pair a, Pair b) {
  const float2 x = both(a), y = both(b), z = both(mul2(a, b));
  return pair(x.x == 0.f || y.x == 0.f ? 0.f : z.x, x.y == 0.f || y.y == 0.f ? 0.f : z.y);
}
// The same of the other lane group's lane
static_assert(kRecGroups == 2, "the lane groups of a warp join in one exchange");
__device__ __forceinline__ Pair rec_other(Pair v) {
  const float2 f = both(v);
  return pair(__shfl_xor_sync(0xffffffffu, f.x, 16), __shfl_xor_sync(0xffffffffu, f.y, 16));
}
// whether a plain product of decays may hide one that is zero: it is zero itself, or no number
__device__ __forceinline__ bool any_zero(Pair a) { const float2 x = both(a); return !(x.x > 0.f) || !(x.y > 0.f); }

// How a tensor's rows are moved: 16, 8 or 4 bytes at a time (everything aligned to them), or by single values (bf16 at odd places)
enum : int { kRecWide = 0, kRecEights = 1, kRecFours = 2, kRecSingle = 3 };
template <class T>
__host__ __device__ __forceinline__ int rec_access(const void* p, long long ld) {
  const unsigned long long at = reinterpret_cast<unsigned long long>(p) | (unsigned long long)ld * sizeof(T);
  return (at & 15) == 0 ? kRecWide : (at & 7) == 0 ? kRecEights : (at & 3) == 0 ? kRecFours : kRecSingle;
}

// Two neighbouring 16-bit values, of which those past `width` are zero
template <class T>
__device__ __forceinline__ uint32_t rec_half_words(const T* row, int c, int width) {
  const uint16_t* p = reinterpret_cast<const uint16_t*>(row);
  const uint32_t lo = c < width ? p[c] : 0u, hi = c + 1 < width ? p[c + 1] : 0u;
  return lo | hi << 16;
}
// A lane's channels c, c + 1 of a row of `width`: those past the last read as zero and are not written.
template <class T>
__device__ __forceinline__ typename RecLane<T>::Raw rec_load(const T* row, int c, int width, int access) {
  if constexpr (sizeof(T) == 4) {
    if (access <= kRecEights && c + 1 < width) return *reinterpret_cast<const uint2*>(row + c);
    return make_uint2(c < width ? __float_as_uint(row[c]) : 0u, c + 1 < width ? __float_as_uint(row[c + 1]) : 0u);
  } else {
    if (access != kRecSingle && c + 1 < width) return *reinterpret_cast<const uint32_t*>(row + c);
    return rec_half_words(row, c, width);
  }
}
template <class T>
__device__ __forceinline__ void rec_store(T* row, int c, int width, int access, Pair v) {
  const typename RecLane<T>::Raw raw = RecLane<T>::pack(v);
  if constexpr (sizeof(T) == 4) {
    if (access <= kRecEights && c + 1 < width) { *reinterpret_cast<uint2*>(row + c) = raw; return; }
    if (c < width) row[c] = __uint_as_float(raw.x);
    if (c + 1 < width) row[c + 1] = __uint_as_float(raw.y);
  } else {
    if (access != kRecSingle && c + 1 < width) { *reinterpret_cast<uint32_t*>(row + c) = raw; return; }
    uint16_t* p = reinterpret_cast<uint16_t*>(row);
    if (c < width) p[c] = (uint16_t)raw;
    if (c + 1 < width) p[c + 1] = (uint16_t)(raw >> 16);
  }
}

__device__ __forceinline__ void rec_copy(uint32_t to, const void* from, int bytes16) {   // 16 bytes, of which those past bytes16 are zero
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes16) : "memory");
}
__device__ __forceinline__ void rec_copy4(uint32_t to, const void* from, int bytes4) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to), "l"(from), "r"(bytes4) : "memory");
}
__device__ __forceinline__ void rec_copy8(uint32_t to, const void* from) { asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(to), "l"(from) : "memory"); }
__device__ __forceinline__ void rec_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void rec_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Where a block stands: a tile of an item, which is a tile (with words) or a whole sequence
struct RecAt {
  int item;            // >= the number of items: none left
  int seq, c0;         // c0: the tile's first channel
  int begin, len;      // the sequence's
  int index, tiles;    // the tile, of how many
  int n;               // its tokens
  bool whole;          // all tokens and channels of a tile
  int tok0;
  int slot;            // of its words
  long long at[5];     // where its first value lies in each tensor, in bytes
};
// The lanes of a warp stand in kRecGroups groups, each of which has TOK tokens behind one another, two channels a lane.  In shared memory a row follows the one before, and a
// group's rows are one row further on, so that the groups' reads meet in no bank.
template <class T, int TOK>
struct RecShape {
  static constexpr int GROUPS = kRecGroups, CHANNELS = kRecChannels, ROW = CHANNELS * (int)sizeof(T), LANES = 32 / GROUPS, GROUP_BYTES = (TOK + 1) * ROW, WARP_BYTES = GROUPS * GROUP_BYTES;
  static constexpr int WARP_TOK = GROUPS * TOK, TILE = kRecWarps * WARP_TOK, TENSOR = kRecWarps * WARP_BYTES;
  static constexpr int AT_ONCE = 512 / ROW;   // rows of a warp's 16-byte copies
  static_assert(TOK % AT_ONCE == 0 || AT_ONCE % TOK == 0, "");
  // of a lane: its group, its first channel, where its values begin in a warp's rows
  static __device__ __forceinline__ int group() { return (threadIdx.x & 31) / LANES; }
  static __device__ __forceinline__ int channel() { return 2 * ((threadIdx.x & 31) % LANES); }
  static __device__ __forceinline__ int place() { return group() * GROUP_BYTES + channel() * (int)sizeof(T); }
  // bytes of a lane's first 16, from the tile's first value on, in memory and in the warp's rows
  static __device__ __forceinline__ long long copy_from(long long ld, int row0) {
    const int lane = threadIdx.x & 31;
    return (row0 + lane * 16 / ROW) * ld * (int)sizeof(T) + lane * 16 % ROW;
  }
  static __device__ __forceinline__ uint32_t copy_to() { const int lane = threadIdx.x & 31; return 16 * lane + lane * 16 / ROW / TOK * ROW; }
  // Asks for a warp's rows of a tile, where every row and channel exists and 16 bytes can be moved; ld in values
  static __device__ __forceinline__ void request_whole(uint32_t warp_smem, const char* from, long long ld) {
    const uint32_t to = warp_smem + copy_to();
#pragma unroll
    for (int i = 0; i < WARP_TOK / AT_ONCE; ++i) {
      rec_copy(to + i * 512 + i * AT_ONCE / TOK * ROW, from, 16);
      from += ld * (AT_ONCE * (int)sizeof(T));
    }
  }
  // ... where BYTES can be moved; at: of the tile's first value, in bytes
  template <int BYTES>
  static __device__ __forceinline__ void request_pieces(uint32_t warp_smem, const char* tile, long long ld_bytes, int row0) {
    constexpr int PER_ROW = ROW / BYTES, ROWS = 32 / PER_ROW;   // lanes of a row, rows at once
    static_assert(TOK % ROWS == 0, "");
    const int lane = threadIdx.x & 31, r = lane / PER_ROW, off = lane % PER_ROW * BYTES;
    const char* from = tile + (row0 + r) * ld_bytes + off;
#pragma unroll
    for (int i = 0; i < WARP_TOK / ROWS; ++i) {
      const uint32_t to = warp_smem + r * ROW + off + i * ROWS * ROW + i * ROWS / TOK * ROW;
      if constexpr (BYTES == 8) rec_copy8(to, from);
      else rec_copy4(to, from, 4);
      from += ROWS * ld_bytes;
    }
  }
  // A whole tile of 16-bit values at odd places comes as the aligned words that hold a row: the row's sixteen and, in `rest` (a warp's, [WARP_TOK]), the one behind them.  The words of the first row's first channels and of the last
  // row's last ones may lie half outside the tensor: those tiles do not come so.
  static __device__ __forceinline__ bool by_words(const RecArgs& a, int tok0, int c0) {
    const long long tokens = a.table ? a.T : (long long)a.n_seqs * a.T;
    return sizeof(T) == 2 && (tok0 > 0 || c0 > 0) && (tok0 + TILE < tokens || c0 + CHANNELS < a.D);
  }
  static __device__ __forceinline__ void request_words(uint32_t warp_smem, uint32_t rest, const char* tile, long long ld_bytes, int row0) {
    const int lane = threadIdx.x & 31, r = group(), off = lane % LANES * 4;
    auto word = [](const char* p) { return reinterpret_cast<const char*>(reinterpret_cast<unsigned long long>(p) & ~3ull); };
    const char* from = tile + (row0 + r * TOK) * ld_bytes;
#pragma unroll
    for (int k = 0; k < TOK; ++k) {
      rec_copy4(warp_smem + place() + k * ROW, word(from) + off, 4);
      from += ld_bytes;
    }
    for (int row = lane; row < WARP_TOK; row += 32) {
      const char* p = tile + (row0 + row) * ld_bytes;   // (a row that is aligned has no word behind it to read)
      const bool odd = reinterpret_cast<unsigned long long>(p) & 2;
      rec_copy4(rest + 4 * row, odd ? word(p) + ROW : p, odd ? 4 : 0);
    }
  }
  static __device__ __forceinline__ void settle_words(unsigned char* warp_smem, const unsigned char* rest, const char* tile, long long ld_bytes, int row0) {   // the rows as they would have come
    const int lane = threadIdx.x & 31, r = group();
    const uint32_t start = (uint32_t)reinterpret_cast<unsigned long long>(tile) + (uint32_t)(row0 + r * TOK) * (uint32_t)ld_bytes;
#pragma unroll
    for (int k = 0; k < TOK; ++k) {
      uint32_t* at = reinterpret_cast<uint32_t*>(warp_smem + place() + k * ROW);
      const uint32_t w = *at;
      uint32_t next = __shfl_down_sync(0xffffffffu, w, 1);
      if (lane % LANES == LANES - 1) next = *reinterpret_cast<const uint32_t*>(rest + 4 * (r * TOK + k));
      if ((start + (uint32_t)k * (uint32_t)ld_bytes) & 2) *at = __funnelshift_r(w, next, 16);
    }
  }
  // A tensor's rows of a whole tile however they lie
  static __device__ __forceinline__ void request_any(uint32_t warp_smem, uint32_t rest, const RecArgs& a, const T* base, const RecAt& t, int tensor, long long ld, int row0, int access) {
    const char* tile = (const char*)base + t.at[tensor];
    if (access == kRecWide) request_whole(warp_smem, tile + copy_from(ld, row0), ld);
    else if (access == kRecEights) request_pieces<8>(warp_smem, tile, ld * (int)sizeof(T), row0);
    else if (access == kRecFours) request_pieces<4>(warp_smem, tile, ld * (int)sizeof(T), row0);
    else if (by_words(a, t.tok0, t.c0)) request_words(warp_smem, rest, tile, ld * (int)sizeof(T), row0);
    else request(warp_smem, base, ld, t.tok0 + row0, TILE, t.c0, a.D, access);
  }
  static __device__ __forceinline__ void settle_any(unsigned char* warp_smem, const unsigned char* rest, const RecArgs& a, const T* base, const RecAt& t, int tensor, long long ld, int row0, int access) {
    if (access == kRecSingle && t.whole && by_words(a, t.tok0, t.c0)) settle_words(warp_smem, rest, (const char*)base + t.at[tensor], ld * (int)sizeof(T), row0);
  }
  // ... where not: rows row0 .. of which `rows` exist, channels c0 .. of `width`; what does not exist reads as zero
  static __device__ __forceinline__ void request(uint32_t warp_smem, const T* base, long long ld, long long row0, int rows, int c0, int width, int access) {
    const int lane = threadIdx.x & 31;
    if (access == kRecWide) {
      const int left = (width - c0) * (int)sizeof(T), at = lane * 16 % ROW, bytes = min(16, left - at), r0 = lane * 16 / ROW;
#pragma unroll
      for (int i = 0; i < WARP_TOK / AT_ONCE; ++i) {
        const bool in = r0 + i * AT_ONCE < rows && bytes > 0;
        rec_copy(warp_smem + copy_to() + i * 512 + i * AT_ONCE / TOK * ROW, in ? base + (row0 + r0 + i * AT_ONCE) * ld + c0 + at / (int)sizeof(T) : base, in ? bytes : 0);
      }
    } else {
      const int first = group() * TOK, c = c0 + channel();
      const uint32_t to = warp_smem + place();
      if (sizeof(T) == 4 || (access != kRecSingle && (width - c0 >= CHANNELS || width % 2 == 0))) {
#pragma unroll
        for (int k = 0; k < TOK; ++k)
#pragma unroll
          for (int j = 0; j < (int)sizeof(T) / 2; ++j) {
            const bool in = first + k < rows && c + j < width;
            rec_copy4(to + k * ROW + 4 * j, in ? base + (row0 + first + k) * ld + c + j : base, in ? 4 : 0);
          }
      } else {
        uint32_t raw[TOK];
#pragma unroll
        for (int k = 0; k < TOK; ++k) raw[k] = first + k < rows ? rec_half_words(base + (row0 + first + k) * ld, c, width) : 0u;
#pragma unroll
        for (int k = 0; k < TOK; ++k) asm volatile("st.shared.b32 [%0], %1;" ::"r"(to + k * ROW), "r"(raw[k]) : "memory");
      }
    }
  }
};

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

// What enters a tile, from the words of the `count` tiles in front of it in its sequence (words of one channel, `step` from one to the one before).  The search goes back to the nearest tile that forgets what came
// before it (P = 0; a tile that knows what leaves it says so with P = 0, the first one always does) and then applies the maps in between in order: the same sums as from tile to tile, whichever words were
// already there.  A word that is missing for the time limit raises the status word, and the NaN that is returned then goes on with this tile's own word, so that no later tile waits as long.
__device__ __forceinline__ float rec_look_back(const unsigned long long* word, long long step, int count, unsigned long long limit, int* status) {
  constexpr int AT_ONCE = 4;   // words that are asked for together
  constexpr unsigned long long NONE = ~0ull;
  {   // mostly one of the nearest two knows
    const unsigned long long v = rec_peek(word), u = count > 1 ? rec_peek(word - step) : NONE;
    const float P = __uint_as_float((uint32_t)v), H = __uint_as_float((uint32_t)(v >> 32));
    if (v != NONE && P == 0.f) return H;
    if (v != NONE && u != NONE && (uint32_t)u << 1 == 0) return rec_step(P, __uint_as_float((uint32_t)(u >> 32)), H);
  }
  unsigned long long begin = 0;
  float h = 0.f;
  bool found = false;
  int base = 0;
  for (unsigned int polls = 1;; ++polls) {
    unsigned long long v[AT_ONCE];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) v[i] = base + i < count ? rec_peek(word - (base + i) * step) : NONE;
    int from = AT_ONCE;   // the maps before this one are applied
    if (!found) {
      int got = 0;
#pragma unroll
      for (int i = 0; i < AT_ONCE; ++i) {
        if (!found && got == i && v[i] != NONE) {
          ++got;
          if (__uint_as_float((uint32_t)v[i]) == 0.f) {
            h = __uint_as_float((uint32_t)(v[i] >> 32));
            found = true;
            from = i;
          }
        }
      }
      if (!found) {
        if (got == AT_ONCE) {
          base += AT_ONCE;
        } else if ((polls & 127) == 0) {
          const unsigned long long now = rec_now();
          if (begin == 0) begin = now;
          else if (now - begin > limit) {
            atomicMax(status, (int)TRI_INV_ERR_DEVICE_TIMEOUT);
            return __uint_as_float(0x7fc00000u);
          }
        }
        continue;
      }
    }
#pragma unroll
    for (int i = AT_ONCE - 1; i >= 0; --i)
      if (i < from) h = rec_step(__uint_as_float((uint32_t)v[i]), h, __uint_as_float((uint32_t)(v[i] >> 32)));
    if (base == 0) return h;
    base -= AT_ONCE;
  }
}

// Waits until the tile of this word has read what it reads: where a final state lies in the place of the one carried in, nothing else may order the tile that writes it behind the tile that reads
// (a decay of zero in between forgets).
__device__ __forceinline__ void rec_await(const unsigned long long* word, unsigned long long limit, int* status) {
  unsigned long long begin = 0;
  for (unsigned int polls = 1; rec_peek(word) == ~0ull; ++polls) {
    if ((polls & 127) != 0) continue;
    const unsigned long long now = rec_now();
    if (begin == 0) begin = now;
    else if (now - begin > limit) {
      atomicMax(status, (int)TRI_INV_ERR_DEVICE_TIMEOUT);
      return;
    }
  }
}

// Where warps meet: those of tokens when their maps are there; all when what enters the tile is there as well.  The barrier is the form that a warp's lanes have to reach together, and they may come from words that
// each waited for by itself, or from stores of half of them.
enum : int { kRecMaps = 1, kRecEntry = 2 };
template <int WHICH, int THREADS>
__device__ __forceinline__ void rec_meet() { __syncwarp(); asm volatile("bar.sync %0, %1;" ::"n"(WHICH), "n"(THREADS) : "memory"); }

// The order of a block's tiles.  The one that it works on, the one before and those that are on their way lie in a ring in shared memory, which one thread keeps ahead.  With words the items are drawn
// from the ticket, so that the tiles in front of a tile are done or in the hands of blocks that run; else they go by a fixed stride.
constexpr int kRecRing = 8;
template <bool WORDS, int TILE, int TENSORS, bool BACK>
struct RecFeed {
  const RecArgs& a;
  int ld[TENSORS];         // bytes
  int width;               // bytes of a value
  int drawn;               // the item whose entry of the table is asked for next
  RecAt last;              // without words: the tile that was given last
  __device__ __forceinline__ bool more() const { return !WORDS && last.item < a.items && (BACK ? last.index > 0 : last.index + 1 < last.tiles); }
  __device__ __forceinline__ RecTile entry(int item) const {
    if (!a.table || item >= a.items) return RecTile{};
    const int r = rec_quotient(item, a.by_cols);
    return a.table[BACK && WORDS ? a.n_segs - 1 - r : r];
  }
  __device__ __forceinline__ void place() {
    last.n = min(TILE, last.len - last.index * TILE);
    last.whole = last.n == TILE && last.c0 + kRecChannels <= a.D;
    last.tok0 = last.begin + last.index * TILE;   // below 2^31
    last.slot = last.begin / TILE + last.seq + last.index;
#pragma unroll
    for (int k = 0; k < TENSORS; ++k) last.at[k] = (long long)last.tok0 * ld[k] + last.c0 * width;
  }
  __device__ __forceinline__ void decode(int item, const RecTile& e) {
    last.item = item;
    if (item >= a.items) return;
    const int r = rec_quotient(item, a.by_cols);
    last.c0 = (item - r * a.cols) * kRecChannels;
    if (a.table) {
      last.begin = e.tok0; last.len = e.n; last.seq = e.seq; last.index = e.index; last.tiles = e.tiles;
    } else {
      const int rank = BACK && WORDS ? a.n_segs - 1 - r : r;
      last.index = WORDS ? rec_quotient(rank, a.by_seqs) : 0;   // the sequences' tiles in turn: the one in front of a tile is n_seqs (times the columns) items ahead of it
      last.tiles = max(1, (int)(((unsigned)a.T + TILE - 1) / TILE));
      last.seq = WORDS ? rank - last.index * a.n_seqs : rank;
      last.begin = last.seq * a.T;
      last.len = a.T;
    }
    if (!WORDS) {
      last.tiles = max(1, (int)(((unsigned)last.len + TILE - 1) / TILE));
      last.index = BACK ? last.tiles - 1 : 0;
    }
    place();
  }
  __device__ __forceinline__ void follow() { last.index += BACK ? -1 : 1; place(); }
  // The first tile
  __device__ __forceinline__ void begin(RecAt* ring) {
    const int item = WORDS ? (int)atomicAdd(a.ticket, 1u) : (int)blockIdx.x;
    decode(item, entry(item));
    ring[0] = last;
    drawn = WORDS ? (int)atomicAdd(a.ticket, 1u) : item + (int)gridDim.x;
  }
  // Early in a round: asks for what `give` needs
  int next_drawn, given;
  RecTile asked;
  __device__ __forceinline__ void ask() {
    given = drawn;
    asked = entry(drawn);
    if (WORDS) next_drawn = (int)atomicAdd(a.ticket, 1u);
  }
  __device__ __forceinline__ void give(RecAt* to) {
    if (more()) {
      follow();
    } else {
      decode(given, asked);
      drawn = WORDS ? next_drawn : given + (int)gridDim.x;
    }
    *to = last;
  }
};
#endif

}  // namespace tri_inv
