// Linear attention with a decay for each head, on the tensor cores: bf16, d_k and d_v up to 128 (the walk's formulas: linear_attention.cuh), in tiles
// of 64 or 128 features, padded with zeros by the copy engine.
//
// A persistent CTA per SM walks (walk, segment, head) items tile after tile of 64 tokens.  As in the delta rule's scan (scan_kernel.cu) everything that carries the state
// lies transposed, value columns as tensor-memory lanes, so that its operands go from registers straight into tensor memory:
//   QK [64 x 64]    = Q . K^T                 both K-major tiles
//   DS [d_v x d_k]  = (V~hi + V~lo)^T . K     V~ = lambda^(n-1-j) v_j as two bf16 numbers; the K tile is read MN-major
//   QS [d_v x 64]   = S^T . Q^T               S^T in bf16
//   PV [d_v x 64]   = V^T . P^T               P = QK * D in bf16, in shared memory
// Unlike there nothing but S <- lambda^n S + DS hangs on the tile before: no product is on a dependent chain, and the tensor cores take one after the other.
// lambda is a constant of the head, so the factors of P, V~ and QS are formed once an item, in the registers of the threads that use them: a thread has
// the same places of every tile.
//
// Warps 0..7 ("state"): lanes 32 (w & 3) .. + 31, half (w >> 2) of the features; S^T in fp32 registers for the whole item.  Warps 8..15 ("value"): V out of its
// tile into tensor memory, transposed by ldmatrix, plain and scaled.  Warps 16..23 ("output"): P, and O one tile behind; in the pass that only wants states they are
// value warps too.  Then one warp each: control A issues DS and QK, control B QS and PV, the copy warp requests the tiles, the store warp has O stored by the copy engine.
// Hand-offs are mbarriers with one phase a tile: a commit for a product that is done, an arrival of each warp for an operand that is written or an accumulator that is read.
//
// Roundings: P, the copy of S that QS reads and O are bf16, as any operand of these products has to be (each 2^-8 relative at most, over sums in fp32; S itself
// stays fp32 from tile to tile).  V~ = V~hi + V~lo keeps 16 bits, so that S is good to about 1e-5 wherever it goes, to the next tile, the next segment or the caller, and O's bits
// depend neither on whether the last state is wanted nor on a segment's place.  (The low half is 256 of a tile's 1,152 cycles of products at d_k = d_v = 128; with it O is 2.3e-3 of its norm
// from 64 bits, without it 2.6e-3, where bf16's own rounding is 1.7e-3.)
//
// What bounds it: a tile's chain of hand-offs while the chip has room, 1.3 us with all 128 value columns and 1.0 with 64 (the same hand-offs without arithmetic and products: three
// quarters of that); from about as many walks as SMs on the memory.  Two slices of 64 columns double the walks and read Q and K twice, the second time mostly from L2.  bf16, d = 128,
// calls in a captured graph, three input sets in turn, on a rested GPU and after 0.3 s of them (the power cap then holds the SM clock at 1.7 to 1.9 GHz): 4 x 4096 x 16 heads (128
// slices) 76 and 80 us, 3.4 TB/s; 4 x 4096 x 37 heads (148 walks of all columns) 114 and 136, 4.6 TB/s; the gradient of 4 x 4096 x 16 (192 walks) 179 and 190; 1 x 32768 x 32 in
// segments 289 and 340.
// Every mbarrier wait is bounded; on expiry the CTA raises the status word, waits for its own products and copies, frees its tensor memory and returns.
#include "linear_attention.cuh"
#include "tc_warps.cuh"

namespace tri_inv {
namespace {

constexpr int L = kLinTile;
constexpr int kStateWarps = 8, kValue = 8, kOutput = 16, kControlA = 24, kControlB = 25, kCopyL = 26, kStoreL = 27, kThreadsL = 28 * 32;
// Registers of a thread of each role's warpgroups: 72 at launch (7 warpgroups), 2 x 104 + 2 x 64 + 2 x 64 + 40 = 7 x 72
template <int N> __device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

struct LinMaps { CUtensorMap q[kLinMaxWalks], k[kLinMaxWalks], v[kLinMaxWalks], o[kLinMaxWalks]; };
struct LinTcArgs {
  LinArgs a;
  int first_walk, n_walks;   // the walks of this launch: those of its head dimensions
  int slices;                // slices of DV value columns
};

template <int DK, int DV>
struct LinCfg {
  static constexpr int LG = DV == 128 ? 2 : 1;            // groups of 16 tensor-memory lanes per quadrant in use
  static constexpr int M = 64 * LG, RPQ = DV / 4;         // value columns (rows here) per quadrant
  static constexpr int KB = DK / 64, VB = DV / 64;        // boxes of 64 features
  static constexpr int SH = DK / 2;                       // features of a state warp's half
  static constexpr int BOX = L * 128;
  static constexpr int OFF_K = KB * BOX, OFF_V = 2 * KB * BOX, STAGE = (2 * KB + VB) * BOX;
  static constexpr int STAGES = 4;
  static constexpr int OFF_P = STAGES * STAGE, OFF_O = OFF_P + L * 128, OFF_BAR = OFF_O + L * DV * 2,
                       OFF_F = OFF_BAR + 256, SMEM = OFF_F + 16 * L * 4;   // F: the value and output warps' factors, a table of each warp
  static constexpr int TM_S = 0, TM_V = TM_S + DK / 2, TM_VH = TM_V + 64, TM_VL = TM_VH + 32, TM_DS = TM_VL + 32, TM_QS = TM_DS + DK, TM_PV = TM_QS + 64, TM_QK = TM_PV + 64;
  static_assert(TM_QK + 64 <= 512 && SMEM <= 232448, "one CTA per SM");
};

// 32 lanes x 16 columns: a lane's row
__device__ __forceinline__ void tmem_ld_row16(float (&r)[16], uint32_t taddr) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
               : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]),
                 "=f"(r[8]), "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15])
               : "r"(taddr));
}
__device__ __forceinline__ void tmem_st_row8(const uint32_t (&r)[8], uint32_t taddr) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};"
               ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(taddr) : "memory");
}

// Two elements in one instruction, each rounded as by the scalar one: what the loops below issue is what bounds them
struct Pair { unsigned long long v; };
__device__ __forceinline__ Pair pair(float x, float y) { Pair p; asm("mov.b64 %0, {%1, %2};" : "=l"(p.v) : "f"(x), "f"(y)); return p; }
__device__ __forceinline__ float2 parts(Pair p) { float2 r; asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(p.v)); return r; }
__device__ __forceinline__ Pair mul2(Pair a, Pair b) { Pair d; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d.v) : "l"(a.v), "l"(b.v)); return d; }
__device__ __forceinline__ Pair add2(Pair a, Pair b) { Pair d; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d.v) : "l"(a.v), "l"(b.v)); return d; }
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) { Pair d; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d.v) : "l"(a.v), "l"(b.v), "l"(c.v)); return d; }
__device__ __forceinline__ uint32_t pack_bf16(Pair p) { const float2 x = parts(p); return pack_bf16(x.x, x.y); }
__device__ __forceinline__ Pair unpack_bf16(uint32_t x) { return pair(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u)); }

// WHOLE: outputs; otherwise the pass that only wants the states (LinArgs::state_only)
template <int DK, int DV, bool WHOLE>
__global__ void __launch_bounds__(kThreadsL, 1) linear_tc_kernel(const __grid_constant__ LinMaps maps, const __grid_constant__ LinTcArgs args) {
  using cfg = LinCfg<DK, DV>;
  constexpr int LG = cfg::LG;
  extern __shared__ __align__(1024) uint8_t smem[];
  const LinArgs& a = args.a;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + cfg::OFF_BAR + 224);
  const uint32_t s0 = smem_u32(smem), sP = s0 + cfg::OFF_P, bars = s0 + cfg::OFF_BAR;
  // copies: bar_full + 8 stage; stage free again: bar_empty + 8 stage (both control warps' commits, value warps)
  // products done (commit): ds, qs, qk, pv.  Operands written: vs (V~, value warps), vr (V), sr (S^T, state warps), pr (P, output warps).
  // Accumulators read: dsf (DS), qkf (QK), acc (QS and PV).  O's tile: o full, os read.  ds, pv, vs, vr and dsf are two barriers each, in turn: V is kept for two
  // tiles, in the pass that only wants states V~ and DS too, so that who writes them may be two tiles ahead of who waits.
  const uint32_t bar_full = bars, bar_empty = bars + 32, b_ds = bars + 64, b_pv = bars + 80, b_qs = bars + 96, b_qk = bars + 104, b_exit = bars + 112, b_exitb = bars + 120,
                 b_vs = bars + 128, b_vr = bars + 144, b_dsf = bars + 160, b_sr = bars + 176, b_pr = bars + 184, b_qkf = bars + 192, b_acc = bars + 200, b_o = bars + 208,
                 b_os = bars + 216;
  const unsigned long long lim = a.wait_limit_ns ? a.wait_limit_ns : kWaitLimitNs;
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;   // warp: uniform for the compiler
  const int quad = warp & 3, half = (warp >> 2) & 1;
  const int gq = lane >> 2, t2 = 2 * (lane & 3), mi = lane >> 3, mr = lane & 7;
  const bool misaligned = (s0 & 1023u) != 0;     // never expected; the swizzle pattern would not match the copies
  wait_for_predecessor();
  if (warp == kControlA) {
    if (lane == 0) {
      for (int b = 0; b < cfg::STAGES; ++b) { mbar_init(bar_full + 8 * b, 1); mbar_init(bar_empty + 8 * b, WHOLE ? 10 : 9); }
      for (uint32_t b = b_ds; b <= b_exitb; b += 8) mbar_init(b, 1);
      for (uint32_t b = b_vs; b <= b_o; b += 8) mbar_init(b, 8);   // eight warps each
      mbar_init(b_os, 1);
      fence_mbar_init();
    }
    __syncwarp();
  }
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_slot, 0);
  const uint32_t tmem_w = tmem + ((uint32_t)(32 * quad) << 16);   // this warp's lanes, column 0
  bool failed = misaligned;
  auto wait = [&](uint32_t bar, uint32_t parity) -> bool {
    // (inline: a call would keep to the launch's registers)
    if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
    const unsigned long long t0 = global_timer_ns();
#pragma unroll 1
    for (uint32_t i = 1; i < kSpinLimit; ++i) {
      if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
      if (__shfl_sync(0xffffffffu, (uint32_t)(global_timer_ns() - t0 > lim), 0)) return false;
    }
    return false;
  };
  const int per_walk = a.H * args.slices, per_seg = per_walk * args.n_walks, n_items = a.n_segs * per_seg;

  // Every role walks the same items: the longest first, dealt to the CTAs back and forth.  f(walk, segment, head, first column, ..) returns false to give up.
  auto for_items = [&](auto&& f) {
    for (int round = 0; round * (int)gridDim.x < n_items && !failed; ++round) {
      const int item = round * (int)gridDim.x + ((round & 1) ? (int)gridDim.x - 1 - (int)blockIdx.x : (int)blockIdx.x);
      if (item >= n_items) continue;
      const int s = item / per_seg, wh = item - s * per_seg, wi = args.first_walk + wh / per_walk, hs = wh % per_walk, h = hs / args.slices, col0 = (hs - h * args.slices) * DV;
      LinSeg g = lin_segment(a, s);
      // All of it uniform for the compiler.  tcgen05.mma takes uniform registers; where the control warp's loop, and so the stage's address, hung on
      // a value that could differ between lanes, each of a tile's 28 products cost about 55 cycles of moves into them, half of a tile's time
      g.tok0 = __shfl_sync(0xffffffffu, g.tok0, 0);
      g.n = __shfl_sync(0xffffffffu, g.n, 0);
      g.seq = __shfl_sync(0xffffffffu, g.seq, 0);
      g.ends = __shfl_sync(0xffffffffu, g.ends, 0);
      const LinWalk& w = a.walk[wi];
      float* s_out = lin_exit_state(a, w, wi, s, g, h);
      if (!WHOLE && !s_out) continue;
      if (!f(w, wi, s, g, h, col0, (g.n + L - 1) / L, s_out)) failed = true;
    }
  };
  auto tile_of = [](const LinWalk& w, int i, int n_tiles) { return w.back ? n_tiles - 1 - i : i; };
  auto rows_of = [](const LinSeg& g, int tile) { return g.n - tile * L < L ? g.n - tile * L : L; };
  uint32_t t = 0;   // tiles of this CTA so far, the same in every role: tile t's barriers are in phase t
  auto stage = [](uint32_t t) { return t % cfg::STAGES; };
  auto lap = [](uint32_t t) { return (t / cfg::STAGES) & 1u; };
  // Barriers in turn: that of tile t, and its phase.  Two of pv and vr always; two of ds, vs and dsf in the pass that only wants states, which keeps V~ and DS for
  // two tiles, the odd ones' where V and QS, PV would be (the control warps' addresses are on a tile's longest path: no turns where none are needed)
  constexpr uint32_t kTurn = WHOLE ? 0 : 1;
  auto turn2 = [](uint32_t bar, uint32_t t) { return bar + 8 * (t & 1); };
  auto wait_turn2 = [&](uint32_t bar, uint32_t t) { return wait(turn2(bar, t), (t >> 1) & 1); };
  auto turn = [](uint32_t bar, uint32_t t) { return bar + 8 * (t & kTurn); };
  auto wait_turn = [&](uint32_t bar, uint32_t t) { return wait(turn(bar, t), (t >> kTurn) & 1); };
  constexpr uint32_t vs_turn = WHOLE ? 0 : (uint32_t)(cfg::TM_V - cfg::TM_VH), ds_turn = WHOLE ? 0 : (uint32_t)(cfg::TM_QS - cfg::TM_DS);

  // (each role changes its registers first of all: nobody waits for a share that another still holds behind a wait)
  if (warp < kStateWarps) {
    // ---------------------------------------------------------------- state warps
    more_registers<104>();
    // S^T as pairs of features.  128 value columns: lane's row 32 quad + lane, features SH half + 2 c, + 1 (S[c]).  64: rows 16 quad + gq and + 8 in
    // lanes 0 .. 15, in accumulator fragments: S[2 nt + e] = row + 8 e, features SH half + 8 nt + t2, + 1.
    constexpr int NP = cfg::SH / 2 * LG / 2, STEP = DV == 128 || NP < 16 ? 8 : 16;
    Pair S[NP];
    auto for_state = [&](auto&& f) {   // f(pair, value column, its first feature)
#pragma unroll
      for (int c = 0; c < NP; ++c) {
        if constexpr (DV == 128) f(S[c], 32 * quad + lane, cfg::SH * half + 2 * c);
        else f(S[c], 16 * quad + 8 * (c & 1) + gq, cfg::SH * half + 8 * (c >> 1) + t2);
      }
    };
    for_items([&](const LinWalk& w, int wi, int s, const LinSeg& g, int h, int col0, int n_tiles, float* s_out) -> bool {
      bool turned;
      const float* s_in = lin_entry_state(a, w, wi, s, g, h, &turned);
      auto inside = [&](int v, int k) { return k < w.d_k && col0 + v < w.d_v; };   // (d_k is even)
      if (!s_in) for_state([&](Pair& x, int, int) { x = pair(0.f, 0.f); });
      else if (turned)
        for_state([&](Pair& x, int v, int k) {
          const float2 y = inside(v, k) ? *reinterpret_cast<const float2*>(s_in + (size_t)(col0 + v) * w.d_k + k) : make_float2(0.f, 0.f);
          x = pair(y.x, y.y);
        });
      else
        for_state([&](Pair& x, int v, int k) {
          const float* at = s_in + (size_t)k * w.d_v + col0 + v;
          const bool in = inside(v, k);
          x = pair(in ? at[0] : 0.f, in ? at[w.d_v] : 0.f);
        });
      const float l2 = lin_log2_decay(a, h);
      const LinFade full = lin_fade(l2, L), last = lin_fade(l2, g.n - (n_tiles - 1) * L);
      for (int i = 0; i < n_tiles; ++i, ++t) {
        const uint32_t ph = t & 1;
        if constexpr (WHOLE) {
          if (t > 0 && !wait(b_qs, ph ^ 1)) return false;   // the operand's last reader
          tc_fence_after();
#pragma unroll
          for (int c = 0; c < NP; c += STEP) {
            uint32_t r[STEP];
#pragma unroll
            for (int q = 0; q < STEP; ++q) r[q] = pack_bf16(S[c + q]);
            const uint32_t at = tmem_w + cfg::TM_S + cfg::SH / 2 * half + c;
            if constexpr (DV == 128) tmem_st_row8(r, at);
            else if constexpr (STEP == 16) tmem_st_packed32(r, at);
            else tmem_st_packed16(r, at);
          }
          tmem_wait_st();
          tc_fence_before();
          warp_arrive(b_sr, lane);
        }
        const LinFade fade = tile_of(w, i, n_tiles) == n_tiles - 1 ? last : full;
        const Pair less = pair(fade.less, fade.less);
        if (!wait_turn(b_ds, t)) return false;
        tc_fence_after();
#pragma unroll
        for (int c = 0; c < NP; c += STEP) {
          float ds[2 * STEP];
          const uint32_t at = tmem_w + cfg::TM_DS + ph * ds_turn + cfg::SH * half + 2 * c;
          if constexpr (DV == 128) tmem_ld_row16(ds, at);
          else if constexpr (STEP == 16) tmem_ld_16x64(reinterpret_cast<float (&)[8][4]>(ds), at);
          else tmem_ld_16x32(reinterpret_cast<float (&)[4][4]>(ds), at);
          tmem_wait_ld();
          if (c + STEP == NP) { tc_fence_before(); warp_arrive(turn(b_dsf, t), lane); }
          if (fade.keep != 0.f) {
#pragma unroll
            for (int q = 0; q < STEP; ++q) S[c + q] = add2(fma2(S[c + q], less, S[c + q]), pair(ds[2 * q], ds[2 * q + 1]));
          } else {
#pragma unroll
            for (int q = 0; q < STEP; ++q) S[c + q] = fma2(S[c + q], less, pair(ds[2 * q], ds[2 * q + 1]));
          }
        }
      }
      if (s_out)
        for_state([&](Pair& x, int v, int k) {
          const float2 y = parts(x);
          if (inside(v, k)) {
            s_out[(size_t)k * w.d_v + col0 + v] = y.x;
            s_out[(size_t)(k + 1) * w.d_v + col0 + v] = y.y;
          }
        });
      return true;
    });
  } else if (WHOLE ? warp < kOutput : warp < kControlA) {
    // ---------------------------------------------------------------- value warps (in the pass that only wants states the output warps too: every second tile each)
    fewer_registers<64>();
    const int row0 = quad * cfg::RPQ;
    float* f = reinterpret_cast<float*>(smem + cfg::OFF_F) + (warp - kValue) * L;   // this warp's table of the tokens' factors
    for_items([&](const LinWalk& w, int, int, const LinSeg& g, int h, int col0, int n_tiles, float*) -> bool {
      const float l2 = lin_log2_decay(a, h);
      int made_for = 0;
      for (int i = 0; i < n_tiles; ++i, ++t) {
        if (!WHOLE && (t & 1) != (uint32_t)(warp >= kOutput)) continue;
        const uint32_t ph = t & 1, base = s0 + stage(t) * cfg::STAGE, sV = base + cfg::OFF_V;
        const int rows = rows_of(g, tile_of(w, i, n_tiles));
        if (rows != made_for) {
          made_for = rows;
          __syncwarp();
#pragma unroll 1
          for (int j = lane; j < L; j += 32) f[j] = j < rows ? w.k_factor * exp2f(l2 * (w.back ? j + 1 : rows - 1 - j)) : 0.f;
          __syncwarp();
        }
        if (!wait(bar_full + 8 * stage(t), lap(t))) return false;
        if (rows < L) {
          // Behind the sequence's end lie a neighbour's rows.  V counts as zero there (below), and zero times a key that is not finite is not zero: the key
          // tile's rows are cleared too (QK may be reading them: those columns of P are left out by selection)
          for (int e = (tid - 32 * kValue) & 255; e < (L - rows) * 8 * cfg::KB; e += 256)
            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(base + cfg::OFF_K + (e / ((L - rows) * 8)) * cfg::BOX + (rows + (e / 8) % (L - rows)) * 128 + (e & 7) * 16), "r"(0) : "memory");
          fence_proxy_async();
        }
        // A warp's part: with 128 value columns 16 of its quadrant's (half) and all tokens, with 64 the quadrant's 16 and 32 tokens (half)
        constexpr int TH = LG;   // blocks of 32 tokens
        const int lg = LG == 2 ? half : 0, th0 = LG == 2 ? 0 : half;
        uint32_t x[TH][8];   // V: pairs of tokens 32 (th0 + th) + 8 nt + t2, + 1 of value columns row0 + 16 lg + gq (2 nt) and + 8 (2 nt + 1)
#pragma unroll
        for (int th = 0; th < TH; ++th)
#pragma unroll
          for (int nt = 0; nt < 4; nt += 2) {
            const int tok = 32 * (th0 + th) + 8 * (nt + (mi >> 1)) + mr, n = row0 + 16 * lg + 8 * (mi & 1);
            ldmatrix_x4_trans(sV + (n >> 6) * cfg::BOX + tok * 128 + ((((n & 63) >> 3) ^ (tok & 7)) << 4), x[th][2 * nt], x[th][2 * nt + 1], x[th][2 * nt + 2], x[th][2 * nt + 3]);
          }
        if (rows < L) {
#pragma unroll
          for (int th = 0; th < TH; ++th)
#pragma unroll
            for (int nt = 0; nt < 4; ++nt) {
              const int j = 32 * (th0 + th) + 8 * nt + t2;
              const uint32_t keep = (j < rows ? 0xffffu : 0u) | (j + 1 < rows ? 0xffff0000u : 0u);
              x[th][2 * nt] &= keep;
              x[th][2 * nt + 1] &= keep;
            }
        }
        if (WHOLE ? t > 0 && !wait_turn(b_ds, t - 1) : t > 1 && !wait_turn(b_ds, t - 2)) return false;   // V~'s place is free
        tc_fence_after();
#pragma unroll
        for (int th = 0; th < TH; ++th) {
          uint32_t hi[8], lo[8];
#pragma unroll
          for (int nt = 0; nt < 4; ++nt) {
            const float2 fj = *reinterpret_cast<const float2*>(f + 32 * (th0 + th) + 8 * nt + t2);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const Pair y = mul2(unpack_bf16(x[th][2 * nt + e]), pair(fj.x, fj.y));
              hi[2 * nt + e] = pack_bf16(y);
              lo[2 * nt + e] = pack_bf16(fma2(unpack_bf16(hi[2 * nt + e]), pair(-1.f, -1.f), y));
            }
          }
          const uint32_t at = tmem_w + ((uint32_t)(16 * lg) << 16) + 16 * (th0 + th) + ph * vs_turn;
          tmem_st_packed16(hi, at + cfg::TM_VH);
          tmem_st_packed16(lo, at + cfg::TM_VL);
        }
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) { mbar_arrive(turn(b_vs, t)); mbar_arrive(bar_empty + 8 * stage(t)); }
        if constexpr (WHOLE) {   // V itself, kept for two tiles in turn
          if (t > 1 && !wait_turn2(b_pv, t - 2)) return false;
          tc_fence_after();
#pragma unroll
          for (int th = 0; th < TH; ++th) tmem_st_packed16(x[th], tmem_w + ((uint32_t)(16 * lg) << 16) + 16 * (th0 + th) + cfg::TM_V + 32 * ph);
          tmem_wait_st();
          tc_fence_before();
          warp_arrive(turn2(b_vr, t), lane);
        }
      }
      return true;
    });
  } else if (WHOLE && warp < kControlA) {
    // ---------------------------------------------------------------- output warps
    fewer_registers<64>();
    if constexpr (WHOLE) {
    const int row0 = quad * cfg::RPQ, ia = 16 * quad + gq, ib = ia + 8;
    float* y = reinterpret_cast<float*>(smem + cfg::OFF_F) + (warp - kValue) * L;   // this warp's table of the tokens' factors of QS
    for_items([&](const LinWalk& w, int, int, const LinSeg& g, int h, int col0, int n_tiles, float*) -> bool {
      const float l2 = lin_log2_decay(a, h), scale = w.k_factor * w.out_factor;
      Pair f[4][2];   // P's factors: columns 32 half + 8 nt + t2, + 1 of rows ia and ib
      // The bits of such a pair that are kept, d rows below its first column.  (Zero factors are not enough where P is masked: a product there may have passed the largest number, or be
      // NaN, and belongs to a token that has not come yet.  Formed at each use: kept in registers they cost a short call 0.2 us more)
      const int da = ia - (32 * half + t2);
      auto kept = [&](int d) { return w.back ? (d <= 1 ? 0xffff0000u : 0u) | (d <= 0 ? 0xffffu : 0u) : (d >= 0 ? 0xffffu : 0u) | (d >= 1 ? 0xffff0000u : 0u); };
#pragma unroll
      for (int nt = 0; nt < 4; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int d = (e ? ib : ia) - (32 * half + 8 * nt + t2), g0 = w.back ? -d : d, g1 = w.back ? 1 - d : d - 1;
          f[nt][e] = pair(g0 >= 0 ? scale * exp2f(l2 * g0) : 0.f, g1 >= 0 ? scale * exp2f(l2 * g1) : 0.f);
        }
      int made_for = 0;
      // O of tile t (its position in the item: i) out of tensor memory into its tile, [token][column]; behind the wait for its PV
      auto put_output = [&](uint32_t t, int rows) -> bool {
        if (rows != made_for) {
          made_for = rows;
          __syncwarp();
#pragma unroll 1
          for (int i = lane; i < L; i += 32) y[i] = i < rows ? w.out_factor * exp2f(l2 * (w.back ? rows - 1 - i : i + 1)) : 0.f;
          __syncwarp();
        }
        if (t > 0 && !wait(b_os, (t - 1) & 1)) return false;   // the last tile's store has read it
        // a warp's part as the value warps': 16 value columns and all tokens, or 32 of them
        constexpr int HF = LG;
        const int lg = LG == 2 ? half : 0, hf0 = LG == 2 ? 0 : half;
#pragma unroll
        for (int hf = 0; hf < HF; ++hf) {
          float pv[4][4], qs[4][4];
          const uint32_t at = tmem_w + ((uint32_t)(16 * lg) << 16) + 32 * (hf0 + hf);
          tmem_ld_16x32(pv, at + cfg::TM_PV);
          tmem_ld_16x32(qs, at + cfg::TM_QS);
          tmem_wait_ld();
          if (hf == HF - 1) { tc_fence_before(); warp_arrive(b_acc, lane); }
          uint32_t o[4][2];
#pragma unroll
          for (int nt = 0; nt < 4; ++nt) {
            const float2 yt = *reinterpret_cast<const float2*>(y + 32 * (hf0 + hf) + 8 * nt + t2);
#pragma unroll
            for (int e = 0; e < 2; ++e)
              o[nt][e] = pack_bf16(fma2(pair(yt.x, yt.y), pair(qs[nt][2 * e], qs[nt][2 * e + 1]), pair(pv[nt][2 * e], pv[nt][2 * e + 1])));
          }
#pragma unroll
          for (int nt = 0; nt < 4; nt += 2) {
            const int tok = 32 * (hf0 + hf) + 8 * (nt + (mi >> 1)) + mr, col = row0 + 16 * lg + 8 * (mi & 1);
            stmatrix_x4_trans(s0 + cfg::OFF_O + (col >> 6) * cfg::BOX + tok * 128 + ((((col >> 3) ^ tok) & 7) << 4), o[nt][0], o[nt][1], o[nt + 1][0], o[nt + 1][1]);
          }
        }
        warp_arrive(b_o, lane);
        return true;
      };
      int last_rows = 0;
      for (int i = 0; i <= n_tiles && n_tiles > 0; ++i, ++t) {
        const uint32_t ph = t & 1;
        const bool more = i < n_tiles;
        uint32_t wa[4], wb[4];
        int rows = 0;
        if (more) {
          rows = rows_of(g, tile_of(w, i, n_tiles));
          if (!wait(b_qk, ph)) return false;
          tc_fence_after();
          float qk[4][4];
          tmem_ld_16x32(qk, tmem_w + cfg::TM_QK + 32 * half);
          tmem_wait_ld();
          tc_fence_before();
          warp_arrive(b_qkf, lane);
          if (rows < L) {   // columns behind the sequence's end: a neighbour's keys, which need not be finite
#pragma unroll
            for (int nt = 0; nt < 4; ++nt) {
              const int j = 32 * half + 8 * nt + t2;
              if (j >= rows) qk[nt][0] = qk[nt][2] = 0.f;
              if (j + 1 >= rows) qk[nt][1] = qk[nt][3] = 0.f;
            }
          }
#pragma unroll
          for (int nt = 0; nt < 4; ++nt) {
            wa[nt] = pack_bf16(mul2(pair(qk[nt][0], qk[nt][1]), f[nt][0])) & kept(da - 8 * nt);
            wb[nt] = pack_bf16(mul2(pair(qk[nt][2], qk[nt][3]), f[nt][1])) & kept(da + 8 - 8 * nt);
          }
        }
        if (t > 0 && !wait_turn2(b_pv, t - 1)) return false;   // PV of the tile before is done: its O can be read, and P's tile is free
        tc_fence_after();
        if (more) {
          const int row = 16 * quad + 8 * (mi & 1) + mr;
#pragma unroll
          for (int nt = 0; nt < 4; nt += 2) stmatrix_x4(sP + row * 128 + (((4 * half + nt + (mi >> 1)) ^ (row & 7)) << 4), wa[nt], wb[nt], wa[nt + 1], wb[nt + 1]);
          warp_arrive(b_pr, lane);   // (the fence for the asynchronous proxy is the control warp's)
        }
        if (i > 0 && !put_output(t - 1, last_rows)) return false;
        last_rows = rows;
        if (!more) break;   // t stays at the next item's first tile
      }
      return true;
    });
    }
  } else {
    // the last warpgroup, a role a warp (setmaxnreg is one instruction for all of it)
    fewer_registers<40>();
    // The descriptors below differ from their bases only in the address field (bits 0 .. 13, units of 16 bytes).
    const uint64_t dQ = umma_desc(s0, 16, 1024), dK = umma_desc(s0 + cfg::OFF_K, 16, 1024), dKm = umma_desc(s0 + cfg::OFF_K, cfg::BOX, 1024), dP = umma_desc(sP, 16, 1024);
    if (warp == kControlA) {
      // ---------------------------------------------------------------- control warp A: DS and QK, which need no state.  (One warp for all the products was what bounded a
      // tile: 28 of them, six commits and seven waits, 2,200 cycles)
      constexpr uint32_t idesc_qk = umma_idesc(64, 64, 0), idesc_ds = umma_idesc(cfg::M, DK, 1);
      auto issue_qk = [&](uint32_t t) {
        const uint32_t st = (stage(t) * cfg::STAGE) >> 4;
#pragma unroll
        for (int ks = 0; ks < DK / 16; ++ks) {
          const uint32_t off = st + (((ks >> 2) * cfg::BOX + (ks & 3) * 32) >> 4);
          umma_bf16(tmem + cfg::TM_QK, dQ + off, dK + off, idesc_qk, ks > 0);
        }
        umma_commit(b_qk);
      };
      for_items([&](const LinWalk& w, int, int, const LinSeg&, int, int, int n_tiles, float*) -> bool {
        for (int i = 0; i < n_tiles; ++i, ++t) {
          const uint32_t ph = t & 1, st = (stage(t) * cfg::STAGE) >> 4;
          if (i == 0) {
            if (!wait(bar_full + 8 * stage(t), lap(t))) return false;
            if constexpr (WHOLE) {
              if (t > 0 && !wait(b_qkf, ph ^ 1)) return false;
              tc_fence_after();
              issue_qk(t);
            }
          }
          if (!wait_turn(b_vs, t) || (WHOLE ? t > 0 && !wait_turn(b_dsf, t - 1) : t > 1 && !wait_turn(b_dsf, t - 2))) return false;
          tc_fence_after();
          // self-test (LinArgs::test_stall): the first CTA leaves out this product of its second tile, so that its waits run out
          const bool stall = a.test_stall && blockIdx.x == 0 && t == 1;
          if (!stall) {
            const uint32_t d = tmem + cfg::TM_DS + ph * ds_turn, v = tmem + ph * vs_turn;
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) umma_bf16_ta(d, v + cfg::TM_VH + 8 * ks, dKm + st + ((ks * 2048) >> 4), idesc_ds, ks > 0);
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) umma_bf16_ta(d, v + cfg::TM_VL + 8 * ks, dKm + st + ((ks * 2048) >> 4), idesc_ds, 1u);
            umma_commit(turn(b_ds, t));
          }
          umma_commit(bar_empty + 8 * stage(t));
          if (i + 1 < n_tiles) {
            if (!wait(bar_full + 8 * stage(t + 1), lap(t + 1))) return false;
            if constexpr (WHOLE) {
              if (!wait(b_qkf, ph)) return false;
              tc_fence_after();
              issue_qk(t + 1);
            }
          }
        }
        return true;
      });
      // every product issued is waited for, with a limit, before the CTA gives up its memory: who reads them may have given up
      umma_commit(b_exit);
      mbar_wait_bounded(b_exit, 0u, lim);
    } else if (warp == kControlB && WHOLE) {
      // ---------------------------------------------------------------- control warp B: QS and PV
      constexpr uint32_t idesc_s = umma_idesc(cfg::M, 64, 0);
      for_items([&](const LinWalk& w, int, int, const LinSeg&, int, int, int n_tiles, float*) -> bool {
        for (int i = 0; i < n_tiles; ++i, ++t) {
          const uint32_t ph = t & 1, st = (stage(t) * cfg::STAGE) >> 4;
          if (!wait(bar_full + 8 * stage(t), lap(t)) || !wait(b_sr, ph) || (t > 0 && !wait(b_acc, ph ^ 1))) return false;
          tc_fence_after();
#pragma unroll
          for (int ks = 0; ks < DK / 16; ++ks)
            umma_bf16_ta(tmem + cfg::TM_QS, tmem + cfg::TM_S + 8 * ks, dQ + st + (((ks >> 2) * cfg::BOX + (ks & 3) * 32) >> 4), idesc_s, ks > 0);
          umma_commit(b_qs);
          umma_commit(bar_empty + 8 * stage(t));
          if (!wait(b_pr, ph) || !wait_turn2(b_vr, t)) return false;
          fence_proxy_async();   // P was written by ordinary stores
          tc_fence_after();
#pragma unroll
          for (int ks = 0; ks < L / 16; ++ks)
            umma_bf16_ta(tmem + cfg::TM_PV, tmem + cfg::TM_V + 32 * ph + 8 * ks, dP + ((ks * 32) >> 4), idesc_s, ks > 0);
          umma_commit(turn2(b_pv, t));
        }
        return true;
      });
      umma_commit(b_exitb);
      mbar_wait_bounded(b_exitb, 0u, lim);
    } else if (warp == kCopyL) {
      // ---------------------------------------------------------------- copy warp
      for_items([&](const LinWalk& w, int wi, int, const LinSeg& g, int h, int col0, int n_tiles, float*) -> bool {
        for (int i = 0; i < n_tiles; ++i, ++t) {
          if (t >= cfg::STAGES && !wait(bar_empty + 8 * stage(t), lap(t) ^ 1)) return false;
          if (lane == 0) {
            const uint32_t base = s0 + stage(t) * cfg::STAGE, bar = bar_full + 8 * stage(t);
            const int tok = g.tok0 + tile_of(w, i, n_tiles) * L;
            mbar_expect_tx(bar, WHOLE ? cfg::STAGE : cfg::STAGE - cfg::KB * cfg::BOX);
#pragma unroll
            for (int b = 0; b < cfg::KB; ++b) tma_load_3d(base + cfg::OFF_K + b * cfg::BOX, &maps.k[wi], bar, 64 * b, h, tok);
#pragma unroll
            for (int b = 0; b < cfg::VB; ++b) tma_load_3d(base + cfg::OFF_V + b * cfg::BOX, &maps.v[wi], bar, col0 + 64 * b, h, tok);
            if constexpr (WHOLE)
#pragma unroll
              for (int b = 0; b < cfg::KB; ++b) tma_load_3d(base + b * cfg::BOX, &maps.q[wi], bar, 64 * b, h, tok);
          }
          __syncwarp();
        }
        return true;
      });
      if (lane == 0)   // and every copy into this CTA's shared memory
        for (uint32_t c = t >= cfg::STAGES ? t - cfg::STAGES : 0; c < t; ++c) mbar_wait_bounded(bar_full + 8 * stage(c), lap(c), lim);
    } else if (warp == kStoreL && WHOLE) {
      // ---------------------------------------------------------------- store warp: O's tile to memory
      for_items([&](const LinWalk& w, int wi, int, const LinSeg& g, int h, int col0, int n_tiles, float*) -> bool {
        for (int i = 0; i < n_tiles; ++i, ++t) {
          if (!wait(b_o, t & 1)) return false;
          const int tile = tile_of(w, i, n_tiles), tok0 = g.tok0 + tile * L, rows = rows_of(g, tile);
          if (rows == L) {
            if (lane == 0) {
              fence_proxy_async();   // the tile was written by ordinary stores
#pragma unroll
              for (int b = 0; b < cfg::VB; ++b) tma_store_3d(&maps.o[wi], s0 + cfg::OFF_O + b * cfg::BOX, col0 + 64 * b, h, tok0);
              bulk_commit();
              bulk_wait_read();
            }
          } else {
            __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(w.out) + ((size_t)tok0 * a.H + h) * w.d_v + col0;
            for (int e = lane; e < rows * (DV / 8); e += 32) {
              const int tok = e / (DV / 8), pc = e % (DV / 8);
              if (col0 + 8 * pc < w.d_v)
                *reinterpret_cast<uint4*>(out + (size_t)tok * a.H * w.d_v + 8 * pc) =
                  *reinterpret_cast<const uint4*>(smem + cfg::OFF_O + (pc >> 3) * cfg::BOX + tok * 128 + (((pc ^ tok) & 7) << 4));
            }
          }
          warp_arrive(b_os, lane);
        }
        return true;
      });
    }
  }
  if (failed) atomicMax(a.status, (int)TRI_INV_ERR_DEVICE_TIMEOUT);
  tc_fence_before();
  __syncthreads();
  if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}

// 3-D view [tokens, H, d] of bf16: a box is 64 features of one head (zeros behind the head's last, which a store leaves out) x 64 tokens, in rows of 128 bytes, swizzled
bool make_head_map(CUtensorMap* tm, const void* base, long long tokens, int H, int d) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[3] = {(cuuint64_t)d, (cuuint64_t)H, (cuuint64_t)tokens};
  cuuint64_t strides[2] = {(cuuint64_t)d * 2, (cuuint64_t)H * d * 2};
  cuuint32_t box[3] = {64, 1, (cuuint32_t)L};
  cuuint32_t estr[3] = {1, 1, 1};
  return fn(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int DK, int DV, bool WHOLE>
cudaError_t launch_form(const LinMaps& maps, const LinTcArgs& args, int sms, cudaStream_t stream) {
  using cfg = LinCfg<DK, DV>;
  static std::mutex mu;
  static bool ready[64] = {false};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  {
    std::lock_guard<std::mutex> lock(mu);
    if (!ready[dev]) {
      if ((e = cudaFuncSetAttribute(linear_tc_kernel<DK, DV, WHOLE>, cudaFuncAttributeMaxDynamicSharedMemorySize, cfg::SMEM)) != cudaSuccess) { (void)cudaGetLastError(); return e; }
      ready[dev] = true;
    }
  }
  const long long items = (long long)args.a.n_segs * args.a.H * args.n_walks * args.slices;
  e = launch_early(linear_tc_kernel<DK, DV, WHOLE>, dim3((unsigned)(items < sms ? items : sms)), kThreadsL, cfg::SMEM, stream, maps, args);
  return e == cudaSuccess ? launched() : e;
}

template <int DK, int DV>
cudaError_t launch_one(const LinMaps& maps, const LinTcArgs& args, int sms, cudaStream_t stream) {
  return args.a.state_only ? launch_form<DK, DV, false>(maps, args, sms, stream) : launch_form<DK, DV, true>(maps, args, sms, stream);
}

}  // namespace

bool linear_tc_fits(int d_k, int d_v, int kv_dtype) {
  return kv_dtype == TRI_INV_BF16 && d_k <= 128 && d_v <= 128;
}

cudaError_t launch_linear_tc(const LinArgs& a, long long tokens, cudaStream_t stream) {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return cudaErrorUnknown;
  LinMaps maps;
  for (int i = 0; i < a.n_walks; ++i) {
    const LinWalk& w = a.walk[i];
    if (!make_head_map(&maps.q[i], w.q, tokens, a.H, w.d_k) || !make_head_map(&maps.k[i], w.k, tokens, a.H, w.d_k) || !make_head_map(&maps.v[i], w.v, tokens, a.H, w.d_v) ||
        !make_head_map(&maps.o[i], w.out, tokens, a.H, w.d_v))
      return cudaErrorUnknown;
  }
  // the walks of one launch take the same form of the kernel: head dimensions up to 64 or up to 128 (the tiles' rest is zeros)
  auto wide_k = [&](int i) { return a.walk[i].d_k > 64; };
  auto wide_v = [&](int i) { return a.walk[i].d_v > 64; };
  LinTcArgs args{a, 0, 0, 1};
  for (int first = 0; first < a.n_walks; first += args.n_walks) {
    args.first_walk = first;
    args.n_walks = 1;
    while (first + args.n_walks < a.n_walks && wide_k(first + args.n_walks) == wide_k(first) && wide_v(first + args.n_walks) == wide_v(first)) ++args.n_walks;
    args.slices = wide_v(first) ? a.slices : 1;
    const bool narrow = !wide_v(first) || args.slices == 2;
    const cudaError_t e = wide_k(first) ? (narrow ? launch_one<128, 64>(maps, args, sms, stream) : launch_one<128, 128>(maps, args, sms, stream))
                                        : (narrow ? launch_one<64, 64>(maps, args, sms, stream) : launch_one<64, 128>(maps, args, sms, stream));
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace tri_inv
