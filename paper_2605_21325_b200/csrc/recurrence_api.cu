// extern "C" boundary of the gated linear recurrence and of the heads' norm with rotation: argument checks, the cut into tiles, dispatch.
#include <algorithm>
#include <cmath>

#include "call_checks.cuh"
#include "gated_recurrence.cuh"
#include "qk_norm_rope.cuh"

namespace tri_inv {
namespace {

size_t round_up(size_t n) { return (n + 255) & ~(size_t)255; }

constexpr int64_t kMostBetweenRows = 1 << 26;

int check_rec(const tri_inv_rec_desc* d) {
  if (!d || d->B < 1 || d->T < 0 || d->D < 1) return TRI_INV_ERR_INVALID_ARG;
  if (d->dtype != TRI_INV_F32 && d->dtype != TRI_INV_BF16) return TRI_INV_ERR_INVALID_ARG;
  if (d->mode != TRI_INV_REC_DECAY && d->mode != TRI_INV_REC_NORMED && d->mode != TRI_INV_REC_GATE) return TRI_INV_ERR_INVALID_ARG;
  if ((long long)d->B * d->T > 0x7fffffffLL) return TRI_INV_ERR_INVALID_ARG;
  if (d->cu_seqlens) {
    if (d->B != 1 || d->n_seqs < 0 || d->cu_seqlens[0] != 0 || d->cu_seqlens[d->n_seqs] != d->T) return TRI_INV_ERR_INVALID_ARG;
    for (int s = 0; s < d->n_seqs; ++s)
      if (d->cu_seqlens[s + 1] < d->cu_seqlens[s]) return TRI_INV_ERR_INVALID_ARG;
  } else if (d->n_seqs != 0) {
    return TRI_INV_ERR_INVALID_ARG;
  }
  return d->D > kMostBetweenRows ? TRI_INV_ERR_UNSUPPORTED : TRI_INV_OK;
}
int seqs_of(const tri_inv_rec_desc* d) { return d->cu_seqlens ? d->n_seqs : d->B; }
long long tokens_of(const tri_inv_rec_desc* d) { return (long long)d->B * d->T; }
long long slots_of(const tri_inv_rec_desc* d, int tile) { return rec_slot(tokens_of(d), seqs_of(d), tile) + 1; }
Rows rows_of(const tri_inv_rec_desc* d, const void* p, int64_t ld) {
  const int es = d->dtype == TRI_INV_F32 ? 4 : 2;
  return Rows{p, tokens_of(d), (__int128)d->D * es, (__int128)ld * es};
}
bool strides_fit(std::initializer_list<int64_t> lds) {   // sixteen rows are counted in 32 bits of bytes
  for (int64_t ld : lds)
    if (ld > kMostBetweenRows) return false;
  return true;
}
Span states_of(const tri_inv_rec_desc* d, const void* p) { return Span{p, (__int128)seqs_of(d) * d->D * 4}; }
Span carries_of(const tri_inv_rec_desc* d, const void* p) { return Span{p, (__int128)slots_of(d, kRecCarry) * d->D * 4}; }

// Sequences of so many tiles are walked whole, whatever the number of channels: the words cost a launch that clears them and, at each tile, the way through the L2 cache.  Longer ones go tile by tile, which
// spreads them over the chip and lets no block be the last for long.  Measured (bf16, us, forward and gradient, tile by tile | whole): 1 x 200 tokens x 2048 channels 7.0 and 7.7 | 5.4 and 7.3; 1 x 333 x 2048 7.3 and 8.1 |
// 6.4 and 9.0; 8 x 333 x 2048 14.6 and 21.4 | 11.2 and 21.0; 1 x 1000 x 2048 10.4 and 12.3 | 11.8 and 18.0; 1 x 4000 x 512 10.7 and 13.3 | 39 and 61; 16 x 1024 x 2048 40.5 and 73.5 | 42.6 and 77.9; 20 x 2048 x 2048
// 88.5 and 163 | 85.6 and 170.  The gradient at three tiles: bf16 (128 tokens a tile) 1 x 333 x 2048 7.7 | 9.7 and 64 x 333 x 2048 120 | 127, against 8 x 333 x 2048 22.4 | 21.4; fp32 (64 tokens) 1 x 180 x 2048 6.7 | 6.3,
// 8 x 180 x 2048 14.9 | 14.2, 64 x 180 x 2048 86 | 81, 200 x 180 x 256 36.4 | 34.5; at four, fp32, 1 x 250 x 2048 7.0 | 7.6, 64 x 250 x 2048 115 | 124, 1 x 250 x 333 7.7 | 12.7, against 16 x 250 x 512 12.5 | 10.0.
constexpr int kMostWalked = 3;
constexpr int most_walked_back(int dtype) { return dtype == TRI_INV_F32 ? 3 : 2; }

// How a walk goes: tile by tile with words between the tiles, or whole sequences.
struct RecPlan {
  int tile;
  bool words;
  int n_segs, cols;
  size_t table_bytes, word_bytes;   // word_bytes: with the ticket in front
  size_t bytes() const { return table_bytes + word_bytes; }
};
int plan(const tri_inv_rec_desc* d, int tile, int most_walked, RecPlan* p) {
  const int n_seqs = seqs_of(d);
  auto tiles_of = [&](long long n) { return std::max(1ll, (n + tile - 1) / tile); };
  long long tiles = 0, longest = 1;
  if (d->cu_seqlens) {
    for (int s = 0; s < n_seqs; ++s) {
      const long long t = tiles_of((long long)d->cu_seqlens[s + 1] - d->cu_seqlens[s]);
      tiles += t;
      longest = std::max(longest, t);
    }
  } else {
    longest = tiles_of(d->T);
    tiles = longest * n_seqs;
  }
  p->tile = tile;
  p->cols = (int)(((long long)d->D + kRecChannels - 1) / kRecChannels);
  p->words = longest > most_walked;
  const long long segs = p->words ? tiles : n_seqs;
  if (segs * p->cols >= 0x3ff00000LL) return TRI_INV_ERR_INVALID_ARG;   // items are counted in 32 bits
  p->n_segs = (int)segs;
  p->table_bytes = d->cu_seqlens ? round_up((size_t)segs * sizeof(RecTile)) : 0;
  p->word_bytes = p->words ? 256 + round_up((size_t)slots_of(d, tile) * d->D * 8) : 0;
  return TRI_INV_OK;
}

// The gradient's walk and, without carries, one in front of it that forms them
struct BackPlan {
  RecPlan back, front;
  size_t carry_bytes;
  size_t bytes() const { return carry_bytes + (carry_bytes ? front.bytes() : 0) + back.bytes(); }
};
int plan_back(const tri_inv_rec_desc* d, bool with_carries, BackPlan* p) {
  p->carry_bytes = with_carries ? 0 : round_up((size_t)slots_of(d, kRecCarry) * d->D * 4);
  const int e = plan(d, rec_back_tile(d->dtype == TRI_INV_F32 ? 4 : 2), most_walked_back(d->dtype), &p->back);
  return e ? e : plan(d, kRecTile, kMostWalked, &p->front);
}

// A walk's share of the arguments, and what is to be set up in its part of the workspace
RecSetup place_walk(RecArgs& a, const RecPlan& p, const tri_inv_rec_desc* d, void* workspace) {
  a.n_seqs = seqs_of(d); a.T = d->T; a.D = d->D; a.cols = p.cols; a.n_segs = p.n_segs; a.mode = d->mode;
  a.items = p.n_segs * p.cols;
  a.by_cols = rec_divide_by(p.cols);
  a.by_seqs = rec_divide_by(std::max(1, a.n_seqs));
  if (d->T == 0) a.x = a.g = a.dy = a.status;   // no row is read, but the copies' addresses are formed
  a.table = d->cu_seqlens ? (RecTile*)workspace : nullptr;
  a.ticket = p.words ? (unsigned int*)((char*)workspace + p.table_bytes) : nullptr;
  a.words = p.words ? (unsigned long long*)((char*)workspace + p.table_bytes + 256) : nullptr;
  return RecSetup{a.ticket, a.words, (RecTile*)a.table, p.words ? slots_of(d, p.tile) * d->D : 0, p.words ? p.tile : 0};
}
int walk_forward(RecArgs& a, const RecPlan& p, const tri_inv_rec_desc* d, void* workspace, cudaStream_t stream) {
  cudaError_t err;
  a.status = status_word_for_current_device(&err);
  if (!a.status) return TRI_INV_ERR_CUDA;
  if (p.n_segs == 0) return TRI_INV_OK;
  const RecSetup setup = place_walk(a, p, d, workspace);
  return launch_rec_setup(&setup, 1, d->cu_seqlens, a.n_seqs, stream) == cudaSuccess && launch_gated_recurrence(a, d->dtype, stream) == cudaSuccess ? TRI_INV_OK : TRI_INV_ERR_CUDA;
}

int check_heads(const tri_inv_heads_desc* d) {
  if (!d || d->tokens < 0 || d->tokens > 0x7fffffffLL || d->H_q < 0 || d->H_k < 0 || d->d < 1 || d->r < 0 || d->r > d->d / 2) return TRI_INV_ERR_INVALID_ARG;
  if (d->dtype != TRI_INV_F32 && d->dtype != TRI_INV_BF16) return TRI_INV_ERR_INVALID_ARG;
  if (!(d->eps >= 0.f) || std::isinf(d->eps) || (d->interleaved != 0 && d->interleaved != 1)) return TRI_INV_ERR_INVALID_ARG;
  if ((long long)d->H_q + d->H_k > 0x100000) return TRI_INV_ERR_INVALID_ARG;   // a token's heads and warps are counted in 32 bits
  return d->d > kHeadsMaxDim ? TRI_INV_ERR_UNSUPPORTED : TRI_INV_OK;
}
Rows heads_of(const tri_inv_heads_desc* d, int H, const void* p, int64_t ld) {
  const int es = d->dtype == TRI_INV_F32 ? 4 : 2;
  return Rows{p, H ? d->tokens : 0, (__int128)H * d->d * es, (__int128)ld * es};
}

}  // namespace
}  // namespace tri_inv

using namespace tri_inv;

extern "C" {

int tri_inv_gated_recurrence_carries(const tri_inv_rec_desc* desc, int64_t* rows) {
  const int rc = check_rec(desc);
  if (rc) return rc;
  if (!rows) return TRI_INV_ERR_INVALID_ARG;
  *rows = slots_of(desc, kRecCarry);
  return TRI_INV_OK;
}

int tri_inv_gated_recurrence_workspace(const tri_inv_rec_desc* desc, size_t* bytes) {
  const int rc = check_rec(desc);
  if (rc) return rc;
  if (!bytes) return TRI_INV_ERR_INVALID_ARG;
  RecPlan p;
  const int e = plan(desc, kRecTile, kMostWalked, &p);
  if (e) return e;
  *bytes = p.bytes();
  return TRI_INV_OK;
}

int tri_inv_gated_recurrence(const void* X, int64_t ldx, const void* G, int64_t ldg, const float* h0, void* Y, int64_t ldy, float* h_out, float* carries,
                             void* workspace, size_t workspace_bytes, const tri_inv_rec_desc* desc, void* cuda_stream) {
  const int rc = check_rec(desc);
  if (rc) return rc;
  const int32_t D = desc->D;
  if ((tokens_of(desc) > 0 && (!X || !G || (!Y && !h_out && !carries))) || ldx < D || ldg < D || (Y && ldy < D)) return TRI_INV_ERR_INVALID_ARG;
  if (!strides_fit({ldx, ldg, ldy})) return TRI_INV_ERR_UNSUPPORTED;
  if (!on_type(desc->dtype, X, G, Y) || !aligned4(h0) || !aligned4(h_out) || !aligned4(carries) || !aligned16(workspace)) return TRI_INV_ERR_INVALID_ARG;
  const Rows x = rows_of(desc, X, ldx), g = rows_of(desc, G, ldg), y = rows_of(desc, Y, ldy);
  const Span s0 = states_of(desc, h0), s1 = states_of(desc, h_out), sc = carries_of(desc, carries);
  if ((meets(y, x) && !same(y, x)) || (meets(y, g) && !same(y, g)) || meets_any(s1, span_of(x), span_of(g), span_of(y), sc) || (h_out != h0 && meets(s1, s0)) ||
      meets(span_of(y), s0) || meets_any(sc, span_of(x), span_of(g), span_of(y), s0))
    return TRI_INV_ERR_INVALID_ARG;
  RecPlan p;
  const int e = plan(desc, kRecTile, kMostWalked, &p);
  if (e) return e;
  const Span work{workspace, (__int128)p.bytes()};
  if (workspace_bytes < p.bytes() || (p.bytes() > 0 && !workspace) || meets_any(work, span_of(x), span_of(g), span_of(y), s0, s1, sc)) return TRI_INV_ERR_INVALID_ARG;
  RecArgs a{};
  a.x = X; a.ld_x = ldx; a.g = G; a.ld_g = ldg; a.y = Y; a.ld_y = ldy;
  a.h0 = h0; a.h_out = h_out; a.carries = carries;
  return walk_forward(a, p, desc, workspace, (cudaStream_t)cuda_stream);
}

int tri_inv_selftest_recurrence_wait_timeout(const void* X, const void* G, void* Y, void* workspace, size_t workspace_bytes, const tri_inv_rec_desc* desc,
                                             uint64_t wait_limit_ns, void* cuda_stream) {
  const int rc = check_rec(desc);
  if (rc) return rc;
  RecPlan p;
  const int e = plan(desc, kRecTile, kMostWalked, &p);
  if (e) return e;
  if (!p.words || desc->cu_seqlens) return TRI_INV_ERR_UNSUPPORTED;
  if (!X || !G || !Y || !on_type(desc->dtype, X, G, Y) || !wait_limit_ns || !workspace || !aligned16(workspace) || workspace_bytes < p.bytes()) return TRI_INV_ERR_INVALID_ARG;
  RecArgs a{};
  a.x = X; a.g = G; a.y = Y;
  a.ld_x = a.ld_g = a.ld_y = desc->D;
  a.wait_limit_ns = wait_limit_ns;
  a.test_stall = 1;
  const int b = walk_forward(a, p, desc, workspace, (cudaStream_t)cuda_stream);
  if (b) return b;
  return cudaStreamSynchronize((cudaStream_t)cuda_stream) == cudaSuccess ? TRI_INV_OK : TRI_INV_ERR_CUDA;
}

int tri_inv_gated_recurrence_backward_workspace(const tri_inv_rec_desc* desc, int with_carries, size_t* bytes) {
  const int rc = check_rec(desc);
  if (rc) return rc;
  if (!bytes) return TRI_INV_ERR_INVALID_ARG;
  BackPlan p;
  const int e = plan_back(desc, with_carries, &p);
  if (e) return e;
  *bytes = p.bytes();
  return TRI_INV_OK;
}

int tri_inv_gated_recurrence_backward(const void* dY, int64_t lddy, const void* X, int64_t ldx, const void* G, int64_t ldg, const float* h0, const float* dh,
                                      const float* carries, void* dX, int64_t lddx, void* dG, int64_t lddg, float* dh0, void* workspace,
                                      size_t workspace_bytes, const tri_inv_rec_desc* desc, void* cuda_stream) {
  const int rc = check_rec(desc);
  if (rc) return rc;
  const int32_t D = desc->D;
  if ((tokens_of(desc) > 0 && (!dY || !X || !G || !dX || !dG)) || lddy < D || ldx < D || ldg < D || lddx < D || lddg < D) return TRI_INV_ERR_INVALID_ARG;
  if (!strides_fit({lddy, ldx, ldg, lddx, lddg})) return TRI_INV_ERR_UNSUPPORTED;
  if (!on_type(desc->dtype, dY, X, G, dX, dG) || !aligned4(h0) || !aligned4(dh) || !aligned4(carries) || !aligned4(dh0) || !aligned16(workspace)) return TRI_INV_ERR_INVALID_ARG;
  const Rows dy = rows_of(desc, dY, lddy), x = rows_of(desc, X, ldx), g = rows_of(desc, G, ldg), dx = rows_of(desc, dX, lddx), dg = rows_of(desc, dG, lddg);
  const Span s0 = states_of(desc, h0), sd = states_of(desc, dh), s1 = states_of(desc, dh0), sc = carries_of(desc, carries);
  if ((meets(dx, dy) && !same(dx, dy)) || (meets(dx, x) && !same(dx, x)) || meets(dx, g) || (meets(dg, dy) && !same(dg, dy)) || (meets(dg, g) && !same(dg, g)) || meets(dg, x) || meets(dx, dg))
    return TRI_INV_ERR_INVALID_ARG;
  if (meets_any(s1, span_of(dy), span_of(x), span_of(g), span_of(dx), span_of(dg), s0, sc) || (dh0 != dh && meets(s1, sd)) || meets_any(span_of(dx), s0, sd, sc) ||
      meets_any(span_of(dg), s0, sd, sc))
    return TRI_INV_ERR_INVALID_ARG;
  BackPlan p;
  const int e = plan_back(desc, carries != nullptr, &p);
  if (e) return e;
  const size_t need = p.bytes();
  if (workspace_bytes < need || (need > 0 && !workspace) ||
      meets_any(Span{workspace, (__int128)need}, span_of(dy), span_of(x), span_of(g), span_of(dx), span_of(dg), s0, sd, s1, sc))
    return TRI_INV_ERR_INVALID_ARG;
  RecArgs a{};
  a.x = X; a.ld_x = ldx; a.g = G; a.ld_g = ldg; a.h0 = h0;
  a.carries = carries ? (float*)carries : (float*)workspace;
  cudaError_t err;
  a.status = status_word_for_current_device(&err);
  if (!a.status) return TRI_INV_ERR_CUDA;
  if (p.back.n_segs == 0) return TRI_INV_OK;
  RecArgs front = a;
  RecSetup setup[2];
  void* control = (char*)workspace + p.carry_bytes;
  if (!carries) setup[1] = place_walk(front, p.front, desc, (char*)control + p.back.bytes());
  a.dy = dY; a.ld_dy = lddy; a.dx = dX; a.ld_dx = lddx; a.dg = dG; a.ld_dg = lddg; a.dh = dh; a.dh0 = dh0;
  setup[0] = place_walk(a, p.back, desc, control);
  const cudaStream_t stream = (cudaStream_t)cuda_stream;
  if (launch_rec_setup(setup, carries ? 1 : 2, desc->cu_seqlens, a.n_seqs, stream) != cudaSuccess) return TRI_INV_ERR_CUDA;
  if (!carries && launch_gated_recurrence(front, desc->dtype, stream) != cudaSuccess) return TRI_INV_ERR_CUDA;
  return launch_gated_recurrence_backward(a, desc->dtype, stream) == cudaSuccess ? TRI_INV_OK : TRI_INV_ERR_CUDA;
}

int tri_inv_gated_recurrence_step(const void* X, int64_t ldx, const void* G, int64_t ldg, float* h, const int32_t* slots, int32_t n_slots, void* Y, int64_t ldy,
                                  const tri_inv_rec_desc* desc, void* cuda_stream) {
  const int rc = check_rec(desc);
  if (rc) return rc;
  if (desc->cu_seqlens || desc->T != 1 || n_slots < 0 || (!slots && n_slots < desc->B)) return TRI_INV_ERR_INVALID_ARG;
  const int32_t D = desc->D;
  if (!X || !G || !h || !Y || ldx < D || ldg < D || ldy < D || !on_type(desc->dtype, X, G, Y) || !aligned4(h) || !aligned4(slots)) return TRI_INV_ERR_INVALID_ARG;
  if ((long long)desc->B * (((long long)D + 127) / 128) > 0x7fffffffLL) return TRI_INV_ERR_INVALID_ARG;   // blocks
  const Rows x = rows_of(desc, X, ldx), g = rows_of(desc, G, ldg), y = rows_of(desc, Y, ldy);
  const Span states{h, (__int128)n_slots * D * 4}, rows{slots, 4ll * desc->B};
  if ((meets(y, x) && !same(y, x)) || (meets(y, g) && !same(y, g)) || meets_any(states, span_of(x), span_of(g), span_of(y), rows) || meets(span_of(y), rows)) return TRI_INV_ERR_INVALID_ARG;
  RecStepArgs a{X, G, Y, ldx, ldg, ldy, h, slots, desc->B, D, n_slots, desc->mode, nullptr};
  cudaError_t err;
  a.status = status_word_for_current_device(&err);
  if (!a.status) return TRI_INV_ERR_CUDA;
  return launch_gated_recurrence_step(a, desc->dtype, (cudaStream_t)cuda_stream) == cudaSuccess ? TRI_INV_OK : TRI_INV_ERR_CUDA;
}

int tri_inv_qk_norm_rope(const void* Q, int64_t ldq, const void* K, int64_t ldk, const void* wq, const void* wk, const float* inv_freq, const int32_t* positions,
                         void* Yq, int64_t ldyq, void* Yk, int64_t ldyk, const tri_inv_heads_desc* desc, void* cuda_stream) {
  const int rc = check_heads(desc);
  if (rc) return rc;
  const long long nq = (long long)desc->H_q * desc->d, nk = (long long)desc->H_k * desc->d;
  if (desc->tokens == 0) return TRI_INV_OK;
  if ((nq && (!Q || !Yq || ldq < nq || ldyq < nq)) || (nk && (!K || !Yk || ldk < nk || ldyk < nk)) || (desc->r && !inv_freq) || (!positions && desc->T < 1)) return TRI_INV_ERR_INVALID_ARG;
  if (!on_type(desc->dtype, Q, K, wq, wk, Yq, Yk) || !aligned4(inv_freq) || !aligned4(positions)) return TRI_INV_ERR_INVALID_ARG;
  const Rows q = heads_of(desc, desc->H_q, Q, ldq), k = heads_of(desc, desc->H_k, K, ldk), yq = heads_of(desc, desc->H_q, Yq, ldyq), yk = heads_of(desc, desc->H_k, Yk, ldyk);
  const int es = desc->dtype == TRI_INV_F32 ? 4 : 2;
  const Span small[4] = {{wq, (__int128)desc->d * es}, {wk, (__int128)desc->d * es}, {inv_freq, 4ll * desc->r}, {positions, 4 * (__int128)desc->tokens}};
  if ((meets(yq, q) && !same(yq, q)) || meets(yq, k) || (meets(yk, k) && !same(yk, k)) || meets(yk, q) || meets(yq, yk)) return TRI_INV_ERR_INVALID_ARG;
  for (const Span& s : small)
    if (meets_any(s, span_of(yq), span_of(yk))) return TRI_INV_ERR_INVALID_ARG;
  HeadsArgs a{};
  a.side[0].x = Q; a.side[0].w = wq; a.side[0].y = Yq; a.side[0].ld_x = ldq; a.side[0].ld_y = ldyq; a.side[0].H = desc->H_q;
  a.side[1].x = K; a.side[1].w = wk; a.side[1].y = Yk; a.side[1].ld_x = ldk; a.side[1].ld_y = ldyk; a.side[1].H = desc->H_k;
  a.inv_freq = inv_freq; a.positions = positions; a.tokens = desc->tokens; a.T = desc->T; a.d = desc->d; a.r = desc->r; a.interleaved = desc->interleaved; a.eps = desc->eps;
  return launch_qk_norm_rope(a, desc->dtype, (cudaStream_t)cuda_stream) == cudaSuccess ? TRI_INV_OK : TRI_INV_ERR_CUDA;
}

int tri_inv_qk_norm_rope_backward_workspace(const tri_inv_heads_desc* desc, size_t* bytes) {
  const int rc = check_heads(desc);
  if (rc) return rc;
  if (!bytes) return TRI_INV_ERR_INVALID_ARG;
  *bytes = (size_t)kHeadsPartials * desc->d * sizeof(float);
  return TRI_INV_OK;
}

int tri_inv_qk_norm_rope_backward(const void* dYq, int64_t lddyq, const void* dYk, int64_t lddyk, const void* Q, int64_t ldq, const void* K, int64_t ldk,
                                  const void* wq, const void* wk, const float* inv_freq, const int32_t* positions, void* dQ, int64_t lddq, void* dK,
                                  int64_t lddk, void* dwq, void* dwk, void* workspace, size_t workspace_bytes, const tri_inv_heads_desc* desc, void* cuda_stream) {
  const int rc = check_heads(desc);
  if (rc) return rc;
  const long long nq = (long long)desc->H_q * desc->d, nk = (long long)desc->H_k * desc->d;
  if (desc->tokens > 0 && ((nq && (!dYq || !Q || !dQ || lddyq < nq || ldq < nq || lddq < nq)) || (nk && (!dYk || !K || !dK || lddyk < nk || ldk < nk || lddk < nk)) ||
                           (desc->r && !inv_freq) || (!positions && desc->T < 1)))
    return TRI_INV_ERR_INVALID_ARG;
  if (!on_type(desc->dtype, dYq, dYk, Q, K, wq, wk, dQ, dK, dwq, dwk) || !aligned4(inv_freq) || !aligned4(positions)) return TRI_INV_ERR_INVALID_ARG;
  const size_t need = (size_t)kHeadsPartials * desc->d * sizeof(float);
  if (!workspace || !aligned16(workspace) || workspace_bytes < need) return TRI_INV_ERR_INVALID_ARG;
  const int es = desc->dtype == TRI_INV_F32 ? 4 : 2;
  const Rows in[4] = {heads_of(desc, desc->H_q, dYq, lddyq), heads_of(desc, desc->H_q, Q, ldq), heads_of(desc, desc->H_k, dYk, lddyk), heads_of(desc, desc->H_k, K, ldk)};
  const Rows out[2] = {heads_of(desc, desc->H_q, dQ, lddq), heads_of(desc, desc->H_k, dK, lddk)};
  const Span small[7] = {{wq, (__int128)desc->d * es}, {wk, (__int128)desc->d * es}, {inv_freq, 4ll * desc->r}, {positions, 4 * (__int128)desc->tokens},
                         {dwq, (__int128)desc->d * es}, {dwk, (__int128)desc->d * es}, {workspace, (__int128)need}};
  for (int o = 0; o < 2; ++o)
    for (int i = 0; i < 4; ++i)
      if (meets(out[o], in[i]) && (i / 2 != o || !same(out[o], in[i]))) return TRI_INV_ERR_INVALID_ARG;
  if (meets(out[0], out[1])) return TRI_INV_ERR_INVALID_ARG;
  for (int i = 0; i < 7; ++i) {
    if (meets_any(small[i], span_of(out[0]), span_of(out[1]))) return TRI_INV_ERR_INVALID_ARG;
    for (int j = std::max(4, i + 1); j < 7; ++j)
      if (meets(small[i], small[j])) return TRI_INV_ERR_INVALID_ARG;
    if (i >= 4)
      for (const Rows& r : in)
        if (meets(small[i], span_of(r))) return TRI_INV_ERR_INVALID_ARG;
  }
  HeadsArgs a{};
  a.side[0].x = Q; a.side[0].w = wq; a.side[0].dy = dYq; a.side[0].dx = dQ; a.side[0].dw = dwq;
  a.side[0].ld_x = ldq; a.side[0].ld_dy = lddyq; a.side[0].ld_dx = lddq; a.side[0].H = desc->H_q;
  a.side[1].x = K; a.side[1].w = wk; a.side[1].dy = dYk; a.side[1].dx = dK; a.side[1].dw = dwk;
  a.side[1].ld_x = ldk; a.side[1].ld_dy = lddyk; a.side[1].ld_dx = lddk; a.side[1].H = desc->H_k;
  a.partial = (float*)workspace;
  a.inv_freq = inv_freq; a.positions = positions; a.tokens = desc->tokens; a.T = desc->T; a.d = desc->d; a.r = desc->r; a.interleaved = desc->interleaved; a.eps = desc->eps;
  return launch_qk_norm_rope_backward(a, desc->dtype, (cudaStream_t)cuda_stream) == cudaSuccess ? TRI_INV_OK : TRI_INV_ERR_CUDA;
}

}  // extern "C"
