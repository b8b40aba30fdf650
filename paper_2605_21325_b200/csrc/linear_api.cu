// extern "C" boundary of linear attention and of the RMS norm: argument checks, the cut into segments, dispatch.
#include <algorithm>
#include <cmath>

#include "call_checks.cuh"
#include "linear_attention.cuh"
#include "rms_norm.cuh"

namespace tri_inv {
namespace {

long long tokens_of(const tri_inv_desc* d) { return d->cu_seqlens ? (long long)d->T : (long long)d->T * d->B; }
// whether the tensor-core kernel takes the call (without a token there is nothing for it to map)
bool on_tensor_cores(const tri_inv_desc* d) { return tokens_of(d) > 0 && linear_tc_fits(d->d_k, d->d_v, d->kv_dtype); }
// the bytes of a tensor of `d` features for each token and head, and of the states
__int128 token_bytes(const tri_inv_desc* d, int features) { return (__int128)tokens_of(d) * d->H * features * (d->kv_dtype == TRI_INV_F32 ? 4 : 2); }
__int128 state_bytes(const tri_inv_desc* d) { return (__int128)(d->cu_seqlens ? d->n_seqs : d->B) * d->H * d->d_k * d->d_v * 4; }
size_t round_up(size_t n) { return (n + 255) & ~(size_t)255; }

// desc->C plays no part: the tiles are the kernels' own.
int check_linear(const tri_inv_desc* d) {
  if (!d) return TRI_INV_ERR_INVALID_ARG;
  tri_inv_desc x = *d;
  x.C = 64;
  const int rc = check_desc(&x, true);
  if (rc) return rc;
  return d->d_k > 256 || d->d_v > 65536 ? TRI_INV_ERR_UNSUPPORTED : TRI_INV_OK;
}

// Times of the tensor-core kernel in units of 1.25 us: a tile (64 tokens, d_k = d_v = 128) of all value columns and of 64, the same of the pass that only wants states, what the
// memory traffic takes for a tile with a block on every SM (less for a gradient's three walks, which read the same tensors), a block's start and end in tiles, a kernel's launch, a
// cut's second launch and join, and a segment's state written, joined and read.  Measured, us, estimate / calls in a captured graph on a rested GPU: 1 x 4096 tokens x 16 heads uncut
// 89 / 85, in halves of the columns 69 / 70, also in four segments 52 / 47, eight of all columns 52 / 45; 1 x 32768 x 8 uncut 649 / 632, 18 segments 102 / 97; 1 x 32768 x 32 in
// halves 494 / 511, four segments 304 / 289, nine 320 / 301; 4 x 4096 x 16 in halves 69 / 76, all columns 89 / 88, two segments 102 / 101; its gradient 173 / 179, in halves 196 / 223;
// the gradient of 1 x 4096 x 16 in halves 69 / 73, uncut 89 / 87, three segments 78 / 78.
constexpr double kTileAll = 1.0, kTileHalf = 0.76, kStateAll = 0.56, kStateHalf = 0.45, kBusyTile = 1.3, kBusyState = 0.65, kShared = 0.75, kBlock = 3.0, kLaunch = 4.0,
                 kCut = 11.0, kSegment = 0.06;

// Cost of a pass over `tiles` tiles in all, in segments of `seg` with `units` blocks a tile: whole rounds of blocks on all SMs and one on what is left, a tile taking `alone`
// where its SM bounds it and `busy` times the share of SMs at work where the memory does.  (Packed segments, the longest first, end about together.)
double pass_cost(double tiles, double seg, double units, bool equal, int sms, double alone, double busy) {
  const double rounds = tiles / seg * units / sms, full = std::floor(rounds), rest = rounds - full;
  const double last = rest <= 0 ? 0 : equal || full == 0 ? std::max(alone, busy * rest) : std::max(alone, busy) * rest;
  return (seg + kBlock) * (full * std::max(alone, busy) + last);
}

// How a call of `walks` walks is cut.  A cut sequence is read twice where it is not the last segment (k and v, for the states), and joining takes two
// launches more, so it pays only where the walk of the longest sequence is long beside what the chip could do with every SM at work.
int plan(const tri_inv_desc* d, int walks, bool tc, LinPlan* p) {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return TRI_INV_ERR_CUDA;
  const int n_seqs = d->cu_seqlens ? d->n_seqs : d->B;
  auto len = [&](int s) -> long long { return d->cu_seqlens ? d->cu_seqlens[s + 1] - d->cu_seqlens[s] : d->T; };   // rounded up to tiles it may pass 2^31 - 1
  long long tiles = 0, longest = 0;
  if (d->cu_seqlens) {
    for (int s = 0; s < n_seqs; ++s) {
      const long long t = (len(s) + kLinTile - 1) / kLinTile;
      tiles += t;
      longest = std::max(longest, t);
    }
  } else {
    longest = ((long long)d->T + kLinTile - 1) / kLinTile;
    tiles = longest * n_seqs;
  }
  long long seg = std::max<long long>(longest, 1);
  p->slices = 1;
  if (tc) {
    const bool wide = std::max(d->d_k, d->d_v) > 64;
    const double shared = walks == 3 ? kShared : 1.0;
    double best = 1e300;
    for (int slices = wide ? 2 : 1; slices >= 1; --slices) {
      const bool half = !wide || slices == 2;
      const double units = (double)d->H * walks * slices;
      for (int n = 1; n <= 64 && (n == 1 || longest >= 4 * n); ++n) {
        const long long s = std::max<long long>(1, (longest + n - 1) / n);
        const bool equal = !d->cu_seqlens;
        // (halves of the columns read q and k twice, from the L2 cache the second time)
        double cost = kLaunch + pass_cost((double)tiles, (double)s, units, equal, sms, half ? kTileHalf : kTileAll, shared * kBusyTile / slices);
        if (n > 1)
          cost += kCut + kSegment * tiles / s * d->H * walks +
                  pass_cost((double)tiles * (n - 1) / n, (double)s, units, equal, sms, half ? kStateHalf : kStateAll, shared * kBusyState / slices);
        if (cost < best) { best = cost; seg = s; p->slices = slices; }
      }
    }
  } else {
    // The CUDA-core kernel, in us, by the key dimension: a tile of a block that has its SM to itself, of one of two or three that share it, the same of the pass that only wants states (one
    // product of four; a cut sequence's last tiles need no increment, which is another), a block's start, and what a cut costs: two launches, and each state written, joined and read.
    // Measured, fp32, estimate / calls in a captured graph: 16 x 64 tokens x 8 heads of 128 uncut 43 / 30; 8 x 512 x 8 of 128 uncut 206 / 167, in tiles 211 / 198, its gradient uncut 468 / 394, in
    // pairs of tiles 532 / 495; 1 x 4096 x 8 of 128 in tiles 211 / 186, in fours 232 / 202; 2 x 2048 x 8 of 64 in tiles 77 / 66, its gradient 162 / 154; gradients of packed sequences: five of up
    // to 1000 x 4 heads of 64 in tiles 55 / 50, twelve of up to 600 x 8 of 128 uncut 388 / 412, in tiles 620 / 520.
    const int slices_v = (d->d_v + 63) / 64, d_most = walks == 3 ? std::max(d->d_k, d->d_v) : d->d_k;
    const double per_tile = (double)d->H * (walks == 3 ? 2 * ((d->d_k + 63) / 64) + slices_v : slices_v), slots = (d_most > 128 ? 1.0 : d_most > 64 ? 2.0 : 3.0) * sms;
    const double alone = 2.5 + 0.175 * d_most, state_alone = std::max(3.0, 0.11 * d_most - 2.0), start = 3.0;
    const double many = d_most > 128 ? 1.0 : d_most > 64 ? 1.3 : 1.85;   // a tile in full rounds of two or three blocks an SM; in a last round by the number there
    auto pass = [&](double tiles_in_all, double s, double a_tile) {
      const double blocks = std::max(1.0, tiles_in_all / s * per_tile), full = std::floor(blocks / slots), rest = blocks - full * slots;
      auto shared = [&](double n) { return n > 2.0 * sms ? 1.9 : n > sms ? 1.45 : n > 0 ? 1.0 : 0.0; };
      // (packed: the longest first, so that the short ones fill what the last round would leave)
      const double rounds = d->cu_seqlens ? std::max(shared(std::min(blocks, slots)), blocks / slots * many) : full * many + shared(rest);
      return s * a_tile * rounds + start * (full + 1);
    };
    double best = 1e300;
    for (int n = 1; n <= 256 && n <= std::max<long long>(longest, 1); ++n) {
      const long long s = std::max<long long>(1, (longest + n - 1) / n);
      double cost = kLaunch + pass((double)tiles, (double)s, alone * (n > 1 ? 1.0 - 0.25 / s : 1.0));
      if (n > 1) cost += 12.0 + pass((double)tiles * (n - 1) / n, (double)s, state_alone) + 2.4e-6 * tiles / s * d->H * walks * d->d_k * d->d_v;
      if (cost < best) { best = cost; seg = s; }
    }
  }
  p->seg_tokens = (int)std::min<long long>(seg * kLinTile, 0x40000000);
  long long n = 0;
  if (d->cu_seqlens) {
    for (int s = 0; s < n_seqs; ++s) n += std::max<long long>(1, (len(s) + p->seg_tokens - 1) / p->seg_tokens);
    p->segs_per_seq = 0;
  } else {
    p->segs_per_seq = (int)std::max<long long>(1, ((long long)d->T + p->seg_tokens - 1) / p->seg_tokens);
    n = (long long)p->segs_per_seq * n_seqs;
  }
  if (n * d->H * walks * ((std::max(d->d_k, d->d_v) + 63) / 64) > 0x40000000LL) return TRI_INV_ERR_INVALID_ARG;   // blocks are counted in 32 bits, and by whole rounds of them
  p->n_segs = (int)n;
  p->cut = longest * kLinTile > p->seg_tokens;
  p->table_bytes = d->cu_seqlens ? round_up((size_t)n * sizeof(LinSeg) + (size_t)n_seqs * sizeof(int32_t)) : 0;
  p->state_bytes = p->cut ? round_up((size_t)walks * n * d->H * d->d_k * d->d_v * sizeof(float)) : 0;
  return TRI_INV_OK;
}

int run_walks(LinArgs& a, const LinPlan& p, const tri_inv_desc* d, bool tc, void* workspace, cudaStream_t stream) {
  cudaError_t err;
  a.status = status_word_for_current_device(&err);
  if (!a.status) return TRI_INV_ERR_CUDA;
  a.H = d->H; a.T = d->T; a.n_seqs = d->cu_seqlens ? d->n_seqs : d->B;
  a.seg_tokens = p.seg_tokens; a.segs_per_seq = p.segs_per_seq; a.n_segs = p.n_segs; a.slices = p.slices;
  if (p.n_segs == 0) return TRI_INV_OK;
  if (d->cu_seqlens) {
    a.table = (const LinSeg*)workspace;
    a.first = (const int32_t*)(a.table + p.n_segs);
    if (launch_linear_table((LinSeg*)workspace, (int32_t*)((LinSeg*)workspace + p.n_segs), p.seg_tokens, d, stream) != cudaSuccess) return TRI_INV_ERR_CUDA;
  }
  auto walk = [&]() { return tc ? launch_linear_tc(a, tokens_of(d), stream) : launch_linear_simt(a, d->kv_dtype, stream); };
  if (p.cut) {
    a.seg_state = (float*)((char*)workspace + p.table_bytes);
    a.state_only = 1;
    if (walk() != cudaSuccess || launch_linear_join(a, stream) != cudaSuccess) return TRI_INV_ERR_CUDA;
    a.state_only = 0;
  }
  return walk() == cudaSuccess ? TRI_INV_OK : TRI_INV_ERR_CUDA;
}

int workspace_of(const tri_inv_desc* d, int walks, size_t* bytes) {
  const int rc = check_linear(d);
  if (rc) return rc;
  if (!bytes) return TRI_INV_ERR_INVALID_ARG;
  LinPlan p;
  const int e = plan(d, walks, on_tensor_cores(d), &p);
  if (e) return e;
  *bytes = p.table_bytes + p.state_bytes;
  return TRI_INV_OK;
}

LinWalk make_walk(const void* q, const void* k, const void* v, void* out, const float* s_in, float* s_out, int d_k, int d_v, int back, int turned, float scale) {
  return LinWalk{q, k, v, out, s_in, s_out, d_k, d_v, back, turned, back ? scale : 1.f, back ? 1.f : scale};
}

int check_norm(int64_t rows, int32_t n, float eps, int dtype) {
  if (rows < 0 || rows > 0x7fffffffLL || n < 1 || !(eps >= 0.f) || std::isinf(eps)) return TRI_INV_ERR_INVALID_ARG;
  if (dtype != TRI_INV_F32 && dtype != TRI_INV_BF16) return TRI_INV_ERR_INVALID_ARG;
  return n > 0x7fffff00 ? TRI_INV_ERR_UNSUPPORTED : TRI_INV_OK;   // columns are counted in 32 bits, and by 256 past the last
}
}  // namespace
}  // namespace tri_inv

using namespace tri_inv;

extern "C" {

int tri_inv_linear_attention_workspace(const tri_inv_desc* desc, size_t* bytes) { return workspace_of(desc, 1, bytes); }

int tri_inv_linear_attention(const void* Q, const void* K, const void* V, const float* log_decay, const float* S0, void* O, float* S_out,
                             float scale, void* workspace, size_t workspace_bytes, const tri_inv_desc* desc, void* cuda_stream) {
  const int rc = check_linear(desc);
  if (rc) return rc;
  if (!log_decay || (tokens_of(desc) > 0 && (!Q || !K || !V || !O)) || !all_aligned(Q, K, V, log_decay, S0, O, S_out, workspace)) return TRI_INV_ERR_INVALID_ARG;
  const __int128 qk = token_bytes(desc, desc->d_k), vo = token_bytes(desc, desc->d_v), state = state_bytes(desc);
  const Span q{Q, qk}, k{K, qk}, v{V, vo}, decay{log_decay, 4ll * desc->H}, s0{S0, state}, o{O, vo}, s_out{S_out, state};
  if (meets_any(o, q, k, v, decay, s0, s_out) || meets_any(s_out, q, k, v, decay) || (S_out != S0 && meets(s_out, s0))) return TRI_INV_ERR_INVALID_ARG;
  const bool tc = on_tensor_cores(desc);
  LinPlan p;
  const int e = plan(desc, 1, tc, &p);
  if (e) return e;
  if (workspace_bytes < p.table_bytes + p.state_bytes || (p.table_bytes + p.state_bytes > 0 && !workspace)) return TRI_INV_ERR_INVALID_ARG;
  LinArgs a{};
  a.log_decay = log_decay;
  a.n_walks = 1;
  a.walk[0] = make_walk(Q, K, V, O, S0, S_out, desc->d_k, desc->d_v, 0, 0, scale);
  return run_walks(a, p, desc, tc, workspace, (cudaStream_t)cuda_stream);
}

int tri_inv_selftest_linear_wait_timeout(const void* Q, const void* K, const void* V, const float* log_decay, void* O, const tri_inv_desc* desc,
                                         uint64_t wait_limit_ns, void* cuda_stream) {
  const int rc = check_linear(desc);
  if (rc) return rc;
  if (!on_tensor_cores(desc) || desc->cu_seqlens || desc->T > 0x40000000) return TRI_INV_ERR_UNSUPPORTED;   // (longer sequences are always cut)
  if (!Q || !K || !V || !log_decay || !O || !wait_limit_ns || !all_aligned(Q, K, V, log_decay, O)) return TRI_INV_ERR_INVALID_ARG;
  const LinPlan p{(desc->T + kLinTile - 1) / kLinTile * kLinTile, 1, desc->B, 1, false, 0, 0};
  LinArgs a{};
  a.log_decay = log_decay;
  a.n_walks = 1;
  a.walk[0] = make_walk(Q, K, V, O, nullptr, nullptr, desc->d_k, desc->d_v, 0, 0, 1.f);
  a.wait_limit_ns = wait_limit_ns;
  a.test_stall = 1;
  const int e = run_walks(a, p, desc, true, nullptr, (cudaStream_t)cuda_stream);
  if (e) return e;
  return cudaStreamSynchronize((cudaStream_t)cuda_stream) == cudaSuccess ? TRI_INV_OK : TRI_INV_ERR_CUDA;
}

int tri_inv_linear_attention_backward_workspace(const tri_inv_desc* desc, size_t* bytes) {
  if (desc && desc->d_v > 256) return TRI_INV_ERR_UNSUPPORTED;
  return workspace_of(desc, 3, bytes);
}

int tri_inv_linear_attention_backward(const void* dO, const void* Q, const void* K, const void* V, const float* log_decay, const float* S0, const float* dS,
                                      void* dQ, void* dK, void* dV, float* dS0, float scale, void* workspace, size_t workspace_bytes,
                                      const tri_inv_desc* desc, void* cuda_stream) {
  const int rc = check_linear(desc);
  if (rc) return rc;
  if (desc->d_v > 256) return TRI_INV_ERR_UNSUPPORTED;   // two of the three walks have the value dimension as their key dimension
  if (!log_decay || (tokens_of(desc) > 0 && (!dO || !Q || !K || !V || !dQ || !dK || !dV)) ||
      !all_aligned(dO, Q, K, V, log_decay, S0, dS, dQ, dK, dV, dS0, workspace))
    return TRI_INV_ERR_INVALID_ARG;
  // the walks run side by side: what one writes another may still have to read
  const __int128 qk = token_bytes(desc, desc->d_k), vo = token_bytes(desc, desc->d_v), state = state_bytes(desc);
  const Span out[4] = {{dQ, qk}, {dK, qk}, {dV, vo}, {dS0, state}};
  for (int i = 0; i < 4; ++i) {
    if (meets_any(out[i], Span{dO, vo}, Span{Q, qk}, Span{K, qk}, Span{V, vo}, Span{log_decay, 4ll * desc->H}, Span{S0, state}, Span{dS, state})) return TRI_INV_ERR_INVALID_ARG;
    for (int j = 0; j < i; ++j)
      if (meets(out[i], out[j])) return TRI_INV_ERR_INVALID_ARG;
  }
  const bool tc = on_tensor_cores(desc);
  LinPlan p;
  const int e = plan(desc, 3, tc, &p);
  if (e) return e;
  if (workspace_bytes < p.table_bytes + p.state_bytes || (p.table_bytes + p.state_bytes > 0 && !workspace)) return TRI_INV_ERR_INVALID_ARG;
  LinArgs a{};
  a.log_decay = log_decay;
  a.n_walks = 3;
  a.walk[0] = make_walk(dO, V, K, dQ, S0, nullptr, desc->d_v, desc->d_k, 0, 1, scale);
  a.walk[1] = make_walk(V, dO, Q, dK, dS, nullptr, desc->d_v, desc->d_k, 1, 1, scale);
  a.walk[2] = make_walk(K, Q, dO, dV, dS, dS0, desc->d_k, desc->d_v, 1, 0, scale);
  return run_walks(a, p, desc, tc, workspace, (cudaStream_t)cuda_stream);
}

int tri_inv_linear_attention_step(const void* Q, const void* K, const void* V, const float* log_decay, float* S, const int32_t* slots, int32_t n_slots,
                                  void* O, float scale, const tri_inv_desc* desc, void* cuda_stream) {
  const int rc = check_linear(desc);
  if (rc) return rc;
  if (desc->cu_seqlens || desc->T != 1 || n_slots < 0) return TRI_INV_ERR_INVALID_ARG;
  if (!slots && n_slots < desc->B) return TRI_INV_ERR_INVALID_ARG;
  if (!Q || !K || !V || !log_decay || !S || !O || !all_aligned(Q, K, V, log_decay, S, O) || (reinterpret_cast<uintptr_t>(slots) & 3u)) return TRI_INV_ERR_INVALID_ARG;
  if ((long long)desc->B * desc->H * ((desc->d_v + 31) / 32) > 0x7fffffffLL) return TRI_INV_ERR_INVALID_ARG;
  // blocks of one row and head read all of q and k while others write their part of the state and of o; of v a block reads what its o takes
  const __int128 qk = token_bytes(desc, desc->d_k), vo = token_bytes(desc, desc->d_v);
  const Span q{Q, qk}, k{K, qk}, v{V, vo}, decay{log_decay, 4ll * desc->H}, states{S, (__int128)n_slots * desc->H * desc->d_k * desc->d_v * 4}, rows{slots, 4ll * desc->B}, o{O, vo};
  if (meets_any(states, q, k, v, decay, rows, o) || meets_any(o, q, k, decay, rows) || (O != V && meets(o, v))) return TRI_INV_ERR_INVALID_ARG;
  LinStepArgs a{Q, K, V, log_decay, S, slots, O, desc->B, desc->H, desc->d_k, desc->d_v, n_slots, desc->kv_dtype == TRI_INV_BF16, scale, nullptr};
  cudaError_t err;
  a.status = status_word_for_current_device(&err);
  if (!a.status) return TRI_INV_ERR_CUDA;
  return launch_linear_step(a, (cudaStream_t)cuda_stream) == cudaSuccess ? TRI_INV_OK : TRI_INV_ERR_CUDA;
}

int tri_inv_rms_norm(const void* X, const void* R, const void* w, void* Y, void* H, float* scales, int64_t rows, int32_t n, int32_t group, float eps,
                     int dtype, int out_dtype, void* cuda_stream) {
  const int rc = check_norm(rows, n, eps, dtype);
  if (rc) return rc;
  if (out_dtype != dtype && out_dtype != TRI_INV_E4M3) return TRI_INV_ERR_INVALID_ARG;
  const bool coded = out_dtype == TRI_INV_E4M3;
  if (coded && group != 0 && group != 128) return TRI_INV_ERR_UNSUPPORTED;
  if (rows == 0) return TRI_INV_OK;
  if (!X || !w || !Y || (coded && !scales) || !on_type(dtype, X, R, w, H) || (!coded && !on_type(dtype, Y)) || (reinterpret_cast<uintptr_t>(scales) & 3u))
    return TRI_INV_ERR_INVALID_ARG;
  RmsNormArgs a{X, R, w, Y, H, scales, rows, n, eps};
  return launch_rms_norm(a, dtype, !coded ? 0 : group == 128 ? 1 : 2, (cudaStream_t)cuda_stream) == cudaSuccess ? TRI_INV_OK : TRI_INV_ERR_CUDA;
}

int tri_inv_rms_norm_backward_workspace(int64_t rows, int32_t n, size_t* bytes) {
  const int rc = check_norm(rows, n, 0.f, TRI_INV_F32);
  if (rc) return rc;
  if (!bytes) return TRI_INV_ERR_INVALID_ARG;
  *bytes = (size_t)kRmsNormPartials * n * sizeof(float);
  return TRI_INV_OK;
}

int tri_inv_rms_norm_backward(const void* dY, const void* X, const void* w, const void* dH, void* dX, void* dw, int64_t rows, int32_t n, float eps, int dtype,
                              void* workspace, size_t workspace_bytes, void* cuda_stream) {
  const int rc = check_norm(rows, n, eps, dtype);
  if (rc) return rc;
  if (!w || !dw || !workspace || !aligned16(workspace) || workspace_bytes < (size_t)kRmsNormPartials * n * sizeof(float)) return TRI_INV_ERR_INVALID_ARG;
  if (rows > 0 && (!dY || !X || !dX)) return TRI_INV_ERR_INVALID_ARG;
  if (!on_type(dtype, dY, X, w, dH, dX, dw)) return TRI_INV_ERR_INVALID_ARG;
  RmsNormBackwardArgs a{dY, X, w, dH, dX, dw, (float*)workspace, rows, n, eps};
  return launch_rms_norm_backward(a, dtype, (cudaStream_t)cuda_stream) == cudaSuccess ? TRI_INV_OK : TRI_INV_ERR_CUDA;
}

}  // extern "C"
