// Linear attention with a decay for each head: what its files share.
//
// Per sequence and head, lambda = exp(log_decay[h]):   S_t = lambda S_{t-1} + k_t v_t^T,   o_t = scale S_t^T q_t.
//
// One WALK is the chunk form of that recurrence over tiles of tokens.  With p the position of a token in the walk (0 .. n-1 inside a tile
// of n), S the state that enters the tile and b = 1 when walking backwards (else 0):
//     out_p = out_factor (sum over p' <= p of lambda^(p - p') k_factor (q_p . k_p') v_p'  +  lambda^(p + 1 - b) S^T q_p)
//     S    <- lambda^n S + sum over p of lambda^(n - 1 - p + b) k_factor k_p v_p^T
// The prompt is one walk.  Its gradient is three, since the same weights lambda^(i - j) (j <= i) join the other operands:
//     dQ = walk(dO, V, K) from S0^T;   dK = walk backwards(V, dO, Q) from dS^T;   dV = walk backwards(K, Q, dO) from dS,
// and the state that the last one leaves is the gradient of S0.  (Forwards the scale is the out_factor, backwards the k_factor: the state
// is then the gradient of S itself.)
//
// A long sequence of few heads is cut into SEGMENTS of whole tiles, walked side by side: first the state that each segment alone
// leaves (state_only), then those are joined in order (join), then every segment is walked from the state that enters it.
#pragma once
#include "common.cuh"

namespace tri_inv {

constexpr int kLinTile = 64;       // tokens of a tile
constexpr int kLinMaxWalks = 3;

struct LinWalk {
  const void* q;        // [tokens, H, d_k]
  const void* k;        // [tokens, H, d_k]
  const void* v;        // [tokens, H, d_v]
  void* out;            // [tokens, H, d_v]
  const float* s_in;    // [n_seqs, H, d_k, d_v] (s_turned: [.., d_v, d_k]) or null: zero
  float* s_out;         // [n_seqs, H, d_k, d_v] or null
  int d_k, d_v;
  int back;
  int s_turned;
  float k_factor, out_factor;
};

// Tokens [tok0, tok0 + n) of sequence seq; n = 0: an empty sequence, whose state only passes through.
struct LinSeg {
  int32_t tok0, n, seq, ends;   // ends: bit 0 first segment of its sequence, bit 1 last
};

struct LinArgs {
  LinWalk walk[kLinMaxWalks];
  int n_walks;
  const float* log_decay;     // [H] device
  const LinSeg* table;        // packed sequences; null: dense
  const int32_t* first;       // with it: each sequence's first segment, in the table's order
  int n_seqs;
  int H, T;                   // T: dense tokens a sequence
  int seg_tokens, segs_per_seq;   // dense: segments of a sequence
  int n_segs;                 // in all
  int slices;                 // tensor cores: 2 where a walk's 128 value columns go as two blocks
  float* seg_state;           // [n_walks][n_segs][H][d_k d_v]: the states that enter the segments; null: no sequence is cut
  int state_only;             // write to seg_state what each segment alone leaves
  int* status;
  unsigned long long wait_limit_ns;
  int test_stall;
};

// How a call is cut.
struct LinPlan {
  int seg_tokens, segs_per_seq, n_segs, slices;
  bool cut;                   // some sequence has more than one segment
  size_t table_bytes, state_bytes;
};

__device__ __forceinline__ LinSeg lin_segment(const LinArgs& a, int s) {
  if (a.table) return a.table[s];
  const int seq = s / a.segs_per_seq, i = s - seq * a.segs_per_seq;
  const int at = i * a.seg_tokens, left = a.T - at;
  return LinSeg{seq * a.T + at, left < a.seg_tokens ? left : a.seg_tokens, seq, (i == 0 ? 1 : 0) | (i == a.segs_per_seq - 1 ? 2 : 0)};
}

// The head's log-decay in units of log 2.  One below -1e4 counts as that: 2^(n x) is then 0 for n > 0 and 1 for n = 0, -inf included.
__device__ __forceinline__ float lin_log2_decay(const LinArgs& a, int h) {
  const float x = a.log_decay[h];
  return 1.4426950408889634f * (x < -1e4f ? -1e4f : x);
}

// lambda^n = keep + less for S <- (keep S + less S) + the increment.  Near 1 as 1 + (lambda^n - 1): a factor that is off by a rounding would be off by it in every tile, always to the same side.
// Where it is at most a half, by itself: lambda^n - 1 rounded is off by up to 2^-25, which against a small lambda^n is not small.
struct LinFade { float keep, less; };
__device__ __forceinline__ LinFade lin_fade(float log2_decay, int n) {
  const float x = log2_decay * n;
  return x > -1.f ? LinFade{1.f, expm1f(x * 0.6931471805599453f)} : LinFade{0.f, exp2f(x)};
}

// The state that enters a segment: null stands for zero; *turned: it lies [d_v][d_k].  In a cut sequence the first segment's comes from seg_state
// as well: s_in is then read before any s_out is written, and the two may be one buffer.
__device__ __forceinline__ const float* lin_entry_state(const LinArgs& a, const LinWalk& w, int walk, int s, const LinSeg& g, int h, bool* turned) {
  const size_t size = (size_t)w.d_k * w.d_v;
  *turned = false;
  if (a.state_only) return nullptr;
  if (a.seg_state && g.ends != 3) return a.seg_state + (((size_t)walk * a.n_segs + s) * a.H + h) * size;
  *turned = w.s_turned;
  return w.s_in ? w.s_in + ((size_t)g.seq * a.H + h) * size : nullptr;
}
// Where the state that a segment leaves goes, or null.
__device__ __forceinline__ float* lin_exit_state(const LinArgs& a, const LinWalk& w, int walk, int s, const LinSeg& g, int h) {
  const size_t size = (size_t)w.d_k * w.d_v;
  const bool last = g.ends & (w.back ? 1 : 2);
  if (a.state_only) return last ? nullptr : a.seg_state + (((size_t)walk * a.n_segs + s) * a.H + h) * size;   // nothing reads the last one's
  return last && w.s_out ? w.s_out + ((size_t)g.seq * a.H + h) * size : nullptr;
}

// Every shape and both storage types, in fp32 on the CUDA cores (d_k and d_v multiples of 8, d_k <= 256).
cudaError_t launch_linear_simt(const LinArgs& a, int kv_dtype, cudaStream_t stream);
// bf16 with head dimensions up to 128, on the tensor cores.
bool linear_tc_fits(int d_k, int d_v, int kv_dtype);
cudaError_t launch_linear_tc(const LinArgs& a, long long tokens, cudaStream_t stream);
// Between the two passes of a call with cut sequences: seg_state[s] from what segment s alone leaves to what enters it.
cudaError_t launch_linear_join(const LinArgs& a, cudaStream_t stream);
// The table of packed sequences, the longest first, from the host offsets of d.
cudaError_t launch_linear_table(LinSeg* dev_tab, int32_t* dev_first, int seg_tokens, const tri_inv_desc* d, cudaStream_t stream);
// One step on states in slots (linear_step_kernel.cu).
struct LinStepArgs {
  const void *q, *k, *v;
  const float* log_decay;
  float* S;                // [n_slots, H, d_k, d_v]
  const int32_t* slots;    // [B] or null: row b has slot b
  void* o;
  int B, H, d_k, d_v, n_slots, bf16;
  float scale;
  int* status;
};
cudaError_t launch_linear_step(const LinStepArgs& a, cudaStream_t stream);

}  // namespace tri_inv
