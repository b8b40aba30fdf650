"""Linear attention with a decay for each head (prompt, single token, gradient) and the RMS norm around it (forward, gradient).

``listed()`` names the cases, ``draw(rng)`` gives further ones of the same ranges, ``prepare`` makes what a program holds before the
call, ``run`` is one pass: with ``own`` the calls of ``paper_2605_21325_b200.binding``, without it the plain form in elementary torch
operations.  ``exact`` is the definition in 64 bits: the recurrence token by token.

With lambda_h = exp(log_decay_h), per sequence and head:
  prompt  S_t = lambda S_{t-1} + k_t v_t^T,  o_t = scale S_t^T q_t                            -> O, the state behind the last token
  token   one step of it on states that lie in slots of a cache, updated in place; slot < 0: a padded row, output zero -> O, S
  grad    the gradients of Q, K, V and of a carried-in state from those of O and of the final state
  norm    H = X + R (stored rounded), Y = H / sqrt(mean H^2 + eps) * w; Y in the type of X, or in 8 bits (e4m3) with a scale for each
          group of columns: scale = max |y| / 448 (1 where that is zero), Y = y / scale          -> Y, H, scales
  normgrad  the gradients of H (with what reaches H past the norm added) and of w
"""
import math
import random

import torch

own = False

_SIZES = {"float32": 4, "bfloat16": 2}
_EPS = 1e-6


def _attn(name, op, B, T, H, dk=128, dv=128, dtype="bfloat16", seqs=0, state=False):
    """``seqs`` > 0: that many packed sequences of lengths uniform in 1..T (B is 1 then); ``state``: states carried in (and, for the
    gradient, a gradient of the final state carried in)."""
    c = {"op": op, "B": B, "T": T, "H": H, "dk": dk, "dv": dv, "dtype": dtype, "seqs": seqs, "state": state}
    if name:
        c["name"] = name
    return c


def _step(name, B, H, dk=128, dv=128, dtype="bfloat16", pad=0):
    """``pad``: padded rows among the B."""
    c = {"op": "token", "B": B, "H": H, "dk": dk, "dv": dv, "dtype": dtype, "pad": pad}
    if name:
        c["name"] = name
    return c


def _norm(name, op, rows, n, dtype="bfloat16", residual=True, out="same", group=128):
    c = {"op": op, "rows": rows, "n": n, "dtype": dtype, "residual": residual, "out": out, "group": group}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one short prompt of no round length: launches and latency
        _attn("attention_short", "prompt", 1, 333, 16),
        # a prefill batch of a layer of 16 heads, continuing carried states
        _attn("attention_prefill", "prompt", 4, 4096, 16, state=True),
        # one long document through a layer of 32 heads: far fewer heads than SMs, a long way to walk
        _attn("attention_long", "prompt", 1, 32768, 32),
        # a batch of prompts of mixed lengths, packed: partial last tiles
        _attn("attention_packed", "prompt", 1, 2048, 16, seqs=64),
        # one new token for each of eight sequences: the smallest call of a serving loop
        _step("token_small", 8, 16),
        # a full serving batch on a cache of states, some rows of it padding
        _step("token_batch", 256, 32, pad=9),
        # the training step of a layer on its prefill shape
        _attn("gradient_prefill", "grad", 4, 4096, 16),
        # the gradient in single precision on a few packed sequences, as it is run for checking and in small models
        _attn("gradient_fp32", "grad", 1, 1000, 4, dk=64, dv=64, dtype="float32", seqs=5, state=True),
        # the norm in front of a layer's projections while tokens are generated: eight rows, residual added
        _norm("norm_token", "norm", 8, 2048),
        # the same over a prefill batch, its output in 8 bits for the projections
        _norm("norm_prefill_e4m3", "norm", 16384, 4096, out="e4m3"),
        # its gradient in training, with what reaches the residual stream past the norm
        _norm("normgrad_prefill", "normgrad", 16384, 2048),
        # the gradient of the norm of each head's output: many short rows, single precision
        _norm("normgrad_heads_fp32", "normgrad", 40000, 128, dtype="float32", residual=False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["prompt", "prompt", "prompt", "token", "token", "grad", "grad", "norm", "norm", "normgrad", "normgrad"])
    dtype = "float32" if rng.random() < 0.3 else "bfloat16"
    if op in ("norm", "normgrad"):
        n = rng.choice([128, 1024, 2048, 2560, 4096, 5120, 7168, 8192]) if rng.random() < 0.6 else _log_int(rng, 64, 8192)
        rows = _log_int(rng, 1, min(65536, (1 << 26) // n))
        if op == "normgrad":
            return _norm(None, op, rows, n, dtype, rng.random() < 0.5)
        return _norm(None, op, rows, n, dtype, rng.random() < 0.7, rng.choice(["same", "e4m3"]), rng.choice([128, 128, 0]))
    H = rng.choice([2, 3, 4, 6, 8, 12, 16, 20, 24, 32])
    dk, dv = rng.choice([(128, 128), (128, 128), (128, 128), (64, 64), (64, 64), (128, 64), (64, 128), (96, 96), (80, 120)])
    if op == "token":
        B = _log_int(rng, 1, 256)
        return _step(None, B, H, dk, dv, dtype, rng.randint(0, B // 4))
    odd = (dk, dv) in ((96, 96), (80, 120))
    most = 1 << (15 if odd or dtype == "float32" else 20 if op == "prompt" else 18)      # (token, head) rows in all
    tokens = max(1, _log_int(rng, 64, most) // H)
    longest = 32768 if op == "prompt" else 8192
    if rng.random() < 0.35 and tokens >= 64:                                              # packed: 2..64 sequences
        seqs = _log_int(rng, 2, min(64, tokens // 16))
        return _attn(None, op, 1, max(1, min(longest, 2 * tokens // seqs)), H, dk, dv, dtype, seqs, rng.random() < 0.5)
    B = _log_int(rng, 1, min(32, tokens))
    return _attn(None, op, B, max(1, min(longest, tokens // B)), H, dk, dv, dtype, 0, rng.random() < 0.5)


def _lengths(case):
    """Tokens of each sequence: a matter of the case, not of the seed."""
    if not case["seqs"]:
        return [case["T"]] * case["B"]
    r = random.Random(1005 * case["seqs"] + case["T"])
    return [r.randint(1, case["T"]) for _ in range(case["seqs"])]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(1000003 * (int(seed) % (1 << 40)) + 29)
    normal = lambda *s: torch.randn(*s, device="cuda", generator=gen)   # noqa: E731
    dt = getattr(torch, case["dtype"])
    s = dict(op=case["op"])
    if case["op"] in ("norm", "normgrad"):
        rows, n = case["rows"], case["n"]
        s.update(X=normal(rows, n).to(dt), w=(1 + 0.1 * normal(n)).to(dt), R=None, group=case["group"], out=case["out"])
        if case["op"] == "norm":
            if case["residual"]:
                s["R"] = (2 * normal(rows, n)).to(dt)
        else:
            s.update(dY=normal(rows, n).to(dt), dH=normal(rows, n).to(dt) if case["residual"] else None)
        return s
    H, dk, dv = case["H"], case["dk"], case["dv"]
    # heads forget at rates spread over powers of two, from half the state a token to a few thousandths
    s.update(log_decay=-(2.0 ** (-8.0 * torch.arange(1, H + 1, device="cuda") / H)), scale=dk ** -0.5)
    if case["op"] == "token":
        B, pad = case["B"], case["pad"]
        n_slots = B + 3
        slots = torch.randperm(n_slots, device="cuda", generator=gen)[:B].to(torch.int32)
        slots[torch.randperm(B, device="cuda", generator=gen)[:pad]] = -1
        s.update(Q=normal(B, H, dk).to(dt), K=normal(B, H, dk).to(dt), V=normal(B, H, dv).to(dt), slots=slots,
                 S=normal(n_slots, H, dk, dv) * 2)
        return s
    lens = _lengths(case)
    B, T = (1, sum(lens)) if case["seqs"] else (case["B"], case["T"])
    s.update(Q=normal(B, T, H, dk).to(dt), K=normal(B, T, H, dk).to(dt), V=normal(B, T, H, dv).to(dt), lens=lens, S0=None, dS=None,
             cu=[sum(lens[:i]) for i in range(len(lens) + 1)] if case["seqs"] else None)
    if case["state"]:
        s["S0"] = normal(len(lens), H, dk, dv) * 2
    if case["op"] == "grad":
        s["dO"] = normal(B, T, H, dv).to(dt)
        s["dS"] = normal(len(lens), H, dk, dv) if case["state"] else None
    return s


# ---- plain form

_L = 64    # tokens of a chunk


class _Chunks:
    """Flat tokens <-> chunks of ``_L`` tokens of each sequence; ``back``: every sequence is walked from its last token to its first."""

    def __init__(self, lens, back, device):
        ln = torch.tensor(lens, device=device)
        beg = ln.cumsum(0) - ln
        per = (ln + _L - 1) // _L
        n = sum((x + _L - 1) // _L for x in lens)
        self.seq = torch.repeat_interleave(torch.arange(len(lens), device=device), per, output_size=n)
        self.start = (torch.arange(n, device=device) - (per.cumsum(0) - per)[self.seq]) * _L        # position of the chunk's first token
        self.count = torch.minimum(ln[self.seq] - self.start, torch.full_like(self.start, _L))
        self.len = ln
        at = torch.arange(_L, device=device)
        self.real = at[None] < self.count[:, None]
        pos = (self.start[:, None] + at).minimum(ln[self.seq][:, None] - 1)
        self.index = beg[self.seq][:, None] + (ln[self.seq][:, None] - 1 - pos if back else pos)
        self.pos = pos

    def cut(self, x):                        # [B, T, H, d] -> [H, chunks, L, d] in 32 bits, zeros where there is no token
        y = x.reshape((-1,) + x.shape[2:])[self.index].float() * self.real[..., None, None]
        return y.permute(2, 0, 1, 3)

    def join(self, y, B, T):
        out = torch.empty((B * T, y.shape[0], y.shape[3]), dtype=y.dtype, device=y.device)
        out[self.index[self.real]] = y.permute(1, 2, 0, 3)[self.real]
        return out.reshape(B, T, y.shape[0], y.shape[3])


def _power(log_decay, n):                    # lambda_h^n for every n: [H, ...]
    return torch.exp(log_decay.double().reshape((-1,) + (1,) * n.dim()) * n).float()


def _linear(q, k, v, log_decay, lens, S0, factor, back=False):
    """out_p = sum over p' <= p of lambda^(p - p') factor (q_p . k_p') v_p' (+ factor lambda^(p+1) q_p S0), p counted from the walk's
    first token, and the state behind its last.  Backwards the carried-in state meets the walk's first token undecayed and unscaled, and
    the state that is left has passed the last one's decay: the gradient's recurrence."""
    B, T = q.shape[:2]
    ch = _Chunks(lens, back, q.device)
    qc, kc, vc = ch.cut(q), ch.cut(k), ch.cut(v)
    b = 1 if back else 0
    at = torch.arange(_L, device=q.device)
    gap = at[:, None] - at[None]
    D = torch.where(gap >= 0, _power(log_decay, gap.clamp(min=0)), 0.0)[:, None]
    out = ((qc @ kc.mT) * D) @ vc
    H, N, dk, dv = qc.shape[0], qc.shape[1], qc.shape[3], vc.shape[3]
    own_state = (kc * _power(log_decay, (ch.count[:, None] - 1 - at).clamp(min=0))[..., None]).mT @ vc       # [H, N, dk, dv]
    far = ch.start[:, None] - (ch.start + ch.count)[None]
    before = (ch.seq[:, None] == ch.seq[None]) & (far >= 0)
    S = torch.where(before, _power(log_decay, far.clamp(min=0)), 0.0) @ own_state.reshape(H, N, dk * dv)
    out = factor * (out + _power(log_decay, at + 1)[:, None, :, None] * (qc @ S.reshape(H, N, dk, dv)))
    first = torch.arange(len(lens), device=q.device)[:, None] == ch.seq[None]
    left = (ch.len[:, None] - (ch.start + ch.count)[None]).clamp(min=0)
    state = torch.where(first, _power(log_decay, left + b), 0.0) @ own_state.reshape(H, N, dk * dv)
    state = state.reshape(H, len(lens), dk, dv).transpose(0, 1) * (factor if back else 1.0)
    if S0 is not None:
        out = out + (1.0 if back else factor) * _power(log_decay, ch.pos + 1 - b)[..., None] * (qc @ S0.transpose(0, 1)[:, ch.seq])
        state = state + _power(log_decay, ch.len).T[..., None, None] * S0
    return ch.join(out.to(q.dtype), B, T), state.contiguous()


def _plain(s):
    op = s["op"]
    if op == "norm":
        h = s["X"].float() if s["R"] is None else s["X"].float() + s["R"].float()
        y = h * torch.rsqrt(h.square().mean(-1, keepdim=True) + _EPS) * s["w"].float()
        H = None if s["R"] is None else h.to(s["X"].dtype)
        if s["out"] == "same":
            return y.to(s["X"].dtype), H, None
        rows, n = y.shape
        group = s["group"] or n
        parts = -(-n // group)
        z = torch.nn.functional.pad(y, (0, parts * group - n)).reshape(rows, parts, group)
        scale = z.abs().amax(-1) / 448.0
        scale = torch.where(scale > 0, scale, 1.0)
        return (z / scale[..., None]).reshape(rows, -1)[:, :n].to(torch.float8_e4m3fn), H, scale
    if op == "normgrad":
        h, dy, w = s["X"].float(), s["dY"].float(), s["w"].float()
        r = torch.rsqrt(h.square().mean(-1, keepdim=True) + _EPS)
        u = dy * w
        dx = r * (u - h * (r * r * (u * h).mean(-1, keepdim=True)))
        if s["dH"] is not None:
            dx = dx + s["dH"].float()
        return dx.to(s["X"].dtype), (dy * h * r).sum(0).to(s["w"].dtype)
    ld, scale = s["log_decay"], s["scale"]
    if op == "token":
        S, real = s["S"], s["slots"] >= 0
        at = s["slots"][real].long()
        q, k, v = s["Q"].float(), s["K"].float()[real], s["V"].float()[real]
        new = torch.exp(ld)[:, None, None] * S[at] + k[..., :, None] * v[..., None, :]
        S[at] = new
        O = torch.zeros_like(s["V"])
        O[real] = (scale * (q[real][..., None, :] @ new)[..., 0, :]).to(O.dtype)
        return O, S
    Q, K, V, lens = s["Q"], s["K"], s["V"], s["lens"]
    if op == "prompt":
        return _linear(Q, K, V, ld, lens, s["S0"], scale)
    turn = lambda x: None if x is None else x.mT   # noqa: E731
    dQ, _ = _linear(s["dO"], V, K, ld, lens, turn(s["S0"]), scale)
    dK, _ = _linear(V, s["dO"], Q, ld, lens, turn(s["dS"]), scale, back=True)
    dV, dS0 = _linear(K, Q, s["dO"], ld, lens, s["dS"], scale, back=True)
    return dQ, dK, dV, (dS0 if s["S0"] is not None else None)


def _own(s):
    from paper_2605_21325_b200 import binding
    op = s["op"]
    if op == "norm":
        return binding.rms_norm(s["X"], s["w"], eps=_EPS, residual=s["R"], out_dtype=torch.float8_e4m3fn if s["out"] == "e4m3" else None, group=s["group"])
    if op == "normgrad":
        return binding.rms_norm_backward(s["dY"], s["X"], s["w"], eps=_EPS, dH=s["dH"])
    if op == "token":
        return binding.linear_attention_step(s["Q"], s["K"], s["V"], s["log_decay"], s["S"], scale=s["scale"], slots=s["slots"]), s["S"]
    if op == "prompt":
        return binding.linear_attention(s["Q"], s["K"], s["V"], s["log_decay"], scale=s["scale"], S0=s["S0"], cu_seqlens=s["cu"])
    return binding.linear_attention_backward(s["dO"], s["Q"], s["K"], s["V"], s["log_decay"], scale=s["scale"], S0=s["S0"], dS=s["dS"], cu_seqlens=s["cu"])


def run(s):
    return _own(s) if own else _plain(s)


def work(case):
    """Each input read once, each output written once; products of the path in chunks of 64 tokens, triangular ones by half."""
    es, op = _SIZES[case["dtype"]], case["op"]
    if op in ("norm", "normgrad"):
        rows, n, res = case["rows"], case["n"], case["residual"]
        if op == "norm":
            out = rows * n * es if case["out"] == "same" else rows * n + 4 * rows * (-(-n // (case["group"] or n)))
            return {"bytes": rows * n * es * (3 if res else 1) + out + n * es, "flops": 5.0 * rows * n}
        return {"bytes": rows * n * es * (4 if res else 3) + 2 * n * es, "flops": 10.0 * rows * n}
    H, dk, dv = case["H"], case["dk"], case["dv"]
    if op == "token":
        rows = (case["B"] - case["pad"]) * H
        return {"bytes": rows * (8.0 * dk * dv + es * (2 * dk + 2 * dv)) + 4 * case["B"], "flops": 5.0 * rows * dk * dv}
    lens = _lengths(case)
    rows, states = sum(lens) * H, len(lens) * H * dk * dv * 4
    if op == "prompt":
        return {"bytes": rows * es * (2 * dk + 2 * dv) + states * (2 if case["state"] else 1), "flops": rows * (64.0 * (dk + dv) + 4.0 * dk * dv)}
    return {"bytes": rows * es * (4 * dk + 3 * dv) + states * (3 if case["state"] else 0), "flops": rows * (64.0 * (3 * dk + 2 * dv) + 10.0 * dk * dv)}


# ---- the definitions in 64 bits, token by token

def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op in ("norm", "normgrad"):
        x, w, n = s["X"].double(), s["w"].double(), case["n"]
        if op == "norm":
            h = x + s["R"].double() if s["R"] is not None else x
            y = w * h / (h.pow(2).sum(1, keepdim=True) / n + _EPS).sqrt()
            kept = h if s["R"] is not None else None
            if case["out"] == "same":
                return y, kept, None
            group = case["group"] or n
            scales = []
            for c in range(0, n, group):
                m = y[:, c:c + group].abs().max(dim=1).values / 448
                m[m == 0] = 1
                y[:, c:c + group] /= m[:, None]
                scales.append(m)
            return y, kept, torch.stack(scales, 1)
        dy = s["dY"].double()
        norm = (x.pow(2).sum(1, keepdim=True) / n + _EPS).sqrt()
        unit = x / norm
        dx = (dy * w - unit * ((dy * w * unit).sum(1, keepdim=True) / n)) / norm
        if s["dH"] is not None:
            dx += s["dH"].double()
        return dx, (dy * unit).sum(0)
    lam = torch.exp(s["log_decay"].double())
    if op == "token":
        S = s["S"].double()
        O = torch.zeros(s["V"].shape, dtype=torch.float64, device="cuda")
        for b, slot in enumerate(s["slots"].tolist()):
            if slot >= 0:
                S[slot] = lam[:, None, None] * S[slot] + torch.einsum("hk,hv->hkv", s["K"][b].double(), s["V"][b].double())
                O[b] = s["scale"] * torch.einsum("hk,hkv->hv", s["Q"][b].double(), S[slot])
        return O, S
    lens, c, H = s["lens"], s["scale"], case["H"]
    beg = torch.tensor([sum(lens[:i]) for i in range(len(lens))], device="cuda")
    ln = torch.tensor(lens, device="cuda")
    dk, dv = case["dk"], case["dv"]
    flat = lambda x: x.reshape((-1,) + x.shape[2:])   # noqa: E731
    Q, K, V = flat(s["Q"]), flat(s["K"]), flat(s["V"])
    zero = torch.zeros(len(lens), H, dk, dv, dtype=torch.float64, device="cuda")
    S = s["S0"].double() if s["S0"] is not None else zero.clone()
    order = torch.argsort(ln, descending=True, stable=True)      # the longest first: sequences that have ended are left out
    sorted_lens = sorted(lens, reverse=True)
    beg, S = beg[order], S[order].contiguous()
    grad = op == "grad"
    out = torch.empty(Q.shape if grad else V.shape, dtype=torch.float64, device="cuda")
    x = flat(s["dO"]) if grad else None
    n = len(lens)
    decay = lam[None, :, None, None]
    for t in range(max(lens)):
        while sorted_lens[n - 1] <= t:
            n -= 1
        at = beg[:n] + t
        S[:n] = decay * S[:n] + K[at].double()[..., :, None] * V[at].double()[..., None, :]
        if grad:
            out[at] = c * (S[:n] @ x[at].double()[..., None])[..., 0]
        else:
            out[at] = c * (Q[at].double()[..., None, :] @ S[:n])[..., 0, :]
    inverse = torch.argsort(order)
    if not grad:
        return out.reshape(s["V"].shape), S[inverse]
    G = (s["dS"].double() if s["dS"] is not None else zero)[order].contiguous()
    dK, dV = torch.empty(K.shape, dtype=torch.float64, device="cuda"), torch.empty(V.shape, dtype=torch.float64, device="cuda")
    n = 0
    for t in range(max(lens) - 1, -1, -1):
        while n < len(lens) and sorted_lens[n] > t:
            n += 1
        at = beg[:n] + t
        G[:n] += c * Q[at].double()[..., :, None] * x[at].double()[..., None, :]
        dK[at] = (G[:n] @ V[at].double()[..., None])[..., 0]
        dV[at] = (K[at].double()[..., None, :] @ G[:n])[..., 0, :]
        G[:n] *= decay
    return out.reshape(s["Q"].shape), dK.reshape(s["K"].shape), dV.reshape(s["V"].shape), (G[inverse] if s["S0"] is not None else None)
