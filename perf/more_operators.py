"""The gated linear recurrence (prompt, single token, training step, gradient) and the norm of each query and key head with the position rotation (forward, gradient).

``listed()`` names the cases, ``draw(rng)`` gives further ones of the same ranges, ``prepare`` makes what a program holds before the
call, ``run`` is one pass: with ``own`` the calls of ``paper_2605_21325_b200.binding``, without it the plain form in elementary torch
operations.  ``exact`` is the definition in 64 bits: the recurrence token by token.

Per sequence and channel, from what the projections give:
  decay   a = exp(g),      u = x
  normed  a = exp(g),      u = sqrt(1 - a^2) x
  gate    a = sigmoid(g),  u = (1 - a) x
  prompt  h_t = a_t h_{t-1} + u_t                                                -> H, the state behind the last token
  token   one step of it on states that lie in slots of a cache, updated in place; slot < 0: a padded row, output zero -> H, states
  train   the prompt, then from the gradients of H and of the final state those of X, G and of a carried-in state        -> all of them
  grad    these gradients alone, where the forward pass was thrown away

Per token and head of queries and keys, with r frequencies f and the token's position p:
  heads      y = x / sqrt(mean x^2 + eps) * w, then the pairs of the first 2 r features turned by the angles p f; the pairs are (i, i + r), or
             (2i, 2i + 1) where they are interleaved; position < 0: a padded token, output zero                -> Q', K'
  headsgrad  the gradients of Q, K and of both weights from those of Q' and K'
"""
import math
import random

import torch

own = False

_SIZES = {"float32": 4, "bfloat16": 2}
_EPS = 1e-6


def _rec(name, op, B, T, D, mode="decay", dtype="bfloat16", seqs=0, state=False):
    """``seqs`` > 0: that many packed sequences of lengths uniform in 1..T (B is 1 then); ``state``: states carried in (and, with
    gradients, a gradient of the final state)."""
    c = {"op": op, "B": B, "T": T, "D": D, "mode": mode, "dtype": dtype, "seqs": seqs, "state": state}
    if name:
        c["name"] = name
    return c


def _token(name, B, D, mode="decay", dtype="bfloat16", pad=0):
    """``pad``: padded rows among the B."""
    c = {"op": "token", "B": B, "D": D, "mode": mode, "dtype": dtype, "pad": pad}
    if name:
        c["name"] = name
    return c


def _heads(name, op, B, T, Hq, Hk, d=128, r=64, interleaved=False, dtype="bfloat16", far=0, pad=0, sliced=True):
    """``far``: positions begin at random below it (0: at zero); ``pad``: padded tokens; ``sliced``: Q and K are slices of one projection's output."""
    c = {"op": op, "B": B, "T": T, "Hq": Hq, "Hk": Hk, "d": d, "r": r, "interleaved": interleaved, "dtype": dtype, "far": far, "pad": pad, "sliced": sliced}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one short prompt of no round length through a layer of 2048 channels: launches and latency
        _rec("recurrence_short", "prompt", 1, 333, 2048, "gate"),
        # a prefill batch that continues carried states
        _rec("recurrence_prefill", "prompt", 4, 4096, 2560, "normed", state=True),
        # one long document: few channels for the chip, a long way to walk
        _rec("recurrence_long", "prompt", 1, 32768, 4096, "decay"),
        # a batch of prompts of mixed lengths, packed: partial last tiles
        _rec("recurrence_packed", "prompt", 1, 2048, 2048, "gate", seqs=64),
        # one new token for each of eight sequences: the smallest call of a serving loop
        _token("recurrence_token", 8, 2048, "normed"),
        # a full serving batch, some rows of it padding
        _token("recurrence_token_batch", 256, 4096, "gate", pad=9),
        # the training step of a layer
        _rec("recurrence_train", "train", 4, 4096, 2048, "normed"),
        # the gradient in single precision on a few packed sequences of an odd width, its forward pass thrown away, as in small models and for checking
        _rec("recurrence_gradient_fp32", "grad", 1, 1000, 333, "decay", dtype="float32", seqs=5, state=True),
        # queries and keys of eight new tokens far into their sequences, one row of them padding
        _heads("heads_token", "heads", 8, 1, 16, 16, far=100000, pad=1),
        # the same over a prefill batch
        _heads("heads_prefill", "heads", 4, 4096, 16, 16),
        # one long document: more query than key heads, half of each head turned, pairs side by side, positions up to a million
        _heads("heads_long", "heads", 1, 32768, 32, 8, r=32, interleaved=True, far=1000000),
        # the gradient of the prefill batch in training
        _heads("headsgrad_prefill", "headsgrad", 4, 4096, 16, 16),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["prompt", "prompt", "prompt", "token", "train", "train", "grad", "heads", "heads", "headsgrad", "headsgrad"])
    dtype = "float32" if rng.random() < 0.3 else "bfloat16"
    if op in ("heads", "headsgrad"):
        Hq = rng.choice([1, 2, 3, 4, 6, 8, 12, 16, 20, 24, 32])
        Hk = rng.choice([h for h in (1, 2, 3, 4, 6, 8, 12, 16, 20, 24, 32) if Hq % h == 0])
        d, r = rng.choice([(128, 64), (128, 64), (128, 32), (64, 32), (64, 32), (64, 16), (96, 48), (96, 20), (80, 40), (120, 59), (256, 128), (256, 32), (128, 0)])
        tokens = _log_int(rng, 1, (1 << 25) // ((Hq + Hk) * d))
        B = _log_int(rng, 1, min(64, tokens))
        T = tokens // B
        return _heads(None, op, B, T, Hq, Hk, d, r, rng.random() < 0.4, dtype, rng.choice([0, 0, 4096, 1000000]),
                      rng.choice([0, 0, rng.randint(0, B * T // 4)]), rng.random() < 0.6)
    mode = rng.choice(["decay", "normed", "gate"])
    D = rng.choice([256, 512, 1024, 2048, 2560, 4096, 5120]) if rng.random() < 0.6 else _log_int(rng, 32, 5120)
    if op == "token":
        B = _log_int(rng, 1, 256)
        return _token(None, B, D, mode, dtype, rng.randint(0, B // 4))
    values = 1 << ((26 if op == "prompt" else 25 if op == "train" else 23) - (dtype == "float32"))
    tokens = max(1, _log_int(rng, 16, max(16, min(1 << 17, values // D))))
    if rng.random() < 0.4 and tokens >= 64:                                              # packed: 2..64 sequences
        seqs = _log_int(rng, 2, min(64, tokens // 16))
        return _rec(None, op, 1, max(1, min(32768, 2 * tokens // seqs)), D, mode, dtype, seqs, rng.random() < 0.5)
    B = _log_int(rng, 1, min(32, tokens))
    return _rec(None, op, B, max(1, min(32768, tokens // B)), D, mode, dtype, 0, rng.random() < 0.5)


def _lengths(case):
    """Tokens of each sequence: a matter of the case, not of the seed."""
    if not case["seqs"]:
        return [case["T"]] * case["B"]
    r = random.Random(911 * case["seqs"] + case["T"])
    return [r.randint(1, case["T"]) for _ in range(case["seqs"])]


def _gates(normal, channel, mode, dt, *shape):
    """What the projection gives for the decays: channels remember for a few tokens up to a few thousand."""
    D = shape[-1]
    spread = 2.0 ** (-9.0 * channel / max(1, D - 1))                  # 1 .. 1/512
    z = normal(*shape)
    return (z - torch.log(spread)).to(dt) if mode == "gate" else (-2.0 * spread * torch.sigmoid(z)).to(dt)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(1000033 * (int(seed) % (1 << 40)) + 71)
    normal = lambda *s: torch.randn(*s, device="cuda", generator=gen)   # noqa: E731
    dt = getattr(torch, case["dtype"])
    s = dict(op=case["op"])
    if case["op"] in ("heads", "headsgrad"):
        B, T, Hq, Hk, d = (case[k] for k in ("B", "T", "Hq", "Hk", "d"))
        if case["sliced"]:                                              # Q, K and V side by side, as one projection writes them
            both = normal(B, T, (Hq + 2 * Hk) * d).to(dt)
            Q, K = both[..., :Hq * d].unflatten(-1, (Hq, d)), both[..., Hq * d:(Hq + Hk) * d].unflatten(-1, (Hk, d))
        else:
            Q, K = normal(B, T, Hq, d).to(dt), normal(B, T, Hk, d).to(dt)
        first = torch.randint(0, case["far"] + 1, (B, 1), device="cuda", generator=gen)
        pos = (first + torch.arange(T, device="cuda")).to(torch.int32)
        pos.view(-1)[torch.randperm(B * T, device="cuda", generator=gen)[:case["pad"]]] = -1
        r = case["r"]
        s.update(Q=Q, K=K, wq=(1 + 0.1 * normal(d)).to(dt), wk=(1 + 0.1 * normal(d)).to(dt), pos=pos, interleaved=case["interleaved"],
                 f=(10000.0 ** (-torch.arange(r, device="cuda", dtype=torch.float64) / max(1, r))).float())
        if case["op"] == "headsgrad":
            s.update(dQ=normal(B, T, Hq, d).to(dt), dK=normal(B, T, Hk, d).to(dt))
        return s
    D, mode = case["D"], case["mode"]
    s.update(mode=mode)
    channel = torch.randperm(D, device="cuda", generator=gen).float()
    if case["op"] == "token":
        B, pad = case["B"], case["pad"]
        n_slots = B + 3
        slots = torch.randperm(n_slots, device="cuda", generator=gen)[:B].to(torch.int32)
        slots[torch.randperm(B, device="cuda", generator=gen)[:pad]] = -1
        s.update(X=normal(B, D).to(dt), G=_gates(normal, channel, mode, dt, B, D), slots=slots, h=normal(n_slots, D))
        return s
    lens = _lengths(case)
    B, T = (1, sum(lens)) if case["seqs"] else (case["B"], case["T"])
    both = torch.empty(B, T, 2 * D, dtype=dt, device="cuda")            # X and G side by side, as one projection writes them
    both[..., :D] = normal(B, T, D)
    both[..., D:] = _gates(normal, channel, mode, dt, B, T, D)
    s.update(X=both[..., :D], G=both[..., D:], lens=lens, h0=None, dh=None, cu=[sum(lens[:i]) for i in range(len(lens) + 1)] if case["seqs"] else None)
    if case["state"]:
        s["h0"] = normal(len(lens), D)
    if case["op"] != "prompt":
        s["dY"] = normal(B, T, D).to(dt)
        s["dh"] = normal(len(lens), D) if case["state"] else None
    return s


# ---- plain form

def _factors(x, g, mode):
    """a and u in 32 bits, and what multiplies x in u."""
    if mode == "gate":
        return torch.sigmoid(g), torch.sigmoid(-g) * x, torch.sigmoid(-g)
    if mode == "normed":
        m = torch.sqrt(-torch.expm1(2 * g))
        return torch.exp(g), m * x, m
    return torch.exp(g), x, None


def _doubling(a, u):
    """h_t = a_t h_{t-1} + u_t over dimension 1 from zero, by doubling the reach of every place."""
    n, k = a.shape[1], 1
    while k < n:
        u = torch.cat([u[:, :k], u[:, k:] + a[:, k:] * u[:, :-k]], 1)
        a = torch.cat([a[:, :k], a[:, k:] * a[:, :-k]], 1)
        k *= 2
    return u


def _ends(s):
    """Where sequences begin and end among the flat tokens."""
    ln = torch.tensor(s["lens"], device=s["X"].device)
    end = ln.cumsum(0)
    return end - ln, end - 1


def _forward(s):
    """In 32 bits, over flat tokens: a, u, what multiplies x, h before and h behind every token."""
    x, g = s["X"].flatten(0, 1).float(), s["G"].flatten(0, 1).float()
    a, u, m = _factors(x, g, s["mode"])
    first, last = _ends(s)
    begin = torch.zeros(len(s["lens"]), x.shape[1], device=x.device) if s["h0"] is None else s["h0"]
    u1, a1 = u.clone(), a.clone()
    u1[first] += a[first] * begin
    a1[first] = 0
    h = _doubling(a1[None], u1[None])[0]
    before = torch.cat([h[:1], h[:-1]])
    before[first] = begin
    return x, a, m, before, h, first, last


def _gradients(s, x, a, m, before, first, last):
    e = s["dY"].flatten(0, 1).float()
    if s["dh"] is not None:
        e = e.index_add(0, last, s["dh"])
    b = torch.cat([a[1:], a[:1]])                                       # the decay that reaches a token from behind it
    b[last] = 0
    e = _doubling(b.flip(0)[None], e.flip(0)[None])[0].flip(0)
    if s["mode"] == "gate":
        dx, dg = e * m, e * (before - x) * a * m
    elif s["mode"] == "normed":
        dx, dg = e * m, e * a * (before - a / m * x)
    else:
        dx, dg = e, e * a * before
    t, shape = s["X"].dtype, s["X"].shape
    return dx.to(t).view(shape), dg.to(t).view(shape), (a * e)[first] if s["h0"] is not None else None


def _turn(y, s, back=False):
    """Turns the pairs of the first 2 r features by the positions' angles (``back``: the other way)."""
    r = s["f"].numel()
    angle = (s["pos"].double()[..., None] * s["f"].double())[:, :, None]
    c, n = torch.cos(angle).float(), torch.sin(angle).float()
    if back:
        n = -n
    if s["interleaved"]:
        p = y[..., :2 * r].unflatten(-1, (r, 2))
        u, v = p[..., 0], p[..., 1]
        turned = torch.stack([u * c - v * n, v * c + u * n], -1).flatten(-2)
    else:
        u, v = y[..., :r], y[..., r:2 * r]
        turned = torch.cat([u * c - v * n, v * c + u * n], -1)
    return torch.where((s["pos"] >= 0)[..., None, None], torch.cat([turned, y[..., 2 * r:]], -1), 0.0)


def _plain(s):
    op = s["op"]
    if op == "heads":
        out = []
        for x, w in ((s["Q"], s["wq"]), (s["K"], s["wk"])):
            x = x.float()
            out.append(_turn(x * torch.rsqrt(x.square().mean(-1, keepdim=True) + _EPS) * w.float(), s).to(s["Q"].dtype))
        return tuple(out)
    if op == "headsgrad":
        dx, dw = [], []
        for x, w, dy in ((s["Q"], s["wq"], s["dQ"]), (s["K"], s["wk"], s["dK"])):
            t, x, dy = x.dtype, x.float(), _turn(dy.float(), s, back=True)
            rstd = torch.rsqrt(x.square().mean(-1, keepdim=True) + _EPS)
            u = dy * w.float()
            dx.append((rstd * (u - x * (rstd * rstd * (u * x).mean(-1, keepdim=True)))).to(t))
            dw.append((dy * x * rstd).sum((0, 1, 2)).to(t))
        return dx[0], dx[1], dw[0], dw[1]
    if op == "token":
        real = s["slots"] >= 0
        at = s["slots"][real].long()
        a, u, _ = _factors(s["X"][real].float(), s["G"][real].float(), s["mode"])
        s["h"][at] = a * s["h"][at] + u
        Y = torch.zeros_like(s["X"])
        Y[real] = s["h"][at].to(Y.dtype)
        return Y, s["h"]
    x, a, m, before, h, first, last = _forward(s)
    state = h[last]
    Y = h.to(s["X"].dtype).view(s["X"].shape)
    if op == "prompt":
        return Y, state
    grads = _gradients(s, x, a, m, before, first, last)
    return grads if op == "grad" else (Y, state) + grads


def _own(s):
    from paper_2605_21325_b200 import binding
    op = s["op"]
    if op == "heads":
        return binding.qk_norm_rope(s["Q"], s["K"], s["wq"], s["wk"], s["f"], positions=s["pos"], eps=_EPS, interleaved=s["interleaved"])
    if op == "headsgrad":
        return binding.qk_norm_rope_backward(s["dQ"], s["dK"], s["Q"], s["K"], s["wq"], s["wk"], s["f"], positions=s["pos"], eps=_EPS, interleaved=s["interleaved"])
    mode = {"decay": binding.REC_DECAY, "normed": binding.REC_NORMED, "gate": binding.REC_GATE}[s["mode"]]
    if op == "token":
        return binding.gated_recurrence_step(s["X"], s["G"], s["h"], mode=mode, slots=s["slots"]), s["h"]
    if op == "grad":
        return binding.gated_recurrence_backward(s["dY"], s["X"], s["G"], mode=mode, h0=s["h0"], dh=s["dh"], cu_seqlens=s["cu"])
    Y, state, carries = binding.gated_recurrence(s["X"], s["G"], mode=mode, h0=s["h0"], cu_seqlens=s["cu"], want_carries=op == "train")
    if op == "prompt":
        return Y, state
    return (Y, state) + binding.gated_recurrence_backward(s["dY"], s["X"], s["G"], mode=mode, h0=s["h0"], dh=s["dh"], carries=carries, cu_seqlens=s["cu"])


def run(s):
    return _own(s) if own else _plain(s)


def work(case):
    """Each input read once, each output written once."""
    es, op = _SIZES[case["dtype"]], case["op"]
    if op in ("heads", "headsgrad"):
        n = (case["B"] * case["T"] - case["pad"]) * (case["Hq"] + case["Hk"]) * case["d"]
        written = case["pad"] * (case["Hq"] + case["Hk"]) * case["d"] * es
        small = 4 * case["B"] * case["T"] + 2 * case["d"] * es * (1 if op == "heads" else 2) + 4 * case["r"]
        return {"bytes": n * es * (2 if op == "heads" else 3) + written + small, "flops": n * (8.0 if op == "heads" else 16.0)}
    D = case["D"]
    if op == "token":
        rows = case["B"] - case["pad"]
        return {"bytes": rows * D * (3 * es + 8) + case["pad"] * D * es + 4 * case["B"], "flops": 6.0 * rows * D}
    lens = _lengths(case)
    n, states = sum(lens) * D, 4 * len(lens) * D
    forward, forward_flops = 3 * n * es + states * (2 if case["state"] else 1), 6.0 * n
    if op == "prompt":
        return {"bytes": forward, "flops": forward_flops}
    back, back_flops = 5 * n * es + states * (3 if case["state"] else 0), 14.0 * n
    return {"bytes": back, "flops": back_flops} if op == "grad" else {"bytes": forward + back, "flops": forward_flops + back_flops}


# ---- the definitions in 64 bits, token by token

def _exact_turn(y, s, sign):
    out, r = y.clone(), s["f"].numel()
    for i in range(r):
        j, k = (2 * i, 2 * i + 1) if s["interleaved"] else (i, i + r)
        t = (s["pos"].double() * float(s["f"][i]))[..., None]
        out[..., j] = y[..., j] * t.cos() - sign * y[..., k] * t.sin()
        out[..., k] = y[..., k] * t.cos() + sign * y[..., j] * t.sin()
    out[s["pos"] < 0] = 0
    return out


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op in ("heads", "headsgrad"):
        outs, weights = [], []
        for x, w, dy in ((s["Q"], s["wq"], s.get("dQ")), (s["K"], s["wk"], s.get("dK"))):
            x, w = x.double(), w.double()
            norm = (x.pow(2).sum(-1, keepdim=True) / case["d"] + _EPS).sqrt()
            unit = x / norm
            if op == "heads":
                outs.append(_exact_turn(unit * w, s, 1))
                continue
            v = _exact_turn(dy.double(), s, -1)
            weights.append((v * unit).sum((0, 1, 2)))
            outs.append((v * w - unit * ((v * w * unit).sum(-1, keepdim=True) / case["d"])) / norm)
        return tuple(outs + weights)
    X, G, mode = s["X"].double(), s["G"].double(), case["mode"]
    a = 1 / (1 + torch.exp(-G)) if mode == "gate" else torch.exp(G)
    m = 1 / (1 + torch.exp(G)) if mode == "gate" else torch.sqrt(-torch.expm1(2 * G)) if mode == "normed" else torch.ones_like(G)
    if op == "token":
        h, Y = s["h"].double(), torch.zeros_like(X)
        for b, slot in enumerate(s["slots"].tolist()):
            if slot >= 0:
                h[slot] = a[b] * h[slot] + m[b] * X[b]
                Y[b] = h[slot]
        return Y, h
    lens, D = s["lens"], case["D"]
    ln = torch.tensor(lens, device="cuda")
    order = torch.argsort(ln, descending=True, stable=True)             # the longest first: sequences that have ended are left out
    sizes = sorted(lens, reverse=True)
    begin = (ln.cumsum(0) - ln)[order]
    A, M, X = a.view(-1, D), m.view(-1, D), X.reshape(-1, D)
    U = M * X
    h = (s["h0"].double() if s["h0"] is not None else torch.zeros(len(lens), D, dtype=torch.float64, device="cuda"))[order].contiguous()
    H, before = torch.empty_like(U), torch.empty_like(U)
    n = len(lens)
    for t in range(sizes[0]):
        while sizes[n - 1] <= t:
            n -= 1
        at = begin[:n] + t
        before[at] = h[:n]
        h[:n] = A[at] * h[:n] + U[at]
        H[at] = h[:n]
    inverse = torch.argsort(order)
    Y, state = H.view(s["X"].shape), h[inverse]
    if op == "prompt":
        return Y, state
    dY = s["dY"].double().view(-1, D)
    c = (s["dh"].double() if s["dh"] is not None else torch.zeros_like(h))[order].contiguous()
    dX, dG = torch.empty_like(X), torch.empty_like(X)
    n = 0
    for t in range(sizes[0] - 1, -1, -1):
        while n < len(lens) and sizes[n] > t:
            n += 1
        at = begin[:n] + t
        e = c[:n] + dY[at]
        c[:n] = A[at] * e
        dX[at] = M[at] * e
        if mode == "gate":                                              # d a / d g = a (1 - a), d (1 - a) / d g = - a (1 - a)
            dG[at] = e * (before[at] - X[at]) * A[at] * M[at]
        elif mode == "normed":                                          # d a / d g = a, d m / d g = - a^2 / m
            dG[at] = e * (A[at] * before[at] - A[at] * A[at] / M[at] * X[at])
        else:
            dG[at] = e * A[at] * before[at]
    grads = dX.view(s["X"].shape), dG.view(s["X"].shape), (c[inverse] if s["h0"] is not None else None)
    return grads if op == "grad" else (Y, state) + grads
