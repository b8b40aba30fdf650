"""The gated linear recurrence and its gradient token by token in 64 bits, with a bound on what fp32 arithmetic may be off by, carried along by the same recurrences.

STEP = 12 roundings of 2^-24 a token: the decay's own error (a power of two 2.8, a reciprocal 2, products and differences 1 each: at most 9 for the logistic form), a fused
product and sum 1, and 2 more for the maps that join tokens, warps and tiles.  The factor of x carries as many (square root form: half of 9, and 3 for the root and its product), its
reciprocal twice as many.  The exponent's product with log2 e rounds to |g| 2^-24 of the decay: beyond |g| = 8, where that alone would pass the rest, the decay leaves less than e^-8 of the state, and the token's input
carries the sum.
"""
import torch

ULP = 2.0 ** -24
STEP = 12 * ULP
STORE = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
DECAY, NORMED, GATE = 0, 1, 2


def factors(G, mode):
    """a, m in 64 bits."""
    G = G.double()
    if mode == GATE:
        return torch.sigmoid(G), torch.sigmoid(-G)
    a = torch.exp(G)
    return a, torch.ones_like(a) if mode == DECAY else torch.sqrt(torch.clamp(-torch.expm1(2 * G), min=0))


def step(a, h, u):
    return torch.where(a == 0, u, a * h + u)


def walk(X, G, mode, lens, h0):
    """Per flat token: h before, h, and their bounds; the final states and theirs."""
    D = X.shape[-1]
    x, (a, m) = X.reshape(-1, D).double(), factors(G.reshape(-1, D), mode)
    u = m * x
    h = torch.zeros(len(lens), D, dtype=torch.float64, device=X.device) if h0 is None else h0.double().clone()
    s, e = h.abs(), torch.zeros_like(h)             # sums of absolute values, bounds
    out = {k: torch.empty_like(u) for k in ("before", "h", "ebefore", "eh")}
    ln = torch.tensor(lens, device=X.device)
    begin = ln.cumsum(0) - ln
    for t in range(max(lens, default=0)):
        r = (ln > t).nonzero()[:, 0]
        at = begin[r] + t
        out["before"][at], out["ebefore"][at] = h[r], e[r]
        s1 = step(a[at], s[r], u[at].abs())
        e[r] = step(a[at], e[r], torch.zeros_like(s1)) + STEP * s1
        h[r], s[r] = step(a[at], h[r], u[at]), s1
        out["h"][at], out["eh"][at] = h[r], e[r]
    out.update(state=h, estate=e, x=x, a=a, m=m, begin=begin, ln=ln)
    return out


def gradient(X, G, mode, lens, h0, dY, dh):
    """((dX, bound), (dG, bound), (dh0, bound)) before they are stored."""
    f = walk(X, G, mode, lens, h0)
    D = X.shape[-1]
    x, a, m, dy = f["x"], f["a"], f["m"], dY.reshape(-1, D).double()
    c = torch.zeros(len(lens), D, dtype=torch.float64, device=X.device) if dh is None else dh.double().clone()
    s, b = c.abs(), torch.zeros_like(c)
    E, EB = torch.empty_like(x), torch.empty_like(x)
    for t in range(max(lens, default=0) - 1, -1, -1):
        r = (f["ln"] > t).nonzero()[:, 0]
        at = f["begin"][r] + t
        e, es = c[r] + dy[at], s[r] + dy[at].abs()
        E[at], EB[at] = e, b[r] + STEP * es
        zero = a[at] == 0
        c[r], s[r], b[r] = (torch.where(zero, 0.0, a[at] * v) for v in (e, es, EB[at]))
        b[r] += STEP * s[r]
    hb, eb = f["before"], f["ebefore"]
    over = torch.where(m > 0, 1 / m, 0.0)
    if mode == GATE:
        w, ws, we = a * m * (hb - x), a * m * (hb.abs() + x.abs()), a * m * eb
    elif mode == NORMED:
        w, ws, we = a * (hb - a * over * x), a * (hb.abs() + a * over * x.abs()), a * eb
    else:
        w, ws, we = a * hb, a * hb.abs(), a * eb
    w, ws, we = (torch.where(a == 0, 0.0, v) for v in (w, ws, we))
    we = we + 2 * STEP * ws
    dg, dgb = E * w, E.abs() * we + w.abs() * EB + EB * we
    dx, dxb = E * m, EB * m + STEP * E.abs() * m
    return (dx, dxb), (dg, dgb), (c, b)


def inside(got, ref, bound):
    """NaN in the same places, infinities equal, the rest within the bound and a rounding of the storage."""
    got64 = got.reshape(ref.shape).double()
    assert bool((torch.isnan(got64) == torch.isnan(ref)).all()), "NaN in other places"
    ok = torch.isnan(ref) | (got64 == ref) | ((got64 - ref).abs() <= 1.01 * (bound + STORE[got.dtype] * ref.abs()) + 1e-37)
    off = ((got64 - ref).abs() / (1.01 * (bound + STORE[got.dtype] * ref.abs()) + 1e-37)).nan_to_num(0)
    assert bool(ok.all()), "%d of %d outside, worst %.3g of its bound" % (int((~ok).sum()), ok.numel(), float(off.max()))
