"""GPU tests of the heads' norm with position rotation and of its gradient against 64-bit arithmetic.

Bounds in roundings of 2^-24 of the same formula over absolute values.  The norm: squares of at most 16 values a lane and five exchanges (half of it counts in the root), the root 2, products 3: 16.  The
rotation: an angle of at most half a turn in fp32 (pi / 2 x 2^-24), sine and cosine 2 each, two products and a sum: 8 of |u| + |v|.  The gradient: both, and the mean of u x with as many as the norm: 48.
Sums for the weights: a lane's terms one after the other, then five exchanges, eight warps and up to 592 blocks in 32 runs.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

ULP = 2.0 ** -24
STORE = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
DTYPES = [torch.float32, torch.bfloat16]
EPS = 1e-6
# tokens (B, T), query heads, key heads, d, r
SHAPES = [(1, 1, 1, 1, 128, 64), (8, 1, 16, 16, 128, 64), (3, 37, 4, 1, 64, 32), (2, 50, 5, 5, 96, 48), (1, 70, 3, 2, 96, 20), (2, 33, 2, 2, 80, 40), (1, 41, 3, 3, 120, 59), (1, 20, 7, 1, 256, 128),
          (1, 20, 2, 1, 256, 32), (2, 9, 3, 3, 128, 0), (1, 13, 2, 1, 7, 3), (1, 5, 2, 2, 2, 1), (1, 3, 1, 1, 1, 0), (1, 11, 3, 1, 255, 127), (4, 700, 8, 2, 128, 64), (1, 3, 40, 8, 64, 16), (3, 21, 6, 0, 64, 32),
          (1, 9, 2, 1, 24, 8), (1, 17, 4, 4, 192, 64)]


@pytest.fixture(scope="module")
def bnd():
    import __graft_entry__ as entry
    entry.build()
    from paper_2605_21325_b200 import binding
    torch.cuda.set_device(0)
    return binding


def make(B, T, Hq, Hk, d, r, dtype, seed=0, far=100000):
    g = torch.Generator(device="cuda").manual_seed(B * T + 100 * d + seed)
    n = lambda *s: torch.randn(*s, device="cuda", generator=g)   # noqa: E731
    pos = torch.randint(0, far, (B, T), device="cuda", generator=g).to(torch.int32)
    s = dict(Q=n(B, T, Hq, d).to(dtype), K=n(B, T, Hk, d).to(dtype) if Hk else None, wq=(1 + 0.2 * n(d)).to(dtype), wk=(1 + 0.2 * n(d)).to(dtype) if Hk else None,
             f=(10000.0 ** (-torch.arange(r, device="cuda", dtype=torch.float64) / max(r, 1))).float() if r else None, pos=pos, dQ=n(B, T, Hq, d).to(dtype), dK=n(B, T, Hk, d).to(dtype) if Hk else None)
    return s


def split(y, r, interleaved):
    if interleaved:
        p = y[..., :2 * r].unflatten(-1, (r, 2))
        return p[..., 0], p[..., 1]
    return y[..., :r], y[..., r:2 * r]


def join(u, v, rest, interleaved):
    return torch.cat([torch.stack([u, v], -1).flatten(-2) if interleaved else torch.cat([u, v], -1), rest], -1)


def turn(y, s, r, interleaved, sign):
    """y turned, and the sums of absolute values that its bound counts."""
    if r == 0:
        return y, y.abs()
    t = (s["pos"].double()[..., None] * s["f"].double())[:, :, None]
    u, v = split(y, r, interleaved)
    rest = y[..., 2 * r:]
    size = u.abs() + v.abs()
    return join(u * t.cos() - sign * v * t.sin(), v * t.cos() + sign * u * t.sin(), rest, interleaved), join(size, size, rest.abs(), interleaved)


def inside(got, ref, bound):
    off = (got.double() - ref).abs() / (1.01 * (bound + STORE[got.dtype] * ref.abs()) + 1e-37)
    assert bool((off <= 1).all()), "%d of %d outside, worst %.3g of its bound" % (int((~(off <= 1)).sum()), off.numel(), float(off.nan_to_num(9e9).max()))


def reference(x, w, s, r, interleaved):
    x = x.double()
    y = x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * (1 if w is None else w.double())
    y, size = turn(y, s, r, interleaved, 1)
    y = torch.where((s["pos"] >= 0)[..., None, None], y, 0.0)
    return y, 24 * ULP * size


def reference_gradient(dy, x, w, s, r, interleaved, heads):
    x, w = x.double(), 1 if w is None else w.double()
    real = (s["pos"] >= 0)[..., None, None]
    rstd = 1 / (x.square().mean(-1, keepdim=True) + EPS).sqrt()
    v, size = turn(dy.double(), s, r, interleaved, -1)
    u, us = v * w, size * abs(w)
    dx = rstd * (u - x * (rstd ** 2 * (u * x).mean(-1, keepdim=True)))
    dxb = 48 * ULP * rstd * (us + x.abs() * (rstd ** 2 * (us * x.abs()).mean(-1, keepdim=True)))
    depth = x.shape[2] + x.shape[0] * x.shape[1] * heads / 1000 + 96
    dw, dwb = torch.where(real, v * x * rstd, 0.0).sum((0, 1, 2)), depth * ULP * torch.where(real, size * x.abs() * rstd, 0.0).sum((0, 1, 2))
    return torch.where(real, dx, 0.0), dxb, dw, dwb


def check(bnd, s, r, interleaved, **kw):
    Yq, Yk = bnd.qk_norm_rope(s["Q"], s["K"], s["wq"], s["wk"], s["f"], positions=s["pos"], eps=EPS, interleaved=interleaved, **kw)
    inside(Yq, *reference(s["Q"], s["wq"], s, r, interleaved))
    if s["K"] is None:
        assert Yk is None
    else:
        inside(Yk, *reference(s["K"], s["wk"], s, r, interleaved))
    return Yq, Yk


def check_gradient(bnd, s, r, interleaved, **kw):
    dQ, dK, dwq, dwk = bnd.qk_norm_rope_backward(s["dQ"], s["dK"], s["Q"], s["K"], s["wq"], s["wk"], s["f"], positions=s["pos"], eps=EPS, interleaved=interleaved, **kw)
    heads = s["Q"].shape[2] + (0 if s["K"] is None else s["K"].shape[2])
    for dy, x, w, gx, gw in ((s["dQ"], s["Q"], s["wq"], dQ, dwq), (s["dK"], s["K"], s["wk"], dK, dwk)):
        if x is None:
            assert gx is None and gw is None
            continue
        rx, bx, rw, bw = reference_gradient(dy, x, w, s, r, interleaved, heads)
        inside(gx, rx, bx)
        if w is not None:
            inside(gw, rw, bw)
        else:
            assert gw is None
    return dQ, dK, dwq, dwk


@pytest.mark.parametrize("interleaved", [False, True], ids=["halves", "interleaved"])
@pytest.mark.parametrize("dtype", DTYPES, ids=["fp32", "bf16"])
@pytest.mark.parametrize("B,T,Hq,Hk,d,r", SHAPES)
def test_forward_and_gradient(bnd, B, T, Hq, Hk, d, r, dtype, interleaved):
    s = make(B, T, Hq, Hk, d, r, dtype)
    if B * T > 2:
        s["pos"].view(-1)[::3] = -1
    check(bnd, s, r, interleaved)
    check_gradient(bnd, s, r, interleaved)
    assert bnd.last_device_status() == 0


@pytest.mark.parametrize("dtype", DTYPES, ids=["fp32", "bf16"])
@pytest.mark.parametrize("offset,pad", [(0, 0), (8, 0), (4, 4), (1, 0), (0, 3)])
def test_slices_in_place_and_gradients_into_slices(bnd, dtype, offset, pad):
    """Queries, keys and values side by side in one projection: read there, normed in place, gradients into the projection's gradient."""
    B, T, Hq, Hk, d, r = 2, 30, 4, 2, 64, 32
    s = make(B, T, Hq, Hk, d, r, dtype)
    width = offset + (Hq + 2 * Hk) * d + pad
    cut = lambda t: (t[..., offset:offset + Hq * d].unflatten(-1, (Hq, d)), t[..., offset + Hq * d:offset + (Hq + Hk) * d].unflatten(-1, (Hk, d)))   # noqa: E731
    both, grad, dy = (torch.full((B, T, width), 7.0, dtype=dtype, device="cuda") for _ in range(3))
    for t, names in ((both, ("Q", "K")), (dy, ("dQ", "dK"))):
        for x, n in zip(cut(t), names):
            x.copy_(s[n])
            s[n] = x
    check_gradient(bnd, s, r, False, out=cut(grad))
    Yq, Yk = check(bnd, s, r, False)
    out = bnd.qk_norm_rope(s["Q"], s["K"], s["wq"], s["wk"], s["f"], positions=s["pos"], eps=EPS, out=(s["Q"], s["K"]))
    assert torch.equal(out[0], Yq) and torch.equal(out[1], Yk)
    for t in (both, grad):
        assert bool((t[..., :offset] == 7).all()) and bool((t[..., offset + (Hq + Hk) * d:] == 7).all())


def test_gradient_in_place(bnd):
    s = make(2, 40, 4, 2, 128, 64, torch.bfloat16)
    want = check_gradient(bnd, s, 64, False)
    for a, b in (("dQ", "dK"), ("Q", "K"), ("dQ", "K")):
        t = {k: v.clone() for k, v in s.items()}
        got = bnd.qk_norm_rope_backward(t["dQ"], t["dK"], t["Q"], t["K"], t["wq"], t["wk"], t["f"], positions=t["pos"], eps=EPS, out=(t[a], t[b]))
        assert got[0] is t[a] and all(torch.equal(x, y) for x, y in zip(got, want))


def test_positions(bnd):
    """Without positions a token's place in its sequence counts; angles hold at the farthest positions."""
    s = make(3, 50, 2, 2, 64, 32, torch.float32)
    s["pos"] = torch.arange(50, device="cuda", dtype=torch.int32).expand(3, 50)
    got = bnd.qk_norm_rope(s["Q"], s["K"], s["wq"], s["wk"], s["f"], eps=EPS)
    for x, y in zip(got, (reference(s["Q"], s["wq"], s, 32, False), reference(s["K"], s["wk"], s, 32, False))):
        inside(x, *y)
    dQ, _, dwq, _ = bnd.qk_norm_rope_backward(s["dQ"], s["dK"], s["Q"], s["K"], s["wq"], s["wk"], s["f"], eps=EPS)
    rx, bx, rw, bw = reference_gradient(s["dQ"], s["Q"], s["wq"], s, 32, False, 4)
    inside(dQ, rx, bx)
    inside(dwq, rw, bw)
    s["pos"] = (2 ** 31 - 1 - torch.randint(0, 1000, (3, 50), device="cuda")).to(torch.int32)
    check(bnd, s, 32, True)
    s["f"] = torch.cat([s["f"][:16], -s["f"][16:]]) * 3
    check(bnd, s, 32, False)


def test_without_weights_and_zero_rows(bnd):
    s = make(1, 20, 3, 2, 64, 16, torch.bfloat16)
    s["wq"] = s["wk"] = None
    s["Q"][0, 3] = 0
    check(bnd, s, 16, False)
    check_gradient(bnd, s, 16, False)
    s["wk"] = torch.ones(64, device="cuda").bfloat16()
    check_gradient(bnd, s, 16, True)


def test_values_that_are_not_finite_stay_in_their_head(bnd):
    s = make(1, 20, 3, 2, 64, 32, torch.bfloat16)
    clean = bnd.qk_norm_rope(s["Q"], s["K"], s["wq"], s["wk"], s["f"], positions=s["pos"])
    s["Q"][0, 5, 1, 7], s["K"][0, 9, 0, 3] = float("nan"), float("inf")
    s["pos"][0, 11] = -1
    s["Q"][0, 11] = float("nan")
    got = bnd.qk_norm_rope(s["Q"], s["K"], s["wq"], s["wk"], s["f"], positions=s["pos"])
    for x, y, (t, h) in ((got[0], clean[0], (5, 1)), (got[1], clean[1], (9, 0))):
        keep = torch.ones(20, x.shape[2], dtype=torch.bool, device="cuda")
        keep[t, h] = keep[11] = False
        assert torch.equal(x[0][keep], y[0][keep]) and bool((x[0, 11] == 0).all())
    s["dQ"][0, 11] = float("inf")
    dQ, dK, dwq, dwk = bnd.qk_norm_rope_backward(s["dQ"], s["dK"], torch.nan_to_num(s["Q"], 0.5, 0.5), torch.nan_to_num(s["K"], 0.5, 0.5), s["wq"], s["wk"], s["f"], positions=s["pos"])
    assert all(bool(torch.isfinite(x).all()) for x in (dQ, dK, dwq, dwk)) and bool((dQ[0, 11] == 0).all())


def test_repeats_streams_and_graphs(bnd):
    s = make(4, 600, 8, 4, 128, 64, torch.bfloat16)
    first = check_gradient(bnd, s, 64, False)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        got = bnd.qk_norm_rope_backward(s["dQ"], s["dK"], s["Q"], s["K"], s["wq"], s["wk"], s["f"], positions=s["pos"], eps=EPS, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(x, y) for x, y in zip(got, first))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y = bnd.qk_norm_rope(s["Q"], s["K"], s["wq"], s["wk"], s["f"], positions=s["pos"], eps=EPS)
        dx = bnd.qk_norm_rope_backward(s["dQ"], s["dK"], s["Q"], s["K"], s["wq"], s["wk"], s["f"], positions=s["pos"], eps=EPS)
    other = make(4, 600, 8, 4, 128, 64, torch.bfloat16, seed=1)
    for k in ("Q", "K", "dQ", "dK", "pos"):
        s[k].copy_(other[k])
    g.replay()
    torch.cuda.synchronize()
    inside(y[0], *reference(s["Q"], s["wq"], s, 64, False))
    want = check_gradient(bnd, s, 64, False)
    assert all(torch.equal(a, b) for a, b in zip(dx, want))


def test_no_tokens(bnd):
    Q, w, f = torch.empty(2, 0, 3, 64, device="cuda"), torch.ones(64, device="cuda"), torch.ones(32, device="cuda")
    Yq, Yk = bnd.qk_norm_rope(Q, Q, w, w, f)
    assert Yq.shape == Q.shape
    dQ, dK, dwq, dwk = bnd.qk_norm_rope_backward(Q, Q, Q, Q, w, w, f)
    assert bool((dwq == 0).all()) and bool((dwk == 0).all())
