"""GPU tests of the RMS norm and its gradient against 64-bit arithmetic.

Bounds: sums of n fp32 terms, all of one sign in mean h^2, in blocks (a thread's own values, then a tree): at most n / 32 + 16 roundings on a term's way, each
2^-24; outputs add their own rounding (bf16 2^-8, fp32 2^-24).  An 8-bit code is off by half a step of e4m3 (2^-4 of the value, or 2^-10 in the subnormal range below 2^-6),
plus what the scale's own roundings move.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

EPS = 1e-6
STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
DTYPES = [torch.float32, torch.bfloat16]
SHAPES = [(1, 1), (3, 7), (2, 64), (5, 128), (1000, 128), (4, 130), (700, 200), (8, 2048), (2000, 512), (700, 1024), (700, 2048), (2, 2056), (400, 4096), (9, 5120),
          (9, 8191), (5, 8192), (400, 8192), (3, 16384), (2, 20000),
          (5000, 127), (700, 333), (700, 801), (700, 2047), (700, 4001), (100, 7001)]   # not whole vectors: more rows than blocks, each width of the rows held value by value


@pytest.fixture(scope="module")
def bnd():
    import __graft_entry__ as entry
    entry.build()
    from paper_2605_21325_b200 import binding
    torch.cuda.set_device(0)
    return binding


def make(rows, n, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(1000 * rows + n + seed)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)   # noqa: E731
    return {"X": r(rows, n).to(dtype), "R": (2 * r(rows, n)).to(dtype), "w": (1 + 0.1 * r(n)).to(dtype), "dY": r(rows, n).to(dtype), "dH": r(rows, n).to(dtype)}


def reference(x, residual):
    h = x["X"].double() + (x["R"].double() if residual else 0)
    return h, h / (h.square().mean(-1, keepdim=True) + EPS).sqrt() * x["w"].double()


def inside(got, ref, bound):
    bad = ~((got.double() - ref).abs() <= bound + 1e-38)
    assert not bool(bad.any()), "%d of %d outside, worst %.3g of its bound" % (int(bad.sum()), bad.numel(), float(((got.double() - ref).abs() / (bound + 1e-38)).max()))


def roundings(n):
    return (n / 32 + 16) * 2.0 ** -24


@pytest.mark.parametrize("residual", [False, True], ids=["plain", "residual"])
@pytest.mark.parametrize("dtype", DTYPES, ids=["fp32", "bf16"])
@pytest.mark.parametrize("rows,n", SHAPES)
def test_forward(bnd, rows, n, dtype, residual):
    x = make(rows, n, dtype)
    y, h, s = bnd.rms_norm(x["X"], x["w"], eps=EPS, residual=x["R"] if residual else None)
    assert s is None and (h is None) == (not residual)
    hr, yr = reference(x, residual)
    inside(y, yr, yr.abs() * (STEP[dtype] + roundings(n)) * 1.01 + (2.0 ** -24 * 4 * hr.abs() if residual else 0))
    if residual:
        inside(h, hr, hr.abs() * STEP[dtype] * 1.01 + 2.0 ** -23 * (x["X"].double().abs() + x["R"].double().abs()))


@pytest.mark.parametrize("group", [128, 0])
@pytest.mark.parametrize("dtype", DTYPES, ids=["fp32", "bf16"])
@pytest.mark.parametrize("rows,n", SHAPES)
def test_eight_bits(bnd, rows, n, dtype, group):
    x = make(rows, n, dtype, seed=1)
    x["w"][: n // 2] *= 1e-3           # groups of different size
    if n > 128:
        x["w"][:128] = 0               # a group of zeros
    c, h, s = bnd.rms_norm(x["X"], x["w"], eps=EPS, residual=x["R"], out_dtype=torch.float8_e4m3fn, group=group)
    hr, yr = reference(x, True)
    parts = -(-n // (group or n))
    assert c.dtype == torch.float8_e4m3fn and s.shape == (rows, parts)
    pad = torch.nn.functional.pad(yr, (0, parts * (group or n) - n)).reshape(rows, parts, -1)
    sr = pad.abs().amax(-1) / 448
    sr = torch.where(sr > 0, sr, 1.0)
    inside(s, sr, sr * (roundings(n) + 4 * 2.0 ** -24 + 2.0 ** -22))
    wide = s.double().repeat_interleave(group or n, 1)[:, :n]
    slack = yr.abs() * (roundings(n) + 2.0 ** -21) + 2.0 ** -22 * hr.abs() * x["w"].double().abs()
    inside(c.double() * wide, yr, torch.maximum(yr.abs() * 2.0 ** -4, wide * 2.0 ** -10) * 1.001 + slack)
    assert not bool(torch.isnan(c.float()).any())
    top = torch.nn.functional.pad(c.float().abs(), (0, parts * (group or n) - n)).reshape(rows, parts, -1).amax(-1)
    assert bool(((top == 448) | (top == 0)).all())     # the whole range is used


@pytest.mark.parametrize("past", [False, True], ids=["plain", "past"])
@pytest.mark.parametrize("dtype", DTYPES, ids=["fp32", "bf16"])
@pytest.mark.parametrize("rows,n", SHAPES)
def test_backward(bnd, rows, n, dtype, past):
    x = make(rows, n, dtype, seed=2)
    dx, dw = bnd.rms_norm_backward(x["dY"], x["X"], x["w"], eps=EPS, dH=x["dH"] if past else None)
    X = x["X"].double().requires_grad_()
    w = x["w"].double().requires_grad_()
    y = X / (X.square().mean(-1, keepdim=True) + EPS).sqrt() * w
    (y * x["dY"].double()).sum().backward()
    ref = X.grad + (x["dH"].double() if past else 0)
    rstd = 1 / (X.detach().square().mean(-1, keepdim=True) + EPS).sqrt()
    u = (x["dY"].double() * w.detach()).abs()
    mag = rstd * (u + X.detach().abs() * rstd ** 2 * (u * X.detach().abs()).mean(-1, keepdim=True)) + (x["dH"].double().abs() if past else 0)
    inside(dx, ref, ref.abs() * STEP[dtype] * 1.01 + mag * 4 * roundings(n))
    wmag = (x["dY"].double() * X.detach() * rstd).abs().sum(0)
    inside(dw, w.grad, w.grad.abs() * STEP[dtype] * 1.01 + wmag * (rows / 100 + 700 + n / 32) * 2.0 ** -24)


def test_gradient_against_differences(bnd):
    """A central difference in 64 bits along random directions: its own error is of third order, 1e-8 of the value at a step of 1e-4."""
    x = make(5, 96, torch.float32, seed=3)
    dx, dw = bnd.rms_norm_backward(x["dY"], x["X"], x["w"], eps=EPS)
    g = torch.Generator(device="cuda").manual_seed(0)
    for _ in range(3):
        d, e = torch.randn(5, 96, device="cuda", generator=g, dtype=torch.float64), torch.randn(96, device="cuda", generator=g, dtype=torch.float64)

        def loss(t):
            h = x["X"].double() + t * d
            return float((h / (h.square().mean(-1, keepdim=True) + EPS).sqrt() * (x["w"].double() + t * e) * x["dY"].double()).sum())

        want, have = (loss(1e-4) - loss(-1e-4)) / 2e-4, float((dx.double() * d).sum() + (dw.double() * e).sum())
        assert abs(want - have) <= 1e-4 * float((dx.double() * d).square().sum().sqrt() + (dw.double() * e).square().sum().sqrt() + 1)


@pytest.mark.parametrize("dtype", DTYPES, ids=["fp32", "bf16"])
@pytest.mark.parametrize("n", [130, 2048])
def test_in_place_unaligned_and_leading_dimensions(bnd, n, dtype):
    """H into X or R, pointers off 16 bytes, more leading dimensions, a weight of zeros and rows of zeros."""
    x = make(6, n, dtype, seed=4)
    y, h, _ = bnd.rms_norm(x["X"], x["w"], residual=x["R"])
    for target in ("X", "R"):
        z = {k: v.clone() for k, v in x.items()}
        y2, h2, _ = bnd.rms_norm(z["X"], z["w"], residual=z["R"], residual_out=z[target])
        assert torch.equal(y, y2) and torch.equal(h, z[target])
    off = {k: torch.empty(v.numel() + 1, dtype=dtype, device="cuda")[1:].reshape(v.shape).copy_(v) for k, v in x.items()}
    y3, h3, _ = bnd.rms_norm(off["X"], off["w"], residual=off["R"])
    step = 2 * STEP[dtype]
    assert torch.equal(h, h3) and float((y3.double() - y.double()).abs().max()) <= step * float(y.abs().max()) * (1 + 1e-3) + 1e-6
    y4, h4, _ = bnd.rms_norm(x["X"].reshape(2, 3, n), x["w"], residual=x["R"].reshape(2, 3, n))
    assert torch.equal(y4.reshape(6, n), y)
    dx, dw = bnd.rms_norm_backward(x["dY"], x["X"], x["w"])
    assert torch.equal(bnd.rms_norm_backward(x["dY"], x["X"], x["w"])[1], dw)       # the same bits each time
    x["X"][2] = 0
    y5, _, _ = bnd.rms_norm(x["X"], x["w"])
    assert not bool(y5[2].any()) and not bool(torch.isnan(y5).any())
    c, _, s = bnd.rms_norm(x["X"], torch.zeros_like(x["w"]), out_dtype=torch.float8_e4m3fn)
    assert bool((s == 1).all()) and not bool(c.float().any())
    if dtype == torch.float32:   # values so small that their scale's reciprocal would overflow: the scale stays a normal number, zeros stay zeros
        tiny = torch.full_like(x["w"], 1e-40)
        tiny[:5] = 0
        for group in (128, 0):
            c, _, s = bnd.rms_norm(x["X"], tiny, out_dtype=torch.float8_e4m3fn, group=group)
            assert bool((s >= 2.0 ** -126).all()) and bool(torch.isfinite(c.float()).all()) and not bool(c.float()[:, :5].any())


def test_a_row_that_is_not_finite_stays_alone(bnd):
    x = make(300, 2048, torch.bfloat16, seed=5)
    y, _, _ = bnd.rms_norm(x["X"], x["w"])
    for bad in (float("nan"), float("inf")):
        z = x["X"].clone()
        z[7, 100] = bad
        y2, _, _ = bnd.rms_norm(z, x["w"])
        keep = [i for i in range(300) if i != 7]
        assert torch.equal(y[keep], y2[keep])
        c, _, s = bnd.rms_norm(z, x["w"], out_dtype=torch.float8_e4m3fn)
        c0, _, s0 = bnd.rms_norm(x["X"], x["w"], out_dtype=torch.float8_e4m3fn)
        assert torch.equal(c.float()[keep], c0.float()[keep]) and torch.equal(s[keep], s0[keep])


def test_no_rows(bnd):
    x = make(1, 256, torch.bfloat16)
    y, _, _ = bnd.rms_norm(x["X"][:0], x["w"])
    assert y.shape == (0, 256)
    dx, dw = bnd.rms_norm_backward(x["dY"][:0], x["X"][:0], x["w"])
    assert dx.shape == (0, 256) and not bool(dw.any())


def test_streams_and_graphs(bnd):
    a, b = make(500, 2048, torch.bfloat16, seed=6), make(500, 2048, torch.bfloat16, seed=7)
    call = lambda x, **k: bnd.rms_norm(x["X"], x["w"], residual=x["R"], **k)[:2] + bnd.rms_norm_backward(x["dY"], x["X"], x["w"], dH=x["dH"], **k)   # noqa: E731
    want = [call(x) for x in (a, b)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        got = [call(x, stream=s) for x, s in zip((a, b), streams)]
    torch.cuda.synchronize()
    for p, q in zip(want, got):
        assert all(torch.equal(u, v) for u, v in zip(p, q))
    buf = {k: v.clone() for k, v in a.items()}
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        out = call(buf)
    for k in buf:
        buf[k].copy_(b[k])
    gr.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(u, v) for u, v in zip(want[1], out))
