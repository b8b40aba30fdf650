"""GPU tests of the gated recurrence and of the heads' norm at the edges of what their header allows."""
from fractions import Fraction

import pytest
import torch

import recurrence_oracle as oracle

pytestmark = pytest.mark.gpu

ULP = 2.0 ** -24
STORE = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
DTYPES = [torch.float32, torch.bfloat16]
MODES = [oracle.DECAY, oracle.NORMED, oracle.GATE]
NAMES = {"ids": ["decay", "normed", "gate"]}


@pytest.fixture(scope="module")
def bnd():
    import __graft_entry__ as entry
    entry.build()
    from paper_2605_21325_b200 import binding
    torch.cuda.set_device(0)
    return binding


def normal(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return lambda *s: torch.randn(*s, device="cuda", generator=g)


@pytest.mark.parametrize("dtype", DTYPES, ids=["fp32", "bf16"])
@pytest.mark.parametrize("Hq,Hk", [(3, 0), (0, 3), (0, 0)])
def test_weights_of_a_side_without_heads_have_zero_gradients(bnd, Hq, Hk, dtype):
    """Sums over no heads, written all the same: whatever the memory held."""
    n, d = normal(1), 64
    Q, K = n(2, 5, Hq, d).to(dtype), n(2, 5, Hk, d).to(dtype)
    w, f = torch.ones(d, device="cuda").to(dtype), torch.rand(32, device="cuda")
    junk = [torch.full((d,), 7.0, dtype=dtype, device="cuda") for _ in range(8)]
    del junk
    for H, got in zip((Hq, Hk), bnd.qk_norm_rope_backward(Q, K, Q, K, w, w, f)[2:]):
        assert bool((got != 0).any()) == (H > 0)
    dw = [torch.full((d,), 7.0, dtype=dtype, device="cuda") for _ in range(2)]
    desc = bnd.HeadsDesc(10, 5, Hq, Hk, d, 32, 0, bnd._dtype_code(w), 1e-6)
    need = bnd._workspace("tri_inv_qk_norm_rope_backward_workspace", desc)
    work, dQ, dK, p = torch.empty(need, dtype=torch.uint8, device="cuda"), torch.empty_like(Q), torch.empty_like(K), lambda t: t.data_ptr()   # noqa: E731
    ld = Hq * d, Hk * d
    assert bnd.load().tri_inv_qk_norm_rope_backward(p(Q), ld[0], p(K), ld[1], p(Q), ld[0], p(K), ld[1], p(w), p(w), p(f), None, p(dQ), ld[0], p(dK), ld[1], *map(p, dw), p(work), need, desc,
                                                    torch.cuda.current_stream().cuda_stream) == bnd.OK
    for H, got in zip((Hq, Hk), dw):
        assert bool((got == 0).all()) == (H == 0) and not bool((got == 7).all())


@pytest.mark.parametrize("dtype", DTYPES, ids=["fp32", "bf16"])
@pytest.mark.parametrize("d", [64, 7])
def test_gradient_of_small_and_large_heads_without_eps(bnd, d, dtype):
    """Heads of 1e-17 to 1e17: squares, their sum and the gradient are normal numbers of fp32, and so is all that lies between.  48 roundings, as the gradient's other tests count them."""
    n = normal(5)
    scale = 10.0 ** torch.tensor([-17.0, -14.0, -13.0, -9.0, 0.0, 9.0, 13.0, 15.0, 17.0], device="cuda")
    Q, dQ = (n(1, 9, 2, d) * scale[:, None, None]).to(dtype), n(1, 9, 2, d).to(dtype)
    w = (1 + 0.2 * n(d)).to(dtype)
    got = bnd.qk_norm_rope_backward(dQ, None, Q, None, w, None, None, eps=0.0)[0]
    x, u = Q.double(), dQ.double() * w.double()
    rstd = 1 / x.square().mean(-1, keepdim=True).sqrt()
    ref = rstd * (u - x * (rstd ** 2 * (u * x).mean(-1, keepdim=True)))
    bound = 48 * ULP * rstd * (u.abs() + x.abs() * (rstd ** 2 * (u * x).abs().mean(-1, keepdim=True)))
    off = (got.double() - ref).abs() / (1.01 * (bound + STORE[dtype] * ref.abs()))
    assert bool((off <= 1).all()), off.amax((0, 2, 3))


def over_two_pi(bits):
    """floor(2^bits / 2 pi), with pi = 16 arctan(1/5) - 4 arctan(1/239) (Machin)."""
    one, pi = 1 << (bits + 64), 0
    for c, x in ((16, 5), (-4, 239)):
        k, term = 0, one // x
        while term:
            pi += c * (term // (2 * k + 1)) * (-1) ** k
            term //= x * x
            k += 1
    return (one << bits) // (2 * pi)


@pytest.mark.parametrize("f", [1e-3, -1e-3, 0.5, 1.0, -3.0, 10.0, 1000.0, -12345.678, 1e9, 3e38])
def test_angles_at_any_position_and_frequency(bnd, f):
    """Angles to 2^-25 of a turn (pi roundings of 2^-24 in radians), against exact ones.  x = (1, 1) without eps: the norm's root 2, two products 2, sine and cosine 2 each of |u| + |v|, two products and a sum 3:
    12 with the angle's."""
    BITS = 420
    g = torch.Generator().manual_seed(6)
    pos = torch.cat([torch.tensor([0, 1, 2 ** 31 - 1]), torch.randint(2 ** 30, 2 ** 31 - 1, (200,), generator=g), torch.randint(0, 100000, (53,), generator=g)]).to(torch.int32)
    freq = torch.tensor([f], dtype=torch.float32)
    exact, by = Fraction(float(freq[0])), over_two_pi(BITS)
    turns = [int(p) * exact * by for p in pos.tolist()]                                # in 2^-BITS of a turn
    angle = torch.tensor([float((t / 2 ** BITS) % 1) for t in turns], dtype=torch.float64) * 2 * torch.pi
    Q = torch.ones(1, len(pos), 1, 2, device="cuda")
    got = bnd.qk_norm_rope(Q, None, None, None, freq.cuda(), positions=pos.cuda()[None], eps=0.0)[0][0, :, 0].double().cpu()
    want = torch.stack([angle.cos() - angle.sin(), angle.cos() + angle.sin()], -1)
    off = (got - want).abs() / (12 * ULP * 2)
    assert bool((off <= 1).all()), float(off.max())
    back = bnd.qk_norm_rope_backward(torch.ones_like(Q), None, 2 * Q + torch.tensor([1.0, -1.0], device="cuda"), None, None, None, freq.cuda(), positions=pos.cuda()[None], eps=0.0)[0]
    # v = R(-p) (1, 1) = (c + s, c - s) at x = (3, 1): mean square 5, dx = (v - x (v . x) / 10) / sqrt 5
    v = torch.stack([angle.cos() + angle.sin(), angle.cos() - angle.sin()], -1)
    x = torch.tensor([3.0, 1.0], dtype=torch.float64)
    dx = (v - x * (v @ x)[:, None] / 10) / 5 ** 0.5
    assert float((back[0, :, 0].double().cpu() - dx).abs().max()) <= 48 * ULP * (2 + 3 * 8 / 10) / 5 ** 0.5


@pytest.mark.parametrize("dtype", DTYPES, ids=["fp32", "bf16"])
def test_gates_that_are_not_numbers_reach_the_input_s_gradient(bnd, dtype):
    """u = sqrt(1 - a^2) x: where a is not a number neither is dx = sqrt(1 - a^2) e, although e is."""
    n = normal(2)
    X, G, dY = n(1, 300, 40).to(dtype), -torch.rand(1, 300, 40, device="cuda").to(dtype), n(1, 300, 40).to(dtype)
    for t, c in ((0, 3), (77, 4), (150, 9), (299, 39)):
        G[0, t, c] = float("nan")
    got = bnd.gated_recurrence_backward(dY, X, G, mode=bnd.REC_NORMED, want_dh0=True)
    for x, (r, e) in zip(got, oracle.gradient(X, G, oracle.NORMED, [300], None, dY, None)):
        oracle.inside(x, r, e)


def faded(a, back=False):
    """Where a state (or, from behind, what reaches a token) is no number because of a decay that is none, and the decays since then come to less than e^-100: below 2^-149 = e^-103 it may be forgotten."""
    out = torch.zeros_like(a, dtype=torch.bool)
    tainted, since = out[0].clone(), torch.zeros_like(a[0])
    for t in reversed(range(len(a))) if back else range(len(a)):
        if back:
            out[t] = tainted & (since < -100)
        bad, reset = torch.isnan(a[t]), a[t] == 0
        tainted = (tainted | bad) & ~reset
        since = torch.where(bad, 0.0, since + torch.where(bad | reset, 1.0, a[t]).log())
        if not back:
            out[t] = tainted & (since < -100)
    return out


@pytest.mark.parametrize("T", [300, 900])
@pytest.mark.parametrize("mode", MODES, **NAMES)
@pytest.mark.parametrize("dtype", DTYPES, ids=["fp32", "bf16"])
def test_resets_forget_gates_that_are_not_numbers(bnd, dtype, mode, T):
    """A decay of zero leaves nothing of what came before it, a decay that is not a number included, and of what comes back from behind it: in the same lane's tokens, other lanes', other warps', and tiles on."""
    D = 70
    n = normal(3)
    X, G, dY, h0, dh = n(1, T, D).to(dtype), n(1, T, D), n(1, T, D).to(dtype), n(1, D), n(1, D)
    G = (G if mode == oracle.GATE else -0.2 * G.abs()).to(dtype)
    for before, bad, reset, c in ((3, 5, 9, 0), (2, 6, 20, 1), (10, 20, 40, 2), (20, 40, 100, 3), (60, 100, 140, 4), (100, 130, 290, 5), (298, 0, 299, 6)):
        G[0, bad, c::7] = float("nan")
        G[0, [before, reset], c::7] = float("-inf")
    if T > 300:
        G[0, 200, 2::7] = float("nan")
        G[0, 850, 2::7] = float("-inf")
    Y, S, carries = bnd.gated_recurrence(X, G, mode=mode, h0=h0, want_carries=True)
    f = oracle.walk(X, G, mode, [T], h0)
    a = oracle.factors(G[0], mode)[0]
    h_faded, e_faded = faded(a), faded(a, back=True)
    before = torch.cat([torch.zeros_like(h_faded[:1]), h_faded[:-1]])
    oracle.inside(torch.where(h_faded, f["h"].to(dtype), Y[0]), f["h"], f["eh"])
    oracle.inside(S, f["state"], f["estate"])
    assert bool(torch.isfinite(S).all()) and bool(torch.isnan(Y).any())
    ref = oracle.gradient(X, G, mode, [T], h0, dY, dh)
    for c in (carries, None):
        for x, (r, e), either in zip(bnd.gated_recurrence_backward(dY, X, G, mode=mode, h0=h0, dh=dh, carries=c, want_dh0=True), ref, (e_faded, e_faded | before, torch.zeros(1, D, dtype=torch.bool, device="cuda"))):
            oracle.inside(torch.where(either, r.to(x.dtype), x.view(r.shape)), r, e)
        assert not bool(torch.isnan(ref[2][0]).view(-1, 7)[:, :6].any())
    assert bnd.last_device_status() == 0


@pytest.mark.parametrize("D", [1, 33, 45])
def test_channels_that_fill_part_of_a_warp(bnd, D):
    """Long walks of channels that leave lanes without one, whose lanes wait for words for different times: right, and the same bits each time."""
    mode, T = oracle.GATE, 4000
    n = normal(4)
    X, G, dY, h0, dh = n(2, T, D).bfloat16(), (n(2, T, D) + 3).bfloat16(), n(2, T, D).bfloat16(), n(2, D), n(2, D)
    call = lambda: bnd.gated_recurrence(X, G, mode=mode, h0=h0)[:2] + bnd.gated_recurrence_backward(dY, X, G, mode=mode, h0=h0, dh=dh)   # noqa: E731
    first = call()
    f = oracle.walk(X, G, mode, [T] * 2, h0)
    for x, (r, e) in zip(first, ((f["h"], f["eh"]), (f["state"], f["estate"]), *oracle.gradient(X, G, mode, [T] * 2, h0, dY, dh))):
        oracle.inside(x, r, e)
    for _ in range(10):
        assert all(torch.equal(x, y) for x, y in zip(call(), first))
    assert bnd.last_device_status() == 0


def test_the_self_test_checks_its_tensors(bnd):
    """Refused on the host: the call has one type and one shape."""
    X = torch.zeros(1, 400, 40, device="cuda")
    for G, out in ((X.bfloat16(), X), (X, X.bfloat16())):
        with pytest.raises(TypeError, match="must be"):
            bnd.selftest_recurrence_wait_timeout(X, G, 1000, out)
    for G, out in ((X[:, :200], X), (X, X[:, :200]), (X.cpu(), X)):
        with pytest.raises(ValueError, match="must"):
            bnd.selftest_recurrence_wait_timeout(X, G, 1000, out)
    assert bnd.last_device_status() == 0


def test_a_wait_that_runs_out_leaves_the_other_tiles_alone(bnd):
    """The first tile of the first 32 channels is never announced: its own 128 tokens and all other channels are as usual, and what its channels hold behind it says so, as long as no product of decays could forget it."""
    n = normal(7)
    X, G = n(1, 400, 100).bfloat16(), (-0.5 * torch.rand(1, 400, 100, device="cuda")).bfloat16()
    Y = torch.zeros_like(X)
    bnd.selftest_recurrence_wait_timeout(X, G, 2_000_000, Y)
    assert bnd.last_device_status() == bnd.ERR_DEVICE_TIMEOUT
    f = oracle.walk(X, G, oracle.DECAY, [400], None)
    oracle.inside(Y[0, :128, :32], f["h"][:128, :32], f["eh"][:128, :32])
    oracle.inside(Y[0, :, 32:], f["h"][:, 32:], f["eh"][:, 32:])
    kept = G[0, 128:, :32].double().cumsum(0) > -80                                   # e^-80 is a normal number
    assert bool(torch.isnan(Y[0, 128:, :32])[kept].all()) and int(kept.sum()) > 5000
