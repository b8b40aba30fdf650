"""GPU tests of how the gated recurrence and the heads' norm are reached: marshalling, streams, memory, offsets past 2^31, and a run of them with the layers around them."""
import ctypes

import numpy as np
import pytest
import torch

import linear_oracle as lo
import recurrence_oracle as oracle

pytestmark = pytest.mark.gpu

EPS = 1e-6


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


def equal(xs, ys):
    for x, y in zip(xs, ys):
        assert (x is None and y is None) or torch.equal(x, y)


def test_native_marshalling_gives_the_python_bodys_bits(bnd):
    """The extension's calls against the ctypes ones (taken where a stream is named), on slices of one projection."""
    cur, n = torch.cuda.current_stream(), normal(1)
    both = n(1, 500, 3 * 96).bfloat16()
    X, G, dY = both[..., :96], both[..., 96:192], both[..., 192:]
    h0, dh, cu = n(4, 96), n(4, 96), [0, 100, 100, 480, 500]
    for kw in (dict(), dict(want_carries=True), dict(want_state=False), dict(h0=h0[:1]), dict(h0=h0, cu_seqlens=cu), dict(h0=h0, cu_seqlens=np.array(cu, np.int32))):
        for mode in (bnd.REC_NORMED, bnd.REC_GATE):
            a, b = bnd.gated_recurrence(X, G, mode=mode, **kw), bnd.gated_recurrence(X, G, mode=mode, stream=cur, **kw)
            equal(a[:2], b[:2])
    c = bnd.gated_recurrence(X, G, mode=bnd.REC_GATE, h0=h0, cu_seqlens=cu, want_carries=True)[2]
    assert c.shape == (bnd.gated_recurrence_carries(X, cu), 96)
    for kw in (dict(), dict(h0=h0, dh=dh, cu_seqlens=cu), dict(h0=h0, dh=dh, cu_seqlens=cu, carries=c), dict(want_dh0=True), dict(h0=h0[:1], want_dh0=False)):
        equal(bnd.gated_recurrence_backward(dY, X, G, mode=bnd.REC_GATE, **kw), bnd.gated_recurrence_backward(dY, X, G, mode=bnd.REC_GATE, stream=cur, **kw))
    a, b = n(7, 96), None
    b = a.clone()
    equal([bnd.gated_recurrence_step(X[0, :5], G[0, :5], a), a], [bnd.gated_recurrence_step(X[0, :5], G[0, :5], b, stream=cur), b])
    Q, K = both[..., :192].unflatten(-1, (3, 64)), both[..., 192:256].unflatten(-1, (1, 64))
    w, f = n(64).bfloat16(), torch.rand(16, device="cuda")
    pos = torch.randint(-2, 10000, (1, 500), device="cuda").to(torch.int32)
    for kw in (dict(), dict(positions=pos), dict(positions=pos, interleaved=True)):
        for k, wk, freq in ((K, w, f), (None, None, f), (K, None, None)):
            equal(bnd.qk_norm_rope(Q, k, w, wk, freq, **kw), bnd.qk_norm_rope(Q, k, w, wk, freq, stream=cur, **kw))
            equal(bnd.qk_norm_rope_backward(Q, k, Q, k, w, wk, freq, **kw), bnd.qk_norm_rope_backward(Q, k, Q, k, w, wk, freq, stream=cur, **kw))
    for bad in (dict(cu_seqlens=[0, 200, 100, 500]), dict(mode=7)):
        with pytest.raises(bnd.TriInvError) as e:
            bnd.gated_recurrence(X, G, **bad)
        assert e.value.status == bnd.ERR_INVALID_ARG
    with pytest.raises(ValueError, match="G must have shape"):
        bnd.gated_recurrence(X, G[:, :5])
    with pytest.raises(ValueError, match="contiguous within a token"):
        bnd.gated_recurrence(both[..., ::3], both[..., ::3])
    with pytest.raises(TypeError, match="positions"):
        bnd.qk_norm_rope(Q, K, w, w, f, positions=pos.long())
    with pytest.raises(bnd.TriInvError):
        bnd.qk_norm_rope(Q, K, w, w, torch.rand(33, device="cuda"))


def test_named_streams_take_their_own_memory(bnd):
    """Outputs and workspaces of a call on another stream come out of that stream's memory, not out of blocks that work queued on the current one may still write."""
    n, side = normal(2), torch.cuda.Stream()
    X, G = n(4, 2000, 512).bfloat16(), -torch.rand(4, 2000, 512, device="cuda").bfloat16()
    want = bnd.gated_recurrence(X, G, mode=bnd.REC_NORMED)
    Q, w, f = n(4, 2000, 8, 64).bfloat16(), torch.ones(64, device="cuda").bfloat16(), torch.rand(32, device="cuda")
    want_heads = bnd.qk_norm_rope_backward(Q, Q, Q, Q, w, w, f)
    torch.cuda.synchronize()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(4):
        junk = [torch.empty_like(X) for _ in range(4)] + [torch.empty(4 << 20, device="cuda")]
        torch.cuda._sleep(2_000_000)
        for t in junk:
            t.fill_(float("nan"))
        del junk, t
        got = bnd.gated_recurrence(X, G, mode=bnd.REC_NORMED, stream=side)
        got_heads = bnd.qk_norm_rope_backward(Q, Q, Q, Q, w, w, f, stream=side)
        torch.cuda.synchronize()
        equal(got[:2], want[:2])
        equal(got_heads, want_heads)


def test_nothing_is_allocated(bnd):
    n, L = normal(3), bnd.load()
    B, T, D, H, d = 2, 1500, 192, 3, 64
    X, G, dY = (n(B, T, D).bfloat16() for _ in range(3))
    Y, dX, dG = (torch.empty_like(X) for _ in range(3))
    h0, h1, dh0, cache = n(B, D), n(B, D), n(B, D), n(T, D)
    w, f = n(d).bfloat16(), torch.rand(32, device="cuda")
    dwq, dwk = torch.empty_like(w), torch.empty_like(w)
    desc, step, heads = bnd.RecDesc(B, T, D, bnd.BF16, bnd.REC_GATE, 0, None), bnd.RecDesc(T, 1, D, bnd.BF16, bnd.REC_GATE, 0, None), bnd.HeadsDesc(B * T, T, H, H, d, 32, 0, bnd.BF16, EPS)
    need = ctypes.c_size_t(0)
    work = []
    for q, a in (("gated_recurrence", (desc,)), ("gated_recurrence_backward", (desc, 0)), ("gated_recurrence_backward", (desc, 1)), ("qk_norm_rope_backward", (heads,))):
        assert getattr(L, "tri_inv_%s_workspace" % q)(*a, need) == 0 and need.value > 0
        work.append((torch.empty(need.value, dtype=torch.uint8, device="cuda").fill_(0xAB), need.value))
    carries = torch.empty(bnd.gated_recurrence_carries(X), D, device="cuda")
    p = lambda t: t.data_ptr()   # noqa: E731

    def calls():
        W = [(t.data_ptr(), m) for t, m in work]
        assert L.tri_inv_gated_recurrence(p(X), D, p(G), D, p(h0), p(Y), D, p(h1), p(carries), *W[0], desc, None) == 0
        assert L.tri_inv_gated_recurrence_backward(p(dY), D, p(X), D, p(G), D, p(h0), p(h1), None, p(dX), D, p(dG), D, p(dh0), *W[1], desc, None) == 0
        assert L.tri_inv_gated_recurrence_backward(p(dY), D, p(X), D, p(G), D, p(h0), p(h1), p(carries), p(dX), D, p(dG), D, p(dh0), *W[2], desc, None) == 0
        assert L.tri_inv_gated_recurrence_step(p(X), D, p(G), D, p(cache), None, T, p(Y), D, step, None) == 0
        assert L.tri_inv_qk_norm_rope(p(X), D, p(G), D, p(w), p(w), p(f), None, p(Y), D, p(dX), D, heads, None) == 0
        assert L.tri_inv_qk_norm_rope_backward(p(dY), D, p(Y), D, p(X), D, p(G), D, p(w), p(w), p(f), None, p(dX), D, p(dG), D, p(dwq), p(dwk), *W[3], heads, None) == 0

    calls()
    torch.cuda.synchronize()
    free, reserved = torch.cuda.mem_get_info()[0], torch.cuda.memory_reserved()
    for _ in range(3):
        calls()
    torch.cuda.synchronize()
    assert torch.cuda.mem_get_info()[0] == free and torch.cuda.memory_reserved() == reserved
    assert bnd.last_device_status() == 0


def test_offsets_past_two_to_the_31st(bnd):
    """Tensors of more than 2^31 elements: the last sequence against the same one alone."""
    B, T, D = 33, 8192, 8192
    n = normal(4)
    x, g = n(1, T, D).bfloat16(), -torch.rand(1, T, D, device="cuda").bfloat16()
    X, G = x.expand(B, T, D).contiguous(), g.expand(B, T, D).contiguous()
    Y, S, c = bnd.gated_recurrence(X, G, want_carries=True)
    y, s, _ = bnd.gated_recurrence(x, g)
    assert torch.equal(Y[-1], y[0]) and torch.equal(Y[0], y[0]) and torch.equal(S[-1], s[0])
    dX, dG, _ = bnd.gated_recurrence_backward(Y, X, G, carries=c)
    dx, dg, _ = bnd.gated_recurrence_backward(y, x, g)
    assert torch.equal(dX[-1], dx[0]) and torch.equal(dG[-1], dg[0])
    del Y, dX, dG, G, c
    w, f = torch.ones(128, device="cuda").bfloat16(), torch.rand(64, device="cuda")
    Q = X.view(B, T, 64, 128)
    out = bnd.qk_norm_rope(Q, None, w, None, f)[0]
    assert torch.equal(out[-1], bnd.qk_norm_rope(x.view(1, T, 64, 128), None, w, None, f)[0][0])
    dQ = bnd.qk_norm_rope_backward(Q, None, Q, None, w, None, f, out=(out, None))[0]
    assert torch.equal(dQ[-1], bnd.qk_norm_rope_backward(x.view(1, T, 64, 128), None, x.view(1, T, 64, 128), None, w, None, f)[0][0])
    assert bnd.last_device_status() == 0


class _Norm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, bnd, X, w):
        ctx.bnd = bnd
        ctx.save_for_backward(X, w)
        return bnd.rms_norm(X, w, eps=EPS)[0]

    @staticmethod
    def backward(ctx, dY):
        return (None, *ctx.bnd.rms_norm_backward(dY.contiguous(), *ctx.saved_tensors, eps=EPS))


class _Heads(torch.autograd.Function):
    @staticmethod
    def forward(ctx, bnd, Q, K, wq, wk, f, pos):
        ctx.bnd = bnd
        ctx.save_for_backward(Q, K, wq, wk, f, pos)
        return bnd.qk_norm_rope(Q, K, wq, wk, f, positions=pos, eps=EPS)

    @staticmethod
    def backward(ctx, dQ, dK):
        Q, K, wq, wk, f, pos = ctx.saved_tensors
        return (None, *ctx.bnd.qk_norm_rope_backward(dQ.contiguous(), dK.contiguous(), Q, K, wq, wk, f, positions=pos, eps=EPS), None, None)


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, bnd, Q, K, V, ld):
        ctx.bnd = bnd
        ctx.save_for_backward(Q, K, V, ld)
        return bnd.linear_attention(Q, K, V, ld, scale=0.2)[0]

    @staticmethod
    def backward(ctx, dO):
        return (None, *ctx.bnd.linear_attention_backward(dO.contiguous(), *ctx.saved_tensors, scale=0.2)[:3], None)


class _Recurrence(torch.autograd.Function):
    @staticmethod
    def forward(ctx, bnd, X, G):
        ctx.bnd = bnd
        Y, _, carries = bnd.gated_recurrence(X, G, mode=bnd.REC_GATE, want_carries=True)
        ctx.save_for_backward(X, G, carries)
        return Y

    @staticmethod
    def backward(ctx, dY):
        X, G, carries = ctx.saved_tensors
        return (None, *ctx.bnd.gated_recurrence_backward(dY.contiguous(), X, G, mode=ctx.bnd.REC_GATE, carries=carries)[:2])


def _layers(x, p, pos, norm, heads, attention, recurrence):
    """A block of a gated recurrence, then one of linear attention on normed and turned heads, each behind a norm and added to its input."""
    B, T, D = x.shape
    H, d = 3, D // 3
    a = norm(x, p["n1"]) @ p["w1"]
    x = x + recurrence(a[..., :D], a[..., D:]) @ p["w2"]
    a = norm(x, p["n2"]) @ p["w3"]
    q, k, v = (a[..., i * D:(i + 1) * D].unflatten(-1, (H, d)) for i in range(3))
    q, k = heads(q, k, p["wq"], p["wk"], pos)
    return x + attention(q, k, v.contiguous()).flatten(-2) @ p["w4"]


def test_layers_together(bnd):
    """Forward and gradients of two layers of these calls in fp32 against the same layers in 64 bits by autograd.  Bound: each of the ten stages in a row rounds to 2^-24 in sums of at most 288 terms and
    passes errors on with factors of a few; 2^-24 x 288 x 10 = 1.7e-4 of the largest value."""
    B, T, D = 2, 150, 96
    n = normal(5)
    p = {"n1": 1 + 0.1 * n(D), "n2": 1 + 0.1 * n(D), "w1": n(D, 2 * D) / 10, "w2": n(D, D) / 10, "w3": n(D, 3 * D) / 10, "w4": n(D, D) / 10, "wq": 1 + 0.1 * n(32), "wk": 1 + 0.1 * n(32)}
    x, dy = n(B, T, D), n(B, T, D)
    pos = (torch.arange(T, device="cuda") + torch.tensor([[0], [5000]], device="cuda")).to(torch.int32)
    f = (100.0 ** (-torch.arange(16, device="cuda") / 16.0)).float()
    ld = -torch.tensor([0.5, 0.1, 0.01], device="cuda")
    leaves = [t.clone().requires_grad_() for t in (x, *p.values())]
    out = _layers(leaves[0], dict(zip(p, leaves[1:])), pos, lambda t, w: _Norm.apply(bnd, t, w), lambda q, k, wq, wk, s: _Heads.apply(bnd, q, k, wq, wk, f, s),
                  lambda q, k, v: _Attention.apply(bnd, q.contiguous(), k.contiguous(), v, ld), lambda a, g: _Recurrence.apply(bnd, a, g))
    grads = torch.autograd.grad(out, leaves, dy)

    def norm64(t, w):
        return t / (t.square().mean(-1, keepdim=True) + EPS).sqrt() * w

    def heads64(q, k, wq, wk, s):
        angle = (s.double()[..., None] * f.double())[:, :, None]
        outs = []
        for t, w in ((q, wq), (k, wk)):
            t = norm64(t, w)
            u, v = t[..., :16], t[..., 16:]
            outs.append(torch.cat([u * angle.cos() - v * angle.sin(), v * angle.cos() + u * angle.sin()], -1))
        return outs

    def attention64(q, k, v):
        i = torch.arange(T, device="cuda")
        w = torch.where(i[:, None] >= i, torch.exp(ld.double()[:, None, None] * (i[:, None] - i).clamp(min=0)), 0.0)
        return 0.2 * torch.einsum("bhij,hij,bjhd->bihd", torch.einsum("bihd,bjhd->bhij", q, k), w, v)

    def recurrence64(a, g):
        h, hs = torch.zeros(B, D, dtype=torch.float64, device="cuda"), []
        for t in range(T):
            s = torch.sigmoid(g[:, t])
            h = s * h + (1 - s) * a[:, t]
            hs.append(h)
        return torch.stack(hs, 1)

    leaves64 = [t.double().requires_grad_() for t in (x, *p.values())]
    out64 = _layers(leaves64[0], dict(zip(p, leaves64[1:])), pos, norm64, heads64, attention64, recurrence64)
    grads64 = torch.autograd.grad(out64, leaves64, dy.double())
    for a, b in zip((out, *grads), (out64, *grads64)):
        assert float((a.double() - b).detach().abs().max()) <= 1.7e-4 * float(b.detach().abs().max())
    assert bnd.last_device_status() == 0


def test_serving_together(bnd):
    """Prompt, then single tokens, through both layers' states: the tokens' outputs are those of one prompt over all of them (fp32: the recurrence to the bound of its steps, the attention as its own tests bound it)."""
    B, T, more, H, d = 3, 200, 4, 2, 64
    n = normal(6)
    X, G = n(B, T + more, H * d), n(B, T + more, H * d)
    Q, K, V = (n(B, T + more, H, d) for _ in range(3))
    w, f = 1 + 0.1 * n(d), (1000.0 ** (-torch.arange(32, device="cuda") / 32.0)).float()
    ld = -torch.tensor([0.3, 0.02], device="cuda")
    pos = torch.arange(T + more, device="cuda", dtype=torch.int32).expand(B, -1).contiguous()
    q, k = bnd.qk_norm_rope(Q, K, w, w, f, positions=pos)
    want = bnd.linear_attention(q, k, V, ld)[0]
    mag = lo.forward(q.abs(), k.abs(), V.abs(), ld, 1.0, None, None)[0]
    cache = torch.zeros(B + 2, H * d, device="cuda")
    slots = torch.tensor([4, 0, 2], dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="one distance"):   # the sequences of a dense batch follow one another
        bnd.gated_recurrence(X[:, :T], G[:, :T], mode=bnd.REC_GATE)
    _, state, _ = bnd.gated_recurrence(X[:, :T].contiguous(), G[:, :T].contiguous(), mode=bnd.REC_GATE)
    cache[slots.long()] = state
    S = bnd.linear_attention(q[:, :T].contiguous(), k[:, :T].contiguous(), V[:, :T].contiguous(), ld)[1]
    ref = oracle.walk(X, G, oracle.GATE, [T + more] * B, None)
    for t in range(T, T + more):
        y = bnd.gated_recurrence_step(X[:, t], G[:, t], cache, mode=bnd.REC_GATE, slots=slots)
        oracle.inside(y, ref["h"].view(B, T + more, -1)[:, t], ref["eh"].view(B, T + more, -1)[:, t])
        qt, kt = bnd.qk_norm_rope(Q[:, t:t + 1], K[:, t:t + 1], w, w, f, positions=pos[:, t:t + 1].contiguous())
        assert torch.equal(qt[:, 0], q[:, t]) and torch.equal(kt[:, 0], k[:, t])
        o = bnd.linear_attention_step(qt[:, 0].contiguous(), kt[:, 0].contiguous(), V[:, t].contiguous(), ld, S)
        assert bool(((o - want[:, t]).double().abs() <= 1000 * 2.0 ** -24 * mag[:, t]).all())   # sums of 64 features and 200 tokens on both sides, each in a few roundings
    assert bnd.last_device_status() == 0
