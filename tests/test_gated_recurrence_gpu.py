"""GPU tests of the gated linear recurrence, its gradient and its single token against the recurrence in 64 bits (bounds: recurrence_oracle)."""
import pytest
import torch

import recurrence_oracle as oracle

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16]
MODES = [oracle.DECAY, oracle.NORMED, oracle.GATE]
NAMES = {"ids": ["decay", "normed", "gate"]}
# (lengths, D, packed): one token, tiles' edges, odd widths, many sequences, long ones
SHAPES = [([1], 1, False), ([1] * 3, 33, False), ([63], 64, False), ([64], 65, False), ([65] * 2, 31, False), ([128] * 3, 128, False), ([333], 200, False), ([1000] * 2, 72, False),
          ([700] * 9, 1100, False), ([5000], 6, False), ([17, 0, 64, 65, 1, 200, 0, 129], 40, True), ([3, 300, 1], 129, True), ([0, 0], 10, True), ([1] * 400, 16, True), ([64] * 40, 257, True),
          ([1000, 5, 0, 450, 129, 640], 40, True), ([400 + i % 3 for i in range(330)], 33, True)]


@pytest.fixture(scope="module")
def bnd():
    import __graft_entry__ as entry
    entry.build()
    from paper_2605_21325_b200 import binding
    torch.cuda.set_device(0)
    return binding


def make(lens, D, packed, dtype, mode, state=True, seed=0):
    g = torch.Generator(device="cuda").manual_seed(1000 * sum(lens) + D + seed)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)   # noqa: E731
    B, T = (1, sum(lens)) if packed else (len(lens), lens[0])
    spread = 2.0 ** (-8.0 * torch.rand(D, device="cuda", generator=g))
    z = r(B, T, D)
    G = z - torch.log(spread) if mode == oracle.GATE else -2 * spread * torch.sigmoid(z)
    n = len(lens)
    return dict(X=r(B, T, D).to(dtype), G=G.to(dtype), dY=r(B, T, D).to(dtype), h0=2 * r(n, D) if state else None, dh=r(n, D) if state else None,
                cu=[sum(lens[:i]) for i in range(n + 1)] if packed else None)


def check_forward(b, s, mode, lens, Y, S, carries=None):
    f = oracle.walk(s["X"], s["G"], mode, lens, s["h0"])
    oracle.inside(Y, f["h"], f["eh"])
    if S is not None:
        oracle.inside(S, f["state"], f["estate"])
    if carries is not None:
        for q, n in enumerate(lens):
            first = int(f["begin"][q])
            k = (n - 1) // b.REC_TILE
            if k > 0:
                at = first + b.REC_TILE * torch.arange(1, k + 1, device="cuda") - 1
                rows = first // b.REC_TILE + q + torch.arange(k, device="cuda")
                oracle.inside(carries[rows], f["h"][at], f["eh"][at])


@pytest.mark.parametrize("state", [False, True], ids=["zero", "states"])
@pytest.mark.parametrize("mode", MODES, **NAMES)
@pytest.mark.parametrize("dtype", DTYPES, ids=["fp32", "bf16"])
@pytest.mark.parametrize("lens,D,packed", SHAPES, ids=["%dx%d%s" % (len(s[0]), max(s[0]), "x%d" % s[1] + "p" * s[2]) for s in SHAPES])
def test_forward_and_gradient(bnd, lens, D, packed, dtype, mode, state):
    s = make(lens, D, packed, dtype, mode, state)
    Y, S, carries = bnd.gated_recurrence(s["X"], s["G"], mode=mode, h0=s["h0"], cu_seqlens=s["cu"], want_carries=True)
    check_forward(bnd, s, mode, lens, Y, S, carries)
    ref = oracle.gradient(s["X"], s["G"], mode, lens, s["h0"], s["dY"], s["dh"])
    for c in (carries, None):
        got = bnd.gated_recurrence_backward(s["dY"], s["X"], s["G"], mode=mode, h0=s["h0"], dh=s["dh"], carries=c, cu_seqlens=s["cu"], want_dh0=True)
        for x, (r, e) in zip(got, ref):
            oracle.inside(x, r, e)
    assert bnd.last_device_status() == 0


@pytest.mark.parametrize("dtype", DTYPES, ids=["fp32", "bf16"])
@pytest.mark.parametrize("offset,pad", [(0, 8), (8, 0), (2, 2), (1, 0), (0, 1), (1, 1)])
def test_strides_and_alignment(bnd, dtype, offset, pad):
    """Slices of one projection's output at any place, outputs into slices of one gradient."""
    B, T, D, mode = 2, 150, 90, oracle.GATE
    s = make([T] * B, D, False, dtype, mode)
    width = 3 * D + pad + offset
    both = torch.zeros(B, T, width, dtype=dtype, device="cuda")
    X, G, dY = both[..., offset:offset + D], both[..., offset + D:offset + 2 * D], both[..., offset + 2 * D:offset + 3 * D]
    for t, v in ((X, s["X"]), (G, s["G"]), (dY, s["dY"])):
        t.copy_(v)
    grads = torch.full((B, T, width), 7.0, dtype=dtype, device="cuda")
    Y, dX, dG = grads[..., offset:offset + D], grads[..., offset + D:offset + 2 * D], grads[..., offset + 2 * D:offset + 3 * D]
    _, S, carries = bnd.gated_recurrence(X, G, mode=mode, h0=s["h0"], out=Y, want_carries=True)
    check_forward(bnd, s, mode, [T] * B, Y, S, carries)
    out = bnd.gated_recurrence_backward(dY, X, G, mode=mode, h0=s["h0"], dh=s["dh"], carries=carries, out=(dX, dG))
    for x, (r, e) in zip(out, oracle.gradient(s["X"], s["G"], mode, [T] * B, s["h0"], s["dY"], s["dh"])):
        oracle.inside(x, r, e)
    assert bool((grads[..., :offset] == 7).all()) and bool((grads[..., offset + 3 * D:] == 7).all())   # what lies between is not written


@pytest.mark.parametrize("D", [64, 50])
def test_in_place(bnd, D):
    lens, mode = [300] * 2, oracle.NORMED
    s = make(lens, D, False, torch.bfloat16, mode)
    f = oracle.walk(s["X"], s["G"], mode, lens, s["h0"])
    for name in ("X", "G"):
        t = {k: s[k].clone() for k in ("X", "G")}
        h = s["h0"].clone()
        Y, S, _ = bnd.gated_recurrence(t["X"], t["G"], mode=mode, h0=h, out=t[name], state_out=h)
        assert Y is t[name] and S is h
        oracle.inside(Y, f["h"], f["eh"])
        oracle.inside(S, f["state"], f["estate"])
    ref = oracle.gradient(s["X"], s["G"], mode, lens, s["h0"], s["dY"], s["dh"])
    for over in (("X", "G"), ("dY", "G"), ("X", "dY")):
        t = {k: s[k].clone() for k in ("X", "G", "dY")}
        got = bnd.gated_recurrence_backward(t["dY"], t["X"], t["G"], mode=mode, h0=s["h0"], dh=s["dh"], out=(t[over[0]], t[over[1]]))
        for x, (r, e) in zip(got, ref):
            oracle.inside(x, r, e)


@pytest.mark.parametrize("mode", MODES, **NAMES)
def test_resets_forget_everything(bnd, mode):
    """A decay of zero: nothing of what came before is left, NaN and infinities included, and no gradient passes."""
    lens, D = [400], 70
    s = make(lens, D, False, torch.float32, mode)
    for t, bad in ((40, float("nan")), (130, float("inf")), (260, float("-inf"))):
        s["X"][0, t, ::3] = bad
    for t in (41, 64, 128, 191, 300, 301, 302):
        s["G"][0, t] = float("-inf")
    Y, S, carries = bnd.gated_recurrence(s["X"], s["G"], mode=mode, h0=s["h0"], want_carries=True)
    check_forward(bnd, s, mode, lens, Y, S)
    assert bool(torch.isfinite(Y[0, 41:64]).all()) and bool(torch.isfinite(Y[0, 300:]).all()) and bool(torch.isnan(Y[0, 40, ::3]).all())
    dY = s["dY"].clone()
    dY[0, 128, 1] = float("nan")
    dY[0, 300, 2] = float("inf")
    clean = make(lens, D, False, torch.float32, mode)["X"]
    got = bnd.gated_recurrence_backward(dY, clean, s["G"], mode=mode, h0=s["h0"], dh=s["dh"])
    for x, (r, e) in zip(got, oracle.gradient(clean, s["G"], mode, lens, s["h0"], dY, s["dh"])):
        oracle.inside(x, r, e)
    assert bool(torch.isfinite(got[0][0, :128]).all())


@pytest.mark.parametrize("mode", MODES, **NAMES)
def test_extreme_gates(bnd, mode):
    """Gates that keep everything or nothing, up to the largest numbers of the type."""
    lens, D = [200], 64
    s = make(lens, D, False, torch.bfloat16, mode)
    v = [0.0, -0.0, -1e-30, -1e-6, -3.0, -90.0, -1000.0, torch.finfo(torch.bfloat16).min] + ([1e-6, 3.0, 90.0, torch.finfo(torch.bfloat16).max, float("inf")] if mode == oracle.GATE else [])
    for i, x in enumerate(v):
        s["G"][0, :, 2 * i] = x
        s["G"][0, 50 + i, 2 * i + 1] = x
    Y, S, _ = bnd.gated_recurrence(s["X"], s["G"], mode=mode, h0=s["h0"])
    check_forward(bnd, s, mode, lens, Y, S)
    if mode == oracle.NORMED:   # 1 / m has no value at 0 and passes the largest number just below it
        s["G"] = torch.where(s["G"] > -1e-20, 0.0, s["G"].float()).to(torch.bfloat16)
    for x, (r, e) in zip(bnd.gated_recurrence_backward(s["dY"], s["X"], s["G"], mode=mode, h0=s["h0"], dh=s["dh"]),
                         oracle.gradient(s["X"], s["G"], mode, lens, s["h0"], s["dY"], s["dh"])):
        oracle.inside(x, r, e)


def test_a_long_memory_over_many_tiles(bnd):
    """A state that remembers thousands of tokens: tiles join in 32 bits, whatever the order they arrive in."""
    for dtype, D in ((torch.bfloat16, 130), (torch.float32, 20)):
        s = make([9000], D, False, dtype, oracle.NORMED)
        s["G"] = (s["G"].float() * 0.01).to(dtype)
        Y, S, _ = bnd.gated_recurrence(s["X"], s["G"], mode=oracle.NORMED, h0=s["h0"])
        check_forward(bnd, s, oracle.NORMED, [9000], Y, S)


def test_gradient_against_differences(bnd):
    """fp32 gradients along random directions against central differences of the 64-bit recurrence."""
    lens, D = [100, 30], 12
    for mode in MODES:
        s = make(lens, D, True, torch.float32, mode)
        dX, dG, dh0 = bnd.gated_recurrence_backward(s["dY"], s["X"], s["G"], mode=mode, h0=s["h0"], dh=s["dh"], cu_seqlens=s["cu"])
        g = torch.Generator(device="cuda").manual_seed(5)
        for which, grad in (("X", dX), ("G", dG), ("h0", dh0)):
            v = torch.randn(s[which].shape, device="cuda", generator=g, dtype=torch.float64)
            if which == "G" and mode != oracle.GATE:
                v = v * s["G"].double().abs()
            loss = []
            for eps in (1e-5, -1e-5):
                t = dict(s)
                t[which] = s[which].double() + eps * v
                f = oracle.walk(t["X"], t["G"], mode, lens, t["h0"])
                loss.append((f["h"] * s["dY"].reshape(-1, D).double()).sum() + (f["state"] * s["dh"].double()).sum())
            want = float(loss[0] - loss[1]) / 2e-5
            got = float((grad.double() * v).sum())
            scale = float((grad.double() * v).abs().sum())
            assert abs(got - want) <= 1e-5 * scale, (mode, which, got, want)   # differences: 1e-10 of the third derivative; fp32 sums: about 1e-6


@pytest.mark.parametrize("mode", MODES, **NAMES)
@pytest.mark.parametrize("dtype", DTYPES, ids=["fp32", "bf16"])
@pytest.mark.parametrize("B,D", [(1, 1), (8, 2048), (3, 33), (200, 257), (5, 1000)])
def test_token(bnd, B, D, dtype, mode):
    s = make([1] * B, D, False, dtype, mode)
    n = B + 4
    g = torch.Generator(device="cuda").manual_seed(B)
    h = torch.randn(n, D, device="cuda", generator=g)
    slots = torch.randperm(n, device="cuda", generator=g)[:B].to(torch.int32)
    if B > 2:
        slots[1] = -1
    X, G = s["X"][:, 0], s["G"][:, 0]
    before = h.clone()
    Y = bnd.gated_recurrence_step(X, G, h, mode=mode, slots=slots)
    real = (slots >= 0).nonzero()[:, 0]
    f = oracle.walk(X[real][:, None], G[real][:, None], mode, [1] * len(real), before[slots[real].long()])
    oracle.inside(Y[real], f["h"], f["eh"])
    oracle.inside(h[slots[real].long()], f["state"], f["estate"])
    left = torch.ones(n, dtype=torch.bool, device="cuda")
    left[slots[real].long()] = False
    assert torch.equal(h[left], before[left])
    assert bool((Y[slots < 0] == 0).all())
    h2 = before.clone()
    X2 = X.clone()
    assert bnd.gated_recurrence_step(X2, G, h2, mode=mode, slots=slots, out=X2) is X2 and torch.equal(X2, Y) and torch.equal(h2, h)
    h3 = before[:B].clone()
    Y3 = bnd.gated_recurrence_step(X, G, h3, mode=mode)
    assert torch.equal(Y3, bnd.gated_recurrence(X[:, None], G[:, None], mode=mode, h0=before[:B])[0][:, 0])
    assert bnd.last_device_status() == 0


def test_token_refuses_slots(bnd):
    X, G, h = torch.randn(4, 40, device="cuda"), -torch.rand(4, 40, device="cuda"), torch.randn(5, 40, device="cuda")
    before = h.clone()
    Y = bnd.gated_recurrence_step(X, G, h, slots=torch.tensor([2, 0, 2, 5], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert bnd.last_device_status() == bnd.ERR_INVALID_ARG and bnd.last_device_status() == 0
    assert bool((Y[2:] == 0).all()) and torch.equal(h[[1, 3, 4]], before[[1, 3, 4]])
    f = oracle.walk(X[:2, None], G[:2, None], oracle.DECAY, [1, 1], before[[2, 0]])
    oracle.inside(Y[:2], f["h"], f["eh"])
    oracle.inside(h[[2, 0]], f["state"], f["estate"])


def test_prompt_then_tokens(bnd):
    """A prompt in two pieces, then single tokens on its final state, give what one walk gives."""
    D, mode = 96, oracle.GATE
    s = make([160], D, False, torch.float32, mode)
    f = oracle.walk(s["X"], s["G"], mode, [160], s["h0"])
    Y1, S1, _ = bnd.gated_recurrence(s["X"][:, :100], s["G"][:, :100], mode=mode, h0=s["h0"])
    Y2, S2, _ = bnd.gated_recurrence(s["X"][:, 100:150], s["G"][:, 100:150], mode=mode, h0=S1)
    ys = [Y1[0], Y2[0]] + [bnd.gated_recurrence_step(s["X"][:, t], s["G"][:, t], S2, mode=mode) for t in range(150, 160)]
    oracle.inside(torch.cat(ys), f["h"], f["eh"])
    oracle.inside(S2, f["state"], f["estate"])


def test_streams_and_graphs(bnd):
    """On another stream than the current one, and captured: replays with new inputs give new outputs; two graphs and eager calls do not share workspaces."""
    lens, D, mode = [500] * 2, 640, oracle.NORMED
    a, b = (make(lens, D, False, torch.bfloat16, mode, seed=i) for i in (1, 2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    Y, S, c = bnd.gated_recurrence(a["X"], a["G"], mode=mode, h0=a["h0"], want_carries=True, stream=side)
    grads = bnd.gated_recurrence_backward(a["dY"], a["X"], a["G"], mode=mode, h0=a["h0"], dh=a["dh"], carries=c, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    check_forward(bnd, a, mode, lens, Y, S, c)
    for x, (r, e) in zip(grads, oracle.gradient(a["X"], a["G"], mode, lens, a["h0"], a["dY"], a["dh"])):
        oracle.inside(x, r, e)
    live = {k: v.clone() for k, v in a.items() if v is not None}
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            Y, S, c = bnd.gated_recurrence(live["X"], live["G"], mode=mode, h0=live["h0"], want_carries=True)
            outs.append((Y, S, c, bnd.gated_recurrence_backward(live["dY"], live["X"], live["G"], mode=mode, h0=live["h0"], dh=live["dh"], carries=c)))
        graphs.append(g)
    for k in live:
        live[k].copy_(b[k])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    ref = oracle.gradient(b["X"], b["G"], mode, lens, b["h0"], b["dY"], b["dh"])
    for Y, S, c, grads in outs:
        check_forward(bnd, b, mode, lens, Y, S, c)
        for x, (r, e) in zip(grads, ref):
            oracle.inside(x, r, e)
    assert bnd.last_device_status() == 0


def test_a_wait_that_runs_out(bnd):
    """The first tile of the first channels never says what leaves it: the status word is raised, the rest of the call ends as usual."""
    s = make([400], 100, False, torch.bfloat16, oracle.DECAY, state=False)
    Y = torch.zeros_like(s["X"])
    bnd.selftest_recurrence_wait_timeout(s["X"], s["G"], 2_000_000, Y)
    assert bnd.last_device_status() == bnd.ERR_DEVICE_TIMEOUT
    f = oracle.walk(s["X"], s["G"], oracle.DECAY, [400], None)
    oracle.inside(Y[0, :64, :64], f["h"][:64, :64], f["eh"][:64, :64])
    oracle.inside(Y[0, :, 64:], f["h"][:, 64:], f["eh"][:, 64:])
    Y2, _, _ = bnd.gated_recurrence(s["X"], s["G"])
    oracle.inside(Y2, f["h"], f["eh"])
    assert bnd.last_device_status() == 0


def test_no_tokens(bnd):
    X = torch.empty(3, 0, 20, device="cuda")
    h0, dh = torch.randn(3, 20, device="cuda"), torch.randn(3, 20, device="cuda")
    Y, S, _ = bnd.gated_recurrence(X, X, h0=h0)
    assert Y.shape == X.shape and torch.equal(S, h0)
    dX, dG, dh0 = bnd.gated_recurrence_backward(X, X, X, h0=h0, dh=dh)
    assert dX.shape == X.shape and torch.equal(dh0, dh)
    assert bool((bnd.gated_recurrence(X, X)[1] == 0).all())


@pytest.mark.parametrize("D", [64, 700, 2048])
def test_two_calls_give_the_same_bits(bnd, D):
    """Whatever order the tiles of a long sequence arrive in, in a batch or alone."""
    for mode in MODES:
        s = make([3000] * 3, D, False, torch.bfloat16, mode)
        call = lambda c: bnd.gated_recurrence_backward(s["dY"], s["X"], s["G"], mode=mode, h0=s["h0"], dh=s["dh"], carries=c)   # noqa: E731
        first = bnd.gated_recurrence(s["X"], s["G"], mode=mode, h0=s["h0"], want_carries=True)
        grads = call(first[2])
        for _ in range(5):
            Y, S, c = bnd.gated_recurrence(s["X"], s["G"], mode=mode, h0=s["h0"], want_carries=True)
            assert torch.equal(Y, first[0]) and torch.equal(S, first[1])
            assert all(torch.equal(a, b) for a, b in zip(call(c), grads)) and all(torch.equal(a, b) for a, b in zip(call(None), grads))
        one = bnd.gated_recurrence(s["X"][1:2], s["G"][1:2], mode=mode, h0=s["h0"][1:2])
        assert torch.equal(one[0][0], first[0][1]) and torch.equal(one[1][0], first[1][1])


@pytest.mark.parametrize("mode", MODES, **NAMES)
def test_states_in_place_across_resets(bnd, mode):
    """The final state in the place of the initial one, its gradient in the place of the final one's: also where decays of zero let no tile of the end wait for one of the beginning."""
    lens, D = [2000] * 3, 300
    s = make(lens, D, False, torch.bfloat16, mode)
    s["G"][:, 5::7] = float("-inf")
    want = bnd.gated_recurrence(s["X"], s["G"], mode=mode, h0=s["h0"], want_carries=True)
    ref = oracle.walk(s["X"], s["G"], mode, lens, s["h0"])
    oracle.inside(want[0], ref["h"], ref["eh"])
    grads = bnd.gated_recurrence_backward(s["dY"], s["X"], s["G"], mode=mode, h0=s["h0"], dh=s["dh"])
    L, p = bnd.load(), lambda t: t.data_ptr()   # noqa: E731
    desc, need = bnd.RecDesc(3, 2000, D, bnd.BF16, mode, 0, None), bnd._workspace("tri_inv_gated_recurrence_backward_workspace", bnd.RecDesc(3, 2000, D, bnd.BF16, mode, 0, None), 1)
    work, dX, dG = torch.empty(need, dtype=torch.uint8, device="cuda"), torch.empty_like(s["X"]), torch.empty_like(s["X"])
    for _ in range(5):
        h, dh = s["h0"].clone(), s["dh"].clone()
        Y, S, _ = bnd.gated_recurrence(s["X"], s["G"], mode=mode, h0=h, state_out=h)
        assert S is h and torch.equal(Y, want[0]) and torch.equal(h, want[1])
        assert L.tri_inv_gated_recurrence_backward(p(s["dY"]), D, p(s["X"]), D, p(s["G"]), D, p(s["h0"]), p(dh), p(want[2]), p(dX), D, p(dG), D, p(dh), p(work), need, desc, None) == 0
        assert torch.equal(dX, grads[0]) and torch.equal(dG, grads[1]) and torch.equal(dh, grads[2])
    assert bnd.last_device_status() == 0
