"""GPU tests of linear attention with a decay for each head: prompt, single token, gradient, against the recurrence in 64 bits.

Bounds are elementwise (linear_oracle.within).  fp32 (CUDA cores): d_k + 64 products and sums in a tile, one rounding a tile in the state, and the
factors lambda^n, n up to 64: the exponent is off by up to 2^-24 of itself (at most 2^-24 * 45 in absolute terms where the factor is above 1e-20; smaller ones do
not matter), which depth = 2 (d_k + 64) + 4 tiles + 128 covers.  bf16 on the tensor cores: each term meets one rounding to bf16 of a computed operand (P, or the
state), the state's increment two numbers of eight bits (2^-16 left).  bf16 on the CUDA cores rounds the output alone: inside the same bounds.
"""
import numpy as np
import pytest
import torch

import linear_oracle as lo

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def bnd():
    import __graft_entry__ as entry
    entry.build()
    from paper_2605_21325_b200 import binding
    torch.cuda.set_device(0)
    return binding


def slopes(H):
    return -(2.0 ** (-8.0 * torch.arange(1, H + 1, device="cuda") / H))


def make(B, T, H, dk, dv, dtype, cu=None, seed=0, state=True):
    if cu is not None:
        B, T = 1, int(cu[-1])
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)   # noqa: E731
    n = B if cu is None else len(cu) - 1
    x = dict(Q=r(B, T, H, dk).to(dtype), K=r(B, T, H, dk).to(dtype), V=r(B, T, H, dv).to(dtype), dO=r(B, T, H, dv).to(dtype),
             S0=r(n, H, dk, dv) if state else None, dS=r(n, H, dk, dv) if state else None)
    return x


def depth(T, dk):
    return 2 * (dk + 64) + 4 * (T // 64 + 1) + 128


def check_forward(bnd, x, ld, cu, scale, O, S):
    refs = lo.forward(x["Q"], x["K"], x["V"], ld, scale, x["S0"], cu)
    mag = lo.forward(x["Q"].abs(), x["K"].abs(), x["V"].abs(), ld, abs(scale), None if x["S0"] is None else x["S0"].abs(), cu)
    bf = x["Q"].dtype == torch.bfloat16
    n = depth(x["Q"].shape[1], x["Q"].shape[3])
    lo.within(O, refs[0], mag[0], int(bf), bf, n)
    lo.within(S, refs[1], mag[1], 2.0 ** -8 if bf else 0, False, n)


PACKED = np.array([0, 0, 64, 65, 65, 300, 428, 531], np.int32)
SHAPES = [   # B, T, H, d_k, d_v, cu
    (1, 1, 1, 128, 128, None),
    (2, 63, 3, 128, 128, None),
    (1, 64, 2, 128, 128, None),
    (3, 65, 2, 128, 128, None),
    (1, 333, 5, 128, 128, None),
    (1, 0, 4, 128, 128, PACKED),
    (1, 333, 3, 64, 64, None),
    (1, 0, 2, 64, 64, PACKED),
    (1, 200, 3, 128, 64, None),
    (1, 0, 3, 64, 128, PACKED),
    (2, 70, 2, 96, 96, None),
    (1, 0, 2, 80, 120, PACKED),
    (1, 130, 1, 8, 8, None),
    (1, 100, 2, 256, 24, None),
    (1, 2500, 1, 128, 128, None),       # cut into segments, the last one partial
    (1, 2500, 1, 64, 128, None),
    (1, 2500, 1, 40, 64, None),
    (1, 0, 1, 128, 128, np.array([0, 1500, 1500, 1501, 3200], np.int32)),   # some sequences cut, some not
]
DTYPES = [torch.float32, torch.bfloat16]


@pytest.mark.parametrize("dtype", DTYPES, ids=["fp32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=["x".join(map(str, s[:5])) + ("_packed" if s[5] is not None else "") for s in SHAPES])
@pytest.mark.parametrize("state", [False, True], ids=["zero", "carried"])
def test_forward(bnd, shape, dtype, state):
    B, T, H, dk, dv, cu = shape
    x = make(B, T, H, dk, dv, dtype, cu, seed=T + dk, state=state)
    ld = slopes(H)
    O, S = bnd.linear_attention(x["Q"], x["K"], x["V"], ld, scale=0.3, S0=x["S0"], cu_seqlens=cu)
    torch.cuda.synchronize()
    assert bnd.last_device_status() == 0
    check_forward(bnd, x, ld, cu, 0.3, O, S)


@pytest.mark.parametrize("dtype", DTYPES, ids=["fp32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=["x".join(map(str, s[:5])) + ("_packed" if s[5] is not None else "") for s in SHAPES])
@pytest.mark.parametrize("state", [False, True], ids=["zero", "carried"])
def test_backward(bnd, shape, dtype, state):
    B, T, H, dk, dv, cu = shape
    x = make(B, T, H, dk, dv, dtype, cu, seed=3 * T + dv, state=state)
    ld, scale = slopes(H), 0.3
    got = bnd.linear_attention_backward(x["dO"], x["Q"], x["K"], x["V"], ld, scale=scale, S0=x["S0"], dS=x["dS"], cu_seqlens=cu, want_dS0=True)
    torch.cuda.synchronize()
    assert bnd.last_device_status() == 0
    ref = lo.backward(x["dO"], x["Q"], x["K"], x["V"], ld, scale, x["S0"], x["dS"], cu)
    a = {k: None if v is None else v.abs() for k, v in x.items()}
    mag = lo.backward(a["dO"], a["Q"], a["K"], a["V"], ld, scale, a["S0"], a["dS"], cu)
    bf = dtype == torch.bfloat16
    n = depth(x["Q"].shape[1], max(dk, dv))
    for i in range(3):
        lo.within(got[i], ref[i], mag[i], int(bf), bf, n)
    lo.within(got[3], ref[3], mag[3], 2.0 ** -8 if bf else 0, False, n)


def test_gradient_against_differences(bnd):
    """Directional differences of the fp64 recurrence: the loss is linear in O and S, and a central difference of a polynomial of degree three (q, k, v move together) is off
    by the third-order term, eps^2 of it; fp32 gradients add their bound, far below the 1e-4 of the norm asked here."""
    B, T, H, dk, dv, scale = 2, 45, 2, 16, 24, 0.5
    x = make(B, T, H, dk, dv, torch.float32, seed=5)
    ld = slopes(H)
    grads = bnd.linear_attention_backward(x["dO"], x["Q"], x["K"], x["V"], ld, scale=scale, S0=x["S0"], dS=x["dS"])
    g = torch.Generator(device="cuda").manual_seed(9)
    for seed in range(3):
        d = {k: torch.randn(x[k].shape, device="cuda", generator=g, dtype=torch.float64) for k in ("Q", "K", "V", "S0")}

        def loss(e):
            p = {k: x[k].double() + e * d[k] for k in d}
            O, S = lo.forward(p["Q"], p["K"], p["V"], ld, scale, p["S0"], None)
            return float((O * x["dO"].double()).sum() + (S * x["dS"].double()).sum())

        eps = 1e-4
        want = (loss(eps) - loss(-eps)) / (2 * eps)
        have = sum(float((a.double() * d[k]).sum()) for a, k in zip(grads, ("Q", "K", "V", "S0")))
        size = sum(float((a.double() * d[k]).square().sum()) for a, k in zip(grads, ("Q", "K", "V", "S0"))) ** 0.5
        assert abs(want - have) <= 1e-4 * size


@pytest.mark.parametrize("dtype", DTYPES, ids=["fp32", "bf16"])
@pytest.mark.parametrize("ld", [0.0, -1e-3, -3.0, -60.0, float("-inf")])
def test_decays(bnd, dtype, ld):
    """No decay, slow and fast ones, and one that forgets everything at once: no factor overflows or becomes NaN."""
    x = make(1, 200, 2, 128, 128, dtype, seed=11)
    d = torch.full((2,), ld, device="cuda")
    O, S = bnd.linear_attention(x["Q"], x["K"], x["V"], d, scale=0.1, S0=x["S0"])
    check_forward(bnd, x, d, None, 0.1, O, S)
    got = bnd.linear_attention_backward(x["dO"], x["Q"], x["K"], x["V"], d, scale=0.1, S0=x["S0"], dS=x["dS"])
    ref = lo.backward(x["dO"], x["Q"], x["K"], x["V"], d, 0.1, x["S0"], x["dS"], None)
    a = {k: v.abs() for k, v in x.items()}
    mag = lo.backward(a["dO"], a["Q"], a["K"], a["V"], d, 0.1, a["S0"], a["dS"], None)
    bf = dtype == torch.bfloat16
    for i in range(4):
        lo.within(got[i], ref[i], mag[i], (int(bf) if i < 3 else 2.0 ** -8 * bf), bf and i < 3, depth(200, 128))


@pytest.mark.parametrize("d", [128, 40])
@pytest.mark.parametrize("dtype", DTYPES, ids=["fp32", "bf16"])
def test_nothing_reaches_another_sequence(bnd, dtype, d):
    """A neighbour of values that are not finite, before and behind sequences that end inside a tile; and rows behind the last token stay as they were."""
    cu = np.array([0, 70, 140, 203], np.int32)
    x = make(1, 0, 2, d, d, dtype, cu, seed=21)
    ld = slopes(2)
    clean = bnd.linear_attention(x["Q"], x["K"], x["V"], ld, S0=x["S0"], cu_seqlens=cu)
    gclean = bnd.linear_attention_backward(x["dO"], x["Q"], x["K"], x["V"], ld, S0=x["S0"], dS=x["dS"], cu_seqlens=cu)
    for bad in (float("nan"), float("inf"), torch.finfo(dtype).min):
        y = {k: v.clone() for k, v in x.items()}
        for k in ("Q", "K", "V", "dO"):
            y[k][:, 70:140] = bad
        y["S0"][1] = bad
        room = torch.full((1, 210, 2, d), 7.0, dtype=dtype, device="cuda")
        O = room[:, :203]
        O, S = bnd.linear_attention(y["Q"], y["K"], y["V"], ld, S0=y["S0"], cu_seqlens=cu, out=O)
        g = bnd.linear_attention_backward(y["dO"], y["Q"], y["K"], y["V"], ld, S0=y["S0"], dS=y["dS"], cu_seqlens=cu)
        assert bool((room[:, 203:] == 7).all())
        for a, b in [(O, clean[0])] + list(zip(g[:3], gclean[:3])):
            assert torch.equal(a[:, :70], b[:, :70]) and torch.equal(a[:, 140:], b[:, 140:])
        for a, b in ((S, clean[1]), (g[3], gclean[3])):
            assert torch.equal(a[0], b[0]) and torch.equal(a[2], b[2])


@pytest.mark.parametrize("dtype", DTYPES, ids=["fp32", "bf16"])
def test_empty_calls(bnd, dtype):
    """No token at all: the states pass through; no sequence at all: nothing happens."""
    S0 = torch.randn(3, 2, 64, 64, device="cuda")
    z = torch.empty(1, 0, 2, 64, device="cuda", dtype=dtype)
    O, S = bnd.linear_attention(z, z, z, slopes(2), S0=S0, cu_seqlens=[0, 0, 0, 0])
    assert O.numel() == 0 and torch.equal(S, S0)
    O, S = bnd.linear_attention(z.expand(3, 0, 2, 64), z.expand(3, 0, 2, 64), z.expand(3, 0, 2, 64), slopes(2), S0=S0)
    assert torch.equal(S, S0)
    assert torch.equal(bnd.linear_attention_backward(z, z, z, z, slopes(2), S0=S0, dS=S0, cu_seqlens=[0, 0, 0, 0])[3], S0)
    O, S = bnd.linear_attention(z, z, z, slopes(2), cu_seqlens=[0])
    assert S.shape[0] == 0


@pytest.mark.parametrize("T,H", [(150, 4), (5000, 1)])
@pytest.mark.parametrize("d", [128, 48])
def test_state_in_place_and_repeatable(bnd, T, H, d):
    """S_out may be S0, cut or not, and the same call gives the same bits."""
    x = make(1, T, H, d, d, torch.bfloat16, seed=2)
    ld = slopes(H)
    O, S = bnd.linear_attention(x["Q"], x["K"], x["V"], ld, S0=x["S0"])
    S2 = x["S0"].clone()
    O2, _ = bnd.linear_attention(x["Q"], x["K"], x["V"], ld, S0=S2, state_out=S2)
    assert torch.equal(S, S2) and torch.equal(O, O2)
    a = bnd.linear_attention_backward(x["dO"], x["Q"], x["K"], x["V"], ld, S0=x["S0"], dS=x["dS"])
    b = bnd.linear_attention_backward(x["dO"], x["Q"], x["K"], x["V"], ld, S0=x["S0"], dS=x["dS"])
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_without_a_final_state(bnd):
    """A training forward asks for no state: O is the same to a rounding of its operands."""
    x = make(2, 500, 3, 128, 128, torch.bfloat16, seed=8)
    ld = slopes(3)
    O, S = bnd.linear_attention(x["Q"], x["K"], x["V"], ld, scale=0.3, S0=x["S0"], want_state=False)
    assert S is None
    ref = lo.forward(x["Q"], x["K"], x["V"], ld, 0.3, x["S0"], None)[0]
    mag = lo.forward(x["Q"].abs(), x["K"].abs(), x["V"].abs(), ld, 0.3, x["S0"].abs(), None)[0]
    # each term meets two roundings to bf16: the increment's and the state's (or P's one)
    lo.within(O, ref, mag, 2, True, depth(500, 128))


def test_streams_and_graphs(bnd):
    """Calls on two streams at once; a captured call replayed on new inputs, twice from two graphs with workspaces of their own."""
    ld = slopes(2)
    xs = [make(1, 3000, 2, 128, 128, torch.bfloat16, seed=s) for s in (31, 32)]
    call = lambda x, **k: bnd.linear_attention(x["Q"], x["K"], x["V"], ld, S0=x["S0"], **k) + bnd.linear_attention_backward(   # noqa: E731
        x["dO"], x["Q"], x["K"], x["V"], ld, S0=x["S0"], dS=x["dS"], **k)
    want = [call(x) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    got = []
    for _ in range(3):
        got = [call(x, stream=st) for x, st in zip(xs, streams)]
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert all(torch.equal(p, q) for p, q in zip(a, b))
    del got
    graphs, outs, ins = [], [], [{k: v.clone() for k, v in x.items()} for x in xs]
    for x in ins:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            outs.append(call(x))
        graphs.append(gr)
    for k in ins[0]:
        ins[0][k].copy_(xs[1][k])
        ins[1][k].copy_(xs[0][k])
    for gr in graphs + graphs:
        gr.replay()
    torch.cuda.synchronize()
    for a, b in ((want[1], outs[0]), (want[0], outs[1])):
        assert all(torch.equal(p, q) for p, q in zip(a, b))
    del graphs


STEP_SHAPES = [(1, 1, 128, 128), (8, 16, 128, 128), (5, 3, 64, 64), (40, 16, 128, 128), (300, 2, 128, 64), (7, 2, 96, 96), (3, 2, 8, 8), (260, 2, 80, 120), (300, 2, 256, 128), (2, 1, 256, 264)]


@pytest.mark.parametrize("dtype", DTYPES, ids=["fp32", "bf16"])
@pytest.mark.parametrize("shape", STEP_SHAPES, ids=["x".join(map(str, s)) for s in STEP_SHAPES])
def test_step(bnd, shape, dtype):
    B, H, dk, dv = shape
    g = torch.Generator(device="cuda").manual_seed(B)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)   # noqa: E731
    Q, K, V, ld = r(B, H, dk).to(dtype), r(B, H, dk).to(dtype), r(B, H, dv).to(dtype), slopes(H)
    n = B + 2
    slots = torch.randperm(n, device="cuda", generator=g)[:B].to(torch.int32)
    if B > 2:
        slots[1] = -1
        slots[B - 1] = -7
    S = r(n, H, dk, dv)
    before = S.clone()
    O = bnd.linear_attention_step(Q, K, V, ld, S, scale=0.4, slots=slots)
    torch.cuda.synchronize()
    assert bnd.last_device_status() == 0
    want, lam, touched = before.double(), torch.exp(ld.double())[:, None, None], []
    for b, s in enumerate(slots.tolist()):
        if s < 0:
            assert not bool(O[b].any())
            continue
        touched.append(s)
        want[s] = lam * want[s] + K[b].double()[:, :, None] * V[b].double()[:, None, :]
        ref = 0.4 * torch.einsum("hk,hkv->hv", Q[b].double(), want[s])
        mag = 0.4 * torch.einsum("hk,hkv->hv", Q[b].double().abs(), want[s].abs())
        lo.within(O[b], ref, mag, 0, dtype == torch.bfloat16, dk + 16)
    lo.within(S, want, want.abs() + before.abs().double() + 10, 0, False, 4)
    rest = [s for s in range(n) if s not in touched]
    assert torch.equal(S[rest], before[rest])
    S2 = before.clone()
    if B > 2:   # without slots, row b has slot b
        O2 = bnd.linear_attention_step(Q, K, V, ld, S2, scale=0.4)
        S3 = before.clone()
        O3 = bnd.linear_attention_step(Q, K, V, ld, S3, scale=0.4, slots=torch.arange(B, dtype=torch.int32, device="cuda"))
        assert torch.equal(O2, O3) and torch.equal(S2, S3)


def test_step_refuses_slots_on_the_device(bnd):
    """The same slot twice: the first row has it; a slot past the cache: no row.  Both show in the status word, once, and nothing else is touched."""
    B, H, d = 6, 2, 128
    g = torch.Generator(device="cuda").manual_seed(1)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)   # noqa: E731
    Q, K, V, S, ld = r(B, H, d), r(B, H, d), r(B, H, d), r(5, H, d, d), slopes(H)
    for slots, dropped in (([0, 3, 1, 3, -1, 2], [3, 4]), ([0, 5, 1, 3, 2 ** 31 - 1, 2], [1, 4])):
        t = torch.tensor(slots, dtype=torch.int32, device="cuda")
        kept = torch.tensor([-1 if b in dropped else s for b, s in enumerate(slots)], dtype=torch.int32, device="cuda")
        S1, S2 = S.clone(), S.clone()
        O1 = bnd.linear_attention_step(Q, K, V, ld, S1, slots=t)
        torch.cuda.synchronize()
        assert bnd.last_device_status() == bnd.ERR_INVALID_ARG and bnd.last_device_status() == 0
        O2 = bnd.linear_attention_step(Q, K, V, ld, S2, slots=kept)
        assert torch.equal(O1, O2) and torch.equal(S1, S2)


@pytest.mark.parametrize("dtype", DTYPES, ids=["fp32", "bf16"])
def test_step_in_a_graph(bnd, dtype):
    """A captured step moves the states on at every replay."""
    B, H, d = 4, 4, 128
    g = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)   # noqa: E731
    Q, K, V, ld = r(B, H, d).to(dtype), r(B, H, d).to(dtype), r(B, H, d).to(dtype), slopes(H)
    S0 = r(B, H, d, d)
    S, want = S0.clone(), S0.clone()
    slots = torch.tensor([2, 0, -1, 3], dtype=torch.int32, device="cuda")
    bnd.linear_attention_step(Q, K, V, ld, S, slots=slots)
    S.copy_(S0)
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        O = bnd.linear_attention_step(Q, K, V, ld, S, slots=slots)
    for _ in range(3):
        gr.replay()
        ref = bnd.linear_attention_step(Q, K, V, ld, want, slots=slots)
        torch.cuda.synchronize()
        assert torch.equal(O, ref) and torch.equal(S, want)


@pytest.mark.parametrize("dtype", DTYPES, ids=["fp32", "bf16"])
def test_prompt_then_tokens(bnd, dtype):
    """A block as it is used: norm with the residual, projections, attention over the prompt, the norm of each head's output; then tokens one by one on
    the carried states, against the whole sequence in one call."""
    T, more, H, d, n = 150, 9, 4, 64, 256
    g = torch.Generator(device="cuda").manual_seed(4)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)   # noqa: E731
    ld, w, wh = slopes(H), (1 + 0.1 * r(n)).to(dtype), (1 + 0.1 * r(d)).to(dtype)
    Wp = (r(n, 3 * H * d) * n ** -0.5).to(dtype)
    x, res = r(1, T + more, n).to(dtype), r(1, T + more, n).to(dtype)

    def project(x, res):
        y, h, _ = bnd.rms_norm(x, w, residual=res)
        qkv = (y @ Wp).reshape(x.shape[0], x.shape[1], 3, H, d)
        return [qkv[:, :, i].contiguous() for i in range(3)] + [h]

    q, k, v, _ = project(x, res)
    whole, S_end = bnd.linear_attention(q, k, v, ld, scale=d ** -0.5)
    whole, _, _ = bnd.rms_norm(whole, wh)
    O, S = bnd.linear_attention(q[:, :T].contiguous(), k[:, :T].contiguous(), v[:, :T].contiguous(), ld, scale=d ** -0.5)
    O, _, _ = bnd.rms_norm(O, wh)
    parts = [O]
    for t in range(T, T + more):
        o = bnd.linear_attention_step(q[:, t].contiguous(), k[:, t].contiguous(), v[:, t].contiguous(), ld, S, scale=d ** -0.5)
        parts.append(bnd.rms_norm(o, wh)[0][:, None])
    got = torch.cat(parts, 1)
    # the states differ by fp32 roundings (bf16: 2^-16 of the increments); a head's output of unit mean square has parts of at most sqrt(d), and
    # in bf16 the outputs of both ways are rounded, the operands of one of them as well: four half steps of a value of at most sqrt(d)
    tol = 4 * 2.0 ** -8 * d ** 0.5 if dtype == torch.bfloat16 else 1e-4
    assert float((got.double() - whole.double()).abs().max()) <= tol
    assert float((S - S_end).abs().max()) <= 1e-4 * float(S_end.abs().max())
    assert bnd.last_device_status() == 0
