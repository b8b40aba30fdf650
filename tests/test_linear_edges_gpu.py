"""GPU tests of linear attention at its edges: outputs that may not depend on what else is asked for, finite values whose products overflow, states far larger than what joins them,
calls from two host threads, memory on the call's own stream, the largest counts of tokens."""
import ctypes
import threading

import pytest
import torch

import linear_oracle as lo
from test_linear_attention_gpu import DTYPES, PACKED, bnd, check_forward, depth, make, slopes   # noqa: F401  (bnd: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", DTYPES, ids=["fp32", "bf16"])
@pytest.mark.parametrize("shape", [(2, 500, 3, 128, 128, None), (1, 5000, 1, 128, 64, None), (1, 5000, 1, 64, 128, None), (1, 0, 2, 48, 64, PACKED)],
                         ids=["uncut", "cut", "cut_turned", "packed"])
def test_outputs_do_not_depend_on_the_state_being_wanted(bnd, shape, dtype):   # noqa: F811
    """O with and without S, dV with and without dS0: the same bits."""
    B, T, H, dk, dv, cu = shape
    x = make(B, T, H, dk, dv, dtype, cu, seed=41)
    ld = slopes(H)
    O, S = bnd.linear_attention(x["Q"], x["K"], x["V"], ld, scale=0.3, S0=x["S0"], cu_seqlens=cu)
    O2, none = bnd.linear_attention(x["Q"], x["K"], x["V"], ld, scale=0.3, S0=x["S0"], cu_seqlens=cu, want_state=False)
    assert none is None and torch.equal(O, O2)
    g = bnd.linear_attention_backward(x["dO"], x["Q"], x["K"], x["V"], ld, scale=0.3, S0=x["S0"], dS=x["dS"], cu_seqlens=cu)
    g2 = bnd.linear_attention_backward(x["dO"], x["Q"], x["K"], x["V"], ld, scale=0.3, S0=x["S0"], dS=x["dS"], cu_seqlens=cu, want_dS0=False)
    assert g2[3] is None and all(torch.equal(a, b) for a, b in zip(g[:3], g2[:3]))


def two_threads(calls, rounds=1500):
    """The last results of each call, made again and again by a thread of its own on a stream of its own."""
    errors, results, start = [], {}, threading.Barrier(len(calls))

    def work(i):
        try:
            torch.cuda.set_device(0)
            with torch.cuda.stream(torch.cuda.Stream()):
                start.wait()
                for _ in range(rounds):
                    results[i] = calls[i]()
                torch.cuda.current_stream().synchronize()
        except Exception as e:   # reported by the test
            errors.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(calls))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors, errors
    return [results[i] for i in range(len(calls))]


def test_two_host_threads(bnd):   # noqa: F811
    """Calls of different sizes from two threads: neither takes away the shared memory that the other's launch of the same kernel needs."""
    ld = slopes(2)
    xs = [make(1, 200, 2, d, d, torch.float32, seed=d) for d in (64, 8)]
    g = torch.Generator(device="cuda").manual_seed(45)
    scans = [[torch.randn(1, 256, 2, d, device="cuda", generator=g) * d ** -0.5 for _ in range(4)] + [-torch.rand(1, 256, 2, device="cuda", generator=g), C] for d, C in ((256, 64), (16, 16))]
    for calls in ([lambda x=x: bnd.linear_attention(x["Q"], x["K"], x["V"], ld) for x in xs], [lambda s=s: bnd.chunk_scan(*s) for s in scans]):
        want = [c() for c in calls]
        torch.cuda.synchronize()
        for a, b in zip(want, two_threads(calls)):
            assert all(torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("dtype", DTYPES, ids=["fp32", "bf16"])
def test_a_step_in_its_values(bnd, dtype):   # noqa: F811
    """O in V's place gives the bits of an O of its own, in blocks of few and of many rows."""
    for B, H, d in ((3, 2, 128), (300, 2, 128), (300, 2, 64)):
        g = torch.Generator(device="cuda").manual_seed(46)
        r = lambda *s: torch.randn(*s, device="cuda", generator=g)   # noqa: E731
        Q, K, V, S, ld = r(B, H, d).to(dtype), r(B, H, d).to(dtype), r(B, H, d).to(dtype), r(B, H, d, d), slopes(H)
        S2 = S.clone()
        O = bnd.linear_attention_step(Q, K, V, ld, S)
        bnd.linear_attention_step(Q, K, V, ld, S2, out=V)
        assert torch.equal(O, V) and torch.equal(S, S2)


@pytest.mark.parametrize("dtype", DTYPES, ids=["fp32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("at", [0, 40, 63, 70])
def test_finite_values_whose_products_overflow(bnd, dtype, d, at):   # noqa: F811
    """A query, key, value or gradient of the type's lowest value at one token: what does not follow from that token is what it is without it."""
    x = make(1, 100, 2, d, d, dtype, seed=42)
    ld = slopes(2)
    O, _ = bnd.linear_attention(x["Q"], x["K"], x["V"], ld, S0=x["S0"])
    g = bnd.linear_attention_backward(x["dO"], x["Q"], x["K"], x["V"], ld, S0=x["S0"], dS=x["dS"])
    before, behind, all_but = slice(0, at), slice(at + 1, 100), [i for i in range(100) if i != at]
    # the tokens of O, dQ, dK, dV that do not see the operand's token (None: all of them, [] : it is the operand's own affair)
    clean = {"Q": (all_but, all_but, behind, behind), "K": (before, before, None, all_but), "V": (before, before, all_but, None), "dO": (None, all_but, behind, behind)}
    for name, rows in clean.items():
        y = dict(x, **{name: x[name].clone()})
        y[name][:, at] = torch.finfo(dtype).min
        O2, _ = bnd.linear_attention(y["Q"], y["K"], y["V"], ld, S0=y["S0"])
        g2 = bnd.linear_attention_backward(y["dO"], y["Q"], y["K"], y["V"], ld, S0=y["S0"], dS=y["dS"])
        for a, b, keep in zip((O, *g[:3]), (O2, *g2[:3]), rows):
            assert torch.equal(a, b) if keep is None else torch.equal(a[:, keep], b[:, keep]), name


@pytest.mark.parametrize("dtype", DTYPES, ids=["fp32", "bf16"])
@pytest.mark.parametrize("T", [64, 100, 128])
@pytest.mark.parametrize("ld", [-0.01, -0.1, -0.2, -0.25, -0.5])
def test_a_large_state_that_fades(bnd, dtype, ld, T):   # noqa: F811
    """States carried in that are a million times what the tokens add, under decays that leave from 0.5 to 1e-14 of them after a tile: what is left is good to its own last bits,
    not to those of what it was."""
    x = make(2, T, 2, 128, 128, dtype, seed=43)
    x["S0"] *= 1e6
    x["dS"] *= 1e6
    d = torch.full((2,), ld, device="cuda")
    O, S = bnd.linear_attention(x["Q"], x["K"], x["V"], d, scale=0.3, S0=x["S0"])
    check_forward(bnd, x, d, None, 0.3, O, S)
    got = bnd.linear_attention_backward(x["dO"], x["Q"], x["K"], x["V"], d, scale=0.3, S0=x["S0"], dS=x["dS"])
    ref = lo.backward(x["dO"], x["Q"], x["K"], x["V"], d, 0.3, x["S0"], x["dS"], None)
    a = {k: v.abs() for k, v in x.items()}
    mag = lo.backward(a["dO"], a["Q"], a["K"], a["V"], d, 0.3, a["S0"], a["dS"], None)
    bf = dtype == torch.bfloat16
    for i in range(4):
        lo.within(got[i], ref[i], mag[i], (int(bf) if i < 3 else 2.0 ** -8 * bf), bf and i < 3, depth(T, 128))


def test_memory_made_for_a_named_stream(bnd):   # noqa: F811
    """Outputs and workspaces of a call on another stream are not memory that work still queued on the current one is going to write: blocks of the outputs' and the workspace's sizes are
    filled there behind a delay, and given back before the call."""
    x = make(1, 3000, 2, 128, 128, torch.bfloat16, seed=44)
    ld, w = slopes(2), torch.ones(128, device="cuda", dtype=torch.bfloat16)
    q, k, v = (x[n][0, :2].contiguous() for n in ("Q", "K", "V"))
    S = torch.randn(2, 2, 128, 128, device="cuda")
    calls = [lambda **s: bnd.linear_attention(x["Q"], x["K"], x["V"], ld, S0=x["S0"], **s),
             lambda **s: bnd.linear_attention_backward(x["dO"], x["Q"], x["K"], x["V"], ld, S0=x["S0"], dS=x["dS"], **s),
             lambda **s: (bnd.linear_attention_step(q, k, v, ld, S.clone() if not s else states, **s),),
             lambda **s: bnd.rms_norm(x["Q"], w, residual=x["K"], **s)[:2],
             lambda **s: bnd.rms_norm(x["Q"], w, residual=x["K"], out_dtype=torch.float8_e4m3fn, **s),
             lambda **s: bnd.rms_norm_backward(x["dO"], x["Q"], w, **s)]
    desc, _ = bnd.make_desc(1, 3000, 2, 128, 128, 64, bnd.BF16)
    need = []
    for f in ("tri_inv_linear_attention_workspace", "tri_inv_linear_attention_backward_workspace"):
        n = ctypes.c_size_t(0)
        assert getattr(bnd.load(), f)(ctypes.byref(desc), ctypes.byref(n)) == 0 and n.value > 0
        need.append(n.value)
    other = torch.cuda.Stream()
    for call in calls:
        want = call()
        states = S.clone()
        torch.cuda.synchronize()
        blocks = [torch.empty(n, dtype=torch.uint8, device="cuda") for t in want for n in [t.numel() * t.element_size()] * 2] + [torch.empty(n, dtype=torch.uint8, device="cuda") for n in need]
        torch.cuda._sleep(100_000_000)   # some 50 ms
        for b in blocks:
            b.fill_(0x7f)
        del blocks, b
        got = call(stream=other)
        torch.cuda.synchronize()
        assert all(torch.equal(a.float(), b.float()) for a, b in zip(want, got))


@pytest.mark.parametrize("packed", [False, True], ids=["dense", "packed"])
def test_the_largest_counts_of_tokens(bnd, packed):   # noqa: F811
    """The cut of a sequence whose tokens, rounded up to tiles, pass 2^31 - 1: the workspace is that of the sequence a few tokens shorter."""
    def size(T):
        desc, keep = bnd.make_desc(1, T, 1, 8, 8, 64, bnd.BF16, [0, T] if packed else None)   # noqa: F841
        n = ctypes.c_size_t(0)
        assert bnd.load().tri_inv_linear_attention_workspace(ctypes.byref(desc), ctypes.byref(n)) == 0
        return n.value
    assert size(2 ** 31 - 1) == size(2 ** 31 - 64) > 0


@pytest.mark.parametrize("dtype", DTYPES, ids=["fp32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("at", [0, 40, 63, 70])
def test_what_is_not_finite_and_not_a_value(bnd, dtype, d, at):   # noqa: F811
    """A query or key (in the gradient what stands in its place) that is not finite at one token: what does not follow from that token is what it is without it."""
    x = make(1, 100, 2, d, d, dtype, seed=47)
    ld = slopes(2)
    O, _ = bnd.linear_attention(x["Q"], x["K"], x["V"], ld, S0=x["S0"])
    g = bnd.linear_attention_backward(x["dO"], x["Q"], x["K"], x["V"], ld, S0=x["S0"], dS=x["dS"])
    before, behind, all_but = slice(0, at), slice(at + 1, 100), [i for i in range(100) if i != at]
    clean = {"Q": {0: all_but, 3: behind}, "K": {0: before, 3: all_but}, "V": {1: before, 2: all_but}, "dO": {1: all_but, 2: behind}}   # of O, dQ, dK, dV
    for bad in (float("nan"), float("inf")):
        for name, rows in clean.items():
            y = dict(x, **{name: x[name].clone()})
            y[name][:, at] = bad
            got = (bnd.linear_attention(y["Q"], y["K"], y["V"], ld, S0=y["S0"])[0],) + bnd.linear_attention_backward(y["dO"], y["Q"], y["K"], y["V"], ld, S0=y["S0"], dS=y["dS"])[:3]
            for i, keep in rows.items():
                assert torch.equal((O, *g)[i][:, keep], got[i][:, keep]), (name, i)


WIDE = [(1, 200, 2, 256, 256, None), (1, 2500, 1, 136, 200, None), (1, 0, 2, 160, 72, PACKED), (1, 0, 2, 72, 160, PACKED), (2, 20, 3, 8, 256, None)]


@pytest.mark.parametrize("dtype", DTYPES, ids=["fp32", "bf16"])
@pytest.mark.parametrize("shape", WIDE, ids=["x".join(map(str, s[:5])) for s in WIDE])
def test_heads_wider_than_the_tensor_cores_tiles(bnd, shape, dtype):   # noqa: F811
    """Key or value dimensions above 128, cut, packed and short: prompt and gradient, inside the bounds of test_linear_attention_gpu.py."""
    B, T, H, dk, dv, cu = shape
    x = make(B, T, H, dk, dv, dtype, cu, seed=48)
    ld, scale, bf = slopes(H), 0.3, dtype == torch.bfloat16
    O, S = bnd.linear_attention(x["Q"], x["K"], x["V"], ld, scale=scale, S0=x["S0"], cu_seqlens=cu)
    check_forward(bnd, x, ld, cu, scale, O, S)
    got = bnd.linear_attention_backward(x["dO"], x["Q"], x["K"], x["V"], ld, scale=scale, S0=x["S0"], dS=x["dS"], cu_seqlens=cu)
    ref = lo.backward(x["dO"], x["Q"], x["K"], x["V"], ld, scale, x["S0"], x["dS"], cu)
    a = {k: v.abs() for k, v in x.items()}
    mag = lo.backward(a["dO"], a["Q"], a["K"], a["V"], ld, scale, a["S0"], a["dS"], cu)
    for i in range(4):
        lo.within(got[i], ref[i], mag[i], (int(bf) if i < 3 else 2.0 ** -8 * bf), bf and i < 3, depth(x["Q"].shape[1], max(dk, dv)))
