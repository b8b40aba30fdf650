"""GPU tests of linear attention's routes: the give-up path of its waits, the two ways of marshalling, both widths of the value columns, many items a block."""
import ctypes

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


def make(B, T, H, dk, dv, dtype=torch.bfloat16, seed=0, n=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)   # noqa: E731
    x = {"Q": r(B, T, H, dk).to(dtype), "K": r(B, T, H, dk).to(dtype), "V": r(B, T, H, dv).to(dtype), "dO": r(B, T, H, dv).to(dtype)}
    x["S0"], x["dS"] = r(n or B, H, dk, dv), r(n or B, H, dk, dv)
    return x, -(2.0 ** (-8.0 * torch.arange(1, H + 1, device="cuda") / H))


def check(x, ld, O, S, cu=None, scale=1.0, S0=None):
    ref = lo.forward(x["Q"], x["K"], x["V"], ld, scale, S0, cu)
    mag = lo.forward(x["Q"].abs(), x["K"].abs(), x["V"].abs(), ld, scale, None if S0 is None else S0.abs(), cu)
    depth = 2 * (x["Q"].shape[3] + 64) + 4 * (x["Q"].shape[1] // 64 + 1) + 128      # as in test_linear_attention_gpu.py
    bf = x["Q"].dtype == torch.bfloat16
    lo.within(O, ref[0], mag[0], int(bf), bf, depth)
    if S is not None:
        lo.within(S, ref[1], mag[1], 2.0 ** -8 * bf, False, depth)


@pytest.mark.parametrize("d", [64, 128])
def test_a_wait_that_runs_out(bnd, d):
    """One block's waits run out: the status word says so, once; every other head's output is as usual, and so is the next call."""
    x, ld = make(2, 320, 3, d, d, seed=1)
    out = torch.zeros_like(x["V"])
    bnd.selftest_linear_wait_timeout(x["Q"], x["K"], x["V"], ld, 5_000_000, out)
    assert bnd.last_device_status() == bnd.ERR_DEVICE_TIMEOUT
    assert bnd.last_device_status() == bnd.OK
    O, S = bnd.linear_attention(x["Q"], x["K"], x["V"], ld)
    torch.cuda.synchronize()
    assert bnd.last_device_status() == bnd.OK
    check(x, ld, O, S)
    keep = torch.ones(2, 320, 3, dtype=torch.bool, device="cuda")
    keep[0, :, 0] = False
    diff = (out.double() - O.double()).abs()[keep]
    # the state is not asked for there, so its increments are rounded to bf16: two roundings a term on one side, one on the other, and both outputs'
    mag = lo.forward(x["Q"].abs(), x["K"].abs(), x["V"].abs(), ld, 1.0, None, None)[0][keep]
    assert bool((diff <= 4 * 2.0 ** -8 * mag + 2 * 2.0 ** -8 * O.double().abs()[keep]).all())


def test_native_marshalling_gives_the_python_bodys_bits(bnd):
    """The extension's calls against the ctypes ones (taken where a stream is named)."""
    cur = torch.cuda.current_stream()
    x, ld = make(1, 300, 3, 128, 64, seed=2, n=3)
    cu = [0, 100, 100, 300]
    fwd = lambda **k: bnd.linear_attention(x["Q"], x["K"], x["V"], ld, scale=0.5, S0=x["S0"], cu_seqlens=cu, **k)   # noqa: E731
    bwd = lambda **k: bnd.linear_attention_backward(x["dO"], x["Q"], x["K"], x["V"], ld, scale=0.5, S0=x["S0"], dS=x["dS"], cu_seqlens=cu, **k)   # noqa: E731
    for f in (fwd, bwd):
        for a, b in zip(f(), f(stream=cur)):
            assert torch.equal(a, b)
    assert fwd(want_state=0)[1] is None and fwd(want_state=1)[1] is not None
    assert bwd(want_dS0=False)[3] is None
    assert torch.equal(fwd()[0], bnd.linear_attention(x["Q"], x["K"], x["V"], ld, scale=0.5, S0=x["S0"], cu_seqlens=np.array(cu, np.int32))[0])
    q, k, v = x["Q"][0, :5].contiguous(), x["K"][0, :5].contiguous(), x["V"][0, :5].contiguous()
    s1 = torch.randn(5, 3, 128, 64, device="cuda")
    s2 = s1.clone()
    assert torch.equal(bnd.linear_attention_step(q, k, v, ld, s1, scale=0.5), bnd.linear_attention_step(q, k, v, ld, s2, scale=0.5, stream=cur)) and torch.equal(s1, s2)
    w = torch.randn(128, device="cuda").bfloat16()
    X = x["Q"]
    for kw in (dict(), dict(residual=x["K"]), dict(residual=x["K"], out_dtype=torch.float8_e4m3fn), dict(out_dtype=torch.float8_e4m3fn, group=0)):
        for a, b in zip(bnd.rms_norm(X, w, **kw), bnd.rms_norm(X, w, stream=cur, **kw)):
            assert (a is None and b is None) or torch.equal(a.float(), b.float())
    for a, b in zip(bnd.rms_norm_backward(x["K"], X, w, dH=X), bnd.rms_norm_backward(x["K"], X, w, dH=X, stream=cur)):
        assert torch.equal(a, b)
    with pytest.raises(bnd.TriInvError) as e:
        bnd.linear_attention(X, X, X, ld, cu_seqlens=[0, 200, 100, 300])
    assert e.value.status == bnd.ERR_INVALID_ARG
    with pytest.raises(ValueError, match="K must have shape"):
        bnd.linear_attention(X, X[:, :5].contiguous(), X, ld)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("shape", [(40, 70, 4, 128, 128), (1, 0, 7, 128, 128), (1, -1, 2, 64, 64), (200, 3, 2, 64, 64), (1, 640, 75, 128, 128)],
                         ids=["short", "packed", "packed_many", "tiny", "heads"])
def test_more_items_than_blocks(bnd, shape, dtype):
    """Blocks that walk several heads and sequences one after the other, of lengths that differ, empty ones among them."""
    B, T, H, dk, dv = shape
    cu, n = None, None
    if T <= 0:
        lens = [(37 * i) % 151 for i in range(60)] if T == 0 else [(5 * i) % 9 for i in range(700)]   # (more than one launch's worth of the table)
        cu = np.cumsum([0] + lens).astype(np.int32)
        B, T, n = 1, int(cu[-1]), len(lens)
    x, ld = make(B, T, H, dk, dv, dtype, seed=3, n=n)
    O, S = bnd.linear_attention(x["Q"], x["K"], x["V"], ld, scale=0.3, S0=x["S0"], cu_seqlens=cu)
    torch.cuda.synchronize()
    assert bnd.last_device_status() == 0
    check(x, ld, O, S, cu, 0.3, x["S0"])
    g = bnd.linear_attention_backward(x["dO"], x["Q"], x["K"], x["V"], ld, scale=0.3, S0=x["S0"], dS=x["dS"], cu_seqlens=cu)
    ref = lo.backward(x["dO"], x["Q"], x["K"], x["V"], ld, 0.3, x["S0"], x["dS"], cu)
    a = {k: v.abs() for k, v in x.items()}
    mag = lo.backward(a["dO"], a["Q"], a["K"], a["V"], ld, 0.3, a["S0"], a["dS"], cu)
    bf = dtype == torch.bfloat16
    for i in range(4):
        lo.within(g[i], ref[i], mag[i], (int(bf) if i < 3 else 2.0 ** -8 * bf), bf and i < 3, 2 * (128 + 64) + 4 * (T // 64 + 1) + 128)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
def test_cut_sequences_among_many(bnd, dtype):
    """More sequences than one launch of the table takes, two of them long enough to be cut, one in each launch's part; forward and gradient."""
    lens = [(7 * i) % 11 for i in range(400)]
    lens[5], lens[390] = 5000, 3001
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    B, T, H, dk, dv, n = 1, cu[-1], 1, 64, 64, len(lens)
    x, ld = make(B, T, H, dk, dv, dtype, seed=4, n=n)
    need = ctypes.c_size_t(0)
    desc, _ = bnd.make_desc(B, T, H, dk, dv, 64, bnd._dtype_code(x["Q"]), cu)
    assert bnd.load().tri_inv_linear_attention_workspace(ctypes.byref(desc), ctypes.byref(need)) == 0
    assert need.value > 400 * 20 + 2 * dk * dv * 4   # states of segments beside the table
    O, S = bnd.linear_attention(x["Q"], x["K"], x["V"], ld, scale=0.3, S0=x["S0"], cu_seqlens=cu)
    check(x, ld, O, S, cu, 0.3, x["S0"])
    g = bnd.linear_attention_backward(x["dO"], x["Q"], x["K"], x["V"], ld, scale=0.3, S0=x["S0"], dS=x["dS"], cu_seqlens=cu)
    ref = lo.backward(x["dO"], x["Q"], x["K"], x["V"], ld, 0.3, x["S0"], x["dS"], cu)
    a = {k: v.abs() for k, v in x.items()}
    mag = lo.backward(a["dO"], a["Q"], a["K"], a["V"], ld, 0.3, a["S0"], a["dS"], cu)
    bf = dtype == torch.bfloat16
    for i in range(4):
        lo.within(g[i], ref[i], mag[i], (int(bf) if i < 3 else 2.0 ** -8 * bf), bf and i < 3, 2 * (128 + 64) + 4 * (5000 // 64 + 1) + 128)


def test_offsets_past_two_to_the_31st(bnd):
    """A tensor of more than 2^31 elements: the last head of the last tokens, against the same sequence alone."""
    B, T, H, d = 33, 8192, 64, 128
    q = torch.randn(1, T, H, d, device="cuda").bfloat16()
    big = q.expand(B, T, H, d).contiguous()
    ld = -(2.0 ** (-8.0 * torch.arange(1, H + 1, device="cuda") / H))
    O, S = bnd.linear_attention(big, big, big, ld, scale=0.01)
    one, S1 = bnd.linear_attention(q, q, q, ld, scale=0.01)
    torch.cuda.synchronize()
    assert bnd.last_device_status() == 0
    # (the single sequence may be cut into segments: roundings of its states at other places)
    assert float((O[-1].float() - one[0].float()).abs().max()) <= 0.02 * float(one.float().abs().max())
    assert torch.equal(O[0], O[-1]) and torch.equal(S[0], S[-1])
