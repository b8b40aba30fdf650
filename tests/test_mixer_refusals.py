"""What the gated recurrence and the heads' norm with rotation refuse on the host, before any device work: no GPU is needed."""
import ctypes

import numpy as np
import pytest
import torch

import __graft_entry__ as entry


@pytest.fixture(scope="module")
def lib():
    entry.build()
    from paper_2605_21325_b200 import binding
    return binding.load(), binding


# pointers that are never followed, far enough apart for the small calls here
P = [1 << 32 | i << 24 for i in range(16)]
BIG = 1 << 40


def rec(b, **kw):
    k = dict(B=2, T=300, D=40, dtype=b.F32, mode=b.REC_DECAY, n_seqs=0, cu=None)
    k.update(kw)
    cu = k.pop("cu")
    keep = None if cu is None else np.array(cu, np.int32)
    return b.RecDesc(*(k[n] for n in ("B", "T", "D", "dtype", "mode")), k["n_seqs"] if cu is None else len(cu) - 1, None if cu is None else keep.ctypes.data), keep


def test_recurrence_refuses(lib):
    L, b = lib
    names = ("X", "G", "h0", "Y", "h", "c", "w")

    def call(d, ld=(40, 40, 40), size=BIG, **over):
        p = dict(zip(names, P))
        p.update(over)
        return L.tri_inv_gated_recurrence(p["X"], ld[0], p["G"], ld[1], p["h0"], p["Y"], ld[2], p["h"], p["c"], p["w"], size, None if d is None else d[0], None)

    d = rec(b, T=3000)   # long enough to be cut, which takes a workspace
    assert call(None) == b.ERR_INVALID_ARG
    for n in ("X", "G", "w"):
        assert call(d, **{n: None}) == b.ERR_INVALID_ARG
    assert call(d, Y=None, h=None, c=None) == b.ERR_INVALID_ARG
    for n in names:
        assert call(d, **{n: P[9] + 2}) == b.ERR_INVALID_ARG, n           # not aligned to fp32 (the workspace to 16 bytes)
    for i in range(3):
        assert call(d, ld=[39 if j == i else 40 for j in range(3)]) == b.ERR_INVALID_ARG
        assert call(d, ld=[2 ** 26 + 1 if j == i else 40 for j in range(3)]) == b.ERR_UNSUPPORTED
    need = ctypes.c_size_t(0)
    assert L.tri_inv_gated_recurrence_workspace(rec(b, T=3000)[0], need) == b.OK and need.value > 0
    assert call(rec(b, T=3000), size=need.value - 1) == b.ERR_INVALID_ARG
    for bad in (dict(B=0), dict(T=-1), dict(D=0), dict(dtype=b.E4M3), dict(mode=3), dict(mode=-1), dict(B=70000, T=70000), dict(n_seqs=1),
                dict(B=1, cu=[0, 10, 5, 300]), dict(B=1, cu=[1, 300]), dict(B=1, cu=[0, 299]), dict(cu=[0, 300])):
        assert call(rec(b, **bad)) == b.ERR_INVALID_ARG, bad
        assert L.tri_inv_gated_recurrence_workspace(rec(b, **bad)[0], need) == b.ERR_INVALID_ARG
    assert call(rec(b, D=2 ** 26 + 1)) == b.ERR_UNSUPPORTED
    assert L.tri_inv_gated_recurrence_workspace(d[0], None) == b.ERR_INVALID_ARG and L.tri_inv_gated_recurrence_carries(d[0], None) == b.ERR_INVALID_ARG
    # outputs over inputs or each other, in part or with other strides
    for n, m in (("Y", "h0"), ("h", "X"), ("h", "Y"), ("c", "G"), ("c", "h"), ("c", "h0"), ("w", "X"), ("w", "Y"), ("w", "c"), ("w", "h0")):
        p = dict(zip(names, P))
        assert call(d, **{n: p[m] if n != "h" or m != "h0" else p[m] + 16}) == b.ERR_INVALID_ARG, (n, m)
    assert call(d, Y=P[0] + 160 * 3) == b.ERR_INVALID_ARG                  # Y in X, three rows on
    assert call(d, ld=(80, 40, 40), Y=P[0]) == b.ERR_INVALID_ARG           # ... with another distance of rows
    assert call(d, ld=(60, 40, 60), Y=P[0] + 100) == b.ERR_INVALID_ARG     # ... in the same rows, but over part of X
    assert call(d, h=P[2] + 16) == b.ERR_INVALID_ARG


def test_recurrence_backward_refuses(lib):
    L, b = lib
    names = ("dY", "X", "G", "h0", "dh", "c", "dX", "dG", "dh0", "w")

    def call(d, ld=(40,) * 5, size=BIG, **over):
        p = dict(zip(names, P))
        p.update(over)
        return L.tri_inv_gated_recurrence_backward(p["dY"], ld[0], p["X"], ld[1], p["G"], ld[2], p["h0"], p["dh"], p["c"], p["dX"], ld[3], p["dG"], ld[4], p["dh0"], p["w"], size, d[0], None)

    d = rec(b)
    for n in ("dY", "X", "G", "dX", "dG", "w"):
        assert call(d, **{n: None}) == b.ERR_INVALID_ARG, n
    for n in names:
        assert call(d, **{n: P[11] + 2}) == b.ERR_INVALID_ARG, n
    for i in range(5):
        assert call(d, ld=[39 if j == i else 40 for j in range(5)]) == b.ERR_INVALID_ARG
        assert call(d, ld=[2 ** 26 + 1 if j == i else 40 for j in range(5)]) == b.ERR_UNSUPPORTED
    p = dict(zip(names, P))
    for n, m in (("dX", "G"), ("dX", "h0"), ("dX", "c"), ("dG", "X"), ("dG", "dX"), ("dG", "dh"), ("dh0", "h0"), ("dh0", "c"), ("dh0", "X"), ("dh0", "dG"), ("w", "dX"), ("w", "c"), ("w", "dY")):
        assert call(d, **{n: p[m]}) == b.ERR_INVALID_ARG, (n, m)
    assert call(d, dX=p["dY"], dG=p["dY"]) == b.ERR_INVALID_ARG
    assert call(d, dX=p["X"] + 4) == b.ERR_INVALID_ARG and call(d, dh0=p["dh"] + 4) == b.ERR_INVALID_ARG
    with_carries, without = ctypes.c_size_t(0), ctypes.c_size_t(0)
    assert L.tri_inv_gated_recurrence_backward_workspace(d[0], 1, with_carries) == b.OK and L.tri_inv_gated_recurrence_backward_workspace(d[0], 0, without) == b.OK
    assert without.value > with_carries.value
    assert call(d, c=None, size=without.value - 1) == b.ERR_INVALID_ARG
    assert L.tri_inv_gated_recurrence_backward_workspace(d[0], 0, None) == b.ERR_INVALID_ARG


def test_recurrence_step_refuses(lib):
    L, b = lib
    names = ("X", "G", "h", "s", "Y")

    def call(d, n=8, ld=(40,) * 3, **over):
        p = dict(zip(names, P))
        p.update(over)
        return L.tri_inv_gated_recurrence_step(p["X"], ld[0], p["G"], ld[1], p["h"], p["s"], n, p["Y"], ld[2], d[0], None)

    d = rec(b, B=8, T=1)
    for n in ("X", "G", "h", "Y"):
        assert call(d, **{n: None}) == b.ERR_INVALID_ARG
    for n in names:
        assert call(d, **{n: P[9] + 2}) == b.ERR_INVALID_ARG
    assert call(d, n=-1) == b.ERR_INVALID_ARG and call(d, n=7, s=None) == b.ERR_INVALID_ARG
    assert call(rec(b, B=8, T=2)) == b.ERR_INVALID_ARG and call(rec(b, B=1, T=1, cu=[0, 1])) == b.ERR_INVALID_ARG
    for n, m in (("Y", "h"), ("Y", "s"), ("h", "X"), ("h", "G"), ("h", "s")):
        assert call(d, **{n: dict(zip(names, P))[m]}) == b.ERR_INVALID_ARG
    assert call(d, Y=P[0] + 4) == b.ERR_INVALID_ARG
    for i in range(3):
        assert call(d, ld=[39 if j == i else 40 for j in range(3)]) == b.ERR_INVALID_ARG


def heads(b, **kw):
    k = dict(tokens=10, T=10, H_q=4, H_k=2, d=64, r=32, interleaved=0, dtype=b.F32, eps=1e-6)
    k.update(kw)
    return b.HeadsDesc(*(k[n] for n in ("tokens", "T", "H_q", "H_k", "d", "r", "interleaved", "dtype", "eps")))


def test_heads_refuse(lib):
    L, b = lib
    names = ("Q", "K", "wq", "wk", "f", "pos", "Yq", "Yk")

    def call(d, ld=(256, 128, 256, 128), **over):
        p = dict(zip(names, P))
        p.update(over)
        return L.tri_inv_qk_norm_rope(p["Q"], ld[0], p["K"], ld[1], p["wq"], p["wk"], p["f"], p["pos"], p["Yq"], ld[2], p["Yk"], ld[3], d, None)

    d = heads(b)
    assert call(None) == b.ERR_INVALID_ARG
    for n in ("Q", "K", "f", "Yq", "Yk"):
        assert call(d, **{n: None}) == b.ERR_INVALID_ARG, n
    for n in names:
        assert call(d, **{n: P[9] + 2}) == b.ERR_INVALID_ARG, n
    for i in range(4):
        assert call(d, ld=[(256, 128, 256, 128)[j] - (j == i) for j in range(4)]) == b.ERR_INVALID_ARG
    for bad in (dict(tokens=-1), dict(tokens=2 ** 31), dict(H_q=-1), dict(H_k=-1), dict(d=0), dict(r=-1), dict(r=33), dict(interleaved=2), dict(dtype=b.E4M3), dict(eps=-1.0),
                dict(eps=float("nan")), dict(eps=float("inf")), dict(H_q=2 ** 20)):
        assert call(heads(b, **bad)) == b.ERR_INVALID_ARG, bad
    assert call(heads(b, T=0), pos=None) == b.ERR_INVALID_ARG
    assert call(heads(b, d=257, r=0), ld=(1028, 514, 1028, 514)) == b.ERR_UNSUPPORTED
    assert call(heads(b, tokens=0), **{n: None for n in names}) == b.OK
    for n, m in (("Yq", "K"), ("Yk", "Q"), ("Yk", "Yq"), ("Yq", "wq"), ("Yq", "f"), ("Yk", "pos"), ("Yk", "wk")):
        assert call(d, **{n: dict(zip(names, P))[m]}) == b.ERR_INVALID_ARG, (n, m)
    assert call(d, Yq=P[0] + 4) == b.ERR_INVALID_ARG and call(d, ld=(512, 128, 256, 128), Yq=P[0]) == b.ERR_INVALID_ARG
    # slices of one buffer beside each other are no overlap, one value further on they are
    assert call(d, ld=(512, 512, 512, 512), K=P[0] + 256 * 4, Yq=P[0] + 4) == b.ERR_INVALID_ARG


def test_heads_backward_refuse(lib):
    L, b = lib
    names = ("dYq", "dYk", "Q", "K", "wq", "wk", "f", "pos", "dQ", "dK", "dwq", "dwk", "w")
    need = ctypes.c_size_t(0)
    d = heads(b)
    assert L.tri_inv_qk_norm_rope_backward_workspace(d, need) == b.OK and L.tri_inv_qk_norm_rope_backward_workspace(d, None) == b.ERR_INVALID_ARG

    def call(d, ld=(256, 128) * 3, size=need.value, **over):
        p = dict(zip(names, P))
        p.update(over)
        return L.tri_inv_qk_norm_rope_backward(p["dYq"], ld[0], p["dYk"], ld[1], p["Q"], ld[2], p["K"], ld[3], p["wq"], p["wk"], p["f"], p["pos"], p["dQ"], ld[4], p["dK"], ld[5], p["dwq"], p["dwk"],
                                               p["w"], size, d, None)

    for n in ("dYq", "dYk", "Q", "K", "f", "dQ", "dK", "w"):
        assert call(d, **{n: None}) == b.ERR_INVALID_ARG, n
    for n in names:
        assert call(d, **{n: P[14] + 2}) == b.ERR_INVALID_ARG, n
    assert call(d, size=need.value - 1) == b.ERR_INVALID_ARG
    for i in range(6):
        assert call(d, ld=[((256, 128) * 3)[j] - (j == i) for j in range(6)]) == b.ERR_INVALID_ARG
    p = dict(zip(names, P))
    for n, m in (("dQ", "K"), ("dQ", "dYk"), ("dQ", "dK"), ("dQ", "w"), ("dQ", "wq"), ("dQ", "dwq"), ("dK", "Q"), ("dK", "pos"), ("dwq", "wq"), ("dwk", "dwq"), ("dwq", "Q"), ("w", "dYq"), ("w", "dwk")):
        assert call(d, **{n: p[m]}) == b.ERR_INVALID_ARG, (n, m)


def test_the_binding_refuses(lib):
    _, b = lib
    x, f = torch.zeros(2, 10, 40), torch.zeros(16)
    with pytest.raises(ValueError):
        b.gated_recurrence(x, x)                                           # not on a GPU
    with pytest.raises(ValueError):
        b.gated_recurrence(x[0], x[0])
    with pytest.raises(TypeError):
        b.gated_recurrence(x.double(), x.double())
    with pytest.raises(ValueError):
        b.gated_recurrence_step(x, x, x)
    with pytest.raises(ValueError):
        b.qk_norm_rope(x[0], None, None, None, f)
    with pytest.raises(ValueError):
        b.qk_norm_rope(x[:, :, None], x[:1, :, None], None, None, f)
