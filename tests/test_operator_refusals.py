"""What linear attention and the RMS norm refuse on the host, before any device work: no GPU is needed."""
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


OK, ODD = 4096, 4100   # pointers that are never followed


def desc(b, **kw):
    k = dict(B=1, T=64, H=1, d_k=64, d_v=64, C=64, kv_dtype=b.F32)
    k.update(kw)
    return b.make_desc(**k)


def test_linear_attention_refuses(lib):
    L, b = lib
    good = [OK] * 7
    call = lambda p, d, work=OK, size=1 << 40: L.tri_inv_linear_attention(*p, 1.0, work, size, d[0], None)   # noqa: E731
    d = desc(b)
    for i in (0, 1, 2, 3, 5):
        assert call(good[:i] + [None] + good[i + 1:], d) == b.ERR_INVALID_ARG
    for i in range(7):
        assert call(good[:i] + [ODD] + good[i + 1:], d) == b.ERR_INVALID_ARG
    assert L.tri_inv_linear_attention(*good, 1.0, OK, 0, None, None) == b.ERR_INVALID_ARG
    for bad in (dict(d_k=12), dict(H=0), dict(kv_dtype=7), dict(B=0), dict(T=-1), dict(d_v=4), dict(B=70000, T=70000)):
        assert call(good, desc(b, **bad)) == b.ERR_INVALID_ARG
    assert call(good, desc(b, d_k=264)) == b.ERR_UNSUPPORTED
    assert call(good, desc(b, d_v=65544)) == b.ERR_UNSUPPORTED
    for cu in ([0, 10, 5, 64], [1, 64], [0, 60]):
        assert call(good, desc(b, cu_seqlens=np.array(cu, np.int32))) == b.ERR_INVALID_ARG
    n = ctypes.c_size_t(0)
    assert L.tri_inv_linear_attention_workspace(d[0], None) == b.ERR_INVALID_ARG
    assert L.tri_inv_linear_attention_workspace(desc(b, d_k=264)[0], n) == b.ERR_UNSUPPORTED


def test_linear_attention_backward_refuses(lib):
    L, b = lib
    good = [OK] * 5 + [OK + 16, OK + 32] + [OK] * 3 + [OK + 48]
    call = lambda p, d: L.tri_inv_linear_attention_backward(*p, 1.0, OK, 1 << 40, d[0], None)   # noqa: E731
    d = desc(b)
    for i in (0, 1, 2, 3, 4, 7, 8, 9):
        assert call(good[:i] + [None] + good[i + 1:], d) == b.ERR_INVALID_ARG
    for i in range(11):
        assert call(good[:i] + [ODD] + good[i + 1:], d) == b.ERR_INVALID_ARG
    assert call(good[:10] + [good[6]], d) == b.ERR_INVALID_ARG          # dS0 in dS
    assert call(good, desc(b, d_v=264)) == b.ERR_UNSUPPORTED
    n = ctypes.c_size_t(0)
    assert L.tri_inv_linear_attention_backward_workspace(desc(b, d_v=264)[0], n) == b.ERR_UNSUPPORTED


def test_step_refuses(lib):
    L, b = lib
    good = [OK] * 6
    call = lambda p, d, n=8, o=OK: L.tri_inv_linear_attention_step(*p, n, o, 1.0, d[0], None)   # noqa: E731
    d = desc(b, B=8, T=1)
    for i in (0, 1, 2, 3, 4):
        assert call(good[:i] + [None] + good[i + 1:], d) == b.ERR_INVALID_ARG
        assert call(good[:i] + [ODD] + good[i + 1:], d) == b.ERR_INVALID_ARG
    assert call(good[:5] + [4098], d) == b.ERR_INVALID_ARG
    assert call(good, d, o=None) == b.ERR_INVALID_ARG
    assert call(good, d, n=-1) == b.ERR_INVALID_ARG
    assert call(good[:5] + [None], d, n=7) == b.ERR_INVALID_ARG         # row 7 would have no slot
    assert call(good, desc(b, B=8, T=2)) == b.ERR_INVALID_ARG
    assert call(good, desc(b, T=1, cu_seqlens=np.array([0, 1], np.int32))) == b.ERR_INVALID_ARG
    assert call(good, desc(b, T=1, d_k=264)) == b.ERR_UNSUPPORTED


def test_rms_norm_refuses(lib):
    L, b = lib
    call = lambda p=(OK,) * 6, rows=4, n=64, group=128, eps=1e-6, dt=b.F32, out=b.F32: L.tri_inv_rms_norm(*p, rows, n, group, eps, dt, out, None)   # noqa: E731
    for i in (0, 2, 3):
        assert call([None if j == i else OK for j in range(6)]) == b.ERR_INVALID_ARG
    for i in range(6):
        assert call([4097 if j == i else OK for j in range(6)], out=b.F32 if i != 5 else b.E4M3) == b.ERR_INVALID_ARG
    assert call([OK] * 5 + [None], out=b.E4M3) == b.ERR_INVALID_ARG
    assert call(rows=-1) == b.ERR_INVALID_ARG and call(n=0) == b.ERR_INVALID_ARG and call(rows=2 ** 31) == b.ERR_INVALID_ARG
    for eps in (-1e-6, float("nan"), float("inf")):
        assert call(eps=eps) == b.ERR_INVALID_ARG
    assert call(dt=b.E4M3, out=b.E4M3) == b.ERR_INVALID_ARG and call(out=b.BF16) == b.ERR_INVALID_ARG and call(dt=9) == b.ERR_INVALID_ARG
    assert call(out=b.E4M3, group=64) == b.ERR_UNSUPPORTED
    assert call((None,) * 6, rows=0) == b.OK
    need = ctypes.c_size_t(0)
    assert L.tri_inv_rms_norm_backward_workspace(4, 64, need) == b.OK and need.value > 0
    back = lambda p=(OK,) * 6, rows=4, n=64, work=OK, size=None: L.tri_inv_rms_norm_backward(*p, rows, n, 1e-6, b.F32, work, need.value if size is None else size, None)   # noqa: E731
    for i in (0, 1, 2, 4, 5):
        assert back([None if j == i else OK for j in range(6)]) == b.ERR_INVALID_ARG
    for i in range(6):
        assert back([4097 if j == i else OK for j in range(6)]) == b.ERR_INVALID_ARG
    assert back(work=None) == b.ERR_INVALID_ARG and back(work=ODD) == b.ERR_INVALID_ARG and back(size=need.value - 1) == b.ERR_INVALID_ARG
    assert back(n=0) == b.ERR_INVALID_ARG and back(rows=-1) == b.ERR_INVALID_ARG


def test_binding_names_what_it_refuses(lib):
    _, b = lib
    q = torch.zeros(1, 8, 2, 64)
    ld = torch.zeros(2)
    with pytest.raises(ValueError, match="Q must be a contiguous"):     # host tensors
        b.linear_attention(q, q, q, ld)
    with pytest.raises(ValueError, match=r"\[B, T, H, d\]"):
        b.linear_attention(q[0], q, q, ld)
    with pytest.raises(TypeError):
        b.linear_attention(q.half(), q, q, ld)
    with pytest.raises(ValueError):
        b.linear_attention_step(q, q, q, ld, torch.zeros(3, 2, 64, 64))
    with pytest.raises(TypeError, match="out_dtype"):
        b.rms_norm(torch.zeros(2, 8), torch.zeros(8), out_dtype=torch.float16)
    with pytest.raises(ValueError, match="X must be a contiguous"):
        b.rms_norm(torch.zeros(2, 8), torch.zeros(8))
