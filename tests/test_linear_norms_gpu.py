"""How far linear attention and its gradient are from 64 bits in the norm of each head: next to the element by element bounds, which leave room for small mistakes in every element.

Bounds.  A rounding to bf16 is off by at most 2^-8 of its value, so by at most 2^-8 / sqrt 3 = 2.3e-3 in the root mean square.  An element of O, dQ, dK or dV is rounded itself and is a sum of terms of which
each met one such rounding (P, or the state); the terms are of either sign and as good as independent, so the two add up to at most sqrt 2 x 2.3e-3 = 3.2e-3 of the norm: 5e-3 over a
thousand values and more.  A state's increments keep 16 bits, 2^-16 = 1.5e-5 at most, and its other roundings are fp32's: 2e-5.  fp32 storage: about 500 roundings on a term's way (depth() of
test_linear_attention_gpu.py), sqrt 500 x 2^-24 / sqrt 3 = 8e-7, and factors whose exponents are off by 2^-24 of up to ten: 2e-6."""
import pytest
import torch

import linear_oracle as lo
from test_linear_attention_gpu import DTYPES, SHAPES, bnd, make, slopes   # noqa: F401  (bnd: the fixture)

OUT = {torch.bfloat16: 5e-3, torch.float32: 2e-6}
STATE = {torch.bfloat16: 2e-5, torch.float32: 2e-6}
LARGE = [s for s in SHAPES if (s[0] * s[1] if s[5] is None else int(s[5][-1])) * min(s[3:5]) >= 1024]
IDS = ["x".join(map(str, s[:5])) + ("_packed" if s[5] is not None else "") for s in LARGE]


def off(got, ref, head):
    """The largest over the heads of |got - ref| / |ref|; ``head``: the heads' dimension."""
    dims = [i for i in range(ref.dim()) if i != head]
    return float(((got.double() - ref).square().sum(dims) / ref.square().sum(dims)).sqrt().max())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES, ids=["fp32", "bf16"])
@pytest.mark.parametrize("shape", LARGE, ids=IDS)
def test_distance(bnd, shape, dtype):   # noqa: F811
    B, T, H, dk, dv, cu = shape
    x = make(B, T, H, dk, dv, dtype, cu, seed=7 * T + dk)
    ld, scale = slopes(H), 0.3
    O, S = bnd.linear_attention(x["Q"], x["K"], x["V"], ld, scale=scale, S0=x["S0"], cu_seqlens=cu)
    refO, refS = lo.forward(x["Q"], x["K"], x["V"], ld, scale, x["S0"], cu)
    assert off(O, refO, 2) <= OUT[dtype] and off(S, refS, 1) <= STATE[dtype]
    got = bnd.linear_attention_backward(x["dO"], x["Q"], x["K"], x["V"], ld, scale=scale, S0=x["S0"], dS=x["dS"], cu_seqlens=cu)
    ref = lo.backward(x["dO"], x["Q"], x["K"], x["V"], ld, scale, x["S0"], x["dS"], cu)
    assert [off(g, r, 2) <= OUT[dtype] for g, r in zip(got[:3], ref)] == [True] * 3 and off(got[3], ref[3], 1) <= STATE[dtype]


@pytest.mark.parametrize("shape", LARGE, ids=IDS)
def test_a_decay_two_per_cent_off_would_show(shape):
    """Of the bounds themselves, on the CPU: a log-decay that is 2 % wrong moves some head's O further than the wider of them (130 tokens of 8 features: 5 %)."""
    B, T, H, dk, dv, cu = shape
    if cu is not None:
        B, T = 1, int(cu[-1])
    g = torch.Generator().manual_seed(T)
    q, k, v = (torch.randn(B, T, H, d, generator=g) for d in (dk, dk, dv))
    ld = -(2.0 ** (-8.0 * torch.arange(1, H + 1) / H))
    right = lo.forward(q, k, v, ld, 0.3, None, cu)[0]
    wrong = lo.forward(q, k, v, ld * (1.02 if dk > 8 else 1.05), 0.3, None, cu)[0]
    assert off(wrong, right, 2) > OUT[torch.bfloat16]
