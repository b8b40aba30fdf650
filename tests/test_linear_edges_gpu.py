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
