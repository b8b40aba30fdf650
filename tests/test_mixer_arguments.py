"""Arguments of the gated recurrence and of the heads' norm that the binding has to turn away itself, because the C call could not see them: no GPU is needed."""
import numpy as np
import pytest
import torch

import __graft_entry__ as entry


@pytest.fixture(scope="module")
def bnd():
    entry.build()
    from paper_2605_21325_b200 import binding
    return binding


@pytest.mark.parametrize("q,k", [(torch.float32, torch.bfloat16), (torch.bfloat16, torch.float32)], ids=["fp32-bf16", "bf16-fp32"])
def test_queries_and_keys_of_different_types(bnd, q, k):
    """One storage type goes with a call: keys of half as many bytes would be read past their end."""
    Q, K, f = torch.zeros(2, 10, 4, 64, dtype=q), torch.zeros(2, 10, 2, 64, dtype=k), torch.zeros(32)
    for call in (lambda **kw: bnd.qk_norm_rope(Q, K, None, None, f, **kw), lambda **kw: bnd.qk_norm_rope_backward(Q, K, Q, K, None, None, f, **kw)):
        for kw in (dict(), dict(out=(Q, K))):
            with pytest.raises(TypeError, match="K must be"):
                call(**kw)


def test_offsets_that_32_bits_do_not_hold(bnd):
    """They wrapped: 2^32 + 100 was a sequence of 100 tokens."""
    X = torch.zeros(1, 300, 40)
    for bad in ([0, 2 ** 32 + 100, 300], np.array([0, 2 ** 32 + 100, 300]), (0, -2 ** 32 + 100, 300), [0, 100.5, 300], [0, float("nan"), 300], [[0, 300]], torch.tensor([0, 2 ** 40, 300])):
        for call in (lambda: bnd.gated_recurrence_carries(X, bad), lambda: bnd.make_desc(1, 300, 2, 64, 64, 64, bnd.F32, cu_seqlens=bad)):
            with pytest.raises(ValueError, match="cu_seqlens"):
                call()
    want = bnd.gated_recurrence_carries(X, [0, 100, 300])
    for good in ((0, 100, 300), np.array([0, 100, 300]), torch.tensor([0, 100, 300]), np.array([0, 100, 300], np.uint64), np.array([0.0, 100.0, 300.0])):
        assert bnd.gated_recurrence_carries(X, good) == want


def test_sizes_that_32_bits_do_not_hold(bnd):
    """They wrapped: 2^32 + 100 tokens were 100, and the others' outputs as the memory was."""
    n, f32 = 2 ** 32 + 100, torch.float32
    e = lambda *s, dtype=f32: torch.empty(*s, dtype=dtype, device="meta")   # noqa: E731
    X, w = e(1, n, 1), e(1)
    long, few = e(n, 1), e(4, 1)
    calls = [lambda: bnd.gated_recurrence_carries(X), lambda: bnd.gated_recurrence(X, X), lambda: bnd.gated_recurrence(e(1, 5, n), e(1, 5, n)), lambda: bnd.gated_recurrence(e(1, 5, 1), e(1, 5, 1), mode=1 << 32),
             lambda: bnd.gated_recurrence_backward(X, X, X), lambda: bnd.gated_recurrence_step(long, long, few), lambda: bnd.gated_recurrence_step(few, few, long),
             lambda: bnd.qk_norm_rope(e(5, n, 1), None, None, None, None), lambda: bnd.qk_norm_rope(e(5, 1, 1), e(5, n, 1), None, None, None), lambda: bnd.qk_norm_rope(e(5, 1, n), None, None, None, None),
             lambda: bnd.qk_norm_rope_backward(e(n, 1, 1), None, e(n, 1, 1), None, None, None, None), lambda: bnd.qk_norm_rope(e(5, 1, 1), None, None, None, e(n)),
             lambda: bnd.make_desc(1, n, 2, 64, 64, 64, bnd.F32), lambda: bnd.linear_attention_step(e(4, 1, 1), e(4, 1, 1), e(4, 1, 1), w, e(n, 1, 1, 1)),
             lambda: bnd.rms_norm(e(1, n), e(n)), lambda: bnd.rms_norm_backward(e(1, n), e(1, n), e(n))]
    for call in calls:
        with pytest.raises(ValueError, match="32 bits"):
            call()
