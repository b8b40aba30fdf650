"""Buffers that may not overlap and sizes that cannot be counted are refused on the host, before any device work: no GPU is needed.  (Only refusals are called here: the pointers are never followed.)"""
import pytest

import __graft_entry__ as entry


@pytest.fixture(scope="module")
def lib():
    entry.build()
    from paper_2605_21325_b200 import binding
    return binding.load(), binding


MB = 1 << 20
TOKENS, STATE = 2 * 64 * 3 * 64 * 4, 2 * 3 * 64 * 64 * 4      # bytes of a tensor of tokens and of the states below


def desc(b, **kw):
    k = dict(B=2, T=64, H=3, d_k=64, d_v=64, C=64, kv_dtype=b.F32)
    k.update(kw)
    return b.make_desc(**k)


def apart(n):
    return [MB * (1 + i) for i in range(n)]


def over(size, other):
    """Where a buffer of ``size`` bytes meets one of ``other`` bytes at 0: at its start, its last 16 bytes, and with its own last 16."""
    return 0, other - 16, 16 - size


def test_a_gradient_in_an_input_state(lib):
    L, b = lib
    p = apart(11)                                    # dO Q K V log_decay S0 dS | dQ dK dV dS0
    call = lambda q: L.tri_inv_linear_attention_backward(*q, 1.0, MB * 64, 1 << 30, desc(b)[0], None)   # noqa: E731
    for other in (5, 6):
        for at in over(STATE, STATE):
            assert call(p[:10] + [p[other] + at]) == b.ERR_INVALID_ARG


def test_linear_attention_backward(lib):
    L, b = lib
    p = apart(11)
    call = lambda q: L.tri_inv_linear_attention_backward(*q, 1.0, MB * 64, 1 << 30, desc(b)[0], None)   # noqa: E731
    sizes = [TOKENS] * 4 + [16] + [STATE] * 2 + [TOKENS] * 3 + [STATE]
    for out in (7, 8, 9, 10):
        for i in range(11):
            if i != out:
                for at in over(sizes[out], sizes[i]):
                    assert call([p[i] + at if j == out else x for j, x in enumerate(p)]) == b.ERR_INVALID_ARG, (out, i, at)


def test_linear_attention(lib):
    L, b = lib
    p = apart(7)                                     # Q K V log_decay S0 | O S_out
    call = lambda q: L.tri_inv_linear_attention(*q, 1.0, MB * 64, 1 << 30, desc(b)[0], None)   # noqa: E731
    sizes = [TOKENS, TOKENS, TOKENS, 12, STATE, TOKENS, STATE]
    for i in (0, 1, 2, 3, 4, 6):
        for at in over(TOKENS, max(sizes[i], 16)):
            assert call(p[:5] + [p[i] + at] + p[6:]) == b.ERR_INVALID_ARG
    for i in (0, 1, 2, 3, 4):
        for at in over(STATE, max(sizes[i], 16)):
            if i != 4 or at:                         # S_out may be S0 itself
                assert call(p[:6] + [p[i] + at]) == b.ERR_INVALID_ARG


def test_step(lib):
    L, b = lib
    p = apart(6)                                     # Q K V log_decay S slots
    row, slots = 8 * 3 * 64 * 4, 8 * 4
    call = lambda o: L.tri_inv_linear_attention_step(*p, 8, o, 1.0, desc(b, B=8, T=1)[0], None)   # noqa: E731
    for i, size in ((0, row), (1, row), (2, row), (3, 16), (4, 8 * 3 * 64 * 64 * 4), (5, slots)):
        for at in over(row, size):
            if i != 2 or at:                         # O may be V itself
                assert call(p[i] + at) == b.ERR_INVALID_ARG, (i, at)


def test_states_of_a_step_over_its_operands(lib):
    L, b = lib
    p = apart(6)                                     # Q K V log_decay S slots
    row, state = 8 * 3 * 64 * 4, 8 * 3 * 64 * 64 * 4
    call = lambda s: L.tri_inv_linear_attention_step(*p[:4], s, p[5], 8, MB * 32, 1.0, desc(b, B=8, T=1)[0], None)   # noqa: E731
    for i, size in ((0, row), (1, row), (2, row), (3, 16), (5, 32)):
        for at in over(state, size):
            assert call(p[i] + at) == b.ERR_INVALID_ARG, (i, at)


def test_rows_too_long_to_count(lib):
    L, b = lib
    for n in (2 ** 31 - 1, 2 ** 31 - 255):
        assert L.tri_inv_rms_norm(4096, None, 4096, 4096, None, None, 1, n, 128, 1e-6, b.F32, b.F32, None) == b.ERR_UNSUPPORTED
        assert L.tri_inv_rms_norm_backward(4096, 4096, 4096, None, 4096, 4096, 1, n, 1e-6, b.F32, 4096, 1 << 60, None) == b.ERR_UNSUPPORTED
