"""Linear attention and the RMS norm allocate no device memory of their own: across calls with the caller's outputs and workspaces (after the first ones on the device) neither the free memory
that the driver reports nor torch's allocator moves."""
import ctypes

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def bnd():
    import __graft_entry__ as entry
    entry.build()
    from paper_2605_21325_b200 import binding
    torch.cuda.set_device(0)
    return binding


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("cu", [None, [0, 0, 70, 3000]], ids=["dense", "packed"])
def test_nothing_is_allocated(bnd, cu, dtype):
    L, T, H, d = bnd.load(), 3000, 2, 64
    n = 1 if cu is None else len(cu) - 1
    new = lambda *s, dt=dtype: torch.randn(*s, device="cuda").to(dt)   # noqa: E731
    p = lambda *t: [x.data_ptr() for x in t]   # noqa: E731
    q, k, v, x, o, dq, dk, dv = (new(1, T, H, d) for _ in range(8))
    s0, s1, ds, ds0 = (new(n, H, d, d, dt=torch.float32) for _ in range(4))
    ld, w, dw, codes, scales = -new(H, dt=torch.float32).abs(), new(d), new(d), torch.empty(T * H, d, dtype=torch.uint8, device="cuda"), new(T * H, dt=torch.float32)
    desc, keep = bnd.make_desc(1, T, H, d, d, 64, bnd._dtype_code(q), cu)   # noqa: F841
    step, _ = bnd.make_desc(n, 1, H, d, d, 64, bnd._dtype_code(q))
    code, need, work = bnd._dtype_code(q), ctypes.c_size_t(0), []
    for f, a in (("linear_attention", (ctypes.byref(desc),)), ("linear_attention_backward", (ctypes.byref(desc),)), ("rms_norm_backward", (T * H, d))):
        assert getattr(L, "tri_inv_%s_workspace" % f)(*a, ctypes.byref(need)) == 0 and need.value > 0
        work.append((torch.empty(need.value, dtype=torch.uint8, device="cuda"), need.value))
    (w1, n1), (w2, n2), (w3, n3) = [(t.data_ptr(), m) for t, m in work]

    def calls():
        assert L.tri_inv_linear_attention(*p(q, k, v, ld, s0, o, s1), 1.0, w1, n1, ctypes.byref(desc), None) == 0
        assert L.tri_inv_linear_attention_backward(*p(x, q, k, v, ld, s0, ds, dq, dk, dv, ds0), 1.0, w2, n2, ctypes.byref(desc), None) == 0
        assert L.tri_inv_linear_attention_step(*p(q, k, v, ld, s0), None, n, o.data_ptr(), 1.0, ctypes.byref(step), None) == 0
        assert L.tri_inv_rms_norm(*p(q, k, w, o, x), None, T * H, d, 128, 1e-6, code, code, None) == 0
        assert L.tri_inv_rms_norm(*p(q, k, w, codes), None, scales.data_ptr(), T * H, d, 0, 1e-6, code, bnd.E4M3, None) == 0
        assert L.tri_inv_rms_norm_backward(*p(v, q, w, k, dq, dw), T * H, d, 1e-6, code, w3, n3, None) == 0

    calls()
    torch.cuda.synchronize()
    free, reserved, allocs = torch.cuda.mem_get_info()[0], torch.cuda.memory_reserved(), torch.cuda.memory_stats().get("allocation.all.allocated", 0)
    for _ in range(3):
        calls()
    torch.cuda.synchronize()
    assert torch.cuda.mem_get_info()[0] == free
    assert torch.cuda.memory_reserved() == reserved and torch.cuda.memory_stats().get("allocation.all.allocated", 0) == allocs
    assert bnd.last_device_status() == 0
