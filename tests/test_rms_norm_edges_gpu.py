"""GPU tests of the RMS norm and its gradient where no eps keeps a row that is not there apart from one of zeros, with row counts that leave a block partly filled.

Bounds: those of test_rms_norm_gpu.py, which counts the roundings."""
import pytest
import torch

from test_rms_norm_gpu import DTYPES, STEP, bnd, inside, make, roundings   # noqa: F401  (bnd: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", DTYPES, ids=["fp32", "bf16"])
@pytest.mark.parametrize("n", [1, 127, 128, 200, 512, 1000, 1024, 2048, 20000])
@pytest.mark.parametrize("rows", [1, 3, 9, 1001])
def test_without_eps(bnd, rows, n, dtype):   # noqa: F811
    if rows * n > 1 << 22:
        rows = 7
    x = make(rows, n, dtype, seed=8)
    h, w, dy, dh = (x[k].double() for k in ("X", "w", "dY", "dH"))
    rstd = 1 / h.square().mean(-1, keepdim=True).sqrt()
    y, _, _ = bnd.rms_norm(x["X"], x["w"], eps=0.0)
    ref = h * rstd * w
    inside(y, ref, ref.abs() * (STEP[dtype] + roundings(n)) * 1.01)
    for past in (False, True):
        dx, dw = bnd.rms_norm_backward(x["dY"], x["X"], x["w"], eps=0.0, dH=x["dH"] if past else None)
        u = dy * w
        ref = rstd * (u - h * rstd ** 2 * (u * h).mean(-1, keepdim=True)) + (dh if past else 0)
        mag = rstd * (u.abs() + h.abs() * rstd ** 2 * (u * h).abs().mean(-1, keepdim=True)) + (dh.abs() if past else 0)
        inside(dx, ref, ref.abs() * STEP[dtype] * 1.01 + mag * 4 * roundings(n))
        ref, wmag = (dy * h * rstd).sum(0), (dy * h * rstd).abs().sum(0)
        inside(dw, ref, ref.abs() * STEP[dtype] * 1.01 + wmag * (rows / 100 + 700 + n / 32) * 2.0 ** -24)
