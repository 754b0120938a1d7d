"""The factor of a scale block in acrl_matmul_fp8, x_scale * w_scale rounded to
fp32: scales of any size whose product lies in fp32's normal range act as the
definition says; past it the result is that of the rounded factor, as
include/acrl.h states."""
import numpy as np
import pytest

from gpu_util import down, torch_dev, up
from operators64 import e4m3_values, product

pytestmark = pytest.mark.gpu
ROWS = [5, 40, 300]  # the kernel for few tokens, small and larger tiles
N = 200              # two blocks of outputs


def _operands(M, K, seed):
    """Codes of whole numbers -4 .. 4; one weight row of zeros in each block of outputs."""
    val = e4m3_values()
    codes = np.array([int(np.flatnonzero(val == v)[0]) for v in range(-4, 5)], np.uint8)
    r = np.random.default_rng(seed)
    xq, wq = codes[r.integers(0, 9, (M, K))], codes[r.integers(0, 9, (N, K))]
    wq[[3, 150]] = codes[4]
    return xq, wq


def _run(xq, xs, wq, ws):
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    return down(acrl.acrl_matmul_fp8(*[up(torch, dev, a) for a in (xq, xs, wq, ws)], out_dtype=torch.float32))


@pytest.mark.parametrize("M", ROWS)
@pytest.mark.parametrize("ex,ew", [(110, -112), (-140, 100), (60, 50), (-70, -50), (-125, 0)])
def test_products_of_normal_size(M, ex, ew):
    # powers of two: every step is exact while the factors, sums and partial sums are normal
    K = 288
    xq, wq = _operands(M, K, abs(M + ex))
    r = np.random.default_rng(abs(ex - ew))
    xs = np.exp2(ex + r.integers(-1, 2, (M, 3))).astype(np.float32)
    ws = np.exp2(ew + r.integers(0, 2, (2, 3))).astype(np.float32)
    want = product(xq, xs, wq, ws)[0]
    assert np.array_equal(_run(xq, xs, wq, ws), want.astype(np.float32))


@pytest.mark.parametrize("M", ROWS)
@pytest.mark.parametrize("sx,sw", [(3e25, 2e19), (1.7e38, 1.9), (7e-23, 9e-23), (1.3e-30, 1.1e-14), (3e-30, 2e-20)])
def test_products_past_it(M, sx, sw):
    # one block of K: the sum t, exact, times the factor rounded to fp32, rounded once
    K = 128
    xq, wq = _operands(M, K, M)
    val = e4m3_values()
    t = val[xq] @ val[wq].T
    xs = np.float32(sx) * np.random.default_rng(M).uniform(0.9, 1.1, (M, 1)).astype(np.float32)
    ws = np.full((2, 1), np.float32(sw))
    with np.errstate(all="ignore"):
        factor = xs * ws[0]
        want = (t * factor.astype(np.float64)).astype(np.float32)
    y = _run(xq, xs, wq, ws)
    assert np.array_equal(y, want, equal_nan=True)
    if sx > 1 and np.isinf(factor).all():
        assert np.isnan(y[:, 3]).all() and np.isinf(y[t != 0]).all()
    if sx < 1:
        assert (np.abs(factor) < np.finfo(np.float32).tiny).all() and not y[:, 3].any()
