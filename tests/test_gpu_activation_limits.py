"""Activations of infinities and of values next to where their formulas end, the
same for every type of y: as the formulas have them, infinity times 0 is NaN."""
import numpy as np
import pytest

from decode64 import ACT_ERROR, HALF, act
from gpu_util import down, torch_dev, up

pytestmark = pytest.mark.gpu

ACTS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3, "gelu_tanh": 4}
OF_MINUS_INFINITY = {"none": -np.inf, "relu": 0.0, "silu": np.nan, "gelu": np.nan, "gelu_tanh": np.nan}


def _of_bias(torch, dev, v, M, name, out):
    """act(v) by way of the bias of a product of zeros."""
    from paper_2607_24062_amd import acrl
    z = lambda n: torch.zeros((n, 128), dtype=torch.uint8, device=dev)  # noqa: E731
    one = lambda n: torch.ones((n, 1), device=dev)  # noqa: E731
    y = acrl.acrl_linear_fp8(z(M), one(M), z(v.size), one((v.size + 127) // 128), bias=up(torch, dev, v), activation=ACTS[name],
                             out_dtype=torch.float32 if out == "f32" else torch.bfloat16)
    return down(y.float())


@pytest.mark.parametrize("M", [1, 16, 20, 300])
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("name", list(ACTS))
def test_infinities_and_nan(name, out, M):
    torch, dev = torch_dev()
    v = np.array([np.inf, -np.inf, np.nan, -1.0] * 9, np.float32)
    got = _of_bias(torch, dev, v, M, name, out)
    assert (got[:, 0::4] == np.inf).all()
    assert np.array_equal(got[:, 1::4], np.full_like(got[:, 1::4], OF_MINUS_INFINITY[name]), equal_nan=True)
    assert np.isnan(got[:, 2::4]).all() and np.isfinite(got[:, 3::4]).all()


@pytest.mark.parametrize("M", [1, 20])
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("name", list(ACTS))
def test_far_from_zero(name, out, M):
    # finite values of every size on both sides: no infinity and no NaN comes of them, and results are within their bounds
    torch, dev = torch_dev()
    v = np.array([s * m for m in (19.0, 19.999998, 20.0, 20.000002, 21.0, 1e2, 1e4, 1e19, 1e20, 1.8e19, 1e25, 1e38, 3.38e38)
                  for s in (1.0, -1.0)], np.float32)
    got = _of_bias(torch, dev, v, M, name, out)
    want = act(name, v)
    assert (np.abs(got - want) <= (ACT_ERROR[out] + HALF[out]) * np.abs(want) + 1.3e-36).all(), name


def test_gate_of_minus_infinity_in_experts():
    # a gate of -infinity is the token's own NaN, whatever the type of y
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    d, F = 32, 32
    w_in = torch.zeros((1, 2 * F, d), dtype=torch.uint8, device=dev)
    w_in[:, :, 0] = 0x38  # 1.0
    w_out = torch.full((1, d, F), 0x38, dtype=torch.uint8, device=dev)
    one = torch.ones((1, 1, 1), device=dev)
    x = torch.zeros((2, d), dtype=torch.bfloat16, device=dev)
    x[0, 0], x[1, 0] = -float("inf"), -2.0
    ids, w = torch.zeros((2, 1), dtype=torch.int32, device=dev), torch.ones((2, 1), device=dev)
    for name in ("silu", "gelu", "gelu_tanh"):
        for out in (torch.float32, torch.bfloat16):
            y = acrl.acrl_moe_fp8(x, w_in, one, w_out, one, 1, ids=ids, weights=w, activation=ACTS[name], out_dtype=out)[0]
            assert bool(torch.isnan(y[0]).all()) and bool(torch.isfinite(y[1]).all()), name
