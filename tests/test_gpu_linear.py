"""acrl_linear_fp8 against its definition in 64 bits.

Tolerance: the product's own (operators64.product: what the matrix instruction
and fp32 sums may lose), through the activation's slope, the epilogue's fp32
roundings, and half a step of the output's type."""
import numpy as np
import pytest

from cases import random_bf16
from decode64 import ACT_ERROR, HALF, act, f64, linear
from gpu_util import bf16_bits, down, torch_dev, up, up_bf16
from operators64 import product, quantize_blocks

pytestmark = pytest.mark.gpu

ACTS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3, "gelu_tanh": 4}


def _operands(torch, dev, M, N, K, seed):
    x, w = random_bf16((M, K), seed), random_bf16((N, K), seed + 1, std=1.5 / np.sqrt(K))
    (xq, xs), (wq, ws) = quantize_blocks(x, 1), quantize_blocks(w, 128)
    return (xq, xs, wq, ws), [up(torch, dev, a) for a in (xq, xs, wq, ws)]


def _values(torch, dev, shape, kind, seed, std=1.0):
    """(values in 64 bits, device tensor) of an array of the type."""
    if kind == "bf16":
        b = random_bf16(shape, seed, std=std)
        return f64(b).reshape(shape), up_bf16(torch, dev, b.reshape(shape))
    a = (np.random.default_rng(seed).normal(size=shape) * std).astype(np.float32)
    return a.astype(np.float64), up(torch, dev, a)


def _check(got, want, tol, kind):
    got = got.astype(np.float64)
    bound = tol * 1.01 + HALF[kind] * (np.abs(want) + tol)
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:3], got[bad][:3], want[bad][:3], bound[bad][:3])


# sizes of every tiling and of the two kernels for up to 16 tokens, odd in all; the last block of K whole or cut
SIZES = [(1, 16, 32), (1, 77, 160), (16, 130, 2080), (7, 5121, 96), (1, 5130, 256), (17, 70, 640), (33, 4641, 224),
         (67, 5460, 128), (131, 5470, 160), (259, 6557, 96), (519, 7190, 64), (1029, 7213, 32)]
EPILOGUES = [("none", "", "bf16", "bf16"), ("relu", "f32", "", "f32"), ("silu", "bf16", "f32", "bf16"),
             ("gelu", "f32", "bf16", "f32"), ("gelu_tanh", "", "", "bf16")]


@pytest.mark.parametrize("M,N,K", SIZES)
def test_sizes(M, N, K):
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    host, t = _operands(torch, dev, M, N, K, 3)
    y, slack = product(*host)
    for name, bias, res, out in EPILOGUES if M * N < 1 << 20 else EPILOGUES[2:4]:
        b, tb = _values(torch, dev, (N,), bias, 5) if bias else (None, None)
        r, tr = _values(torch, dev, (M, N), res, 6, 3.0) if res else (None, None)
        got = acrl.acrl_linear_fp8(*t, bias=tb, activation=ACTS[name], residual=tr,
                                   out_dtype=torch.bfloat16 if out == "bf16" else torch.float32)
        _check(down(got.float()), *linear(y, slack, name, b, r, out), out)


@pytest.mark.parametrize("M", [3, 40, 300])
def test_nothing_asked_for_is_the_plain_product(M):
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    _, t = _operands(torch, dev, M, 200, 512, 8)
    for dtype in (torch.bfloat16, torch.float32):
        a, b = acrl.acrl_matmul_fp8(*t, out_dtype=dtype), acrl.acrl_linear_fp8(*t, out_dtype=dtype)
        assert torch.equal(a, b)


@pytest.mark.parametrize("M,N", [(5, 100), (60, 515), (1500, 4100)])
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_in_place_and_beside(M, N, kind):
    # the residual is y itself; y and the residual are columns of one matrix, of every alignment of rows
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    dtype = torch.bfloat16 if kind == "bf16" else torch.float32
    K = 256
    host, t = _operands(torch, dev, M, N, K, 9)
    y, slack = product(*host)
    b, tb = _values(torch, dev, (N,), "f32", 5)
    r, tr = _values(torch, dev, (M, N), kind, 6, 3.0)
    want, tol = linear(y, slack, "none", b, r)
    own = tr.clone()
    got = acrl.acrl_linear_fp8(*t, bias=tb, residual=own, out=own)
    assert got is own
    _check(down(own.float()), want, tol, kind)
    ref = acrl.acrl_linear_fp8(*t, bias=tb, residual=tr, out_dtype=dtype)
    assert torch.equal(ref, own)
    first = (N + 7) // 8 * 8
    for extra in (0, 1, 2, 4, 8):
        wide = torch.full((M, first + N + extra), 7.0, dtype=dtype, device=dev)
        wide[:, first:first + N] = tr
        acrl.acrl_linear_fp8(*t, bias=tb, residual=wide[:, first:first + N], out=wide[:, :N])
        assert torch.equal(wide[:, :N], ref)
        assert torch.equal(wide[:, first:first + N], tr)
        rest = torch.cat([wide[:, N:first], wide[:, first + N:]], 1)
        assert bool((rest == 7.0).all())


def test_activations_over_their_range():
    # one row, K of one block, the operands 0: y = act(bias) alone, exact but for the activation's own error
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    r = np.random.default_rng(1)
    v = np.concatenate([np.linspace(-30, 30, 4001), r.normal(size=2000) * 1e-3, [0.0, -0.0, 1e-30, -1e-30, 1e30, -1e30, 88.0,
                        -88.0, -87.0, -13.0, -14.2, 3e38, -3e38]]).astype(np.float32)
    N = v.size
    z = lambda n: torch.zeros((n, 128), dtype=torch.uint8, device=dev)  # noqa: E731
    one = lambda n: torch.ones((n, 1), device=dev)  # noqa: E731
    for M in (1, 20):
        for name in ACTS:
            want = act(name, v)
            for kind, dtype in (("f32", torch.float32), ("bf16", torch.bfloat16)):
                got = down(acrl.acrl_linear_fp8(z(M), one(M), z(N), one((N + 127) // 128), bias=up(torch, dev, v),
                                                activation=ACTS[name], out_dtype=dtype).float())
                # (as documented, and half a step; bf16 overflows to infinity from 3.39e38 on)
                bound = (ACT_ERROR[kind] + HALF[kind]) * np.abs(want) + 1.3e-36
                assert (np.abs(got - want) <= bound).all(), (name, kind)
                assert (got == got[:1]).all()


def test_nan_and_infinities():
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    inf, nan = np.inf, np.nan
    v = np.array([inf, -inf, nan, 1.0] * 5, np.float32)
    z = torch.zeros((2, 32), dtype=torch.uint8, device=dev)
    w = torch.zeros((20, 32), dtype=torch.uint8, device=dev)
    one = torch.ones((2, 1), device=dev)
    for name in ACTS:
        got = down(acrl.acrl_linear_fp8(z, one, w, one[:1], bias=up(torch, dev, v), activation=ACTS[name],
                                        out_dtype=torch.float32))
        assert (got[:, 0] == inf).all() and np.isnan(got[:, 2]).all() and np.isfinite(got[:, 3]).all()
        if name in ("none", "relu"):
            assert (got[:, 1] == (0.0 if name == "relu" else -inf)).all()
    res = up(torch, dev, np.tile(v, (2, 1)))
    got = down(acrl.acrl_linear_fp8(z, one, w, one[:1], residual=res, out_dtype=torch.float32))
    assert np.array_equal(got, np.tile(v, (2, 1)), equal_nan=True)


def test_no_rows_and_other_streams():
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    _, t = _operands(torch, dev, 6, 64, 256, 4)
    empty = acrl.acrl_linear_fp8(t[0][:0], t[1][:0], *t[2:], residual=torch.zeros((0, 64), device=dev))
    assert empty.shape == (0, 64)
    res = torch.randn((6, 64), device=dev)
    want = acrl.acrl_linear_fp8(*t, residual=res, activation=acrl.ACT_SILU)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = acrl.acrl_linear_fp8(*t, residual=res, activation=acrl.ACT_SILU, stream=s)
    s.synchronize()
    assert torch.equal(got, want)


def test_graph_replays():
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    _, t = _operands(torch, dev, 9, 300, 512, 4)
    res = torch.randn((9, 300), device=dev)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y = acrl.acrl_linear_fp8(*t, residual=res, activation=acrl.ACT_GELU, out_dtype=torch.float32)
    for k in range(3):
        res.normal_()
        want = acrl.acrl_linear_fp8(*t, residual=res, activation=acrl.ACT_GELU, out_dtype=torch.float32)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)


def test_refusals():
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    _, t = _operands(torch, dev, 6, 64, 256, 4)
    z = lambda *shape, dtype=torch.float32: torch.zeros(shape, dtype=dtype, device=dev)  # noqa: E731
    for kw in (dict(bias=z(63)), dict(bias=z(64, dtype=torch.float16)), dict(residual=z(6, 65)), dict(residual=z(5, 64)),
               dict(residual=z(64, 6).t()), dict(residual=z(6, 64, dtype=torch.float64)), dict(bias=torch.zeros(64)),
               dict(out_dtype=torch.float16)):
        with pytest.raises(ValueError):
            acrl.acrl_linear_fp8(*t, **kw)
    wide = z(6, 200)
    for kw in (dict(activation=5), dict(activation=-1), dict(bias=z(65)[1:]), dict(residual=z(6, 65)[:, 1:]),
               dict(residual=wide[:, 32:96], out=wide[:, :64]), dict(residual=wide[:, :64], out=wide[:, 32:96]),
               dict(residual=wide.view(torch.bfloat16)[:, :64], out=wide[:, :64]),
               dict(residual=z(7, 64)[1:], out=None, activation=9)):
        with pytest.raises(acrl.AcrlError):
            acrl.acrl_linear_fp8(*t, **kw)
    big = z(7, 64)
    with pytest.raises(acrl.AcrlError, match="overlap"):
        acrl.acrl_linear_fp8(*t, residual=big[1:], out=big[:6])
