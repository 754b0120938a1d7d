"""acrl_moe_fp8 where one property alone decides the result: what lies between the
products (one-hot weights hand it through to y) and which pairs of a given routing
count (tokens that are masked out, among few pairs)."""
import numpy as np
import pytest

from cases import random_bf16
from decode64 import HALF, experts, f64
from gpu_util import down, torch_dev, up, up_bf16
from test_gpu_moe import Layer, _check, _x

pytestmark = pytest.mark.gpu

ONE = 0x38  # the E4M3 code of 1


# T, d, E, k: the second product of few pairs; tiles of two and four rows, one block of columns, two and four; a pair a
# workgroup, few of them and more
SHAPES = [(1, 64, 1, 1), (16, 96, 1, 1), (9, 64, 3, 1), (17, 64, 3, 1), (17, 96, 3, 1), (36, 64, 1, 1), (36, 96, 1, 1), (100, 64, 1, 1),
          (128, 96, 2, 1), (5, 64, 200, 2), (20, 96, 200, 2)]


@pytest.mark.parametrize("T,d,E,k", SHAPES)
@pytest.mark.parametrize("routed", [False, True])
def test_fp32_results_keep_what_lies_between_the_products(T, d, E, k, routed):
    # gate f is s x[f], up f is s x[32 + f] and y[r] = h[r % 32] times a weight that is a power of two: y is a product of
    # three fp32 roundings, within 3 half steps and their products (two bf16 parts would leave 2^-17 and more)
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    F, s = 32, np.float32(0.7182818)
    w_in = torch.zeros((E, 2 * F, d), dtype=torch.uint8, device=dev)
    w_out = torch.zeros((E, d, F), dtype=torch.uint8, device=dev)
    w_in[:, torch.arange(2 * F), torch.arange(2 * F)] = ONE
    w_out[:, torch.arange(d), torch.arange(d) % F] = ONE
    scale = lambda v: torch.full((E, 1, 1), float(v), device=dev)  # noqa: E731
    x, tx = _x(torch, dev, T, d, 5)
    if routed:  # (all scores equal: weights of 1 / k)
        kw = dict(router=torch.zeros((E, d), dtype=torch.bfloat16, device=dev))
    else:
        r = np.random.default_rng(3)
        ids = np.stack([r.permutation(E)[:k] for _ in range(T)]).astype(np.int32)
        kw = dict(ids=up(torch, dev, ids), weights=torch.full((T, k), 1.0 / k, device=dev))
    y = down(acrl.acrl_moe_fp8(tx, w_in, scale(s), w_out, scale(1), k, activation=acrl.ACT_NONE, out_dtype=torch.float32, **kw)[0])
    want = x[:, np.arange(d) % F] * x[:, F + np.arange(d) % F] * float(s) ** 2
    assert (np.abs(y - want) <= 3.01 * HALF["f32"] * np.abs(want)).all()


# T k < E with at most 16 pairs and with more
@pytest.mark.parametrize("T,k,E,d,F", [(4, 3, 40, 96, 64), (7, 2, 17, 160, 96), (8, 3, 40, 96, 64), (12, 4, 60, 64, 160),
                                       (30, 2, 64, 96, 64)])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_given_routing_of_few_pairs_with_a_mask(T, k, E, d, F, out):
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    layer = Layer(torch, dev, d, E, F, 17)
    x, tx = _x(torch, dev, T, d, 4)
    res = random_bf16((T, d), 6, std=2.0).reshape(T, d)
    r = np.random.default_rng(T)
    dtype = torch.float32 if out == "f32" else torch.bfloat16
    for n in range(4):
        # the tokens share three experts, the first of a call belongs to a token that is masked out
        ids = r.choice([1, E - 1, E // 2], (T, k)).astype(np.int32)
        if n == 1:
            ids[:, 0] = E - 1  # one for all
        if n == 2:
            ids[r.random((T, k)) < 0.4] = -1
            ids[1] = (E, -7, 2 ** 31 - 1, 3)[:k]
        mask = (r.random(T) < 0.5).astype(np.uint8)
        mask[0], mask[T - 1] = 0, 1
        if n == 3:
            mask[:] = 0
            mask[T - 1] = 1
        w = r.normal(size=(T, k)).astype(np.float32)
        t2, w2 = tx.clone(), w.copy()
        t2[up(torch, dev, mask) == 0] = float("nan")
        w2[mask == 0] = np.nan
        ti, tw = up(torch, dev, ids), up(torch, dev, w2)
        y = acrl.acrl_moe_fp8(t2, *layer.t, k, ids=ti, weights=tw, mask=up(torch, dev, mask), residual=up_bf16(torch, dev, res),
                              out_dtype=dtype)[0]
        counted = np.where(mask[:, None] != 0, ids, -1)
        _check(down(y.float()), *experts(x, counted, w, layer.win, layer.wout, residual=f64(res)), out)
        assert np.array_equal(down(y.float())[mask == 0], f64(res)[mask == 0])
        assert np.array_equal(down(ti), ids) and np.array_equal(down(tw), w2, equal_nan=True)
        # the same call without the masked tokens: each token alone is what it was among them
        live = np.flatnonzero(mask)
        pick = lambda a: up(torch, dev, np.ascontiguousarray(a[live]))  # noqa: E731
        alone = acrl.acrl_moe_fp8(tx[up(torch, dev, live)], *layer.t, k, ids=pick(ids), weights=pick(w), out_dtype=torch.float32)[0]
        _check(down(alone), *experts(x[live], ids[live], w[live], layer.win, layer.wout), "f32")
