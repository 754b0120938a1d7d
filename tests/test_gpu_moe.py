"""acrl_moe_fp8 against its definition in 64 bits (tests/decode64.py, where the
tolerances are derived): the choices are equal, the weights are off by half a
step of fp32, y by what fp32 sums may lose and half a step of its type."""
import numpy as np
import pytest

from cases import random_bf16
from decode64 import HALF, experts, f64, routing, spread
from gpu_util import down, torch_dev, up, up_bf16
from operators64 import e4m3_values, quantize_blocks

pytestmark = pytest.mark.gpu

ACTS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3, "gelu_tanh": 4}


class Layer:
    """Weights of a layer on the host (values in 64 bits) and the device."""

    def __init__(self, torch, dev, d, E, F, seed):
        val = e4m3_values()

        def make(rows, cols, s):
            q = [quantize_blocks(random_bf16((rows, cols), s + 7 * e, std=1.5 / np.sqrt(cols)), 128) for e in range(E)]
            codes, scales = np.stack([a for a, _ in q]), np.stack([b for _, b in q])
            return codes, scales, np.stack([val[a] * spread(b, rows, cols) for a, b in q])

        self.cin, self.sin, self.win = make(2 * F, d, seed)
        self.cout, self.sout, self.wout = make(d, F, seed + 3)
        r = random_bf16((E, d), seed + 5, std=1.0 / np.sqrt(d)).reshape(E, d)
        self.router = f64(r)
        self.t = [up(torch, dev, a) for a in (self.cin, self.sin, self.cout, self.sout)]
        self.t_router = up_bf16(torch, dev, r)


def _check(got, want, tol, kind):
    got = got.astype(np.float64)
    bound = tol * 1.01 + HALF[kind] * (np.abs(want) + tol)
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:3], got[bad][:3], want[bad][:3], bound[bad][:3])


def _x(torch, dev, T, d, seed):
    b = random_bf16((T, d), seed).reshape(T, d)
    return f64(b), up_bf16(torch, dev, b)


# T, d, E, k, F: one token and one expert; odd widths; every expert of a token; more tokens of an expert than a block of
# columns has, than all its blocks have; the most of everything; one and two tokens among many experts, with long rows of
# Wout that waves share; as many pairs as the kernel for few takes, and one more
SIZES = [(1, 32, 1, 1, 32), (1, 256, 8, 2, 96), (3, 160, 5, 5, 64), (2, 416, 70, 6, 32), (16, 96, 4, 2, 160), (17, 288, 12, 3, 160),
         (33, 128, 2, 1, 416), (70, 512, 3, 2, 256), (128, 64, 1, 1, 96), (128, 32, 512, 16, 32), (5, 1312, 9, 4, 1184), (2, 96, 300, 3, 64), (1, 64, 129, 16, 160), (1, 96, 4, 2, 1184), (2, 1056, 40, 8, 32),
         (16, 64, 20, 1, 64), (17, 64, 20, 1, 64), (30, 2080, 2, 1, 544)]


@pytest.mark.parametrize("n,size", list(enumerate(SIZES)))
def test_sizes(n, size):
    T, d, E, k, F = size
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    layer = Layer(torch, dev, d, E, F, 11)
    x, tx = _x(torch, dev, T, d, 2)
    r = np.random.default_rng(n)
    for score, renorm, with_bias, masked, res, out, act in (("softmax", True, False, False, "", "f32", "silu"),
                                                           ("sigmoid", False, True, True, "bf16", "bf16", "gelu")):
        bias = (0.1 * r.normal(size=E)).astype(np.float32) if with_bias else None
        mask = (r.random(T) < 0.7).astype(np.uint8) if masked else None
        resid = random_bf16((T, d), 9, std=2.0).reshape(T, d) if res else None
        ids, w = routing(x, layer.router, k, score, bias, renorm, 1.5, mask)
        y, gi, gw = acrl.acrl_moe_fp8(
            tx, *layer.t, k, router=layer.t_router, score={"softmax": 0, "sigmoid": 1}[score], renormalize=renorm, scale=1.5,
            select_bias=None if bias is None else up(torch, dev, bias), mask=None if mask is None else up(torch, dev, mask),
            residual=None if resid is None else up_bf16(torch, dev, resid), activation=ACTS[act],
            out_dtype=torch.float32 if out == "f32" else torch.bfloat16)
        assert np.array_equal(down(gi), ids)
        assert (np.abs(down(gw) - w) <= (HALF["f32"] + 1e-12) * np.abs(w)).all()
        _check(down(y.float()), *experts(x, ids, w, layer.win, layer.wout, act, None if resid is None else f64(resid)), out)


# tokens that hardly share experts, a pair a workgroup: up to 128 experts and more, pairs for either second product, as many
# pairs as that takes and one expert too few for it
FEW = [(3, 96, 70, 2, 64), (8, 64, 64, 2, 96), (8, 64, 63, 2, 96), (8, 160, 300, 9, 64), (5, 288, 128, 6, 1184), (4, 1312, 512, 16, 32),
       (9, 64, 512, 2, 64)]


@pytest.mark.parametrize("n,size", list(enumerate(FEW)))
def test_few_tokens(n, size):
    test_sizes(n + 100, size)


# long rows of Wout and few of them: workgroups share a row, by expert and by pair, odd parts among them
LONG = [(8, 64, 2, 2, 4160), (3, 96, 5, 4, 4480), (2, 96, 8, 6, 4512), (40, 64, 2, 1, 4128), (1, 32, 3, 3, 5152), (17, 32, 20, 1, 8224),
        (70, 64, 2, 2, 6144)]


@pytest.mark.parametrize("n,size", list(enumerate(LONG)))
def test_long_rows(n, size):
    test_sizes(n + 200, size)


@pytest.mark.parametrize("act", list(ACTS))
def test_activations(act):
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    layer = Layer(torch, dev, 128, 4, 64, 5)
    x, tx = _x(torch, dev, 9, 128, 3)
    ids, w = routing(x, layer.router, 2)
    y, _, _ = acrl.acrl_moe_fp8(tx, *layer.t, 2, router=layer.t_router, activation=ACTS[act], out_dtype=torch.float32)
    _check(down(y), *experts(x, ids, w, layer.win, layer.wout, act), "f32")


def test_equal_scores_go_to_the_lower_index():
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    layer = Layer(torch, dev, 64, 70, 32, 5)
    _, tx = _x(torch, dev, 4, 64, 3)
    for router in (torch.zeros_like(layer.t_router), layer.t_router[:1].expand(70, 64).contiguous()):
        for score in (0, 1):
            _, ids, w = acrl.acrl_moe_fp8(tx, *layer.t, 6, router=router, score=score)
            assert ids.tolist() == [list(range(6))] * 4
            assert torch.equal(w, torch.full_like(w, np.float32(1 / 6)))
    bias = torch.zeros(70, device=dev)
    bias[[64, 3, 69]] = 1.0
    _, ids, _ = acrl.acrl_moe_fp8(tx, *layer.t, 5, router=torch.zeros_like(layer.t_router), select_bias=bias)
    assert ids.tolist() == [[3, 64, 69, 0, 1]] * 4


def test_what_is_not_chosen_has_no_influence():
    # NaN and infinities in experts that no token chose, in experts of other tokens, and in masked rows of x
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    T, d, E, k, F = 6, 160, 12, 2, 96
    layer = Layer(torch, dev, d, E, F, 21)
    x, tx = _x(torch, dev, T, d, 2)
    clean, ids, w = acrl.acrl_moe_fp8(tx, *layer.t, k, router=layer.t_router, out_dtype=torch.float32)
    chosen = set(ids.flatten().tolist())
    t = [a.clone() for a in layer.t]
    for e in set(range(E)) - chosen:
        t[0][e], t[2][e], t[1][e], t[3][e] = 0x7F, 0x7F, float("nan"), float("inf")
    y, _, _ = acrl.acrl_moe_fp8(tx, *t, k, router=layer.t_router, out_dtype=torch.float32)
    assert len(chosen) < E and torch.equal(y, clean)
    bad = int(ids[2, 0])
    t[0][bad] = 0x7F
    y, _, _ = acrl.acrl_moe_fp8(tx, *t, k, router=layer.t_router, out_dtype=torch.float32)
    hit = (ids == bad).any(1)
    assert bool(hit.any()) and bool(torch.isnan(y[hit]).all()) and torch.equal(y[~hit], clean[~hit])
    mask = torch.tensor([1, 0, 1, 1, 0, 1], dtype=torch.uint8, device=dev)
    tx2 = tx.clone()
    tx2[mask == 0] = float("nan")
    res = torch.randn((T, d), device=dev)
    want, _, _ = acrl.acrl_moe_fp8(tx, *layer.t, k, router=layer.t_router, residual=res, out_dtype=torch.float32)
    y, gi, gw = acrl.acrl_moe_fp8(tx2, *layer.t, k, router=layer.t_router, mask=mask, residual=res, out_dtype=torch.float32)
    dead = mask == 0
    assert torch.equal(y[~dead], want[~dead]) and torch.equal(y[dead], res[dead])
    assert bool((gi[dead] == -1).all()) and bool((gw[dead] == 0).all()) and torch.equal(gi[~dead], ids[~dead])
    y, gi, _ = acrl.acrl_moe_fp8(tx2, *layer.t, k, router=layer.t_router, mask=torch.zeros_like(mask), out_dtype=torch.float32)
    assert bool((y == 0).all()) and bool((gi == -1).all())
    # a NaN score is the lowest; a token whose scores are all NaN still has its own experts, and NaN
    rt = layer.t_router.clone()
    rt[ids[0, 0]] = float("nan")
    _, gi, gw = acrl.acrl_moe_fp8(tx, *layer.t, k, router=rt, score=1)
    assert int(ids[0, 0]) not in gi[0].tolist() and bool(torch.isfinite(gw).all())
    y, gi, gw = acrl.acrl_moe_fp8(torch.full_like(tx, float("nan")), *layer.t, k, router=layer.t_router)
    assert gi.tolist() == [[0, 1]] * T and bool(torch.isnan(y).all())


@pytest.mark.parametrize("T", [3, 5, 21, 60])
def test_given_routing(T):
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    d, E, k, F = 96, 7, 3, 64
    layer = Layer(torch, dev, d, E, F, 31)
    x, tx = _x(torch, dev, T, d, 2)
    y, ids, w = acrl.acrl_moe_fp8(tx, *layer.t, k, router=layer.t_router)
    again, i2, w2 = acrl.acrl_moe_fp8(tx, *layer.t, k, ids=ids, weights=w)
    assert torch.equal(again, y) and i2 is ids and w2 is w
    # the same expert twice, none, out of range, masked
    r = np.random.default_rng(3)
    gi = r.integers(-2, E + 2, (T, k)).astype(np.int32)
    gi[0], gi[1], gi[2] = 4, -1, (2 ** 31 - 1, -2 ** 31, 5)
    gw = r.normal(size=(T, k)).astype(np.float32)
    gw[1] = np.nan
    mask = (r.random(T) < 0.8).astype(np.uint8)
    mask[:3] = 1
    ti, tw = up(torch, dev, gi), up(torch, dev, gw)
    y, _, _ = acrl.acrl_moe_fp8(tx, *layer.t, k, ids=ti, weights=tw, mask=up(torch, dev, mask), out_dtype=torch.float32)
    assert np.array_equal(down(ti), gi) and np.array_equal(down(tw), gw, equal_nan=True)
    want, tol = experts(x, np.where(mask[:, None] != 0, gi, -1), np.nan_to_num(gw), layer.win, layer.wout)
    _check(down(y), want, tol, "f32")


def test_strides_and_in_place():
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    T, d, E, k, F = 10, 96, 6, 2, 64
    layer = Layer(torch, dev, d, E, F, 41)
    x, tx = _x(torch, dev, T, d, 2)
    want, _, _ = acrl.acrl_moe_fp8(tx, *layer.t, k, router=layer.t_router, residual=tx)
    wide = torch.full((T, d + 40), 3.0, dtype=torch.bfloat16, device=dev)
    wide[:, 8:8 + d] = tx
    out = torch.full((T, d + 7), 5.0, dtype=torch.bfloat16, device=dev)
    y, _, _ = acrl.acrl_moe_fp8(wide[:, 8:8 + d], *layer.t, k, router=layer.t_router, residual=wide[:, 8:8 + d], out=out[:, :d])
    assert torch.equal(y, want) and bool((out[:, d:] == 5.0).all())
    own = tx.clone()
    y, _, _ = acrl.acrl_moe_fp8(own, *layer.t, k, router=layer.t_router, residual=own, out=own)
    assert torch.equal(own, want)


def test_given_routing_of_one_token():
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    d, E, k, F = 160, 7, 4, 96
    layer = Layer(torch, dev, d, E, F, 33)
    x, tx = _x(torch, dev, 1, d, 2)
    y, ids, w = acrl.acrl_moe_fp8(tx, *layer.t, k, router=layer.t_router, out_dtype=torch.float32)
    assert torch.equal(acrl.acrl_moe_fp8(tx, *layer.t, k, ids=ids, weights=w, out_dtype=torch.float32)[0], y)
    for row in ([3, 3, -1, 9], [-5, 7, 8, 100], [6, 0, 6, 6]):
        gi, gw = np.array([row], np.int32), np.array([[0.5, -1.0, 2.0, 0.25]], np.float32)
        got = acrl.acrl_moe_fp8(tx, *layer.t, k, ids=up(torch, dev, gi), weights=up(torch, dev, gw), residual=tx,
                                out_dtype=torch.float32)[0]
        _check(down(got), *experts(x, gi, gw.astype(np.float64), layer.win, layer.wout, residual=x), "f32")


@pytest.mark.parametrize("T", [1, 2, 6, 20])
def test_streams_graphs_and_no_tokens(T):
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    d, E, k, F = 160, 9, 2, 96
    layer = Layer(torch, dev, d, E, F, 51)
    x, tx = _x(torch, dev, T, d, 2)
    call = lambda **kw: acrl.acrl_moe_fp8(tx, *layer.t, k, router=layer.t_router, out_dtype=torch.float32, **kw)  # noqa: E731
    y0, i0, w0 = acrl.acrl_moe_fp8(tx[:0], *layer.t, k, router=layer.t_router)
    assert y0.shape == (0, d) and i0.shape == w0.shape == (0, k)
    want = call()
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = call(stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graphs = []
    for _ in range(2):  # two graphs of the same call, replayed in turn: each has its own workspace
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            o = call()
        graphs.append((g, o))
    for n in range(4):
        tx.copy_(_x(torch, dev, T, d, 70 + n)[1])
        want = call()
        for g, o in graphs:
            g.replay()
        torch.cuda.synchronize()
        for g, o in graphs:
            assert all(torch.equal(a, b) for a, b in zip(o, want)), n


def test_alone_and_among_others():
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    T, d, E, k, F = 40, 256, 8, 2, 128
    layer = Layer(torch, dev, d, E, F, 61)
    x, tx = _x(torch, dev, T, d, 2)
    y, ids, w = acrl.acrl_moe_fp8(tx, *layer.t, k, router=layer.t_router, out_dtype=torch.float32)
    tol = experts(x, down(ids), down(w).astype(np.float64), layer.win, layer.wout)[1]
    for t in (0, 17, 39):
        one, i1, w1 = acrl.acrl_moe_fp8(tx[t:t + 1], *layer.t, k, router=layer.t_router, out_dtype=torch.float32)
        assert torch.equal(i1[0], ids[t]) and torch.equal(w1[0], w[t])
        assert (np.abs(down(one[0]) - down(y[t])) <= 2.02 * tol[t]).all()


def test_refusals():
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    d, E, F = 64, 4, 32
    layer = Layer(torch, dev, d, E, F, 5)
    _, tx = _x(torch, dev, 4, d, 3)
    z = lambda *shape, dtype=torch.float32: torch.zeros(shape, dtype=dtype, device=dev)  # noqa: E731
    rt = layer.t_router
    i2, w2 = z(4, 2, dtype=torch.int32), z(4, 2)
    for args, kw in (((tx.float(), *layer.t, 2), dict(router=rt)), ((tx[:, :32], *layer.t, 2), dict(router=rt)),
                     ((tx, *layer.t, 2), {}), ((tx, *layer.t, 2), dict(ids=i2)), ((tx, *layer.t, 2), dict(router=rt[:3])),
                     ((tx, *layer.t, 2), dict(router=rt.float())), ((tx, *layer.t, 2), dict(router=rt, mask=z(4))),
                     ((tx, *layer.t, 2), dict(router=rt, select_bias=z(5))), ((tx, *layer.t, 2), dict(router=rt, residual=z(4, 65))),
                     ((tx, *layer.t, 2), dict(router=rt, out=z(4, 64, dtype=torch.float16))),
                     ((tx, *layer.t, 2), dict(ids=i2.long(), weights=w2)), ((tx, *layer.t, 2), dict(ids=i2[:3], weights=w2)),
                     ((tx, layer.t[0], layer.t[1][:3], *layer.t[2:], 2), dict(router=rt)),
                     ((tx, layer.t[0].cpu(), *layer.t[1:], 2), dict(router=rt))):
        with pytest.raises(ValueError):
            acrl.acrl_moe_fp8(*args, **kw)
    wide = z(4, 200)
    for args, kw in (((tx, *layer.t, 5), {}), ((tx, *layer.t, 0), {}), ((tx, *layer.t, 2), dict(score=2)),
                     ((tx, *layer.t, 2), dict(activation=9)), ((tx, *layer.t, 2), dict(scale=float("nan"))),
                     ((z(129, 64, dtype=torch.bfloat16), *layer.t, 2), {}),
                     ((tx, *layer.t, 2), dict(residual=wide[:, 32:96], out=wide[:, :64]))):
        with pytest.raises(acrl.AcrlError):
            acrl.acrl_moe_fp8(*args, router=rt, **kw)
    odd = z(4, 70, dtype=torch.bfloat16)
    with pytest.raises(acrl.AcrlError, match="ldx"):
        acrl.acrl_moe_fp8(odd[:, :64], *layer.t, 2, router=rt)
