"""A decode step's operators over memory past 2^31 elements and 2^32 bytes: rows
far apart, states and weights of many GB."""
import numpy as np
import pytest

from cases import random_bf16
from decode64 import HALF, beam, experts, f64, linear, spread
from gpu_util import down, torch_dev, up, up_bf16
from operators64 import e4m3_values, product, quantize_blocks

pytestmark = pytest.mark.gpu

FAR = 1 << 30  # elements between rows


def test_rows_far_apart():
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    M, N, K = 5, 77, 160
    host = (*quantize_blocks(random_bf16((M, K), 1), 1), *quantize_blocks(random_bf16((N, K), 2, std=0.1), 128))
    t = [up(torch, dev, a) for a in host]
    wide = torch.empty((M, FAR), dtype=torch.bfloat16, device=dev)
    res = random_bf16((M, N), 3, std=3.0).reshape(M, N)
    wide[:, :N], wide[:, 96:96 + 8] = up_bf16(torch, dev, res), 7.0
    got = acrl.acrl_linear_fp8(*t, residual=wide[:, :N], out=wide[:, :N])
    want, tol = linear(*product(*host), "none", residual=f64(res).reshape(M, N))
    assert (np.abs(down(got.float()) - want) <= tol * 1.01 + HALF["bf16"] * (np.abs(want) + tol)).all()
    assert bool((wide[:, 96:104] == 7.0).all())

    V = 5001
    r = np.random.default_rng(4)
    z = torch.from_numpy((2.5 * r.normal(size=(M, V))).astype(np.float32)).to(dev).to(torch.bfloat16)
    wide[:, 8:8 + V] = z
    scores = (-4 * r.random((1, M))).astype(np.float32)
    ids, parents, best = acrl.acrl_beam_step(wide[:, 8:8 + V], up(torch, dev, scores), 7)
    want = beam(down(z.float())[None], scores, 7)
    assert np.array_equal(down(ids), want[0]) and np.array_equal(down(parents), want[1])
    assert (np.abs(down(best) - want[2]) <= HALF["f32"] * np.abs(want[2]) + 1e-11).all()

    back = up(torch, dev, np.array([[4, 0, 4, 3, 1]], np.int32))
    state = wide[None, :, 8:8 + V]
    assert torch.equal(acrl.acrl_beam_reorder(state, back), z[back[0].long()][None])
    acrl.acrl_beam_reorder(state, back, out=state)
    assert torch.equal(state[0], z[back[0].long()])


def test_long_rows_of_states():
    # 2 x 2 beams of 1.5 GB each, read and written past 2^32 bytes
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    n = 1500 * (1 << 20) // 2
    state = torch.empty((2, 2, n), dtype=torch.bfloat16, device=dev)
    for b in range(2):
        for k in range(2):
            state[b, k] = float(2 * b + k + 1)
            state[b, k, -5:] = torch.arange(5, device=dev) + 10.0 * (2 * b + k)
    parents = torch.tensor([[1, 1], [1, 0]], dtype=torch.int32, device=dev)
    for out in (acrl.acrl_beam_reorder(state, parents), acrl.acrl_beam_reorder(state, parents, out=state)):
        for b, row in enumerate([[1, 1], [1, 0]]):
            for k, p in enumerate(row):
                i = 2 * b + p
                assert bool((out[b, k, :-5] == i + 1).all())
                assert out[b, k, -5:].tolist() == [10.0 * i + j for j in range(5)]


def test_many_experts():
    # 5.4 GB of weights, the last experts chosen; the others hold NaN
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    T, d, E, k, F = 3, 4096, 400, 2, 1088
    val = e4m3_values()
    w_in = torch.full((E, 2 * F, d), 0x7F, dtype=torch.uint8, device=dev)
    w_out = torch.full((E, d, F), 0x7F, dtype=torch.uint8, device=dev)
    s_in = torch.full((E, 17, 32), float("nan"), device=dev)
    s_out = torch.full((E, 32, 9), float("nan"), device=dev)
    used, values = (398, 399), {}
    for e in used:
        (q, s), (qo, so) = (quantize_blocks(random_bf16(shape, e + n, std=1.5 / np.sqrt(shape[1])), 128)
                            for n, shape in ((0, (2 * F, d)), (5, (d, F))))
        w_in[e], s_in[e], w_out[e], s_out[e] = (up(torch, dev, a) for a in (q, s, qo, so))
        values[e] = val[q] * spread(s, 2 * F, d), val[qo] * spread(so, d, F)
    b = random_bf16((T, d), 3).reshape(T, d)
    ids = np.array([[398, 399], [399, -1], [399, 398]], np.int32)
    w = np.array([[0.25, 0.75], [1.0, 0.0], [0.5, 0.5]], np.float32)
    y, _, _ = acrl.acrl_moe_fp8(up_bf16(torch, dev, b), w_in, s_in, w_out, s_out, k, ids=up(torch, dev, ids),
                                weights=up(torch, dev, w), out_dtype=torch.float32)
    small = np.where(ids >= 0, ids - 398, -1)
    want, tol = experts(f64(b), small, w.astype(np.float64), np.stack([values[e][0] for e in used]),
                        np.stack([values[e][1] for e in used]))
    assert (np.abs(down(y) - want) <= tol * 1.01 + HALF["f32"] * (np.abs(want) + tol)).all()
