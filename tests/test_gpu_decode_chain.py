"""A decode step of the rollout policy with its operators one after another, as a
program runs it: a layer's product with bias and activation, the next one's with
the residual stream in place, a mixture of experts, the head's logits, beam
search's choice and the states of the chosen beams -- eagerly and as a replayed
graph.  Every operator is compared with its definition in 64 bits on the inputs
that it was given (tolerances in tests/decode64.py and tests/operators64.py)."""
import numpy as np
import pytest

from cases import random_bf16
from decode64 import HALF, beam, experts, f64, linear, routing, spread
from gpu_util import bf16_bits, down, torch_dev, up, up_bf16
from operators64 import e4m3_values, product, quantize_blocks

pytestmark = pytest.mark.gpu

B, K, D, WIDE, E, TOP, F, V = 2, 4, 160, 352, 9, 3, 96, 3001


def _close(got, want, tol, kind):
    got = down(got.float()).astype(np.float64)
    assert (np.abs(got - want) <= tol * 1.01 + HALF[kind] * (np.abs(want) + tol)).all()


class Model:
    def __init__(self, torch, dev):
        val = e4m3_values()

        def weights(rows, cols, seed):
            q, s = quantize_blocks(random_bf16((rows, cols), seed, std=1.5 / np.sqrt(cols)), 128)
            return (q, s), (up(torch, dev, q), up(torch, dev, s)), val[q] * spread(s, rows, cols)

        self.up, self.down, self.head = weights(WIDE, D, 1), weights(D, WIDE, 2), weights(V, D, 3)
        win, wout = [weights(2 * F, D, 10 + e) for e in range(E)], [weights(D, F, 40 + e) for e in range(E)]
        self.experts = [torch.stack([m[1][i] for m in ms]) for ms in (win, wout) for i in (0, 1)]
        self.win, self.wout = np.stack([m[2] for m in win]), np.stack([m[2] for m in wout])
        r = random_bf16((E, D), 70, std=1.0 / np.sqrt(D)).reshape(E, D)
        self.router, self.t_router = f64(r), up_bf16(torch, dev, r)
        self.bias = (0.1 * np.random.default_rng(5).normal(size=WIDE)).astype(np.float32)
        self.t_bias = up(torch, dev, self.bias)


def _step(acrl, m, h, scores, done, state):
    """One step; every intermediate by name.  h is updated in place."""
    r = {}
    r["x"] = acrl.acrl_quantize_fp8(h, acrl.SCALE_ROW128)
    r["wide"] = acrl.acrl_linear_fp8(*r["x"], *m.up[1], bias=m.t_bias, activation=acrl.ACT_SILU)
    r["wq"] = acrl.acrl_quantize_fp8(r["wide"], acrl.SCALE_ROW128)
    r["before"] = h.clone()
    acrl.acrl_linear_fp8(*r["wq"], *m.down[1], residual=h, out=h)
    r["h"] = h.clone()
    r["y"], r["ids"], r["weights"] = acrl.acrl_moe_fp8(h, *m.experts, TOP, router=m.t_router, residual=h)
    r["yq"] = acrl.acrl_quantize_fp8(r["y"], acrl.SCALE_ROW128)
    r["logits"] = acrl.acrl_matmul_fp8(*r["yq"], *m.head[1])
    r["tokens"], r["parents"], r["scores"] = acrl.acrl_beam_step(r["logits"], scores, K, finished=done, eos_id=2)
    r["state"] = acrl.acrl_beam_reorder(state, r["parents"], dim=1)
    return r


def test_decode_step():
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    m = Model(torch, dev)
    h = up_bf16(torch, dev, random_bf16((B * K, D), 7).reshape(B * K, D))
    scores = -5.0 * torch.rand((B, K), device=dev, generator=torch.Generator(device=dev).manual_seed(2))
    done = torch.tensor([[0, 1, 0, 0], [0, 0, 0, 0]], dtype=torch.uint8, device=dev)
    state = torch.randn((3, B, K, 5, 24), device=dev).to(torch.bfloat16)
    first = h.clone()
    r = _step(acrl, m, h, scores, done, state)

    codes = lambda q: (down(q[0]), down(q[1]))  # noqa: E731
    want, slack = product(*codes(r["x"]), *m.up[0])
    _close(r["wide"], *linear(want, slack, "silu", m.bias.astype(np.float64)[None]), "bf16")
    want, slack = product(*codes(r["wq"]), *m.down[0])
    _close(r["h"], *linear(want, slack, "none", residual=f64(bf16_bits(r["before"]))), "bf16")
    x = f64(bf16_bits(r["h"]))
    ids, w = routing(x, m.router, TOP)
    assert np.array_equal(down(r["ids"]), ids)
    _close(r["y"], *experts(x, ids, w, m.win, m.wout, residual=x), "bf16")
    z = f64(bf16_bits(r["logits"])).reshape(B, K, V)
    tokens, parents, best = beam(z, down(scores), K, 1.0, down(done), 2)
    assert np.array_equal(down(r["tokens"]), tokens) and np.array_equal(down(r["parents"]), parents)
    assert (np.abs(down(r["scores"]) - best) <= HALF["f32"] * np.abs(best) + 1e-11).all()
    assert torch.equal(r["state"], torch.stack([state[:, b, r["parents"][b].long()] for b in range(B)], 1))

    # the same step as a graph, replayed with eager steps between
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c = _step(acrl, m, h, scores, done, state)
    for k in range(3):
        h.copy_(first * (1.0 + 0.25 * k))
        state.normal_()
        own = h.clone()
        want = _step(acrl, m, own, scores, done, state)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(h, own)
        for n in ("wide", "h", "y", "ids", "weights", "logits", "tokens", "parents", "scores", "state"):
            assert torch.equal(c[n], want[n]), (k, n)


def test_two_calls_at_once():
    # on two streams: nothing is shared between calls
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    m = Model(torch, dev)
    hs = [up_bf16(torch, dev, random_bf16((B * K, D), s).reshape(B * K, D)) for s in (7, 8)]
    scores = -torch.rand((B, K), device=dev)
    call = lambda h, s=None: (*acrl.acrl_moe_fp8(h, *m.experts, TOP, router=m.t_router, residual=h, stream=s),  # noqa: E731
                              *acrl.acrl_beam_step(h, scores, K, stream=s))
    want = [call(h) for h in hs]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        got = [call(h, s) for h, s in zip(hs, streams)]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_stream_of_another_device_and_ownership():
    import types
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    m = Model(torch, dev)
    h = torch.zeros((B * K, D), dtype=torch.bfloat16, device=dev)
    x = acrl.acrl_quantize_fp8(h, acrl.SCALE_ROW128)
    scores, parents = torch.zeros((B, K), device=dev), torch.zeros((B, K), dtype=torch.int32, device=dev)
    calls = dict(linear=lambda s: [acrl.acrl_linear_fp8(*x, *m.up[1], stream=s)],
                 moe=lambda s: acrl.acrl_moe_fp8(h, *m.experts, TOP, router=m.t_router, stream=s),
                 beam=lambda s: acrl.acrl_beam_step(h, scores, K, stream=s),
                 reorder=lambda s: [acrl.acrl_beam_reorder(h.view(B, K, D), parents, stream=s)])
    other = types.SimpleNamespace(device_index=torch.cuda.current_device() + 1, cuda_stream=0)  # (refused before its use)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    for name, call in calls.items():
        with pytest.raises(ValueError, match="stream"):
            call(other)
        out = call(s)
        held = [(t.data_ptr(), t.shape, t.dtype) for t in out]
        del out
        fresh = [torch.empty(shape, dtype=dtype, device=dev) for _, shape, dtype in held for _ in range(3)]
        assert not {a for a, _, _ in held} & {t.data_ptr() for t in fresh}, name
    torch.cuda.synchronize()
