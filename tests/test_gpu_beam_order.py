"""The order of acrl_beam_step's candidates where scores do not tell them apart:
temperatures so high, or scores so large, that the tokens of a beam have the same c
in 64 bits.  Equal c go by beam, and a beam's tokens by logit, then token, over all
segments that a row is cut into and all lists that the choice walks.  The expected
choice is exact: the beam comes from scores that lie far apart or are equal, the
tokens from a stable sort of the logits themselves."""
import numpy as np
import pytest

from gpu_util import down, torch_dev, up

pytestmark = pytest.mark.gpu

LOWEST = float(np.finfo(np.float32).min)


def _by_logit(z, n):
    return np.argsort(-z.astype(np.float64) + 0.0, kind="stable")[:n]


def _step(torch, dev, z, s, n, kind, **kw):
    """(ids, parents, scores) and the logits as the type has them."""
    from paper_2607_24062_amd import acrl
    t = up(torch, dev, z)
    if kind == "bf16":
        t = t.to(torch.bfloat16)
    return [down(o) for o in acrl.acrl_beam_step(t, up(torch, dev, s), n, **kw)], down(t.float())


# rows of one segment and of many; more than one wave's lists (24 beams of 10 segments: a beam lies across two waves)
SHAPES = [(2, 1, 8192, 6), (1, 3, 8192, 6), (3, 5, 3001, 20), (1, 24, 151936, 4), (2, 2, 151936, 64), (1, 4, 60000, 24)]


@pytest.mark.parametrize("B,K,V,n", SHAPES)
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("inv_t", [1e-15, 1e-20, 2e-30])
def test_high_temperatures(B, K, V, n, kind, inv_t):
    torch, dev = torch_dev()
    r = np.random.default_rng(V + K)
    z = (3.0 * r.normal(size=(B * K, V))).astype(np.float32)
    s = np.stack([r.permutation(K) for _ in range(B)]).astype(np.float32) * -1.0 - 1.0
    (ids, parents, scores), z = _step(torch, dev, z, s, n, kind, inv_temperature=inv_t)
    for b in range(B):
        j = int(s[b].argmax())
        assert (parents[b] == j).all()
        assert np.array_equal(ids[b], _by_logit(z[b * K + j], n)), (b, j)
        assert (np.abs(scores[b] - (s[b, j] - np.log(V))) <= 2.0 ** -24 * 20 + 1e-11).all()


@pytest.mark.parametrize("B,K,V,n", SHAPES)
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_scores_that_leave_logits_no_bits(B, K, V, n, kind):
    # beams masked by the type's lowest value, scores of 1e18: score + lp is the score, for all tokens
    torch, dev = torch_dev()
    r = np.random.default_rng(V)
    z = r.normal(size=(B * K, V)).astype(np.float32)
    z[:, ::7] = r.integers(-1, 3, z[:, ::7].shape)  # (equal ones, zeros of both signs among them)
    z[:, 3::7] *= np.where(r.random(z[:, 3::7].shape) < 0.1, -0.0, 1.0)
    for size in (LOWEST, -1e18):
        s = np.full((B, K), size, np.float32)
        (ids, parents, scores), seen = _step(torch, dev, z, s, n, kind)
        assert not parents.any() and (scores == np.float32(size)).all()
        for b in range(B):
            assert np.array_equal(ids[b], _by_logit(seen[b * K], n))
        if K > 1:  # one beam less far down; and a finished one of the same score before the others
            s[:, K - 1] = np.float32(size * 0.5)
            (ids, parents, scores), seen = _step(torch, dev, z, s, n, kind)
            assert (parents == K - 1).all() and (scores == np.float32(size * 0.5)).all()
            for b in range(B):
                assert np.array_equal(ids[b], _by_logit(seen[b * K + K - 1], n))
            s[:] = size
            done = np.zeros((B, K), np.uint8)
            done[:, 0] = 1
            (ids, parents, scores), seen = _step(torch, dev, z, s, n, kind, finished=up(torch, dev, done), eos_id=11)
            assert (scores == np.float32(size)).all()
            for b in range(B):
                assert parents[b].tolist() == [0] + [1] * (n - 1)
                assert ids[b].tolist() == [11] + _by_logit(seen[b * K + 1], n - 1).tolist()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_small_vocabularies_go_on_with_the_next_beam(kind):
    # all candidates of a sequence are chosen, beams of equal scores among them
    torch, dev = torch_dev()
    z = np.array([[0.5, 2.0, -1.0], [3.0, 3.0, 4.0], [-2.0, -0.0, 0.0], [1.0, 0.5, 2.0]], np.float32)
    s = np.array([[-2.0, -1.0, -1.0, -2.0]], np.float32)
    (ids, parents, _), z = _step(torch, dev, z, s, 12, kind, inv_temperature=1e-20)
    assert parents[0].tolist() == [1] * 3 + [2] * 3 + [0] * 3 + [3] * 3
    assert ids[0].tolist() == [t for j in (1, 2, 0, 3) for t in _by_logit(z[j], 3)]


def test_differences_of_a_few_steps():
    # some tokens of a row have equal c and some do not: with logits of 1e-12 and less about one token in eight of those that
    # are chosen shares c with another (c lies at 12, whose step is 1.8e-15)
    torch, dev = torch_dev()
    V, n = 151936, 64
    r = np.random.default_rng(8)
    z = (1e-14 * r.normal(size=(2, V))).astype(np.float32)
    s = np.array([[-0.25], [-0.25]], np.float32)
    (ids, parents, scores), _ = _step(torch, dev, z, s, n, "f32")
    for b in range(2):
        assert np.array_equal(ids[b], _by_logit(z[b], n))
    assert (np.diff(scores) <= 0).all()


def test_states_whose_layers_sequences_and_beams_lie_in_any_order():
    # the strides that rows of dst may have: every order of the three, holes among them
    torch, dev = torch_dev()
    from itertools import permutations

    from paper_2607_24062_amd import acrl
    L, B, K, n = 2, 3, 4, 40
    state = torch.randn((L, B, K, n), device=dev)
    parents = torch.tensor([[3, 0, 0, 2], [1, 1, 2, 0], [0, 1, 2, 3]], dtype=torch.int32, device=dev)
    want = torch.stack([state[:, b, parents[b].long()] for b in range(B)], 1)
    for order in permutations(range(3)):
        shape = [(L, B, K)[i] for i in order]
        wide = torch.full((*shape[:2], shape[2] + 1, n + 4), 7.0, device=dev)
        out = wide[:, :, :shape[2], :n].permute(*(order.index(i) for i in range(3)), 3)
        assert out.shape == state.shape
        acrl.acrl_beam_reorder(state, parents, dim=1, out=out)
        assert torch.equal(out, want)
        assert bool((wide[..., n:] == 7.0).all()) and bool((wide[:, :, shape[2]:] == 7.0).all())
        own = out.clone(memory_format=torch.preserve_format)
        out.copy_(state)
        acrl.acrl_beam_reorder(out, parents, dim=1, out=out)
        assert torch.equal(out, want) and torch.equal(own, want)
    # rows of two sequences on each other: refused
    flat = torch.zeros(L * B * K * n, device=dev)
    both = flat.as_strided((1, 2, 3, n), (0, n, n, 1))
    with pytest.raises(acrl.AcrlError, match="overlap"):
        acrl.acrl_beam_reorder(state[:1, :2, :3].contiguous(), parents[:2, :3].contiguous(), dim=1, out=both)
