"""The normaliser of acrl_beam_step where nothing hides its error: scores of 0 and
logits that leave one token all or nearly all of the weight, so that the exact
result is 0 or far below 1, and ties with a finished beam.

Tolerance: 2^f is within 1.07e-12 of its value and exact at f = 0.  A term of the
sum has that error once and passes up to three factors of the same kind (a lane's
sum to its wave's, that to the workgroup's, that to the row's), so the logarithm of
the sum is within 4.3e-12; exponents of up to 60 and sums of up to 2^12 terms a
lane, rounded to 53 bits, add less than (2 * 60 + 2^12) 2^-53 = 5e-13."""
import numpy as np
import pytest

from decode64 import HALF, beam
from gpu_util import down, torch_dev, up

pytestmark = pytest.mark.gpu

SLACK = 5e-12


def _step(torch, dev, z, s, n, kind, **kw):
    from paper_2607_24062_amd import acrl
    t = up(torch, dev, z)
    if kind == "bf16":
        t = t.to(torch.bfloat16)
    return [down(o) for o in acrl.acrl_beam_step(t, up(torch, dev, s), n, **kw)]


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 300, 4097, 40000, 151936])
@pytest.mark.parametrize("inv_t", [1.0, 1 / 0.7])
def test_the_only_token_costs_nothing(V, inv_t, kind):
    # every place of the token among lanes, waves and segments; the others -infinity or far below
    torch, dev = torch_dev()
    at = sorted({0, V // 3, V // 2, V - 1})
    for rest in (-np.inf, -3000.0):
        z = np.full((len(at), V), rest, np.float32)
        for j, v in enumerate(at):
            z[j, v] = (7.25, -3.5, 0.0, 40.0)[j]
        for score in (0.0, -3.0):
            s = np.full((len(at), 1), score, np.float32)
            ids, parents, scores = _step(torch, dev, z, s, 1, kind, inv_temperature=inv_t)
            assert ids[:, 0].tolist() == at and not parents.any()
            assert (scores == score).all(), scores


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 700, 20000])
def test_ties_of_finished_and_forced_beams(V, kind):
    # a finished beam and one that has a single token left, of equal scores: the first beam is the better one
    torch, dev = torch_dev()
    z = np.full((6, V), -np.inf, np.float32)
    z[:, V // 2] = 3.0
    for score in (0.0, -1.5, -40.0):
        s = np.full((2, 3), score, np.float32)
        done = np.array([[1, 0, 0], [0, 1, 0]], np.uint8)
        for n in (1, 3):
            ids, parents, scores = _step(torch, dev, z, s, n, kind, finished=up(torch, dev, done), eos_id=0)
            assert parents.tolist() == [list(range(n))] * 2
            assert ids.tolist() == [[0, V // 2, V // 2][:n], [V // 2, 0, V // 2][:n]]
            assert (scores == score).all()


@pytest.mark.parametrize("V", [2, 777, 30000, 151936])
def test_scores_near_zero(V):
    # one token holds all but 1e-3 .. 1e-9 of the weight: its score is as far below 0
    torch, dev = torch_dev()
    r = np.random.default_rng(V)
    for ahead in (8.0, 13.0, 21.0):
        z = r.normal(size=(4, V)).astype(np.float32)
        z[np.arange(4), r.integers(0, V, 4)] = ahead + np.log(V)
        s = np.zeros((1, 4), np.float32)
        want = beam(z[None], s, 4)
        ids, parents, scores = _step(torch, dev, z, s, 4, "f32")
        # (The best of each beam, by beam: where they hold all but 1e-9, and V values average out to 3e-3 of that, beams lie
        # 3e-12 apart and less, and two normalisers that are each off by SLACK may order them either way.)
        assert sorted(parents[0]) == sorted(want[1][0]) == [0, 1, 2, 3]
        mine, other = np.argsort(parents[0]), np.argsort(want[1][0])
        assert np.array_equal(ids[0][mine], want[0][0][other])
        got, exact = scores[0][mine], want[2][0][other]
        assert (np.abs(exact) < 2e-2).all()
        assert (np.abs(got - exact) <= HALF["f32"] * np.abs(exact) + SLACK).all()
        assert (np.diff(scores[0]) <= 0).all()
