"""acrl_beam_step against a stable sort of all candidates in 64 bits: the choices
are equal, the scores off by half a step of fp32 (and 1e-11: fp64 sums, terms
within 1.1e-12); acrl_beam_reorder against an indexed copy, bit for bit."""
import numpy as np
import pytest

from cases import random_bf16
from decode64 import HALF, beam, f64
from gpu_util import down, torch_dev, up, up_bf16

pytestmark = pytest.mark.gpu


def _same(got, want):
    ids, parents, scores = (down(t) for t in got)
    assert np.array_equal(parents, want[1]) and np.array_equal(ids, want[0])
    with np.errstate(invalid="ignore"):
        off = np.where(np.isneginf(want[2]), np.where(np.isneginf(scores), 0.0, np.inf), np.abs(scores - want[2]))
    assert (off <= HALF["f32"] * np.abs(np.where(np.isneginf(want[2]), 0.0, want[2])) + 1e-11).all()


def _inputs(torch, dev, B, K, V, kind, seed, std=2.5):
    r = np.random.default_rng(seed)
    scores = (-5.0 * r.random((B, K)) - 2.0).astype(np.float32)
    if kind == "bf16":
        bits = random_bf16((B * K, V), seed, std=std).reshape(B * K, V)
        return f64(bits).reshape(B, K, V), up_bf16(torch, dev, bits), scores, up(torch, dev, scores)
    z = (r.normal(size=(B * K, V)) * std).astype(np.float32)
    return z.reshape(B, K, V), up(torch, dev, z), scores, up(torch, dev, scores)


# a single candidate; all candidates of a sequence; odd rows; more rows than workgroups; many beams; more lists than a wave's
SIZES = [(1, 1, 1, 1), (1, 3, 5, 15), (2, 5, 2049, 10), (3, 2, 1000, 1), (1, 64, 300, 64), (2, 1, 40000, 64), (1, 2, 151936, 8),
         (600, 1, 130, 3), (1, 16, 70001, 32), (5, 4, 17, 8), (2, 8, 8193, 16)]


@pytest.mark.parametrize("B,K,V,N", SIZES)
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_sizes(B, K, V, N, kind):
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    z, tz, s, ts = _inputs(torch, dev, B, K, V, kind, B + V)
    r = np.random.default_rng(5)
    _same(acrl.acrl_beam_step(tz, ts, N), beam(z, s, N))
    done = (r.random((B, K)) < 0.4).astype(np.uint8)
    s[r.random((B, K)) < 0.3] = -np.inf
    _same(acrl.acrl_beam_step(tz, up(torch, dev, s), N, inv_temperature=1 / 0.7, finished=up(torch, dev, done), eos_id=V // 2),
          beam(z, s, N, 1 / 0.7, done, V // 2))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_ties_and_orders(kind):
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    V, N = 5003, 24
    r = np.random.default_rng(2)
    rows = [np.zeros(V), np.arange(V) * 0.01, -np.arange(V) * 0.01, r.integers(-2, 3, V), -0.0 * np.ones(V),
            np.where(np.arange(V) % 700 == 3, 1.0, -1.0)]
    for n, z in enumerate(rows):
        z = np.stack([z, z, z]).astype(np.float32)
        t = up(torch, dev, z)
        if kind == "bf16":
            t = t.to(torch.bfloat16)
            z = down(t.float())
        for s in ([-1.0, -1.0, -1.0], [-2.0, -1.0, -1.5]):
            s = np.array([s], np.float32)
            _same(acrl.acrl_beam_step(t, up(torch, dev, s), N), beam(z[None], s, N))


def test_logits_of_any_size():
    # far below and above the first ones a lane meets: its reference moves; what is far below adds nothing
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    V, N = 30000, 9
    r = np.random.default_rng(4)
    rows = [np.linspace(-4000, 4000, V), np.linspace(4000, -4000, V), r.normal(size=V) * 1e4, r.normal(size=V) * 1e30,
            np.where(np.arange(V) == 29999, 3000.0, -3000.0), -1e38 * r.random(V)]
    for z in rows:
        z = np.stack([z, z[::-1]]).astype(np.float32)
        s = np.array([[-1.0, -1.0]], np.float32)
        ids, parents, scores = beam(z[None], s, N)
        got = acrl.acrl_beam_step(up(torch, dev, z), up(torch, dev, s), N)
        assert np.array_equal(down(got[0]), ids) and np.array_equal(down(got[1]), parents)
        # the score is a difference of numbers as large as the logits, in 64 bits
        tol = HALF["f32"] * np.abs(scores) + 2.0 ** -50 * np.abs(z).max() + 1e-11
        assert (np.abs(down(got[2]) - scores) <= tol).all()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_ties_over_many_tiles(kind):
    # a workgroup meets the same values again and again: the first tokens are the ones to keep
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    V, N = 151936, 40
    r = np.random.default_rng(12)
    rows = [np.zeros(V), r.integers(-2, 3, V), np.arange(V) // 20000, -(np.arange(V) // 20000), np.where(np.arange(V) > 9000, -0.0, 0.0)]
    for z in rows:
        z = np.stack([z, z]).astype(np.float32)
        t = up(torch, dev, z)
        t = t.to(torch.bfloat16) if kind == "bf16" else t
        s = np.array([[-1.0, -1.5]], np.float32)
        _same(acrl.acrl_beam_step(t, up(torch, dev, s), N), beam(z[None], s, N))


@pytest.mark.parametrize("size", [1e10, 1e20, 1e30])
def test_scores_of_large_logits(size):
    # differences are of the logits themselves: those of the same size keep theirs, and the largest has all the weight
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    V, N = 40000, 5
    r = np.random.default_rng(13)
    z = (r.normal(size=(6, V)) * size).astype(np.float32)
    s = np.array([[-1.0, -2.0, -3.0], [-2.5, -0.5, -1.5]], np.float32)
    ids, parents, scores = beam(z.reshape(2, 3, V), s, N)
    got = acrl.acrl_beam_step(up(torch, dev, z), up(torch, dev, s), N)
    assert np.array_equal(down(got[0]), ids) and np.array_equal(down(got[1]), parents)
    # fp64 roundings of z, of the normaliser (1e-10) and of two sums, and the one to fp32
    assert (np.abs(down(got[2]) - scores) <= (HALF["f32"] + 4 * 2.0 ** -53) * np.abs(scores) + 1e-9).all()


@pytest.mark.parametrize("inv_t", [1e-3, 50.0, 1e20])
def test_temperatures(inv_t):
    # from nearly even weights to all of it on the largest logit
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    V, N = 30000, 6
    r = np.random.default_rng(15)
    z = (r.normal(size=(6, V)) * 3).astype(np.float32)
    s = np.array([[-1.0, -1.001, -1.002], [-2.5, -0.5, -1.5]], np.float32)
    ids, parents, scores = beam(z.reshape(2, 3, V), s, N, inv_t)
    got = acrl.acrl_beam_step(up(torch, dev, z), up(torch, dev, s), N, inv_temperature=inv_t)
    assert np.array_equal(down(got[0]), ids) and np.array_equal(down(got[1]), parents)
    assert (np.abs(down(got[2]) - scores) <= (HALF["f32"] + 4 * 2.0 ** -53) * np.abs(scores) + 1e-9).all()


def test_masked_logits_and_lost_rows():
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    inf, nan = np.inf, np.nan
    K, V, N = 4, 3001, 20
    z, _, s, ts = _inputs(torch, dev, 1, K, V, "f32", 3)
    for change in range(8):
        a, sc = z[0].copy(), s.copy()
        if change == 0:
            a[:, 7:] = -inf           # 28 candidates for 20
        elif change == 1:
            a[:, 3:2999] = -inf
            a[:, :3] = -inf           # 8 candidates: the others by beam and token
        elif change == 2:
            a[:] = -inf               # none
        elif change == 3:
            a[1, 5], a[2, 2999] = nan, inf
            a[0, 9] = -inf
        elif change == 4:
            a[:] = nan
        elif change == 5:
            sc[0] = (-inf, nan, inf, -3.0)
        elif change == 6:
            sc[0] = -inf
        else:
            a[1:] = -inf
            a[0, 1:] = -inf           # one
        ref = a.copy()
        _same(acrl.acrl_beam_step(up(torch, dev, a), up(torch, dev, sc), N), beam(ref[None], sc, N))
    # vocabularies smaller than what is chosen, their beams half lost
    a = np.full((4, 3), -inf, np.float32)
    a[2, 1] = 0.5
    _same(acrl.acrl_beam_step(up(torch, dev, a), ts, 12), beam(a[None], s, 12))
    # what a row that is not read holds has no influence
    done = np.array([[0, 1, 0, 1]], np.uint8)
    want = beam(z, s, N, 1.0, done, 11)
    z[0, 1], z[0, 3] = nan, inf
    _same(acrl.acrl_beam_step(up(torch, dev, z[0]), ts, N, finished=up(torch, dev, done), eos_id=11), want)


def test_rows_apart_streams_and_graphs():
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    B, K, V, N = 3, 3, 4001, 6
    for kind, dtype in (("f32", torch.float32), ("bf16", torch.bfloat16)):
        z, tz, s, ts = _inputs(torch, dev, B, K, V, kind, 8)
        want = acrl.acrl_beam_step(tz, ts, N)
        for extra, first in ((1, 0), (3, 1), (64, 7)):
            wide = torch.full((B * K, V + extra + first), 99.0, dtype=dtype, device=dev)
            wide[:, first:first + V] = tz
            got = acrl.acrl_beam_step(wide[:, first:first + V], ts, N)
            assert all(torch.equal(a, b) for a, b in zip(got, want))
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = acrl.acrl_beam_step(tz, ts, N, stream=st)
    st.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    state = torch.randn((2, B, K, 33), device=dev)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            o = acrl.acrl_beam_step(tz, ts, K)
            moved = acrl.acrl_beam_reorder(state, o[1], dim=1)
        graphs.append((g, o, moved))
    for n in range(3):
        tz.normal_()
        state.normal_()
        want = acrl.acrl_beam_step(tz, ts, K)
        for g, _, _ in graphs:
            g.replay()
        torch.cuda.synchronize()
        for _, o, moved in graphs:
            assert all(torch.equal(a, b) for a, b in zip(o, want))
            assert torch.equal(moved, torch.stack([state[:, b, want[1][b].long()] for b in range(B)], 1))
    none = acrl.acrl_beam_step(tz[:0], ts[:0], 2)
    assert [tuple(t.shape) for t in none] == [(0, 2)] * 3


@pytest.mark.parametrize("K,V,N", [(4, 3000, 4), (64, 20000, 64), (8, 5, 8)])
def test_scores_in_place(K, V, N):
    # a step's scores take the place of the last one's
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    _, tz, _, ts = _inputs(torch, dev, 5, K, V, "f32", 14)
    want = acrl.acrl_beam_step(tz, ts, N)
    got = acrl.acrl_beam_step(tz, ts, N, out_scores=ts)
    assert got[2] is ts and all(torch.equal(a, b) for a, b in zip(got, want))


# ------------------------------------------------------------------ states
def _gather(state, parents, dim):
    torch = __import__("torch")
    rows = [state.select(dim, b).index_select(dim, parents[b].long()) for b in range(state.shape[dim])]
    return torch.stack(rows, dim)


@pytest.mark.parametrize("shape,dim,N,dtype", [
    ((1, 1, 1), 0, 1, "float32"), ((3, 5, 2048), 0, 5, "bfloat16"), ((4, 3, 8, 7, 64), 1, 8, "bfloat16"), ((2, 4, 33), 0, 9, "uint8"),
    ((2, 3, 2, 64, 5), 2, 64, "float16"), ((2, 64, 4096), 0, 64, "float32"), ((2, 17, 100), 0, 3, "int64"), ((1, 3, 13), 0, 3, "bfloat16"),
    ((2, 16, 20000), 0, 16, "uint8")])
def test_reorder(shape, dim, N, dtype):
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    g = torch.Generator(device=dev).manual_seed(3)
    K = shape[dim + 1]
    state = torch.randint(0, 120, shape, generator=g, device=dev).to(getattr(torch, dtype))
    parents = torch.randint(0, K, (shape[dim], N), generator=g, device=dev, dtype=torch.int32)
    want = _gather(state, parents, dim)
    assert torch.equal(acrl.acrl_beam_reorder(state, parents, dim=dim), want)
    if N == K:
        for p in (parents, torch.arange(K, dtype=torch.int32, device=dev).expand(shape[dim], K).contiguous(),
                  torch.arange(K, dtype=torch.int32, device=dev).flip(0).expand(shape[dim], K).contiguous()):
            want = _gather(state, p, dim)
            own = state.clone()
            assert acrl.acrl_beam_reorder(own, p, dim=dim, out=own) is own and torch.equal(own, want)


def test_reorder_prefixes_and_what_lies_beside():
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    L, B, K, tokens, width, live = 3, 2, 4, 20, 24, 13
    for dtype in (torch.bfloat16, torch.uint8):
        state = torch.randint(0, 100, (L, B, K, tokens, width), device=dev).to(dtype)
        parents = torch.tensor([[1, 1, 3, 0], [0, 2, 2, 2]], dtype=torch.int32, device=dev)
        want = _gather(state, parents, 1)[:, :, :, :live]
        assert torch.equal(acrl.acrl_beam_reorder(state[:, :, :, :live], parents, dim=1), want)
        other = torch.full_like(state, 7)
        acrl.acrl_beam_reorder(state[:, :, :, :live], parents, dim=1, out=other[:, :, :, :live])
        assert torch.equal(other[:, :, :, :live], want) and bool((other[:, :, :, live:] == 7).all())
        own = state.clone()
        acrl.acrl_beam_reorder(own[:, :, :, :live], parents, dim=1, out=own[:, :, :, :live])
        assert torch.equal(own[:, :, :, :live], want) and torch.equal(own[:, :, :, live:], state[:, :, :, live:])
        odd = state.reshape(-1)[1:1 + B * K * 15].view(B, K, 15)
        assert torch.equal(acrl.acrl_beam_reorder(odd, parents), _gather(odd, parents, 0))


def test_reorder_parents_that_are_no_beam():
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    state = torch.randn((2, 3, 50), device=dev)
    parents = torch.tensor([[-1, 2, 0], [3, 2 ** 31 - 1, 1]], dtype=torch.int32, device=dev)
    want = torch.zeros_like(state)
    want[0, 1], want[0, 2], want[1, 2] = state[0, 2], state[0, 0], state[1, 1]
    assert torch.equal(acrl.acrl_beam_reorder(state, parents), want)
    own = state.clone()
    acrl.acrl_beam_reorder(own, parents, out=own)
    assert torch.equal(own, want)
    for empty in (torch.zeros((0, 3, 5), device=dev), torch.zeros((2, 3, 0), device=dev)):
        assert acrl.acrl_beam_reorder(empty, parents[:empty.shape[0]]).shape == empty.shape


def test_refusals():
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    z = lambda *shape, dtype=torch.float32: torch.zeros(shape, dtype=dtype, device=dev)  # noqa: E731
    i = lambda *shape: z(*shape, dtype=torch.int32)  # noqa: E731
    for args, kw in (((z(6, 10), z(2, 4), 2), {}), ((z(6, 10, dtype=torch.float16), z(2, 3), 2), {}), ((z(6, 10).cpu(), z(2, 3), 2), {}),
                     ((z(6, 10), z(2, 3).double(), 2), {}), ((z(10, 6).t(), z(2, 3), 2), {}),
                     ((z(6, 10), z(2, 3), 2), dict(finished=z(2, 3))), ((z(6, 10), z(2, 3), 2), dict(ids=i(2, 3)))):
        with pytest.raises(ValueError):
            acrl.acrl_beam_step(*args, **kw)
    done = z(2, 3, dtype=torch.uint8)
    for args, kw in (((z(6, 10), z(2, 3), 0), {}), ((z(6, 10), z(2, 3), 31), {}), ((z(6, 100), z(2, 3), 65), {}),
                     ((z(130, 10), z(2, 65), 2), {}), ((z(6, 10), z(2, 3), 2), dict(inv_temperature=0.0)),
                     ((z(6, 10), z(2, 3), 2), dict(inv_temperature=float("nan"))),
                     ((z(6, 10), z(2, 3), 2), dict(finished=done)), ((z(6, 10), z(2, 3), 2), dict(finished=done, eos_id=10))):
        with pytest.raises(acrl.AcrlError):
            acrl.acrl_beam_step(*args, **kw)
    s = z(2, 3, 8)
    for args, kw in (((s.cpu(), i(2, 3)), {}), ((s, i(2, 3).long()), {}), ((s, i(3, 3)), {}), ((s, i(2, 3)), dict(dim=2)),
                     ((s, i(2, 3)), dict(out=z(2, 3, 7))), ((s, i(2, 3)), dict(out=z(2, 3, 8, dtype=torch.int32))),
                     ((z(2, 3, 8, 4)[..., :2], i(2, 3)), {}), ((z(4, 5, 2, 3, 8)[:, :3], i(2, 3)), dict(dim=2))):
        with pytest.raises(ValueError):
            acrl.acrl_beam_reorder(*args, **kw)
    big = z(2, 4, 8)
    for args, kw in (((s, i(2, 65)), {}), ((z(2, 65, 8), i(2, 3)), {}), ((big[:, :3], i(2, 3)), dict(out=big[:, 1:])),
                     ((big, i(2, 3)), dict(out=big[:, :3])), ((s, i(2, 3)), dict(out=z(2, 1, 8).expand(2, 3, 8)))):
        with pytest.raises(acrl.AcrlError):
            acrl.acrl_beam_reorder(*args, **kw)
