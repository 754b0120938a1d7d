"""acrl_policy_loss and acrl_preference_loss against their definitions in 64
bits.  Sums and terms are fp64: losses and statistics may be off by the
roundings of a few thousand fp64 operations (1e-12 of the magnitudes added),
gradients by those and half an fp32 step."""
import numpy as np
import pytest

from gpu_util import down, torch_dev, up
from operators64 import policy_loss, preference_loss

pytestmark = pytest.mark.gpu

HALF32 = 2.0 ** -24
AGG = ["group", "sequence", "token", "constant"]
KL = ["k1", "k2", "k3"]


def _batch(B, L, seed, n_groups, holes=0.1, std=0.3):
    r = np.random.default_rng(seed)
    mask = (np.arange(L)[None] < r.integers(0, L + 1, size=B)[:, None]) & (r.random((B, L)) >= holes)
    if B > 2:
        mask[r.integers(0, B)] = False
        mask[0] = True
    old = np.log(r.uniform(1e-5, 1, B * L)).astype(np.float32)
    lp = {"old": old, "new": (old + r.normal(0, std, B * L)).astype(np.float32),
          "ref": (old + r.normal(0, std, B * L)).astype(np.float32)}
    return r, mask.astype(np.uint8).reshape(-1), lp, r.permutation(np.arange(B) % max(1, n_groups)).astype(np.int32)


def _garbage(mask, *arrays):
    """What masked slots hold must not matter."""
    junk = np.array([np.nan, np.inf, -np.inf, -3.4e38], np.float32)
    for k, a in enumerate(arrays):
        at = np.flatnonzero(mask == 0)
        a[at] = junk[(at + k) % 4]


def _policy(B, L, n_groups, mask, groups, lp, adv, per_token, aggregate="group", kl="k3", use_ref=True, weight=None,
            kl_coef=0.05, dual_clip=0.0, eps=(0.2, 0.28), norm=31.0, place=None, **kw):
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    t = place or (lambda a: up(torch, dev, a))
    return acrl.acrl_policy_loss(
        B, L, n_groups, t(mask), t(groups), t(lp["new"]), t(lp["old"]), t(adv), per_token,
        logp_ref=t(lp["ref"]) if use_ref else None, weight=None if weight is None else t(weight), eps_low=eps[0],
        eps_high=eps[1], dual_clip=dual_clip, kl_coef=kl_coef if use_ref else 0.0,
        kl_estimator={"k1": acrl.KL_K1, "k2": acrl.KL_K2, "k3": acrl.KL_K3}[kl],
        aggregate={"group": acrl.AGG_GROUP, "sequence": acrl.AGG_SEQUENCE, "token": acrl.AGG_TOKEN,
                   "constant": acrl.AGG_CONSTANT}[aggregate], norm=norm, **kw)


def _check(coef, want, ref_size):
    got = down(coef).astype(np.float64)
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(got), nan)
    slack = HALF32 * np.abs(want) + 1e-12 * ref_size + 2.0 ** -150
    assert (np.abs(got - want) <= slack)[~nan].all()


def _check_policy(got, ref, B, L):
    coef, loss, stats = got
    _check(coef, ref["coef"], np.abs(ref["coef"]))
    assert abs(float(down(loss)[0]) - ref["loss"]) <= 1e-12 * ref["size"]
    s = down(stats)
    assert (np.abs(s - ref["stats"]) <= 1e-11 * np.maximum(np.abs(ref["stats"]), ref["size"])).all(), (s, ref["stats"])


@pytest.mark.parametrize("B,L,n_groups", [(1, 1, 1), (3, 5, 2), (4, 64, 1), (6, 1000, 3), (5, 1024, 5), (16, 67, 4),
                                          (2, 4099, 1), (70, 36, 40), (1100, 12, 300)])
@pytest.mark.parametrize("aggregate", AGG)
def test_policy_shapes(B, L, n_groups, aggregate):
    r, mask, lp, groups = _batch(B, L, B + L, n_groups)
    per_token = (B + L) % 2 == 0
    adv = r.normal(size=B * L if per_token else B).astype(np.float32)
    w = r.uniform(0.2, 3, B * L).astype(np.float32) if B % 2 else None
    kl = KL[(B + L) % 3]
    kw = dict(ref=lp["ref"], weight=w, eps_low=0.2, eps_high=0.28, dual_clip=1.5, kl_coef=0.05, kl=kl, norm=31.0)
    ref = policy_loss(B, L, mask, lp["new"], lp["old"], adv, per_token, aggregate, groups, n_groups, **kw)
    _garbage(mask, *lp.values(), *([w] if w is not None else []))
    got = _policy(B, L, n_groups, mask, groups, lp, adv, per_token, aggregate, kl, weight=w, dual_clip=1.5)
    _check_policy(got, ref, B, L)
    assert not down(got[0])[mask == 0].any()


@pytest.mark.parametrize("kl", KL)
@pytest.mark.parametrize("dual", [0.0, 1.01])
@pytest.mark.parametrize("use_ref", [True, False])
def test_policy_terms(kl, dual, use_ref):
    # ratios far from 1, next to 1 and exactly 1, at and next to the clip's borders
    B, L = 4, 512
    r, mask, lp, groups = _batch(B, L, 3, 2, std=2.0)
    lp["new"][::5] = lp["old"][::5]
    lp["ref"][1::7] = lp["new"][1::7]
    lp["ref"][2::7] = np.nextafter(lp["new"][2::7], np.float32(0))
    for k, b in enumerate((0.8, 1.28, max(dual, 1.0))):
        lp["new"][k::11] = lp["old"][k::11] + np.float32(np.log(b))
    adv = r.normal(size=B * L).astype(np.float32)
    adv[::13] = 0
    ref = policy_loss(B, L, mask, lp["new"], lp["old"], adv, True, "token", eps_high=0.28, dual_clip=dual, kl=kl,
                      kl_coef=0.05, ref=lp["ref"] if use_ref else None)
    got = _policy(B, L, 2, mask, groups, lp, adv, True, "token", kl, use_ref, dual_clip=dual)
    _check_policy(got, ref, B, L)


@pytest.mark.parametrize("B,L", [(4, 64), (3, 4096)])
@pytest.mark.parametrize("kl", KL)
def test_policy_reference_far_below_and_above(B, L, kl):
    # a reference that gives a token next to nothing: k' = 1 - exp(q) is 1 there, whatever k is
    r, mask, lp, groups = _batch(B, L, 5, 1)
    mask[:] = 1
    far = np.array([-1.0, -1.5, -40, -745, -800, -1e9, -1e30, -3.4e38, 5, 40, 60], np.float32)
    lp["ref"][:far.size] = far
    adv = r.normal(size=B).astype(np.float32)
    ref = policy_loss(B, L, mask, lp["new"], lp["old"], adv, False, "constant", eps_high=0.28, kl=kl, kl_coef=0.05,
                      ref=lp["ref"], norm=31.0)
    coef, loss, stats = _policy(B, L, 1, mask, groups, lp, adv, False, "constant", kl)
    _check(coef, ref["coef"], np.abs(ref["coef"]))
    assert abs(float(down(loss)[0]) - ref["loss"]) <= 1e-12 * ref["size"]


@pytest.mark.parametrize("B,L", [(4, 64), (3, 4096)])
def test_policy_infinite_divergence(B, L):
    # k is infinite where the reference rules a token out: the loss too, but not the gradient of k3, and without
    # kl_coef the statistics alone
    r, mask, lp, groups = _batch(B, L, 5, 1)
    mask[:] = 1
    lp["ref"][3] = -np.inf
    adv = r.normal(size=B).astype(np.float32)
    for kl in ("k1", "k3"):
        for kl_coef in (0.05, 0.0):
            q = lp["ref"].astype(np.float64) - lp["new"]
            coef, loss, stats = _policy(B, L, 1, mask, groups, lp, adv, False, "token", kl, kl_coef=kl_coef)
            finite = dict(lp, ref=np.where(q == -np.inf, np.float32(-1e30), lp["ref"]))
            ref = policy_loss(B, L, mask, lp["new"], lp["old"], adv, False, "token", eps_high=0.28, kl=kl,
                              kl_coef=kl_coef, ref=finite["ref"])
            _check(coef, ref["coef"], np.abs(ref["coef"]))
            s = down(stats)
            assert s[1] == np.inf and np.isfinite(s[[0, 2, 3, 4, 5]]).all()
            if kl_coef:
                assert down(loss)[0] == np.inf
            else:
                assert abs(float(down(loss)[0]) - ref["loss"]) <= 1e-12 * ref["size"]


def test_policy_matches_the_surrogate():
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    B, L, n = 12, 130, 4
    r, mask, lp, groups = _batch(B, L, 8, n)
    adv = r.normal(size=B).astype(np.float32)
    w = r.uniform(0.2, 3, B * L).astype(np.float32)
    t = lambda a: up(torch, dev, a)
    coef, loss, _ = _policy(B, L, n, mask, groups, lp, adv, False, use_ref=False, weight=w, eps=(0.2, 0.2))
    c2, l2 = acrl.acrl_surrogate(B, L, n, t(mask), t(groups), t(lp["new"]), t(lp["old"]), t(adv), False, 0.2, 0.2,
                                 weight=t(w))
    np.testing.assert_allclose(down(coef), down(c2), rtol=2.0 ** -23, atol=0)
    np.testing.assert_allclose(down(loss), down(l2), rtol=1e-12)


@pytest.mark.parametrize("aggregate", AGG)
def test_policy_many_groups_and_large_batch(aggregate):
    # more groups than one workgroup counts; more slots than its workgroups share out the norms of
    for B, L, n_groups in ((40, 200, 3000), (33, 33000, 5)):
        if L > 1000 and aggregate in ("sequence", "constant"):
            continue
        r, mask, lp, groups = _batch(B, L, 70 + B, n_groups, holes=0.4)
        adv = r.normal(size=B).astype(np.float32)
        ref = policy_loss(B, L, mask, lp["new"], lp["old"], adv, False, aggregate, groups, n_groups, ref=lp["ref"],
                          kl_coef=0.05, eps_high=0.28, norm=31.0)
        _check_policy(_policy(B, L, n_groups, mask, groups, lp, adv, False, aggregate), ref, B, L)


def test_policy_any_nonzero_mask():
    for B, L in ((3, 90), (7, 4099), (12, 90000)):
        r, mask, lp, groups = _batch(B, L, 90 + B, 2)
        adv = r.normal(size=B).astype(np.float32)
        a = _policy(B, L, 2, mask, groups, lp, adv, False, "token")
        b = _policy(B, L, 2, mask * r.choice([1, 2, 127, 128, 255], mask.size).astype(np.uint8), groups, lp, adv, False,
                    "token")
        assert all((down(x) == down(y)).all() for x, y in zip(a, b))


@pytest.mark.parametrize("aggregate", AGG)
def test_policy_nothing_valid(aggregate):
    for B, L in ((3, 40), (2, 5000), (0, 8), (4, 0)):
        mask = np.zeros(B * L, np.uint8)
        lp = {k: np.full(B * L, np.nan, np.float32) for k in ("new", "old", "ref")}
        coef, loss, stats = _policy(B, L, 2, mask, np.zeros(B, np.int32), lp, np.ones(B, np.float32), False, aggregate)
        assert not down(coef).any() and down(loss)[0] == 0 and not down(stats).any()


def test_policy_group_out_of_range():
    B, L, n = 9, 70, 3
    r, mask, lp, groups = _batch(B, L, 4, n)
    mask[:] = 1
    groups[2], groups[5] = -1, n
    adv = r.normal(size=B).astype(np.float32)
    ref = policy_loss(B, L, mask, lp["new"], lp["old"], adv, False, "group", groups, n, ref=lp["ref"], kl_coef=0.05,
                      eps_high=0.28)
    _check_policy(_policy(B, L, n, mask, groups, lp, adv, False), ref, B, L)


def test_policy_nan_stays_in_its_slot():
    B, L = 4, 300
    r, mask, lp, groups = _batch(B, L, 6, 2)
    mask[:] = 1
    lp["new"][333] = np.nan
    adv = np.ones(B, np.float32)
    coef, loss, _ = _policy(B, L, 2, mask, groups, lp, adv, False)
    assert list(np.flatnonzero(np.isnan(down(coef)))) == [333] and np.isnan(down(loss)[0])


def _unaligned(torch, dev):
    """Tensors whose first element is not 16-byte aligned."""
    def place(a):
        buf = torch.empty(a.size + 1, dtype=torch.from_numpy(a).dtype, device=dev)
        buf[1:] = torch.from_numpy(a).to(dev)
        return buf[1:]
    return place


@pytest.mark.parametrize("L", [64, 4096])
def test_policy_unaligned_and_aligned_agree(L):
    torch, dev = torch_dev()
    B = 6
    r, mask, lp, groups = _batch(B, L, 14, 2)
    adv = r.normal(size=B * L).astype(np.float32)
    a = _policy(B, L, 2, mask, groups, lp, adv, True, "sequence")
    b = _policy(B, L, 2, mask, groups, lp, adv, True, "sequence", place=_unaligned(torch, dev))
    assert torch.equal(a[0], b[0])
    np.testing.assert_allclose(down(a[1]), down(b[1]), rtol=1e-13)
    np.testing.assert_allclose(down(a[2]), down(b[2]), rtol=1e-12)


def test_policy_large_batch_against_its_responses():
    # several turns a workgroup and many units: response by response, CONSTANT, gives the same gradient and sums
    torch, dev = torch_dev()
    B, L = 96, 12300
    r, mask, lp, groups = _batch(B, L, 15, 2, holes=0.3)
    adv = r.normal(size=B).astype(np.float32)
    coef, loss, stats = _policy(B, L, 2, mask, groups, lp, adv, False, "constant", norm=3.0)
    parts, total, tokens = [], 0.0, 0.0
    for i in range(0, B, 12):
        at = slice(i * L, (i + 12) * L)
        c, l, s = _policy(12, L, 2, mask[at], groups[i:i + 12], {k: v[at] for k, v in lp.items()}, adv[i:i + 12],
                          False, "constant", norm=3.0)
        parts.append(c)
        total += float(l)
        tokens += float(s[5])
    assert torch.equal(coef, torch.cat(parts)) and tokens == float(stats[5]) == mask.sum()
    assert abs(total - float(loss)) <= 1e-12 * abs(total) + 1e-9


# ------------------------------------------------------------------ preference
def _preference(B, L, mask, lp, chosen, rejected, use_ref=True, weight=None, form="sigmoid", mean=False, beta=0.1,
                margin=0.0, smoothing=0.0, place=None, **kw):
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    t = place or (lambda a: up(torch, dev, a))
    return acrl.acrl_preference_loss(
        B, L, t(mask), t(lp["new"]), t(chosen), t(rejected), logp_ref=t(lp["ref"]) if use_ref else None,
        pair_weight=None if weight is None else t(weight), beta=beta, margin=margin, label_smoothing=smoothing,
        form={"sigmoid": acrl.PREF_SIGMOID, "hinge": acrl.PREF_HINGE, "squared": acrl.PREF_SQUARED}[form],
        mean_logp=mean, **kw)


def _check_preference(got, ref):
    coef, loss, rewards = got
    _check(coef, ref["coef"], np.abs(ref["coef"]) + 1.0 / max(1, ref["rewards"].shape[1]))
    if np.isnan(ref["loss"]):
        assert np.isnan(down(loss)[0])
    else:
        assert abs(float(down(loss)[0]) - ref["loss"]) <= 1e-11 * max(ref["size"], 1e-3)
    w = ref["rewards"]
    g = down(rewards).astype(np.float64)
    assert np.array_equal(np.isnan(g), np.isnan(w))
    assert (np.abs(g - w) <= HALF32 * np.abs(w) + 1e-11)[~np.isnan(w)].all()


@pytest.mark.parametrize("B,L,P", [(2, 1, 1), (4, 64, 2), (8, 67, 4), (5, 1023, 9), (6, 4100, 3), (64, 40, 300),
                                   (3, 1024, 1), (1200, 8, 700)])
@pytest.mark.parametrize("form", ["sigmoid", "hinge", "squared"])
@pytest.mark.parametrize("mean", [False, True])
def test_preference_shapes(B, L, P, form, mean):
    r, mask, lp, _ = _batch(B, L, B + L + P, 1)
    chosen, rejected = (r.integers(0, B, P).astype(np.int32) for _ in range(2))  # shared, repeated, c == r among them
    u = r.uniform(0.1, 2, P).astype(np.float32) if P % 2 else None
    use_ref = B % 3 != 0
    sm = 0.1 if form == "sigmoid" else 0.0
    ref = preference_loss(B, L, mask, lp["new"], chosen, rejected, lp["ref"] if use_ref else None, u, 0.3, 0.25, sm,
                          form, mean)
    _garbage(mask, *lp.values())
    got = _preference(B, L, mask, lp, chosen, rejected, use_ref, u, form, mean, 0.3, 0.25, sm)
    _check_preference(got, ref)
    assert not down(got[0])[mask == 0].any()


def test_preference_far_apart():
    # log-ratios of hundreds: the sigmoid's tails keep their relative precision
    B, L = 6, 900
    r, mask, lp, _ = _batch(B, L, 2, 1, std=0.1)
    mask[:] = 1
    lp["new"] = (lp["ref"] + np.repeat([1.0, -1.0, 0.1, 0.3, -0.4, 0.0], L)).astype(np.float32)
    chosen, rejected = np.array([0, 1, 2, 4, 5, 5], np.int32), np.array([1, 0, 3, 2, 0, 5], np.int32)
    ref = preference_loss(B, L, mask, lp["new"], chosen, rejected, lp["ref"], None, 0.3)
    coef, loss, _ = _preference(B, L, mask, lp, chosen, rejected, beta=0.3)
    got, want = down(coef).astype(np.float64), ref["coef"]
    # h is a difference of sums of size 900, off by 1e-12: exp(h) by that, relative
    assert (np.abs(got - want) <= (HALF32 + 1e-10) * np.abs(want)).all()
    assert abs(float(down(loss)[0]) - ref["loss"]) <= 1e-11 * ref["size"]


def test_preference_no_pairs_and_no_tokens():
    torch, dev = torch_dev()
    none = np.zeros(0, np.int32)
    r, mask, lp, _ = _batch(4, 50, 1, 1)
    coef, loss, rewards = _preference(4, 50, mask, lp, none, none)
    assert not down(coef).any() and down(loss)[0] == 0 and rewards.shape == (2, 0)
    mask[:] = 0
    c = np.array([1, 2], np.int32)
    coef, loss, rewards = _preference(4, 50, mask, lp, c, c[::-1].copy(), mean=True)
    assert not down(coef).any() and abs(down(loss)[0] - np.log(2)) < 1e-15 and not down(rewards).any()
    for B, L in ((0, 8), (3, 0)):
        lp0 = {k: np.zeros(B * L, np.float32) for k in lp}
        coef, loss, _ = _preference(B, L, np.zeros(B * L, np.uint8), lp0, none, none)
        assert coef.numel() == 0 and down(loss)[0] == 0


def test_preference_index_out_of_range():
    B, L = 5, 60
    r, mask, lp, _ = _batch(B, L, 12, 1)
    mask[:] = 1
    chosen, rejected = np.array([0, 5, 3], np.int32), np.array([1, 2, -1], np.int32)
    ref = preference_loss(B, L, mask, lp["new"], chosen, rejected, lp["ref"])
    _check_preference(_preference(B, L, mask, lp, chosen, rejected), ref)


def test_preference_unaligned():
    torch, dev = torch_dev()
    B, L = 5, 1024
    r, mask, lp, _ = _batch(B, L, 13, 1)
    c, j = np.array([0, 1], np.int32), np.array([2, 3], np.int32)
    a = _preference(B, L, mask, lp, c, j)
    b = _preference(B, L, mask, lp, c, j, place=_unaligned(torch, dev))
    np.testing.assert_allclose(down(a[0]), down(b[0]), rtol=2.0 ** -22)
    np.testing.assert_allclose(down(a[1]), down(b[1]), rtol=1e-12)


def test_more_slots_than_31_bits():
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    B, L = 140000, 16384
    mask = torch.zeros((B, L), dtype=torch.uint8, device=dev)
    mask[:, :3] = 1
    new, old = torch.zeros((B, L), device=dev), torch.zeros((B, L), device=dev)
    new[-1, 1] = 0.125
    groups, adv = torch.zeros(B, dtype=torch.int32, device=dev), torch.ones(B, device=dev)
    coef, loss, stats = acrl.acrl_policy_loss(B, L, 1, mask, groups, new, old, adv, False, aggregate=acrl.AGG_TOKEN)
    n, c = 3 * B, coef.view(B, L)
    assert float(stats[5]) == n and abs(float(loss) + (n - 1 + np.exp(0.125)) / n) <= 1e-12
    want = np.array([-1 / n, -np.exp(0.125) / n, -1 / n, 0])
    assert (np.abs(down(c[-1, :4]) - want) <= HALF32 * np.abs(want)).all() and not c[:, 3:].any()
    pair = lambda *i: torch.tensor(i, dtype=torch.int32, device=dev)
    coef, loss, rewards = acrl.acrl_preference_loss(B, L, mask, new, pair(B - 1, 0), pair(0, B - 2), beta=0.5)
    up1, up0 = 1 / (1 + np.exp(0.0625)), 0.5  # sigmoid(-h) of the two pairs
    want = np.array([-up1, up0, up1 - up0]) * 0.25  # (response 0: rejected in the first pair, preferred in the second)
    got = down(coef.view(B, L)[[B - 1, B - 2, 0], 0])
    assert (np.abs(got - want) <= HALF32 * np.abs(want) + 1e-15).all()


# ------------------------------------------------------------------ refusals
def test_refusals():
    # tensors that do not fit B, L and the number of pairs are refused before anything is launched
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    B, L = 3, 2000
    n = B * L
    m, lp = torch.ones(n, dtype=torch.uint8, device=dev), torch.zeros(n, device=dev)
    i = torch.zeros(B, dtype=torch.int32, device=dev)
    ok = dict(mask=m, group_of_seq=i, logp_new=lp, logp_old=lp, adv=lp[:B], adv_per_token=False, logp_ref=lp, kl_coef=0.1)
    for bad in (dict(mask=m[1:]), dict(mask=m.bool()), dict(mask=m.cpu()), dict(mask=None), dict(group_of_seq=i[1:]),
                dict(group_of_seq=i.long()), dict(logp_new=lp[1:]), dict(logp_new=lp.double()), dict(logp_old=None),
                dict(logp_old=lp.view(L, B).t()), dict(adv=lp), dict(adv_per_token=True), dict(logp_ref=lp.half()),
                dict(weight=lp[:B]), dict(coef=lp[:5]), dict(coef=lp.double())):
        with pytest.raises(ValueError):
            acrl.acrl_policy_loss(B, L, 1, **{**ok, **bad})
    for bad in (dict(eps_low=1.0), dict(kl_coef=-1.0), dict(logp_ref=None), dict(dual_clip=0.9), dict(aggregate=7),
                dict(group_of_seq=None)):
        with pytest.raises(acrl.AcrlError):
            acrl.acrl_policy_loss(B, L, 1, **{**ok, **bad})
    ok = dict(mask=m, logp_new=lp, chosen=i, rejected=i, logp_ref=lp)
    for bad in (dict(mask=m[1:]), dict(logp_new=lp[1:]), dict(chosen=i[1:]), dict(chosen=i.long()), dict(rejected=None),
                dict(rejected=i.cpu()), dict(pair_weight=lp[:2]), dict(logp_ref=lp[:B]), dict(coef=lp[:5])):
        with pytest.raises(ValueError):
            acrl.acrl_preference_loss(B, L, **{**ok, **bad})
    for bad in (dict(beta=0.0), dict(label_smoothing=1.0), dict(form=1, label_smoothing=0.1), dict(form=3)):
        with pytest.raises(acrl.AcrlError):
            acrl.acrl_preference_loss(B, L, **{**ok, **bad})


# ------------------------------------------------------------------ streams and graphs
def _both(B, L, t, stream=None):
    from paper_2607_24062_amd import acrl
    p = acrl.acrl_policy_loss(B, L, 2, t["mask"], t["groups"], t["new"], t["old"], t["adv"], False, logp_ref=t["ref"],
                              kl_coef=0.05, stream=stream)
    q = acrl.acrl_preference_loss(B, L, t["mask"], t["new"], t["chosen"], t["rejected"], logp_ref=t["ref"], stream=stream)
    return [*p, *q]


def _tensors(B, L, seed):
    torch, dev = torch_dev()
    r, mask, lp, groups = _batch(B, L, seed, 2)
    c = r.integers(0, B, 5).astype(np.int32)
    a = dict(mask=mask, groups=groups, adv=r.normal(size=B).astype(np.float32), chosen=c,
             rejected=((c + 1) % B).astype(np.int32), **lp)
    return {k: up(torch, dev, v) for k, v in a.items()}


@pytest.mark.parametrize("B,L", [(4, 64), (6, 4096), (40, 30000)])
def test_captured_and_replayed(B, L):
    # two graphs of the same calls, each with its own workspace, replayed at once on two streams, eager calls between
    torch, dev = torch_dev()
    ins = [_tensors(B, L, 40), _tensors(B, L, 41)]
    _both(B, L, ins[0])
    torch.cuda.synchronize()
    graphs, outs = [], []
    for t in ins:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(_both(B, L, t))
        graphs.append(g)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for k in range(3):
        for t in ins:
            t["new"].copy_(_tensors(B, L, 50 + k)["new"])
        want = [[x.clone() for x in _both(B, L, t)] for t in ins]
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert all(torch.equal(x, y) for x, y in zip(o, w))


def test_two_streams_at_once():
    torch, dev = torch_dev()
    ins = [_tensors(24, 5000, 60), _tensors(24, 5000, 61)]
    want = [[x.clone() for x in _both(24, 5000, t)] for t in ins]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(4):
        for k in range(2):
            got[k].append(_both(24, 5000, ins[k], stream=streams[k]))
    torch.cuda.synchronize()
    for k in range(2):
        for o in got[k]:
            assert all(torch.equal(x, y) for x, y in zip(o, want[k]))
