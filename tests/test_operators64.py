"""The 64-bit definitions that the GPU tests compare with, checked on the host:
their gradients against differences, against autograd of the formulas, and the
policy loss against the oracle's surrogate where the two are the same."""
import numpy as np
import pytest
import torch

import oracle
from operators64 import policy_loss, preference_loss, shares


def _batch(B, L, seed, n_groups):
    r = np.random.default_rng(seed)
    mask = (np.arange(L)[None] < r.integers(0, L + 1, size=B)[:, None]) & (r.random((B, L)) > 0.1)
    mask[0] = False
    lp = {k: np.log(r.uniform(1e-3, 1, B * L)).astype(np.float32) for k in ("old",)}
    lp["new"] = (lp["old"] + r.normal(0, 0.3, B * L)).astype(np.float32)
    lp["ref"] = (lp["old"] + r.normal(0, 0.3, B * L)).astype(np.float32)
    return r, mask.astype(np.uint8).reshape(-1), lp, (np.arange(B) * n_groups // B).astype(np.int32)


@pytest.mark.parametrize("kl", ["k1", "k2", "k3"])
@pytest.mark.parametrize("aggregate", ["group", "sequence", "token", "constant"])
@pytest.mark.parametrize("dual", [0.0, 1.5])
def test_policy_gradient(kl, aggregate, dual):
    B, L = 6, 7
    r, mask, lp, groups = _batch(B, L, 3, 2)
    adv = r.normal(size=B).astype(np.float32)
    w = r.uniform(0.2, 2, B * L).astype(np.float32)
    kw = dict(groups=groups, n_groups=2, ref=lp["ref"], weight=w, eps_low=0.2, eps_high=0.3, dual_clip=dual,
              kl_coef=0.05, kl=kl, norm=17.0)
    got = policy_loss(B, L, mask, lp["new"], lp["old"], adv, False, aggregate, **kw)
    # autograd of the formula in 64 bits
    a = torch.from_numpy(np.repeat(shares(B, L, mask, aggregate, groups, 2, 17.0), L))
    new = torch.from_numpy(lp["new"]).double().requires_grad_()
    old, ref = (torch.from_numpy(lp[k]).double() for k in ("old", "ref"))
    A, W = torch.from_numpy(adv).double().repeat_interleave(L), torch.from_numpy(w).double()
    f = lambda v: float(np.float32(v))  # noqa: E731
    ratio = torch.exp(new - old)
    m = torch.minimum(ratio * A, ratio.clamp(1 - f(0.2), 1 + f(0.3)) * A)
    if dual:
        m = torch.where(A < 0, torch.maximum(m, f(dual) * A), m)
    q = ref - new
    k = {"k1": -q, "k2": q * q / 2, "k3": torch.expm1(q) - q}[kl]
    loss = (torch.from_numpy(mask).double() * a * (-W * m + f(0.05) * k)).sum()
    loss.backward()
    assert abs(got["loss"] - loss.item()) <= 1e-14 * max(1, got["size"])
    np.testing.assert_allclose(got["coef"], new.grad.numpy(), rtol=1e-12, atol=1e-16)
    # and differences, away from the borders: the step 2^-10 is exact in the fp32 log-probs used
    for t in np.flatnonzero(mask)[:8]:
        h = 2.0 ** -10
        side = []
        for s in (-h, h):
            moved = lp["new"].astype(np.float64)
            moved[t] += s
            side.append(policy_loss(B, L, mask, moved, lp["old"], adv, False, aggregate, **kw)["loss"])
        if abs(got["coef"][t]) > 1e-6 and np.sign(side[0] - got["loss"]) == -np.sign(side[1] - got["loss"]):
            slope = (side[1] - side[0]) / (2 * h)
            if abs(slope - got["coef"][t]) > 1e-3 * abs(slope):  # a border of the clip within the step
                edge = np.exp(float(lp["new"][t]) - float(lp["old"][t]))
                assert min(abs(edge / b - 1) for b in (0.8, 1.3, max(dual, 1e-9))) < 2 * h


def test_policy_is_the_surrogate_without_its_additions():
    B, L = 8, 9
    r, mask, lp, groups = _batch(B, L, 5, 3)
    adv = r.normal(size=B).astype(np.float32)
    w = r.uniform(0.2, 2, B * L).astype(np.float32)
    got = policy_loss(B, L, mask, lp["new"], lp["old"], adv, False, "group", groups=groups, n_groups=3, weight=w)
    coef, loss = oracle.surrogate(B, L, mask, groups, 3, lp["new"], lp["old"], adv, False, w, float(np.float32(0.2)),
                                  float(np.float32(0.2)))
    assert abs(got["loss"] - loss) < 1e-13
    np.testing.assert_allclose(got["coef"], coef, rtol=1e-12, atol=1e-16)


@pytest.mark.parametrize("form", ["sigmoid", "hinge", "squared"])
@pytest.mark.parametrize("mean", [False, True])
def test_preference_gradient(form, mean):
    B, L = 5, 6
    r, mask, lp, _ = _batch(B, L, 7, 1)
    chosen, rejected = np.array([1, 2, 1, 4]), np.array([2, 3, 0, 4])
    u = r.uniform(0.5, 2, 4).astype(np.float32)
    sm = 0.1 if form == "sigmoid" else 0.0
    kw = dict(ref=lp["ref"], weight=u, beta=0.3, margin=0.2, smoothing=sm, form=form, mean=mean)
    got = preference_loss(B, L, mask, lp["new"], chosen, rejected, **kw)
    f = lambda v: float(np.float32(v))  # noqa: E731
    new = torch.from_numpy(lp["new"]).double().requires_grad_()
    valid = torch.from_numpy(mask.reshape(B, L)).double()
    x = ((new - torch.from_numpy(lp["ref"]).double()).reshape(B, L) * valid).sum(1)
    if mean:
        x = x / valid.sum(1).clamp(min=1)
    h = f(0.3) * (x[chosen] - x[rejected]) - f(0.2)
    ls = torch.nn.functional.logsigmoid
    l = {"sigmoid": -(1 - f(sm)) * ls(h) - f(sm) * ls(-h), "hinge": torch.relu(1 - h),
         "squared": ((h - 0.5) / f(0.3)) ** 2}[form]
    loss = (torch.from_numpy(u).double() * l).mean()
    loss.backward()
    assert abs(got["loss"] - loss.item()) < 1e-13 * max(1, got["size"])
    np.testing.assert_allclose(got["coef"], new.grad.numpy(), rtol=1e-12, atol=1e-16)
    t = int(np.flatnonzero(mask.reshape(B, L)[1])[0]) + L
    side = []
    for s in (-1e-6, 1e-6):
        moved = lp["new"].astype(np.float64)
        moved[t] += s
        side.append(preference_loss(B, L, mask, moved, chosen, rejected, **kw)["loss"])
    assert abs((side[1] - side[0]) / 2e-6 - got["coef"][t]) < 1e-6 * max(1, abs(got["coef"][t]))
