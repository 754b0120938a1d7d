"""The operators together, as a training step uses them: the rollout policy's
last layer in block-scaled FP8 gives mu's hidden states; both policies are
scored; the discrepancy controls the weights; the clipped policy loss with its
KL term to a reference policy, and a preference loss on the same responses, give
coef; acrl_lm_head_backward turns coef into dH and dW.

Compared with the same chain in 64 bits on the host.  The log-probs that enter
the losses are the library's own (their accuracy has its tests elsewhere), so
what is compared is the loss's and the gradient's part:
 - d loss / d Z is rounded to bf16, half a step = 2^-8 of each value, before the
   products: |dH - ref| <= 2^-8 |dZ| |W| elementwise, and dW likewise;
 - softmax and coef are off by the log-probs' error (2e-3 bound of the scoring
   tests, taken relative to the probability): another 2e-3 of the same sums;
 - fp32 accumulation: 2^-20 of the same sums covers 2048 additions' random walk."""
import types

import numpy as np
import pytest

import inputs
import oracle
from cases import random_bf16
from gpu_util import down, torch_dev, up, up_bf16
from operators64 import policy_loss, preference_loss, product, quantize_blocks

pytestmark = pytest.mark.gpu


def _f64(bits):
    return (bits.astype(np.uint32) << 16).view(np.float32).astype(np.float64)


@pytest.mark.parametrize("kl,aggregate", [("k3", "token"), ("k1", "group"), ("k2", "sequence")])
def test_step(kl, aggregate):
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    B, L, n_groups, d_in, d, V = 6, 48, 2, 352, 256, 1500
    r = np.random.default_rng(11)
    lens = np.array([48, 31, 0, 17, 40, 5])
    mask = (np.arange(L)[None] < lens[:, None]).astype(np.uint8).reshape(-1)
    slots = np.flatnonzero(mask).astype(np.int32)
    groups = np.array([0, 0, 0, 1, 1, 1], np.int32)
    T = slots.size
    x, layer = random_bf16((T, d_in), 1), random_bf16((d, d_in), 2, std=0.06)
    head, head_ref = random_bf16((V, d), 3, std=0.1), random_bf16((V, d), 4, std=0.1)
    ids = r.integers(0, V, T).astype(np.int32)
    adv = r.normal(size=B).astype(np.float32)
    t_x, t_layer, w, w_ref = (up_bf16(torch, dev, a) for a in (x, layer, head, head_ref))
    t_ids, t_slots, t_mask, t_groups, t_adv = (up(torch, dev, a) for a in (ids, slots, mask, groups, adv))

    # pi's layer in bf16, mu's in block-scaled FP8
    h = (t_x.float() @ t_layer.float().t()).to(torch.bfloat16)
    lq, ls = acrl.acrl_quantize_fp8(t_layer, acrl.SCALE_BLOCK128)
    xq, xs = acrl.acrl_quantize_fp8(t_x, acrl.SCALE_ROW128)
    h_mu = acrl.acrl_matmul_fp8(xq, xs, lq, ls)
    want, slack = product(*quantize_blocks(x, 1), *quantize_blocks(layer, 128))
    assert (np.abs(down(h_mu.float()) - want) <= slack * 1.01 + 2.0 ** -8 * np.abs(want)).all()

    # scores of pi, mu and the reference policy, discrepancy, weights
    hq, hs = acrl.acrl_quantize_fp8(h_mu, acrl.SCALE_PER_ROW)
    wq, ws = acrl.acrl_quantize_fp8(w, acrl.SCALE_PER_ROW)
    n = B * L
    sc = acrl.acrl_score_pi_mu(h, w, hq, hs, wq, ws, acrl.SCALE_PER_ROW, t_ids, out_slot=t_slots, n_slots=n,
                               want=("entropy", "lse"))
    rf = acrl.acrl_score_pi_mu(h, w_ref, hq, hs, wq, ws, acrl.SCALE_PER_ROW, t_ids, out_slot=t_slots, n_slots=n,
                               want=(), policies=acrl.POLICY_PI)
    red = acrl.acrl_discrepancy_reduce(B, L, n_groups, sc["logp_pi"], sc["logp_mu"], t_mask, t_groups)
    _, weight = acrl.acrl_controller_step(B, L, n_groups, t_mask, t_groups, sc["logp_pi"], sc["logp_mu"], t_adv, False,
                                          acrl.Y_GROUP, red["seq_mean_d"], red["group_y"], red["stats"], 1e-3, 0.65, 3.0)
    old = sc["logp_pi"] + 0.2 * torch.randn(n, generator=torch.Generator(device=dev).manual_seed(5), device=dev)

    coef, loss, stats = acrl.acrl_policy_loss(
        B, L, n_groups, t_mask, t_groups, sc["logp_pi"], old, t_adv, False, logp_ref=rf["logp_pi"], weight=weight,
        eps_high=0.28, dual_clip=3.0, kl_coef=0.05, kl_estimator={"k1": 0, "k2": 1, "k3": 2}[kl],
        aggregate={"group": acrl.AGG_GROUP, "sequence": acrl.AGG_SEQUENCE, "token": acrl.AGG_TOKEN}[aggregate])
    a = {k: down(v) for k, v in dict(new=sc["logp_pi"], old=old, ref=rf["logp_pi"], w=weight).items()}
    ref = policy_loss(B, L, mask, a["new"], a["old"], adv, False, aggregate, groups, n_groups, ref=a["ref"],
                      weight=a["w"], eps_high=0.28, dual_clip=3.0, kl_coef=0.05, kl=kl)
    assert abs(float(loss) - ref["loss"]) <= 1e-12 * ref["size"]

    chosen, rejected = np.array([0, 3, 0], np.int32), np.array([1, 4, 4], np.int32)
    p_coef, p_loss, _ = acrl.acrl_preference_loss(B, L, t_mask, sc["logp_pi"], up(torch, dev, chosen),
                                                  up(torch, dev, rejected), logp_ref=rf["logp_pi"], beta=0.1)
    p_ref = preference_loss(B, L, mask, a["new"], chosen, rejected, a["ref"], None, 0.1)
    assert abs(float(p_loss) - p_ref["loss"]) <= 1e-11 * max(1, p_ref["size"])

    H, W = _f64(down(h.view(torch.int16)).view(np.uint16)), _f64(head)
    z = H @ W.T
    p = np.exp(z - z.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    one = np.zeros_like(p)
    one[np.arange(T), ids] = 1
    for c, cref in ((coef, ref["coef"]), (p_coef, p_ref["coef"])):
        dh, dw = acrl.acrl_lm_head_backward(h, w, t_ids, c, sc["lse_pi"], row_slot=t_slots)
        g = cref[slots][:, None]
        dz, mag = g * (one - p), np.abs(g) * (one + p)
        tol = 2.0 ** -8 + 2e-3 + 2.0 ** -20
        assert (np.abs(down(dh) - dz @ W) <= tol * (mag @ np.abs(W)) + 1e-12).all()
        assert (np.abs(down(dw) - dz.T @ H) <= tol * (mag.T @ np.abs(H)) + 1e-12).all()
        assert np.abs(down(dw)).max() > 0


def _calls(torch, dev, acrl, stream=None):
    """One call of each operator: name -> outputs."""
    x, w = (up_bf16(torch, dev, random_bf16(shape, k)) for k, shape in enumerate(((40, 256), (192, 256))))
    n, m = torch.zeros(4000, device=dev), torch.ones(4000, dtype=torch.uint8, device=dev)
    i = torch.zeros(2, dtype=torch.int32, device=dev)
    xq, xs = acrl.acrl_quantize_fp8(x, acrl.SCALE_ROW128)
    wq, ws = acrl.acrl_quantize_fp8(w, acrl.SCALE_BLOCK128)
    torch.cuda.synchronize()
    return dict(rows=lambda: acrl.acrl_quantize_fp8(x, acrl.SCALE_ROW128, stream=stream),
                blocks=lambda: acrl.acrl_quantize_fp8(w, acrl.SCALE_BLOCK128, stream=stream),
                matmul=lambda: [acrl.acrl_matmul_fp8(xq, xs, wq, ws, stream=stream)],
                policy=lambda: acrl.acrl_policy_loss(2, 2000, 1, m, i, n, n, n[:2], False, stream=stream),
                preference=lambda: acrl.acrl_preference_loss(2, 2000, m, n, i, i, stream=stream))


def test_stream_of_another_device():
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    other = types.SimpleNamespace(device_index=torch.cuda.current_device() + 1, cuda_stream=0)  # (refused before its use)
    for name, call in _calls(torch, dev, acrl, other).items():
        with pytest.raises(ValueError, match="stream"):
            call()


def test_outputs_belong_to_the_stream():
    # memory of outputs that are dropped while the stream may still use them goes back to that stream, not to the
    # current one's next allocation
    torch, dev = torch_dev()
    from paper_2607_24062_amd import acrl
    s = torch.cuda.Stream()
    for name, call in _calls(torch, dev, acrl, s).items():
        out = call()
        held = [(t.data_ptr(), t.shape, t.dtype) for t in out]
        del out
        fresh = [torch.empty(shape, dtype=dtype, device=dev) for _, shape, dtype in held for _ in range(3)]
        assert not {a for a, _, _ in held} & {t.data_ptr() for t in fresh}, name
    torch.cuda.synchronize()
