"""Refusals of the block-scaled FP8 operators and the losses: out-of-contract
calls return a status before any HIP call, on the host and without a device."""
import ctypes

import pytest

INT_MAX = 2 ** 31 - 1


@pytest.fixture(scope="module")
def acrl():
    from paper_2607_24062_amd import acrl
    try:
        acrl.lib()
    except (RuntimeError, OSError) as e:
        pytest.skip("libacrl.so not available: %s" % e)
    return acrl


@pytest.fixture(scope="module")
def p():
    buf = (ctypes.c_uint8 * 4096)()  # never dereferenced: validation fails before any launch
    yield ctypes.c_void_p(ctypes.addressof(buf) + (-ctypes.addressof(buf)) % 256)
    del buf


def _off(p, n):
    return ctypes.c_void_p(p.value + n)


def test_descriptor_sizes(acrl):
    sizes = [ctypes.c_size_t() for _ in range(3)]
    acrl.lib().acrl_abi_operator_struct_sizes(*[ctypes.byref(s) for s in sizes])
    assert [s.value for s in sizes] == [ctypes.sizeof(x) for x in (acrl.MatmulDesc, acrl.PolicyLossDesc,
                                                                  acrl.PreferenceDesc)]
    acrl.lib().acrl_abi_operator_struct_sizes(None, None, None)


def test_quantize_blocks(acrl, p):
    L = acrl.lib()
    nb = ctypes.c_size_t(7)
    for scaling in (acrl.SCALE_ROW128, acrl.SCALE_BLOCK128):
        assert L.acrl_quantize_workspace_size(4, 64, scaling, ctypes.byref(nb)) == 0 and nb.value == 0
        for rows, cols, ld in ((4, 33, 64), (-1, 64, 64), (4, 64, 60), (4, 0, 64), (4, 64, 68)):
            assert L.acrl_quantize_fp8(p, rows, cols, ld, scaling, 0, p, p, None, 0, None) == 1
        assert L.acrl_quantize_fp8(p, 4, 64, 64, scaling, 3, p, p, None, 0, None) == 1
        assert L.acrl_quantize_fp8(p, 4, 64, 64, scaling, 0, p, None, None, 0, None) == 1
        assert L.acrl_quantize_fp8(p, 4, 64, 64, scaling, 0, _off(p, 8), p, None, 0, None) == 1
    assert L.acrl_quantize_workspace_size(4, 64, 5, ctypes.byref(nb)) == 1


@pytest.mark.parametrize("scaling", [3, 4])
def test_scorers_take_no_block_scales(acrl, p, scaling):
    # mu's LM-head kernels know the first three scalings only
    L = acrl.lib()
    nb = ctypes.c_size_t()
    assert L.acrl_score_workspace_size(4, 256, 1000, scaling, ctypes.byref(nb)) == 1
    assert L.acrl_packed_weights_size(1000, 256, scaling, ctypes.byref(nb)) == 1
    d = acrl.ScoreDesc(n_rows=4, d=256, V=1000, h=p, w=p, hq=p, hq_scales=p, wq=p, wq_scales=p, mu_scaling=scaling,
                       inv_temperature=1.0, token_ids=p, logp_pi=p, logp_mu=p, workspace=p, workspace_bytes=1 << 40)
    assert L.acrl_score_pi_mu(ctypes.byref(d), None) == 1
    s = acrl.SampleDesc(n_rows=4, d=256, V=1000, hq=p, hq_scales=p, wq=p, wq_scales=p, mu_scaling=scaling,
                        inv_temperature=1.0, ids=p, workspace=p, workspace_bytes=1 << 40)
    assert L.acrl_sample_mu(ctypes.byref(s), None) == 1


def test_matmul(acrl, p):
    L = acrl.lib()
    ok = dict(M=4, N=64, K=256, xq=p, x_scales=p, wq=p, w_scales=p, y=p, ldy=64, y_type=0)
    for bad in (dict(M=-1), dict(M=1 << 26), dict(N=0), dict(N=-5), dict(N=1 << 26, ldy=1 << 26), dict(K=0),
                dict(K=-32), dict(K=100), dict(K=(1 << 22) + 32), dict(ldy=63), dict(y_type=2), dict(y_type=-1),
                dict(xq=None), dict(x_scales=None), dict(wq=None), dict(w_scales=None), dict(y=None),
                dict(xq=_off(p, 8)), dict(wq=_off(p, 4)), dict(y=_off(p, 2)), dict(x_scales=_off(p, 2)),
                dict(w_scales=_off(p, 1)), dict(M=1 << 25, N=1 << 20, ldy=1 << 20)):
        d = acrl.MatmulDesc(**{**ok, **bad})
        assert L.acrl_matmul_fp8(ctypes.byref(d), None) == acrl.ACRL_ERR_INVALID_ARG, bad
        assert L.acrl_last_error()
    assert L.acrl_matmul_fp8(None, None) == acrl.ACRL_ERR_INVALID_ARG


def test_policy_loss(acrl, p):
    L = acrl.lib()
    ok = dict(B=2, L=4096, n_groups=1, mask=p, group_of_seq=p, logp_new=p, logp_old=p, logp_ref=p, adv=p, eps_low=0.2,
              eps_high=0.2, kl_coef=0.1, kl_estimator=2, coef=p, loss=p, workspace=p, workspace_bytes=1 << 30)
    nan = float("nan")
    for bad in (dict(B=-1), dict(L=-1), dict(n_groups=-1), dict(n_groups=0), dict(group_of_seq=None), dict(mask=None),
                dict(logp_new=None), dict(logp_old=None), dict(adv=None), dict(coef=None), dict(loss=None),
                dict(eps_low=1.0), dict(eps_low=-0.1), dict(eps_low=nan), dict(eps_high=-0.1), dict(eps_high=nan),
                dict(dual_clip=1.0), dict(dual_clip=-1.0), dict(dual_clip=0.5), dict(dual_clip=nan), dict(kl_coef=-1.0),
                dict(kl_coef=nan), dict(logp_ref=None), dict(kl_estimator=3), dict(kl_estimator=-1), dict(aggregate=4),
                dict(aggregate=-1), dict(aggregate=3, norm=0.0), dict(aggregate=3, norm=-1.0),
                dict(aggregate=3, norm=float("inf")), dict(aggregate=3, norm=nan), dict(B=1 << 22), dict(L=INT_MAX),
                dict(B=1 << 21, L=1 << 20), dict(workspace=_off(p, 8))):
        d = acrl.PolicyLossDesc(**{**ok, **bad})
        assert L.acrl_policy_loss(ctypes.byref(d), None) == acrl.ACRL_ERR_INVALID_ARG, bad
    for bad in (dict(workspace=None), dict(workspace_bytes=16)):
        d = acrl.PolicyLossDesc(**{**ok, **bad})
        assert L.acrl_policy_loss(ctypes.byref(d), None) == acrl.ACRL_ERR_WORKSPACE, bad
    assert L.acrl_policy_loss(None, None) == acrl.ACRL_ERR_INVALID_ARG
    nb = ctypes.c_size_t()
    assert L.acrl_policy_loss_workspace_size(64, 4096, 8, ctypes.byref(nb)) == 0 and nb.value >= 64 * 12
    assert L.acrl_policy_loss_workspace_size(4, 64, 1, ctypes.byref(nb)) == 0 and nb.value == 0  # one workgroup's batch
    for B, n, g in ((-1, 4, 1), (4, -1, 1), (4, 4, -1), (1 << 22, 4, 1)):
        assert L.acrl_policy_loss_workspace_size(B, n, g, ctypes.byref(nb)) == acrl.ACRL_ERR_INVALID_ARG
    assert L.acrl_policy_loss_workspace_size(4, 4, 1, None) == acrl.ACRL_ERR_INVALID_ARG


def test_preference_loss(acrl, p):
    L = acrl.lib()
    ok = dict(B=2, L=4096, n_pairs=1, mask=p, logp_new=p, logp_ref=p, chosen=p, rejected=p, beta=0.1, coef=p, loss=p,
              workspace=p, workspace_bytes=1 << 30)
    nan, inf = float("nan"), float("inf")
    for bad in (dict(B=-1), dict(L=-1), dict(n_pairs=-1), dict(mask=None), dict(logp_new=None), dict(coef=None),
                dict(loss=None), dict(chosen=None), dict(rejected=None), dict(beta=0.0), dict(beta=-1.0),
                dict(beta=nan), dict(beta=inf), dict(margin=nan), dict(margin=inf), dict(label_smoothing=1.0),
                dict(label_smoothing=-0.1), dict(label_smoothing=nan), dict(form=1, label_smoothing=0.1),
                dict(form=2, label_smoothing=0.1), dict(form=3), dict(form=-1), dict(mean_logp=2), dict(B=1 << 22),
                dict(L=INT_MAX), dict(n_pairs=INT_MAX), dict(n_pairs=1 << 24), dict(B=1 << 20, n_pairs=1 << 20),
                dict(workspace=_off(p, 8))):
        d = acrl.PreferenceDesc(**{**ok, **bad})
        assert L.acrl_preference_loss(ctypes.byref(d), None) == acrl.ACRL_ERR_INVALID_ARG, bad
    for bad in (dict(workspace=None), dict(workspace_bytes=16)):
        d = acrl.PreferenceDesc(**{**ok, **bad})
        assert L.acrl_preference_loss(ctypes.byref(d), None) == acrl.ACRL_ERR_WORKSPACE, bad
    assert L.acrl_preference_loss(None, None) == acrl.ACRL_ERR_INVALID_ARG
    nb = ctypes.c_size_t()
    assert L.acrl_preference_loss_workspace_size(64, 4096, 8, ctypes.byref(nb)) == 0 and nb.value >= 64 * 16
    assert L.acrl_preference_loss_workspace_size(-1, 4096, 8, ctypes.byref(nb)) == acrl.ACRL_ERR_INVALID_ARG
    assert L.acrl_preference_loss_workspace_size(4, 4, 4, None) == acrl.ACRL_ERR_INVALID_ARG


def test_binding_refuses_host_tensors(acrl):
    import torch
    q, s = torch.zeros((4, 128), dtype=torch.uint8), torch.ones((4, 1))
    with pytest.raises(ValueError, match="device tensor"):
        acrl.acrl_matmul_fp8(q, s, q, s)
    f, m, g = torch.zeros(8), torch.ones(8, dtype=torch.uint8), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="device tensor"):
        acrl.acrl_policy_loss(2, 4, 1, m, g, f, f, f[:2], False)
    with pytest.raises(ValueError, match="device tensor"):
        acrl.acrl_preference_loss(2, 4, m, f, g, g)


def test_bounds_of_the_losses_are_named(acrl, p):
    # what the header's requirements allow is sized, what they do not is refused with the bound
    L, nb = acrl.lib(), ctypes.c_size_t()
    last = lambda: L.acrl_last_error().decode()  # noqa: E731
    for B, n, g in ((1, INT_MAX - 1, 1), (15, INT_MAX - 1, 1), ((1 << 22) - 1, 6144, 0), (4, 64, INT_MAX - 1), (4, 64, 0)):
        assert L.acrl_policy_loss_workspace_size(B, n, g, ctypes.byref(nb)) == 0, (B, n, g)
    for B, n, g, bound in ((1, INT_MAX, 1, "2^31"), (4, 64, INT_MAX, "2^31"), (1 << 22, 64, 1, "2^22"),
                           (16, INT_MAX - 1, 1, "2^24"), ((1 << 22) - 1, 8193, 1, "2^24")):
        assert L.acrl_policy_loss_workspace_size(B, n, g, ctypes.byref(nb)) == acrl.ACRL_ERR_INVALID_ARG
        assert bound in last(), last()
    for B, n, P in ((1, INT_MAX - 1, 1), ((1 << 22) - 1, 64, 1 << 18), (1 << 16, 64, (1 << 24) - 1), (0, 0, 0)):
        assert L.acrl_preference_loss_workspace_size(B, n, P, ctypes.byref(nb)) == 0, (B, n, P)
    for B, n, P, bound in ((1, INT_MAX, 1, "2^31"), (1 << 22, 64, 1, "2^22"), (1, 64, 1 << 24, "2^24"),
                           (1 << 16, 64, 1 << 24, "2^24"), (1 << 21, 64, 1 << 19, "2^40")):
        assert L.acrl_preference_loss_workspace_size(B, n, P, ctypes.byref(nb)) == acrl.ACRL_ERR_INVALID_ARG
        assert bound in last(), last()
    ok = dict(B=2, L=4096, n_groups=1, mask=p, group_of_seq=p, logp_new=p, logp_old=p, logp_ref=p, adv=p, eps_low=0.2,
              eps_high=0.2, kl_coef=0.1, kl_estimator=2, coef=p, loss=p, workspace=p, workspace_bytes=1 << 30)
    for bad in (dict(eps_high=float("inf")), dict(eps_high=1e30), dict(dual_clip=1e30), dict(kl_coef=1e30)):
        d = acrl.PolicyLossDesc(**{**ok, **bad})
        assert L.acrl_policy_loss(ctypes.byref(d), None) == acrl.ACRL_ERR_INVALID_ARG and "1e30" in last(), bad
    d = acrl.PolicyLossDesc(**{**ok, "aggregate": 3, "norm": float("inf")})
    assert L.acrl_policy_loss(ctypes.byref(d), None) == acrl.ACRL_ERR_INVALID_ARG and "finite" in last()
    d = acrl.PreferenceDesc(B=2, L=4096, n_pairs=1, mask=p, logp_new=p, chosen=p, rejected=p, beta=1e30, coef=p, loss=p,
                            workspace=p, workspace_bytes=1 << 30)
    assert L.acrl_preference_loss(ctypes.byref(d), None) == acrl.ACRL_ERR_INVALID_ARG and "1e30" in last()
