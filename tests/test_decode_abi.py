"""Refusals of the operators of a decode step: out-of-contract calls return a
status before any HIP call, on the host and without a device."""
import ctypes

import pytest

from test_operators_abi import _off, acrl, p  # noqa: F401  (fixtures)


def test_descriptor_sizes(acrl):  # noqa: F811
    descs = (acrl.LinearDesc, acrl.MoeDesc, acrl.BeamDesc, acrl.ReorderDesc)
    sizes = [ctypes.c_size_t() for _ in descs]
    acrl.lib().acrl_abi_decode_struct_sizes(*[ctypes.byref(s) for s in sizes])
    assert [s.value for s in sizes] == [ctypes.sizeof(x) for x in descs]
    acrl.lib().acrl_abi_decode_struct_sizes(*[None] * len(descs))


def test_linear(acrl, p):  # noqa: F811
    L = acrl.lib()
    product = dict(M=4, N=64, K=256, xq=p, x_scales=p, wq=p, w_scales=p, y=p, ldy=64, y_type=0)
    ok = dict(bias=p, residual=_off(p, 2048), ldr=64)
    for bad in (dict(M=-1), dict(K=100), dict(ldy=63), dict(y=None), dict(wq=None), dict(y_type=2), dict(ldy=1 << 34)):
        d = acrl.LinearDesc(acrl.MatmulDesc(**{**product, **bad}), **ok)
        assert L.acrl_linear_fp8(ctypes.byref(d), None) == acrl.ACRL_ERR_INVALID_ARG, bad
    for bad in (dict(activation=-1), dict(activation=5), dict(bias_type=2), dict(bias=_off(p, 8)), dict(residual_type=3),
                dict(residual=_off(p, 2052)), dict(ldr=63), dict(ldr=-1), dict(ldr=1 << 34),
                # y is 4 rows of 128 bytes from p on
                dict(residual=_off(p, 16)), dict(residual=_off(p, 128)), dict(residual=_off(p, 496)),
                dict(residual=p, ldr=72), dict(residual=p, residual_type=1)):
        d = acrl.LinearDesc(acrl.MatmulDesc(**product), **{**ok, **bad})
        assert L.acrl_linear_fp8(ctypes.byref(d), None) == acrl.ACRL_ERR_INVALID_ARG, bad
        assert L.acrl_last_error()
    assert L.acrl_linear_fp8(None, None) == acrl.ACRL_ERR_INVALID_ARG


def test_moe(acrl, p):  # noqa: F811
    L, nb = acrl.lib(), ctypes.c_size_t()
    ok = dict(T=4, d=64, E=8, top_k=2, F=32, x=p, ldx=64, router=p, w_in=p, s_in=p, w_out=p, s_out=p, y=p, ldy=64,
              residual=_off(p, 2048), ldr=64, ids=p, weights=p, scale=1.0, workspace=p, workspace_bytes=1 << 30)
    sizes = [dict(T=-1), dict(T=129), dict(d=0), dict(d=48), dict(d=65568), dict(E=0), dict(E=513), dict(top_k=0), dict(top_k=9),
             dict(E=32, top_k=17), dict(F=0), dict(F=16), dict(F=65568)]
    for bad in sizes:
        s = {**ok, **bad}
        assert L.acrl_moe_workspace_size(*[s[n] for n in ("T", "d", "E", "top_k", "F")], ctypes.byref(nb)) == 1, bad
    for bad in sizes + [dict(score=-1), dict(score=2), dict(activation=5), dict(y_type=2), dict(residual_type=2),
                        dict(scale=float("inf")), dict(scale=float("nan")), dict(ldx=63), dict(ldx=68), dict(ldx=1 << 34),
                        dict(ldy=63), dict(ldy=1 << 34), dict(ldr=63), dict(ldr=1 << 34), dict(x=None), dict(w_in=None),
                        dict(s_in=None), dict(w_out=None), dict(s_out=None), dict(y=None), dict(ids=None), dict(weights=None),
                        dict(x=_off(p, 8)), dict(w_in=_off(p, 8)), dict(w_out=_off(p, 8)), dict(router=_off(p, 8)),
                        dict(s_in=_off(p, 2)), dict(s_out=_off(p, 2)), dict(select_bias=_off(p, 2)), dict(y=_off(p, 2)),
                        dict(ids=_off(p, 1)), dict(weights=_off(p, 2)), dict(residual=_off(p, 2050)), dict(residual=_off(p, 64)),
                        dict(residual=p, ldr=72), dict(workspace=_off(p, 8))]:
        d = acrl.MoeDesc(**{**ok, **bad})
        assert L.acrl_moe_fp8(ctypes.byref(d), None) == acrl.ACRL_ERR_INVALID_ARG, bad
        assert L.acrl_last_error()
    for bad in (dict(workspace=None), dict(workspace_bytes=100)):
        d = acrl.MoeDesc(**{**ok, **bad})
        assert L.acrl_moe_fp8(ctypes.byref(d), None) == acrl.ACRL_ERR_WORKSPACE, bad
    assert L.acrl_moe_fp8(None, None) == acrl.ACRL_ERR_INVALID_ARG
    assert L.acrl_moe_workspace_size(4, 64, 8, 2, 32, None) == acrl.ACRL_ERR_INVALID_ARG
    assert L.acrl_moe_workspace_size(0, 64, 8, 2, 32, ctypes.byref(nb)) == 0 and nb.value == 0
    assert L.acrl_moe_workspace_size(128, 65536, 512, 16, 65536, ctypes.byref(nb)) == 0 and nb.value > 2048 * 65536 * 8


def test_beam(acrl, p):  # noqa: F811
    L, nb = acrl.lib(), ctypes.c_size_t()
    ok = dict(B=2, K=3, V=1000, n_out=4, logits=p, ldl=1000, scores=p, finished=p, eos_id=5, inv_temperature=1.0, ids=p, parents=p,
              out_scores=p, workspace=p, workspace_bytes=1 << 30)
    sizes = [dict(B=-1), dict(B=(1 << 20) + 1), dict(K=0), dict(K=65), dict(B=1 << 19, K=8), dict(V=0), dict(V=1 << 30, ldl=1 << 30),
             dict(n_out=0), dict(n_out=65), dict(V=2, n_out=7)]
    for bad in sizes:
        s = {**ok, **bad}
        assert L.acrl_beam_workspace_size(*[s[n] for n in ("B", "K", "V", "n_out")], ctypes.byref(nb)) == 1, bad
    for bad in sizes + [dict(ldl=999), dict(ldl=1 << 34), dict(logits_type=2), dict(logits_type=-1), dict(eos_id=-1), dict(eos_id=1000),
                        dict(inv_temperature=0.0), dict(inv_temperature=-1.0), dict(inv_temperature=float("nan")),
                        dict(inv_temperature=float("inf")), dict(logits=None), dict(scores=None), dict(ids=None), dict(parents=None),
                        dict(out_scores=None), dict(logits=_off(p, 1)), dict(logits=_off(p, 2), logits_type=1), dict(scores=_off(p, 2)),
                        dict(ids=_off(p, 2)), dict(parents=_off(p, 1)), dict(out_scores=_off(p, 3)), dict(workspace=_off(p, 8))]:
        d = acrl.BeamDesc(**{**ok, **bad})
        assert L.acrl_beam_step(ctypes.byref(d), None) == acrl.ACRL_ERR_INVALID_ARG, bad
        assert L.acrl_last_error()
    for bad in (dict(workspace=None), dict(workspace_bytes=100)):
        d = acrl.BeamDesc(**{**ok, **bad})
        assert L.acrl_beam_step(ctypes.byref(d), None) == acrl.ACRL_ERR_WORKSPACE, bad
    assert L.acrl_beam_step(None, None) == acrl.ACRL_ERR_INVALID_ARG


def test_reorder(acrl, p):  # noqa: F811
    L = acrl.lib()
    ok = dict(outer=2, B=2, K=3, n_out=3, row_bytes=64, src=p, src_outer=384, src_seq=192, src_beam=64, dst=_off(p, 2048), dst_outer=384,
              dst_seq=192, dst_beam=64, parents=p)
    for bad in (dict(K=0), dict(K=65), dict(n_out=0), dict(n_out=65), dict(B=-1), dict(B=(1 << 20) + 1), dict(outer=-1),
                dict(outer=(1 << 20) + 1), dict(row_bytes=-1), dict(row_bytes=1 << 40), dict(src_beam=-64), dict(src_seq=1 << 42),
                dict(dst_outer=-1), dict(src=None), dict(dst=None), dict(parents=None), dict(parents=_off(p, 2)), dict(dst_beam=63),
                dict(dst_seq=0), dict(dst_outer=63), dict(dst=_off(p, 64)), dict(dst=p, dst_beam=128, dst_seq=384, dst_outer=768),
                dict(dst=p, n_out=2), dict(src=_off(p, 2048), dst=p, row_bytes=64, dst_outer=2048)):
        d = acrl.ReorderDesc(**{**ok, **bad})
        assert L.acrl_beam_reorder(ctypes.byref(d), None) == acrl.ACRL_ERR_INVALID_ARG, bad
        assert L.acrl_last_error()
    assert L.acrl_beam_reorder(None, None) == acrl.ACRL_ERR_INVALID_ARG


def test_binding_refuses_host_tensors(acrl):  # noqa: F811
    import torch
    q, s = torch.zeros((4, 128), dtype=torch.uint8), torch.ones((4, 1))
    with pytest.raises(ValueError, match="device tensor"):
        acrl.acrl_linear_fp8(q, s, q, s)
    x, w = torch.zeros((2, 32), dtype=torch.bfloat16), torch.zeros((1, 64, 32), dtype=torch.uint8)
    with pytest.raises(ValueError, match="device tensor"):
        acrl.acrl_moe_fp8(x, w, s[:1], w[:, :32], s[:1], 1, router=x[:1])
    z, i = torch.zeros((4, 8)), torch.zeros((2, 2), dtype=torch.int32)
    with pytest.raises(ValueError, match="device tensor"):
        acrl.acrl_beam_step(z, z[:2, :2], 2)
    with pytest.raises(ValueError, match="device tensor"):
        acrl.acrl_beam_reorder(z.view(2, 2, 8), i)
