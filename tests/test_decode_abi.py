"""Refusals of the operators of a decode step: out-of-contract calls return a
status before any HIP call, on the host and without a device."""
import ctypes

import pytest

from test_operators_abi import _off, acrl, p  # noqa: F401  (fixtures)


def test_descriptor_sizes(acrl):  # noqa: F811
    descs = (acrl.LinearDesc,)
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


def test_binding_refuses_host_tensors(acrl):  # noqa: F811
    import torch
    q, s = torch.zeros((4, 128), dtype=torch.uint8), torch.ones((4, 1))
    with pytest.raises(ValueError, match="device tensor"):
        acrl.acrl_linear_fp8(q, s, q, s)
