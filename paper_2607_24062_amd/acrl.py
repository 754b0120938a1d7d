"""Thin Python binding of libacrl (ctypes).

Every entry point of include/acrl.h is exposed under the same name; the
wrappers only marshal arguments (torch tensors supply device memory, the
current torch stream supplies the HIP stream).  All computation runs in the
library's HIP kernels.  If libacrl.so is missing or cannot be loaded, every
call raises: there is no fallback path.
"""
from __future__ import annotations

import ctypes
import functools
import math
import os
from typing import Dict, Optional

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libacrl.so")

ACRL_OK, ACRL_ERR_INVALID_ARG, ACRL_ERR_UNSUPPORTED, ACRL_ERR_WORKSPACE, ACRL_ERR_HIP = range(5)
SCALE_PER_TENSOR, SCALE_PER_ROW, SCALE_MX32, SCALE_ROW128, SCALE_BLOCK128 = 0, 1, 2, 3, 4
ROUND_NEAREST_EVEN, ROUND_TOWARD_ZERO = 0, 1
Y_GROUP, Y_SEQUENCE, Y_BATCH = 0, 1, 2
CTRL_ACRL, CTRL_TIS, CTRL_MIS, CTRL_CONTINUOUS, CTRL_FALLBACK = 0, 1, 2, 3, 4
POLICY_BOTH, POLICY_PI, POLICY_MU = 0, 1, 2
OUT_BF16, OUT_F32 = 0, 1
KL_K1, KL_K2, KL_K3 = 0, 1, 2
AGG_GROUP, AGG_SEQUENCE, AGG_TOKEN, AGG_CONSTANT = 0, 1, 2, 3
PREF_SIGMOID, PREF_HINGE, PREF_SQUARED = 0, 1, 2
MOE_SOFTMAX, MOE_SIGMOID = 0, 1
ACT_NONE, ACT_RELU, ACT_SILU, ACT_GELU, ACT_GELU_TANH = 0, 1, 2, 3, 4
N_STATS = 10
STAT_NAMES = ["y_batch", "tok_mean_d", "tok_max_d", "tok_std_d", "mean_h_pi", "mean_h_mu",
              "n_tokens", "n_groups", "tok_mean_logratio", "n_seqs"]
N_PSTATS = 6
PSTAT_NAMES = ["policy", "kl", "clipped", "dual", "moved", "n_tokens"]

EXPORTED = [
    "acrl_status_string", "acrl_last_error", "acrl_abi_version", "acrl_abi_struct_sizes",
    "acrl_quantize_workspace_size", "acrl_quantize_fp8", "acrl_fp8_encode",
    "acrl_score_workspace_size", "acrl_score_div_workspace_size", "acrl_score_workspace_query", "acrl_score_pi_mu",
    "acrl_packed_weights_size", "acrl_pack_weights",
    "acrl_reduce_workspace_size", "acrl_discrepancy_reduce", "acrl_discrepancy_reduce_noalloc",
    "acrl_controller_step", "acrl_reference_from_groups", "acrl_sample_mu",
    "acrl_surrogate_workspace_size", "acrl_surrogate",
    "acrl_backward_workspace_size", "acrl_lm_head_backward",
    "acrl_matmul_fp8", "acrl_policy_loss_workspace_size", "acrl_policy_loss",
    "acrl_preference_loss_workspace_size", "acrl_preference_loss", "acrl_abi_operator_struct_sizes",
    "acrl_linear_fp8", "acrl_moe_workspace_size", "acrl_moe_fp8", "acrl_beam_workspace_size",
    "acrl_beam_step", "acrl_beam_reorder", "acrl_abi_decode_struct_sizes",
]

_P = ctypes.c_void_p
_I64 = ctypes.c_int64
_I32 = ctypes.c_int32
_F32 = ctypes.c_float
_SZ = ctypes.c_size_t


class ScoreDesc(ctypes.Structure):
    _fields_ = [("n_rows", _I64), ("d", _I64), ("V", _I64),
                ("h", _P), ("w", _P), ("hq", _P), ("hq_scales", _P), ("wq", _P), ("wq_scales", _P),
                ("mu_scaling", _I32), ("inv_temperature", _F32),
                ("token_ids", _P), ("mask", _P), ("out_slot", _P),
                ("logp_pi", _P), ("logp_mu", _P), ("entropy_pi", _P), ("entropy_mu", _P),
                ("lse_pi", _P), ("lse_mu", _P), ("logit_pi", _P), ("logit_mu", _P),
                ("error_flag", _P), ("workspace", _P), ("workspace_bytes", _SZ),
                ("kl_pi_mu", _P), ("kl_mu_pi", _P), ("l2", _P), ("div_chunk", _I64),
                ("policies", _I32), ("packed_weights", _P), ("packed_weights_bytes", _SZ)]


class ReduceDesc(ctypes.Structure):
    _fields_ = [("B", _I64), ("L", _I64), ("n_groups", _I64),
                ("logp_pi", _P), ("logp_mu", _P), ("entropy_pi", _P), ("entropy_mu", _P),
                ("mask", _P), ("group_of_seq", _P),
                ("d_tok", _P), ("seq_len", _P), ("seq_sum_d", _P), ("seq_sum_logratio", _P),
                ("seq_mean_d", _P), ("group_y", _P), ("group_nseq", _P), ("stats", _P),
                ("workspace", _P), ("workspace_bytes", _SZ)]


class ControllerDesc(ctypes.Structure):
    _fields_ = [("B", _I64), ("L", _I64), ("n_groups", _I64),
                ("mask", _P), ("group_of_seq", _P), ("logp_pi", _P), ("logp_mu", _P),
                ("adv", _P), ("adv_per_token", _I32), ("y_level", _I32),
                ("seq_mean_d", _P), ("group_y", _P), ("stats", _P),
                ("X", _F32), ("gamma", _F32), ("C", _F32),
                ("alpha", _P), ("weight", _P), ("mode", _I32), ("k", _F32),
                ("seq_sum_logratio", _P)]


class SurrogateDesc(ctypes.Structure):
    _fields_ = [("B", _I64), ("L", _I64), ("n_groups", _I64),
                ("mask", _P), ("group_of_seq", _P), ("logp_new", _P), ("logp_old", _P),
                ("adv", _P), ("adv_per_token", _I32), ("eps_low", _F32), ("eps_high", _F32),
                ("weight", _P), ("coef", _P), ("loss", _P), ("workspace", _P), ("workspace_bytes", _SZ)]


class BackwardDesc(ctypes.Structure):
    _fields_ = [("n_rows", _I64), ("d", _I64), ("V", _I64), ("h", _P), ("w", _P),
                ("token_ids", _P), ("row_slot", _P), ("coef", _P), ("lse", _P),
                ("inv_temperature", _F32), ("dh", _P), ("dw", _P), ("accumulate_dw", _I32),
                ("token_chunk", _I64), ("workspace", _P), ("workspace_bytes", _SZ)]


class SampleDesc(ctypes.Structure):
    _fields_ = [("n_rows", _I64), ("d", _I64), ("V", _I64),
                ("hq", _P), ("hq_scales", _P), ("wq", _P), ("wq_scales", _P),
                ("mu_scaling", _I32), ("inv_temperature", _F32),
                ("seed", ctypes.c_uint64), ("row_offset", _I64),
                ("ids", _P), ("logp_mu", _P), ("workspace", _P), ("workspace_bytes", _SZ),
                ("packed_weights", _P), ("packed_weights_bytes", _SZ)]


class MatmulDesc(ctypes.Structure):
    _fields_ = [("M", _I64), ("N", _I64), ("K", _I64), ("xq", _P), ("x_scales", _P), ("wq", _P), ("w_scales", _P),
                ("y", _P), ("ldy", _I64), ("y_type", _I32)]


class LinearDesc(ctypes.Structure):
    _fields_ = [("product", MatmulDesc), ("bias", _P), ("residual", _P), ("ldr", _I64), ("bias_type", _I32),
                ("residual_type", _I32), ("activation", _I32)]


class MoeDesc(ctypes.Structure):
    _fields_ = [("T", _I64), ("d", _I64), ("E", _I64), ("top_k", _I64), ("F", _I64), ("x", _P), ("ldx", _I64),
                ("router", _P), ("select_bias", _P), ("mask", _P), ("w_in", _P), ("s_in", _P), ("w_out", _P), ("s_out", _P),
                ("residual", _P), ("ldr", _I64), ("y", _P), ("ldy", _I64), ("ids", _P), ("weights", _P),
                ("residual_type", _I32), ("y_type", _I32), ("score", _I32), ("renormalize", _I32), ("activation", _I32),
                ("scale", _F32), ("workspace", _P), ("workspace_bytes", _SZ)]


class BeamDesc(ctypes.Structure):
    _fields_ = [("B", _I64), ("K", _I64), ("V", _I64), ("n_out", _I64), ("logits", _P), ("ldl", _I64), ("scores", _P),
                ("finished", _P), ("logits_type", _I32), ("eos_id", _I32), ("inv_temperature", _F32), ("ids", _P),
                ("parents", _P), ("out_scores", _P), ("workspace", _P), ("workspace_bytes", _SZ)]


class ReorderDesc(ctypes.Structure):
    _fields_ = [("outer", _I64), ("B", _I64), ("K", _I64), ("n_out", _I64), ("row_bytes", _I64), ("src", _P),
                ("src_outer", _I64), ("src_seq", _I64), ("src_beam", _I64), ("dst", _P), ("dst_outer", _I64),
                ("dst_seq", _I64), ("dst_beam", _I64), ("parents", _P)]


class PolicyLossDesc(ctypes.Structure):
    _fields_ = [("B", _I64), ("L", _I64), ("n_groups", _I64), ("mask", _P), ("group_of_seq", _P),
                ("logp_new", _P), ("logp_old", _P), ("logp_ref", _P), ("adv", _P), ("weight", _P),
                ("adv_per_token", _I32), ("kl_estimator", _I32), ("aggregate", _I32),
                ("eps_low", _F32), ("eps_high", _F32), ("dual_clip", _F32), ("kl_coef", _F32), ("norm", _F32),
                ("coef", _P), ("loss", _P), ("stats", _P), ("workspace", _P), ("workspace_bytes", _SZ)]


class PreferenceDesc(ctypes.Structure):
    _fields_ = [("B", _I64), ("L", _I64), ("n_pairs", _I64), ("mask", _P), ("logp_new", _P), ("logp_ref", _P),
                ("chosen", _P), ("rejected", _P), ("pair_weight", _P), ("form", _I32), ("mean_logp", _I32),
                ("beta", _F32), ("margin", _F32), ("label_smoothing", _F32),
                ("coef", _P), ("loss", _P), ("rewards", _P), ("workspace", _P), ("workspace_bytes", _SZ)]


class AcrlError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str):
        super().__init__("%s failed: %s (%s)" % (where, _status_names.get(status, status), detail))
        self.status = status


_status_names = {0: "ok", 1: "invalid argument", 2: "unsupported", 3: "workspace too small",
                 4: "HIP runtime error"}

_lib: Optional[ctypes.CDLL] = None


def lib() -> ctypes.CDLL:
    """Load libacrl.so (built in-tree by paper_2607_24062_amd.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libacrl.so is not built (%s); run python -m paper_2607_24062_amd.build"
                               % LIB_PATH)
        L = ctypes.CDLL(LIB_PATH)
        L.acrl_status_string.restype = ctypes.c_char_p
        L.acrl_status_string.argtypes = [_I32]
        L.acrl_last_error.restype = ctypes.c_char_p
        L.acrl_last_error.argtypes = []
        L.acrl_abi_version.restype = _I32
        L.acrl_abi_struct_sizes.restype = None
        L.acrl_abi_struct_sizes.argtypes = [ctypes.POINTER(_SZ)] * 6
        L.acrl_quantize_workspace_size.restype = _I32
        L.acrl_quantize_workspace_size.argtypes = [_I64, _I64, _I32, ctypes.POINTER(_SZ)]
        L.acrl_quantize_fp8.restype = _I32
        L.acrl_quantize_fp8.argtypes = [_P, _I64, _I64, _I64, _I32, _I32, _P, _P, _P, _SZ, _P]
        L.acrl_fp8_encode.restype = _I32
        L.acrl_fp8_encode.argtypes = [_P, _I64, _I32, _P, _P]
        L.acrl_score_workspace_size.restype = _I32
        L.acrl_score_workspace_size.argtypes = [_I64, _I64, _I64, _I32, ctypes.POINTER(_SZ)]
        L.acrl_score_div_workspace_size.restype = _I32
        L.acrl_score_div_workspace_size.argtypes = [_I64, _I64, _I64, _I32, _I64, ctypes.POINTER(_SZ)]
        L.acrl_score_pi_mu.restype = _I32
        L.acrl_score_pi_mu.argtypes = [ctypes.POINTER(ScoreDesc), _P]
        L.acrl_score_workspace_query.restype = _I32
        L.acrl_score_workspace_query.argtypes = [ctypes.POINTER(ScoreDesc), ctypes.POINTER(_SZ)]
        L.acrl_packed_weights_size.restype = _I32
        L.acrl_packed_weights_size.argtypes = [_I64, _I64, _I32, ctypes.POINTER(_SZ)]
        L.acrl_pack_weights.restype = _I32
        L.acrl_pack_weights.argtypes = [_P, _P, _P, _I64, _I64, _I32, _P, _SZ, _P]
        L.acrl_reduce_workspace_size.restype = _I32
        L.acrl_reduce_workspace_size.argtypes = [_I64, _I64, _I64, ctypes.POINTER(_SZ)]
        L.acrl_discrepancy_reduce.restype = _I32
        L.acrl_discrepancy_reduce.argtypes = [ctypes.POINTER(ReduceDesc), _P]
        L.acrl_discrepancy_reduce_noalloc.restype = _I32
        L.acrl_discrepancy_reduce_noalloc.argtypes = [ctypes.POINTER(ReduceDesc), _P]
        L.acrl_controller_step.restype = _I32
        L.acrl_controller_step.argtypes = [ctypes.POINTER(ControllerDesc), _P]
        L.acrl_reference_from_groups.restype = _I32
        L.acrl_reference_from_groups.argtypes = [_P, _P, _I64, ctypes.POINTER(_F32)]
        L.acrl_sample_mu.restype = _I32
        L.acrl_sample_mu.argtypes = [ctypes.POINTER(SampleDesc), _P]
        L.acrl_surrogate_workspace_size.restype = _I32
        L.acrl_surrogate_workspace_size.argtypes = [_I64, _I64, ctypes.POINTER(_SZ)]
        L.acrl_surrogate.restype = _I32
        L.acrl_surrogate.argtypes = [ctypes.POINTER(SurrogateDesc), _P]
        L.acrl_backward_workspace_size.restype = _I32
        L.acrl_backward_workspace_size.argtypes = [_I64, _I64, _I64, _I64, ctypes.POINTER(_SZ)]
        L.acrl_lm_head_backward.restype = _I32
        L.acrl_lm_head_backward.argtypes = [ctypes.POINTER(BackwardDesc), _P]
        L.acrl_matmul_fp8.restype = _I32
        L.acrl_matmul_fp8.argtypes = [ctypes.POINTER(MatmulDesc), _P]
        L.acrl_policy_loss_workspace_size.restype = _I32
        L.acrl_policy_loss_workspace_size.argtypes = [_I64, _I64, _I64, ctypes.POINTER(_SZ)]
        L.acrl_policy_loss.restype = _I32
        L.acrl_policy_loss.argtypes = [ctypes.POINTER(PolicyLossDesc), _P]
        L.acrl_preference_loss_workspace_size.restype = _I32
        L.acrl_preference_loss_workspace_size.argtypes = [_I64, _I64, _I64, ctypes.POINTER(_SZ)]
        L.acrl_preference_loss.restype = _I32
        L.acrl_preference_loss.argtypes = [ctypes.POINTER(PreferenceDesc), _P]
        L.acrl_abi_operator_struct_sizes.restype = None
        L.acrl_abi_operator_struct_sizes.argtypes = [ctypes.POINTER(_SZ)] * 3
        L.acrl_linear_fp8.restype = _I32
        L.acrl_linear_fp8.argtypes = [ctypes.POINTER(LinearDesc), _P]
        L.acrl_abi_decode_struct_sizes.restype = None
        L.acrl_abi_decode_struct_sizes.argtypes = [ctypes.POINTER(_SZ)] * 4
        L.acrl_beam_workspace_size.restype = _I32
        L.acrl_beam_workspace_size.argtypes = [_I64] * 4 + [ctypes.POINTER(_SZ)]
        L.acrl_beam_step.restype = _I32
        L.acrl_beam_step.argtypes = [ctypes.POINTER(BeamDesc), _P]
        L.acrl_beam_reorder.restype = _I32
        L.acrl_beam_reorder.argtypes = [ctypes.POINTER(ReorderDesc), _P]
        L.acrl_moe_workspace_size.restype = _I32
        L.acrl_moe_workspace_size.argtypes = [_I64] * 5 + [ctypes.POINTER(_SZ)]
        L.acrl_moe_fp8.restype = _I32
        L.acrl_moe_fp8.argtypes = [ctypes.POINTER(MoeDesc), _P]
        sizes = [_SZ() for _ in range(13)]
        L.acrl_abi_struct_sizes(*[ctypes.byref(s) for s in sizes[:6]])
        L.acrl_abi_operator_struct_sizes(*[ctypes.byref(s) for s in sizes[6:9]])
        L.acrl_abi_decode_struct_sizes(*[ctypes.byref(s) for s in sizes[9:]])
        want = [ctypes.sizeof(ScoreDesc), ctypes.sizeof(ReduceDesc), ctypes.sizeof(ControllerDesc),
                ctypes.sizeof(SampleDesc), ctypes.sizeof(SurrogateDesc), ctypes.sizeof(BackwardDesc),
                ctypes.sizeof(MatmulDesc), ctypes.sizeof(PolicyLossDesc), ctypes.sizeof(PreferenceDesc),
                ctypes.sizeof(LinearDesc), ctypes.sizeof(MoeDesc), ctypes.sizeof(BeamDesc), ctypes.sizeof(ReorderDesc)]
        got = [s.value for s in sizes]
        if got != want:
            raise RuntimeError("libacrl descriptor layout mismatch: library %s, binding %s" % (got, want))
        _lib = L
    return _lib


def _check(status: int, where: str) -> None:
    if status != ACRL_OK:
        raise AcrlError(status, where, lib().acrl_last_error().decode(errors="replace"))


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


# the current stream's handle alone, where torch has it: making its Stream
# object takes 2.7 us, twice per call, and the handle 0.1
_current_raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
# likewise the current device's index, once there is a device tensor
_current_index = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_zero_all = getattr(torch, "_foreach_zero_", None)


def _raw_stream(stream=None, device=None) -> int:
    """The HIP stream of `stream`, or the current one of `device` (None: of
    the current device)."""
    if stream is not None:
        return stream.cuda_stream
    index = torch.cuda.current_device() if device is None else device.index
    if _current_raw is None or index is None:
        return torch.cuda.current_stream(device).cuda_stream  # (raises on other devices)
    return _current_raw(index)


def _zero(tensors) -> None:
    """Clear device tensors, by one launch where torch can."""
    if _zero_all is not None:
        _zero_all(tensors)
    else:
        for t in tensors:
            t.zero_()


def _stream(stream=None):
    return ctypes.c_void_p(_raw_stream(stream))


def _dev(t: torch.Tensor, dtype, name: str):
    if not t.is_cuda:
        raise ValueError("%s must be a device tensor" % name)
    if t.dtype != dtype:
        raise ValueError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    return t


def _want(t, dtype, numel: int, index: int, name: str, optional: bool = False):
    """Device address of a contiguous tensor of numel elements on device
    `index`.  (A call takes up to ten of them: the checks are one expression,
    0.4 us each, and the reason is found afterwards.)"""
    if t is None and optional:
        return None
    if t is None or t.dtype is not dtype or t.get_device() != index or t.numel() != numel or not t.is_contiguous():
        if t is None:
            raise ValueError("%s is required" % name)
        _dev(t, dtype, name)
        if t.get_device() != index:
            raise ValueError("%s is on %s, not on cuda:%d" % (name, t.device, index))
        raise ValueError("%s must have %d elements, got %d" % (name, numel, t.numel()))
    return t.data_ptr()


def _index_of(t, dtype, name: str, stream=None) -> int:
    """The device index of a device tensor, which is to be the current one (the
    library launches there) and the stream's."""
    index = t.get_device()
    if index < 0 or t.dtype is not dtype or not t.is_contiguous():
        _dev(t, dtype, name)
    if stream is not None and stream.device_index != index:
        raise ValueError("%s is on cuda:%d, the stream belongs to cuda:%d" % (name, index, stream.device_index))
    if index != _current_index():
        raise ValueError("%s is on cuda:%d, the current device is cuda:%d" % (name, index, _current_index()))
    return index


def _raw_of(stream, index: int) -> int:
    """The HIP stream of `stream`, or the current one of the device `index`."""
    if stream is not None or _current_raw is None:
        return _raw_stream(stream, torch.device("cuda", index))
    return _current_raw(index)


@functools.lru_cache(maxsize=256)
def _size(query: str, *sizes) -> int:
    """Workspace bytes by a library query of plain sizes."""
    nb = _SZ()
    _check(getattr(lib(), query)(*sizes, ctypes.byref(nb)), query)
    return nb.value


def _empty(shape, dtype, device, stream=None):
    """A fresh device tensor that belongs to the stream the call runs on.
    Outputs and workspaces of a captured call then live in its graph's memory:
    graphs share none, and nothing else takes it while the graph lives."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


_ws_cache: Dict[tuple, torch.Tensor] = {}


def _workspace(nbytes: int, device, stream=None) -> torch.Tensor:
    """A cached device byte buffer of at least nbytes for calls on `stream`
    (the current stream if None), grown on demand.  One buffer per (device,
    stream): calls on one stream run in order, so they may share it, and a
    buffer is allocated on the stream that uses it, so torch's allocator
    recycles a replaced one only after that stream's earlier work."""
    key = (device, _raw_stream(stream, device))
    buf = _ws_cache.get(key)
    if buf is None or buf.numel() < nbytes:
        s = stream if stream is not None else torch.cuda.current_stream(device)
        _ws_cache.pop(key, None)
        with torch.cuda.stream(s):
            buf = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)
        _ws_cache[key] = buf
    return buf


# ------------------------------------------------------------------ a1/a2
def acrl_quantize_fp8(x: torch.Tensor, scaling: int, rounding: int = ROUND_NEAREST_EVEN,
                      q: Optional[torch.Tensor] = None, scales: Optional[torch.Tensor] = None,
                      stream=None):
    """x: bf16 [rows, cols] -> (q uint8 [rows, cols], scales).  x may be a
    column slice of a wider matrix (unit column stride, row stride = ld)."""
    if x.dim() != 2:
        raise ValueError("x must be 2-D")
    rows, cols = x.shape
    if x.is_contiguous():
        _dev(x, torch.bfloat16, "x")
        ld = cols
    else:
        if not x.is_cuda or x.dtype != torch.bfloat16 or x.stride(1) != 1 or x.stride(0) < cols:
            raise ValueError("x must be a bf16 device matrix with unit column stride")
        ld = x.stride(0)
    if scaling == SCALE_ROW128 or scaling == SCALE_BLOCK128:
        return _quantize_blocks(x, rows, cols, ld, scaling, rounding, q, scales, stream)
    if q is None:
        q = torch.empty((rows, cols), dtype=torch.uint8, device=x.device)
    if scales is None:
        if scaling == SCALE_PER_TENSOR:
            scales = torch.empty(1, dtype=torch.float32, device=x.device)
        elif scaling == SCALE_PER_ROW:
            scales = torch.empty(rows, dtype=torch.float32, device=x.device)
        else:
            scales = torch.empty((rows, cols // 32), dtype=torch.uint8, device=x.device)
    nbytes = _size("acrl_quantize_workspace_size", rows, cols, scaling)
    ws = _workspace(nbytes, x.device, stream) if nbytes else None
    _check(lib().acrl_quantize_fp8(x.data_ptr(), rows, cols, ld, scaling, rounding, q.data_ptr(), scales.data_ptr(),
                                   _ptr(ws), nbytes, _raw_stream(stream)), "acrl_quantize_fp8")
    return q, scales


def _room(t, dtype, numel: int, index: int, name: str):
    if t.dtype is not dtype or t.get_device() != index or t.numel() < numel or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor of %d elements or more on cuda:%d" % (name, dtype, numel, index))


def _quantize_blocks(x, rows: int, cols: int, ld: int, scaling: int, rounding: int, q, scales, stream):
    """ROW128 and BLOCK128: outputs and stream as for acrl_matmul_fp8."""
    index, groups = x.get_device(), (cols + 127) // 128
    if index != torch.cuda.current_device() or (stream is not None and stream.device_index != index):
        raise ValueError("x is on %s, not on the current device or the stream's" % x.device)
    n = rows if scaling == SCALE_ROW128 else (rows + 127) // 128
    if q is None:
        q = _empty((rows, cols), torch.uint8, x.device, stream)
    else:
        _room(q, torch.uint8, rows * cols, index, "q")
    if scales is None:
        scales = _empty((n, groups), torch.float32, x.device, stream)
    else:
        _room(scales, torch.float32, n * groups, index, "scales")
    _check(lib().acrl_quantize_fp8(x.data_ptr(), rows, cols, ld, scaling, rounding, q.data_ptr(), scales.data_ptr(),
                                   None, 0, _raw_stream(stream, x.device)), "acrl_quantize_fp8")
    return q, scales


def acrl_fp8_encode(x: torch.Tensor, rounding: int = ROUND_NEAREST_EVEN, q=None, stream=None):
    _dev(x, torch.float32, "x")
    if q is None:
        q = torch.empty(x.shape, dtype=torch.uint8, device=x.device)
    _check(lib().acrl_fp8_encode(_ptr(x), x.numel(), rounding, _ptr(q), _stream(stream)),
           "acrl_fp8_encode")
    return q


# ------------------------------------------------------------------ a3..a5
def acrl_pack_weights(w, wq, wq_scales, mu_scaling: int, packed=None, stream=None):
    """The tiled copy of W and Wq (and Wq's MX scales) the scorers stream
    from, once per weight version; returns the uint8 device buffer to pass
    as packed_weights."""
    _dev(w, torch.bfloat16, "w")
    _dev(wq, torch.uint8, "wq")
    V, d = w.shape
    nb = _SZ()
    _check(lib().acrl_packed_weights_size(V, d, mu_scaling, ctypes.byref(nb)), "acrl_packed_weights_size")
    if packed is None:
        packed = torch.empty(nb.value, dtype=torch.uint8, device=w.device)
    _check(lib().acrl_pack_weights(_ptr(w), _ptr(wq), _ptr(wq_scales), V, d, mu_scaling, _ptr(packed),
                                   packed.numel(), _stream(stream)), "acrl_pack_weights")
    return packed


def acrl_score_pi_mu(h, w, hq, hq_scales, wq, wq_scales, mu_scaling: int, token_ids,
                     inv_temperature: float = 1.0, mask=None, out_slot=None, n_slots=None,
                     outputs: Optional[dict] = None, want=("entropy", "lse", "logit"),
                     error_flag=None, stream=None, divergence: bool = False, div_chunk: int = 0,
                     policies: int = POLICY_BOTH, packed_weights=None) -> dict:
    """Score every row of h under pi (bf16) and mu (fp8/mxfp8).

    Returns a dict of float32 [n_slots] tensors: logp_pi, logp_mu and, per
    `want`, entropy_pi/mu, lse_pi/mu, logit_pi/mu; with divergence=True also
    the full-vocabulary kl_pi_mu, kl_mu_pi and l2.  Pass `outputs` to reuse
    preallocated tensors.  policies = POLICY_PI / POLICY_MU scores one
    policy only (the other's outputs are left untouched); packed_weights is
    the buffer acrl_pack_weights returned for these w, wq."""
    _dev(h, torch.bfloat16, "h")
    _dev(w, torch.bfloat16, "w")
    _dev(hq, torch.uint8, "hq")
    _dev(wq, torch.uint8, "wq")
    _dev(token_ids, torch.int32, "token_ids")
    n_rows, d = h.shape
    V = w.shape[0]
    if n_slots is None:
        n_slots = n_rows
    dev = h.device
    out = {} if outputs is None else dict(outputs)
    names = ["logp_pi", "logp_mu"]
    for k in want:
        names += [k + "_pi", k + "_mu"]
    if divergence:
        names += ["kl_pi_mu", "kl_mu_pi", "l2"]
    # The call writes every slot of the policies it scores when there is one per
    # row; other slots read 0, cleared by one launch (8 of 3 us GPU time and 5 us
    # host time each before: 20 us of 490 for 133 rows, d = 4096).
    unscored = {POLICY_PI: "_mu", POLICY_MU: "_pi"}.get(policies)
    clear = []
    for k in names:
        if k not in out:
            out[k] = torch.empty(n_slots, dtype=torch.float32, device=dev)
            if out_slot is not None or n_slots != n_rows or (unscored and k.endswith(unscored)):
                clear.append(out[k])
    if clear:
        _zero(clear)
    desc = ScoreDesc(n_rows=n_rows, d=d, V=V, h=_ptr(h), w=_ptr(w), hq=_ptr(hq),
                     hq_scales=_ptr(hq_scales), wq=_ptr(wq), wq_scales=_ptr(wq_scales),
                     mu_scaling=mu_scaling, inv_temperature=float(inv_temperature),
                     token_ids=_ptr(token_ids), mask=_ptr(mask), out_slot=_ptr(out_slot),
                     logp_pi=_ptr(out["logp_pi"]), logp_mu=_ptr(out["logp_mu"]),
                     entropy_pi=_ptr(out.get("entropy_pi")), entropy_mu=_ptr(out.get("entropy_mu")),
                     lse_pi=_ptr(out.get("lse_pi")), lse_mu=_ptr(out.get("lse_mu")),
                     logit_pi=_ptr(out.get("logit_pi")), logit_mu=_ptr(out.get("logit_mu")),
                     error_flag=_ptr(error_flag),
                     kl_pi_mu=_ptr(out.get("kl_pi_mu") if divergence else None),
                     kl_mu_pi=_ptr(out.get("kl_mu_pi") if divergence else None),
                     l2=_ptr(out.get("l2") if divergence else None), div_chunk=int(div_chunk),
                     policies=int(policies), packed_weights=_ptr(packed_weights),
                     packed_weights_bytes=0 if packed_weights is None else packed_weights.numel())
    nb = _SZ()
    _check(lib().acrl_score_workspace_query(ctypes.byref(desc), ctypes.byref(nb)), "acrl_score_workspace_query")
    ws = _workspace(nb.value, dev, stream)
    desc.workspace, desc.workspace_bytes = _ptr(ws), nb.value
    _check(lib().acrl_score_pi_mu(ctypes.byref(desc), _stream(stream)), "acrl_score_pi_mu")
    return out


def acrl_sample_mu(hq, hq_scales, wq, wq_scales, mu_scaling: int, seed: int, row_offset: int = 0,
                   inv_temperature: float = 1.0, ids=None, logp_mu=None, want_logp: bool = True,
                   stream=None, packed_weights=None):
    """Draw one token per row of hq from mu (Gumbel-max in the mu kernel).

    Returns (ids int32 [n_rows], logp_mu float32 [n_rows] or None)."""
    _dev(hq, torch.uint8, "hq")
    _dev(wq, torch.uint8, "wq")
    n_rows, d = hq.shape
    V = wq.shape[0]
    dev = hq.device
    if ids is None:
        ids = torch.empty(n_rows, dtype=torch.int32, device=dev)
    if logp_mu is None and want_logp:
        logp_mu = torch.empty(n_rows, dtype=torch.float32, device=dev)
    nb = _SZ()
    probe = ScoreDesc(n_rows=n_rows, d=d, V=V, mu_scaling=mu_scaling, packed_weights=_ptr(packed_weights))
    _check(lib().acrl_score_workspace_query(ctypes.byref(probe), ctypes.byref(nb)), "acrl_score_workspace_query")
    ws = _workspace(nb.value, dev, stream)
    desc = SampleDesc(n_rows=n_rows, d=d, V=V, hq=_ptr(hq), hq_scales=_ptr(hq_scales), wq=_ptr(wq),
                      wq_scales=_ptr(wq_scales), mu_scaling=mu_scaling,
                      inv_temperature=float(inv_temperature), seed=int(seed) & (2 ** 64 - 1),
                      row_offset=int(row_offset), ids=_ptr(ids), logp_mu=_ptr(logp_mu),
                      workspace=_ptr(ws), workspace_bytes=nb.value, packed_weights=_ptr(packed_weights),
                      packed_weights_bytes=0 if packed_weights is None else packed_weights.numel())
    _check(lib().acrl_sample_mu(ctypes.byref(desc), _stream(stream)), "acrl_sample_mu")
    return ids, logp_mu


# ------------------------------------------------------------------ a6/a7
def _reduce(fn_name: str, B: int, L: int, n_groups: int, logp_pi, logp_mu, mask, group_of_seq,
            entropy_pi, entropy_mu, want_d_tok: bool, stream, use_workspace: bool, out=None) -> dict:
    dev = logp_pi.device
    if out is None:
        out = dict(
            d_tok=torch.empty(B * L, dtype=torch.float32, device=dev) if want_d_tok else None,
            seq_len=torch.empty(B, dtype=torch.int32, device=dev),
            seq_sum_d=torch.empty(B, dtype=torch.float64, device=dev),
            seq_sum_logratio=torch.empty(B, dtype=torch.float64, device=dev),
            seq_mean_d=torch.empty(B, dtype=torch.float32, device=dev),
            group_y=torch.empty(n_groups, dtype=torch.float32, device=dev),
            group_nseq=torch.empty(n_groups, dtype=torch.int32, device=dev),
            stats=torch.empty(N_STATS, dtype=torch.float64, device=dev),
        )
    ws = None
    nbytes = 0
    if use_workspace:
        nb = _SZ()
        _check(lib().acrl_reduce_workspace_size(B, L, n_groups, ctypes.byref(nb)), "acrl_reduce_workspace_size")
        ws = _workspace(nb.value, dev, stream)
        nbytes = nb.value
    desc = ReduceDesc(B=B, L=L, n_groups=n_groups, logp_pi=_ptr(logp_pi), logp_mu=_ptr(logp_mu),
                      entropy_pi=_ptr(entropy_pi), entropy_mu=_ptr(entropy_mu), mask=_ptr(mask),
                      group_of_seq=_ptr(group_of_seq), d_tok=_ptr(out["d_tok"]),
                      seq_len=_ptr(out["seq_len"]), seq_sum_d=_ptr(out["seq_sum_d"]),
                      seq_sum_logratio=_ptr(out["seq_sum_logratio"]), seq_mean_d=_ptr(out["seq_mean_d"]),
                      group_y=_ptr(out["group_y"]), group_nseq=_ptr(out["group_nseq"]),
                      stats=_ptr(out["stats"]), workspace=_ptr(ws), workspace_bytes=nbytes)
    _check(getattr(lib(), fn_name)(ctypes.byref(desc), _stream(stream)), fn_name)
    return out


def acrl_discrepancy_reduce(B: int, L: int, n_groups: int, logp_pi, logp_mu, mask, group_of_seq,
                            entropy_pi=None, entropy_mu=None, want_d_tok: bool = True,
                            stream=None) -> dict:
    """Per-token d, per-response / per-group / batch reductions (a6/a7).
    Returns a dict of device tensors (d_tok, seq_len, seq_sum_d,
    seq_sum_logratio, seq_mean_d, group_y, group_nseq, stats)."""
    return _reduce("acrl_discrepancy_reduce", B, L, n_groups, logp_pi, logp_mu, mask, group_of_seq,
                   entropy_pi, entropy_mu, want_d_tok, stream, True)


def acrl_discrepancy_reduce_noalloc(B: int, L: int, n_groups: int, logp_pi, logp_mu, mask, group_of_seq,
                                    entropy_pi=None, entropy_mu=None, want_d_tok: bool = True,
                                    stream=None, out: Optional[dict] = None) -> dict:
    """The same reduce on the library's fixed per-device scratch (no
    workspace).  With `out` (a dict of preallocated output tensors as
    acrl_discrepancy_reduce returns) nothing is allocated on this path."""
    return _reduce("acrl_discrepancy_reduce_noalloc", B, L, n_groups, logp_pi, logp_mu, mask, group_of_seq,
                   entropy_pi, entropy_mu, want_d_tok, stream, False, out)


# ------------------------------------------------------------------ a8
def acrl_controller_step(B: int, L: int, n_groups: int, mask, group_of_seq, logp_pi, logp_mu, adv,
                         adv_per_token: bool, y_level: int, seq_mean_d, group_y, stats,
                         X: float, gamma: float, C: float, want_alpha: bool = True, stream=None,
                         mode: int = 0, k: float = 1.0, seq_sum_logratio=None):
    dev = logp_pi.device
    alpha = torch.empty(B * L, dtype=torch.float32, device=dev) if want_alpha else None
    weight = torch.empty(B * L, dtype=torch.float32, device=dev)
    desc = ControllerDesc(B=B, L=L, n_groups=n_groups, mask=_ptr(mask), group_of_seq=_ptr(group_of_seq),
                          logp_pi=_ptr(logp_pi), logp_mu=_ptr(logp_mu), adv=_ptr(adv),
                          adv_per_token=int(bool(adv_per_token)), y_level=y_level,
                          seq_mean_d=_ptr(seq_mean_d), group_y=_ptr(group_y), stats=_ptr(stats),
                          X=float(X), gamma=float(gamma), C=float(C), alpha=_ptr(alpha),
                          weight=_ptr(weight), mode=int(mode), k=float(k),
                          seq_sum_logratio=_ptr(seq_sum_logratio))
    _check(lib().acrl_controller_step(ctypes.byref(desc), _stream(stream)), "acrl_controller_step")
    return alpha, weight


def acrl_reference_from_groups(group_y, group_nseq) -> float:
    """Host helper: X = mean of Y_g over non-empty groups (host arrays)."""
    import numpy as np
    gy = np.ascontiguousarray(group_y, np.float32)
    gn = np.ascontiguousarray(group_nseq, np.int32)
    X = _F32()
    _check(lib().acrl_reference_from_groups(gy.ctypes.data_as(_P), gn.ctypes.data_as(_P), gy.size,
                                            ctypes.byref(X)), "acrl_reference_from_groups")
    return float(X.value)


# ------------------------------------------------------------------ surrogate and its backward
def acrl_surrogate(B: int, L: int, n_groups: int, mask, group_of_seq, logp_new, logp_old, adv,
                   adv_per_token: bool, eps_low: float = 0.2, eps_high: float = 0.2, weight=None,
                   coef=None, stream=None):
    """ACRL-weighted clipped surrogate: returns (coef float32 [B*L], loss float64 [1])."""
    dev = logp_new.device
    if coef is None:
        coef = torch.empty(B * L, dtype=torch.float32, device=dev)
    loss = torch.empty(1, dtype=torch.float64, device=dev)
    nb = _SZ()
    _check(lib().acrl_surrogate_workspace_size(B, n_groups, ctypes.byref(nb)), "acrl_surrogate_workspace_size")
    ws = _workspace(nb.value, dev, stream)
    desc = SurrogateDesc(B=B, L=L, n_groups=n_groups, mask=_ptr(mask), group_of_seq=_ptr(group_of_seq),
                         logp_new=_ptr(logp_new), logp_old=_ptr(logp_old), adv=_ptr(adv),
                         adv_per_token=int(bool(adv_per_token)), eps_low=float(eps_low),
                         eps_high=float(eps_high), weight=_ptr(weight), coef=_ptr(coef), loss=_ptr(loss),
                         workspace=_ptr(ws), workspace_bytes=nb.value)
    _check(lib().acrl_surrogate(ctypes.byref(desc), _stream(stream)), "acrl_surrogate")
    return coef, loss


def acrl_lm_head_backward(h, w, token_ids, coef, lse, inv_temperature: float = 1.0, row_slot=None,
                          want_dh: bool = True, want_dw: bool = True, dh=None, dw=None,
                          accumulate_dw: bool = False, token_chunk: int = 0, stream=None):
    """Gradient of the surrogate w.r.t. h [n_rows, d] and w [V, d] (bf16):
    returns (dh float32 [n_rows, d] or None, dw float32 [V, d] or None)."""
    _dev(h, torch.bfloat16, "h")
    _dev(w, torch.bfloat16, "w")
    _dev(token_ids, torch.int32, "token_ids")
    _dev(coef, torch.float32, "coef")
    _dev(lse, torch.float32, "lse")
    n_rows, d = h.shape
    V = w.shape[0]
    dev = h.device
    if want_dh and dh is None:
        dh = torch.empty((n_rows, d), dtype=torch.float32, device=dev)
    if want_dw and dw is None:
        dw = torch.empty((V, d), dtype=torch.float32, device=dev)
    nb = _SZ()
    _check(lib().acrl_backward_workspace_size(n_rows, d, V, int(token_chunk), ctypes.byref(nb)),
           "acrl_backward_workspace_size")
    ws = _workspace(nb.value, dev, stream)
    desc = BackwardDesc(n_rows=n_rows, d=d, V=V, h=_ptr(h), w=_ptr(w), token_ids=_ptr(token_ids),
                        row_slot=_ptr(row_slot), coef=_ptr(coef), lse=_ptr(lse),
                        inv_temperature=float(inv_temperature), dh=_ptr(dh if want_dh else None),
                        dw=_ptr(dw if want_dw else None), accumulate_dw=int(bool(accumulate_dw)),
                        token_chunk=int(token_chunk), workspace=_ptr(ws), workspace_bytes=nb.value)
    _check(lib().acrl_lm_head_backward(ctypes.byref(desc), _stream(stream)), "acrl_lm_head_backward")
    return (dh if want_dh else None), (dw if want_dw else None)


# ------------------------------------------------------------------ block-scaled FP8 product
_OUT_TYPES = {torch.bfloat16: OUT_BF16, torch.float32: OUT_F32}


def acrl_matmul_fp8(xq, x_scales, wq, w_scales, out=None, out_dtype=torch.bfloat16, stream=None):
    """y = x W^T [M, N] of FP8 operands with one scale per 128 elements:
    xq uint8 [M, K] with SCALE_ROW128 scales, wq uint8 [N, K] with
    SCALE_BLOCK128 scales (acrl_quantize_fp8); a block's x_scale * w_scale is
    rounded to float32 before its use.  `out` (bf16 or float32) may be
    a column slice of a wider matrix: unit column stride, any row stride, its
    first element 16-byte aligned."""
    index, out, desc = _product(xq, x_scales, wq, w_scales, out, out_dtype, stream)
    _check(lib().acrl_matmul_fp8(ctypes.byref(desc), _raw_stream(stream, xq.device)), "acrl_matmul_fp8")
    return out


def _product(xq, x_scales, wq, w_scales, out, out_dtype, stream):
    """(device index, out, descriptor) of a product of block-scaled operands."""
    if xq.dim() != 2 or wq.dim() != 2 or xq.shape[1] != wq.shape[1]:
        raise ValueError("xq [M, K] and wq [N, K] must be 2-D with the same K")
    index = _index_of(xq, torch.uint8, "xq", stream)
    M, K = xq.shape
    N = wq.shape[0]
    kb = (K + 127) // 128
    if out is None:
        if out_dtype not in _OUT_TYPES:
            raise ValueError("out_dtype must be torch.bfloat16 or torch.float32, got %s" % out_dtype)
        out, ldy = _empty((M, N), out_dtype, xq.device, stream), N
    else:
        ldy = _matrix(out, M, N, index, "out")
        out_dtype = out.dtype
    return index, out, MatmulDesc(M, N, K, xq.data_ptr(), _want(x_scales, torch.float32, M * kb, index, "x_scales"),
                                  _want(wq, torch.uint8, N * K, index, "wq"),
                                  _want(w_scales, torch.float32, (N + 127) // 128 * kb, index, "w_scales"),
                                  out.data_ptr(), ldy, _OUT_TYPES[out_dtype])


def _matrix(t, rows: int, cols: int, index: int, name: str) -> int:
    """The row distance of a bf16 or float32 matrix that may be a column slice of a wider one."""
    if (t.dtype not in _OUT_TYPES or t.get_device() != index or tuple(t.shape) != (rows, cols) or
            (cols > 1 and t.stride(1) != 1) or (rows > 1 and t.stride(0) < cols)):
        raise ValueError("%s must be a bf16 or float32 device matrix [%d, %d] on cuda:%d with unit column stride"
                         % (name, rows, cols, index))
    return t.stride(0) if rows > 1 else cols


def acrl_linear_fp8(xq, x_scales, wq, w_scales, bias=None, activation: int = ACT_NONE, residual=None, out=None,
                    out_dtype=torch.bfloat16, stream=None):
    """y = act(x W^T + bias) + residual [M, N], operands and `out` as for
    acrl_matmul_fp8, rounded once.  bias [N] and residual [M, N] are bf16 or
    float32; the residual may be a column slice of a wider matrix (first element
    16-byte aligned), and may be `out` itself."""
    index, out, product = _product(xq, x_scales, wq, w_scales, out, out_dtype, stream)
    M, N = out.shape
    desc = LinearDesc(product, activation=activation)
    if bias is not None:
        if bias.dtype not in _OUT_TYPES:
            raise ValueError("bias must be bf16 or float32, got %s" % bias.dtype)
        desc.bias, desc.bias_type = _want(bias, bias.dtype, N, index, "bias"), _OUT_TYPES[bias.dtype]
    if residual is not None:
        desc.ldr = _matrix(residual, M, N, index, "residual")
        desc.residual, desc.residual_type = residual.data_ptr(), _OUT_TYPES[residual.dtype]
    _check(lib().acrl_linear_fp8(ctypes.byref(desc), _raw_of(stream, index)), "acrl_linear_fp8")
    return out


# ------------------------------------------------------------------ mixture of experts
def acrl_moe_fp8(x, w_in, s_in, w_out, s_out, top_k: int, router=None, score: int = MOE_SOFTMAX, select_bias=None,
                 renormalize: bool = True, scale: float = 1.0, activation: int = ACT_SILU, mask=None, residual=None,
                 ids=None, weights=None, out=None, out_dtype=torch.bfloat16, stream=None):
    """A mixture-of-experts layer for up to 128 tokens: x bf16 [T, d] (rows may
    lie apart), w_in uint8 [E, 2 F, d] (gate rows, then up rows) and w_out uint8
    [E, d, F] with the SCALE_BLOCK128 scales of each expert's matrix, router bf16
    [E, d].  Returns (y [T, d], ids int32 [T, top_k], weights float32 [T, top_k]);
    without a router `ids` and `weights` are inputs (the routing of an earlier
    call).  `out` and `residual` may be column slices of wider matrices, and the
    same tensor."""
    if x.dim() != 2 or w_in.dim() != 3 or w_out.dim() != 3:
        raise ValueError("x [T, d], w_in [E, 2 F, d] and w_out [E, d, F] are required")
    T, d = x.shape
    E, F = w_in.shape[0], w_out.shape[2]
    if tuple(w_in.shape) != (E, 2 * F, d) or tuple(w_out.shape) != (E, d, F):
        raise ValueError("w_in %s and w_out %s do not fit x's %d columns" % (tuple(w_in.shape), tuple(w_out.shape), d))
    index, dev, f32, kb = _index_of(w_in, torch.uint8, "w_in", stream), x.device, torch.float32, (d + 127) // 128
    if x.dtype is not torch.bfloat16 or x.get_device() != index or (d > 1 and x.stride(1) != 1) or (T > 1 and x.stride(0) < d):
        raise ValueError("x must be a bf16 matrix on cuda:%d with unit column stride" % index)
    if router is None and (ids is None or weights is None):
        raise ValueError("a router, or ids and weights, are required")
    nbytes = _size("acrl_moe_workspace_size", T, d, E, top_k, F)
    ldr = ldy = d
    if residual is not None:
        ldr = _matrix(residual, T, d, index, "residual")
    if out is None:
        if out_dtype not in _OUT_TYPES:
            raise ValueError("out_dtype must be torch.bfloat16 or torch.float32, got %s" % out_dtype)
        out = _empty((T, d), out_dtype, dev, stream)
    else:
        ldy = _matrix(out, T, d, index, "out")
    if ids is None:
        ids = _empty((T, top_k), torch.int32, dev, stream)
    if weights is None:
        weights = _empty((T, top_k), f32, dev, stream)
    ws = _empty(nbytes, torch.uint8, dev, stream) if nbytes else None
    desc = MoeDesc(
        T, d, E, top_k, F, x.data_ptr(), x.stride(0) if T > 1 else (d + 7) // 8 * 8,
        _want(router, torch.bfloat16, E * d, index, "router", True), _want(select_bias, f32, E, index, "select_bias", True),
        _want(mask, torch.uint8, T, index, "mask", True), w_in.data_ptr(),
        _want(s_in, f32, E * ((2 * F + 127) // 128) * kb, index, "s_in"),
        _want(w_out, torch.uint8, E * d * F, index, "w_out"), _want(s_out, f32, E * kb * ((F + 127) // 128), index, "s_out"),
        None if residual is None else residual.data_ptr(), ldr, out.data_ptr(), ldy,
        _want(ids, torch.int32, T * top_k, index, "ids"), _want(weights, f32, T * top_k, index, "weights"),
        0 if residual is None else _OUT_TYPES[residual.dtype], _OUT_TYPES[out.dtype], score, 1 if renormalize else 0,
        activation, scale, ws.data_ptr() if nbytes else None, nbytes)
    _check(lib().acrl_moe_fp8(ctypes.byref(desc), _raw_of(stream, index)), "acrl_moe_fp8")
    return out, ids, weights


# ------------------------------------------------------------------ beam search
def acrl_beam_step(logits, scores, n_out: int, inv_temperature: float = 1.0, finished=None, eos_id: int = -1, ids=None,
                   parents=None, out_scores=None, stream=None):
    """The n_out best continuations of every sequence: logits [B K, V] (bf16 or
    float32, rows may lie apart), scores float32 [B, K], finished uint8 [B, K].
    Returns (ids int32, parents int32, scores float32), each [B, n_out]."""
    if scores.dim() != 2 or logits.dim() != 2 or logits.shape[0] != scores.numel():
        raise ValueError("scores [B, K] and logits [B K, V] are required")
    B, K = scores.shape
    V = logits.shape[1]
    index, dev, f32 = _index_of(scores, torch.float32, "scores", stream), scores.device, torch.float32
    ldl = _matrix(logits, B * K, V, index, "logits")
    nbytes = _size("acrl_beam_workspace_size", B, K, V, n_out)
    outputs = []
    for t, dtype, name in ((ids, torch.int32, "ids"), (parents, torch.int32, "parents"), (out_scores, f32, "out_scores")):
        if t is None:
            t = _empty((B, n_out), dtype, dev, stream)
        else:
            _want(t, dtype, B * n_out, index, name)
        outputs.append(t)
    ws = _empty(nbytes, torch.uint8, dev, stream) if nbytes else None
    desc = BeamDesc(B, K, V, n_out, logits.data_ptr(), ldl, scores.data_ptr(),
                    _want(finished, torch.uint8, B * K, index, "finished", True), _OUT_TYPES[logits.dtype], eos_id,
                    inv_temperature, *[t.data_ptr() for t in outputs], ws.data_ptr() if nbytes else None, nbytes)
    _check(lib().acrl_beam_step(ctypes.byref(desc), _raw_of(stream, index)), "acrl_beam_step")
    return tuple(outputs)


def acrl_beam_reorder(state, parents, dim: int = 0, out=None, stream=None):
    """The states of the chosen beams: state has the sequences B in dimension `dim`
    and their K beams in the next; parents int32 [B, n_out] (acrl_beam_step).
    Returns `out`, of state's shape with n_out beams.  What follows the beams'
    dimension is one dense row a beam (a prefix of a longer one, as state[..., :n,
    :], where the rows lie apart); what precedes `dim` is collapsed.  `out` may be
    `state` itself (n_out = K)."""
    index = state.get_device()
    if not state.is_cuda or state.dim() < dim + 2 or dim < 0:
        raise ValueError("state must be a device tensor with sequences in dimension %d and beams in the next" % dim)
    _index_of(parents, torch.int32, "parents", stream)
    shape, size = state.shape, state.element_size()
    B, K = shape[dim], shape[dim + 1]
    if parents.dim() != 2 or parents.shape[0] != B or parents.get_device() != index:
        raise ValueError("parents must be [%d, n_out] on %s" % (B, state.device))
    n_out = parents.shape[1]
    shape_out = (*shape[:dim + 1], n_out, *shape[dim + 2:])
    if out is None:
        out = _empty(shape_out, state.dtype, state.device, stream)
    elif tuple(out.shape) != shape_out or out.dtype != state.dtype or out.get_device() != index:
        raise ValueError("out must be %s of %s on %s" % (shape_out, state.dtype, state.device))
    outer, row, *src = _rows(shape, state.stride(), dim, size, "state")
    _, _, *dst = _rows(shape_out, out.stride(), dim, size, "out")
    desc = ReorderDesc(outer, B, K, n_out, row, state.data_ptr(), *src, out.data_ptr(), *dst, parents.data_ptr())
    _check(lib().acrl_beam_reorder(ctypes.byref(desc), _raw_of(stream, index)), "acrl_beam_reorder")
    return out


@functools.lru_cache(maxsize=256)
def _rows(shape, strides, dim: int, size: int, name: str):
    """(outer, bytes of a beam's row, bytes between outer ones, sequences, beams)
    of a tensor of states with elements of `size` bytes."""
    if 0 in shape:
        return 0, 0, 0, 0, 0
    row = 1
    for n, s in zip(reversed(shape[dim + 2:]), reversed(strides[dim + 2:])):
        if n != 1 and s != row:
            raise ValueError("%s: a beam's row must be dense" % name)
        row *= n
    outer, step = 0, None
    for n, s in zip(reversed(shape[:dim]), reversed(strides[:dim])):
        if n == 1:
            continue
        if step is not None and s != step:
            raise ValueError("%s: the dimensions before the sequences must collapse into one" % name)
        outer, step = outer if step is not None else s, s * n
    return (math.prod(shape[:dim]), row * size, outer * size, strides[dim] * size if shape[dim] > 1 else 0,
            strides[dim + 1] * size if shape[dim + 1] > 1 else 0)


# ------------------------------------------------------------------ losses beside the surrogate
def acrl_policy_loss(B: int, L: int, n_groups: int, mask, group_of_seq, logp_new, logp_old, adv,
                     adv_per_token: bool, logp_ref=None, weight=None, eps_low: float = 0.2, eps_high: float = 0.2,
                     dual_clip: float = 0.0, kl_coef: float = 0.0, kl_estimator: int = KL_K3,
                     aggregate: int = AGG_GROUP, norm: float = 1.0, coef=None, stream=None):
    """Clipped policy loss with a KL term to a reference policy: returns
    (coef float32 [B*L] = d loss / d logp_new, loss float64 [1], stats float64
    [N_PSTATS], PSTAT_NAMES).  coef goes to acrl_lm_head_backward."""
    n, index, dev, f32 = B * L, _index_of(logp_new, torch.float32, "logp_new", stream), logp_new.device, torch.float32
    nbytes = _size("acrl_policy_loss_workspace_size", B, L, n_groups)
    if coef is None:
        coef = _empty(n, f32, dev, stream)
    loss = _empty(1, torch.float64, dev, stream)
    stats = _empty(N_PSTATS, torch.float64, dev, stream)
    ws = _empty(nbytes, torch.uint8, dev, stream) if nbytes else None
    desc = PolicyLossDesc(
        B, L, n_groups, _want(mask, torch.uint8, n, index, "mask"),
        _want(group_of_seq, torch.int32, B, index, "group_of_seq", True), _want(logp_new, f32, n, index, "logp_new"),
        _want(logp_old, f32, n, index, "logp_old"), _want(logp_ref, f32, n, index, "logp_ref", True),
        _want(adv, f32, n if adv_per_token else B, index, "adv"), _want(weight, f32, n, index, "weight", True),
        1 if adv_per_token else 0, kl_estimator, aggregate, eps_low, eps_high, dual_clip, kl_coef, norm,
        _want(coef, f32, n, index, "coef"), loss.data_ptr(), stats.data_ptr(), ws.data_ptr() if nbytes else None, nbytes)
    _check(lib().acrl_policy_loss(ctypes.byref(desc), _raw_stream(stream, dev)), "acrl_policy_loss")
    return coef, loss, stats


def acrl_preference_loss(B: int, L: int, mask, logp_new, chosen, rejected, logp_ref=None, pair_weight=None,
                         beta: float = 0.1, margin: float = 0.0, label_smoothing: float = 0.0,
                         form: int = PREF_SIGMOID, mean_logp: bool = False, coef=None, stream=None):
    """Loss of preferred / rejected response pairs (int32 response indexes
    chosen, rejected [n_pairs]): returns (coef float32 [B*L] = d loss / d
    logp_new, loss float64 [1], rewards float32 [2, n_pairs])."""
    n, index, dev, f32 = B * L, _index_of(logp_new, torch.float32, "logp_new", stream), logp_new.device, torch.float32
    P = chosen.numel()
    nbytes = _size("acrl_preference_loss_workspace_size", B, L, P)
    if coef is None:
        coef = _empty(n, f32, dev, stream)
    loss = _empty(1, torch.float64, dev, stream)
    rewards = _empty((2, P), f32, dev, stream)
    ws = _empty(nbytes, torch.uint8, dev, stream) if nbytes else None
    desc = PreferenceDesc(
        B, L, P, _want(mask, torch.uint8, n, index, "mask"), _want(logp_new, f32, n, index, "logp_new"),
        _want(logp_ref, f32, n, index, "logp_ref", True), _want(chosen, torch.int32, P, index, "chosen"),
        _want(rejected, torch.int32, P, index, "rejected"), _want(pair_weight, f32, P, index, "pair_weight", True),
        form, 1 if mean_logp else 0, beta, margin, label_smoothing, _want(coef, f32, n, index, "coef"),
        loss.data_ptr(), rewards.data_ptr(), ws.data_ptr() if nbytes else None, nbytes)
    _check(lib().acrl_preference_loss(ctypes.byref(desc), _raw_stream(stream, dev)), "acrl_preference_loss")
    return coef, loss, rewards
