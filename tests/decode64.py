"""The operators of a decode step by their definitions, in 64 bits on the host:
what the GPU tests compare with.  Nothing here comes from the HIP path."""
import math

import numpy as np
from scipy.special import ndtr

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}  # half a step, relative to the value


def f64(bits):
    """The values of bf16 patterns."""
    return (np.asarray(bits).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


# ------------------------------------------------------------------ activations
def _sigmoid(u):
    e = np.exp(-np.abs(u))
    return np.where(u >= 0, 1 / (1 + e), e / (1 + e))


def act(name, v):
    v = np.asarray(v, np.float64)
    if name == "relu":
        return np.where(v < 0, 0.0, v)
    if name == "silu":
        return v * _sigmoid(v)
    if name == "gelu":
        return v * ndtr(v)
    if name == "gelu_tanh":
        return v * _sigmoid(2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3))
    return v


# |act'| is nowhere above these (silu 1.0998, gelu 1.1290, gelu_tanh 1.1292)
SLOPE = {"none": 1.0, "relu": 1.0, "silu": 1.11, "gelu": 1.13, "gelu_tanh": 1.14}
ACT_ERROR = 6e-7  # of act at a given fp32 value, relative to act


def linear(y, slack, name, bias=None, residual=None):
    """(value, bound on the error before y is rounded) of act(y + bias) + residual
    for a product y that is off by up to `slack`: the bias enters by one fp32 sum,
    the residual by another, half a step each."""
    e = HALF["f32"]
    s = y if bias is None else y + bias
    slack = slack + (0 if bias is None else e * (np.abs(s) + slack))
    a = act(name, s)
    tol = SLOPE[name] * slack + (0 if name in ("none", "relu") else ACT_ERROR * (np.abs(a) + slack) + 1.3e-36)
    out = a if residual is None else a + residual
    return out, tol + (0 if residual is None else e * (np.abs(out) + tol))
