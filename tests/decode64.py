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
ACT_ERROR = {"f32": 6e-7, "bf16": 5e-5}  # of act at a given fp32 value, relative to act, by the output's type


def linear(y, slack, name, bias=None, residual=None, out="bf16"):
    """(value, bound on the error before y is rounded) of act(y + bias) + residual
    for a product y that is off by up to `slack`: the bias enters by one fp32 sum,
    the residual by another, half a step each."""
    e = HALF["f32"]
    s = y if bias is None else y + bias
    slack = slack + (0 if bias is None else e * (np.abs(s) + slack))
    a = act(name, s)
    tol = SLOPE[name] * slack + (0 if name in ("none", "relu") else ACT_ERROR[out] * (np.abs(a) + slack) + 1.3e-36)
    out = a if residual is None else a + residual
    return out, tol + (0 if residual is None else e * (np.abs(out) + tol))


# ------------------------------------------------------------------ mixture of experts
def spread(scales, rows, cols):
    """The scale of every element of a matrix with one per 128 x 128 block."""
    return np.repeat(np.repeat(scales.astype(np.float64), 128, 0)[:rows], 128, 1)[:, :cols]


def routing(x, router, k, score="softmax", bias=None, renorm=True, scale=1.0, mask=None):
    """(ids, weights) in 64 bits; ids -1 and weights 0 for masked tokens."""
    T, E = x.shape[0], router.shape[0]
    ids, w = np.full((T, k), -1), np.zeros((T, k))
    for t in range(T):
        if mask is not None and not mask[t]:
            continue
        l = np.array([math.fsum(x[t] * router[e]) for e in range(E)])
        if score == "softmax":
            s = np.exp(l - l.max())
            s /= s.sum()
        else:
            s = _sigmoid(l)
        by = l if bias is None else s + bias.astype(np.float64)
        ids[t] = sorted(range(E), key=lambda e: (-by[e], e))[:k]
        w[t] = s[ids[t]]
        if renorm:
            w[t] = w[t] / w[t].sum() if w[t].sum() else 0.0
        w[t] *= float(np.float32(scale))
    return ids, w


def experts(x, ids, w, w_in, w_out, activation="silu", residual=None):
    """(y, bound on the error before y is rounded).  w_in [E, 2F, d] and w_out
    [E, d, F] are values.  The bound takes every sum in the worst order: n terms in
    fp32 lose at most n 2^-23 of the sum of their sizes (twice half a step: the
    matrix instruction may cut); what lies between the products keeps 2^-16."""
    T, d = x.shape
    E, F = w_out.shape[0], w_out.shape[2]
    y, tol, size = np.zeros((T, d)), np.zeros((T, d)), np.zeros((T, d))
    e1, e2 = (128 + d / 128 + 4) * 2.0 ** -23, (256 + F / 128 + 4) * 2.0 ** -23
    for t in range(T):
        for e, weight in zip(ids[t], w[t]):
            if not 0 <= e < E:
                continue
            u, mag = w_in[e] @ x[t], np.abs(w_in[e]) @ np.abs(x[t])
            g, v, eg, ev = u[:F], u[F:], e1 * mag[:F], e1 * mag[F:]
            a = act(activation, g)
            h = a * v
            ea = SLOPE[activation] * eg + ACT_ERROR["f32"] * (np.abs(a) + eg) + 1.3e-36
            eh = ea * (np.abs(v) + ev) + np.abs(a) * ev
            eh = eh + 2.0 ** -16 * (np.abs(h) + eh) * 1.01
            z, ez = w_out[e] @ h, np.abs(w_out[e]) @ (eh + e2 * (np.abs(h) + eh))
            y[t] += weight * z
            size[t] += abs(weight) * (np.abs(z) + ez)
            tol[t] += abs(weight) * ez
    tol = tol + (ids.shape[1] + 3) * 2.0 ** -23 * size
    if residual is None:
        return y, tol
    return y + residual, tol + HALF["f32"] * (np.abs(y + residual) + tol)


# ------------------------------------------------------------------ beam search
def beam(logits, scores, n, inv_t=1.0, finished=None, eos=-1):
    """(ids, parents, scores) of logits [B, K, V] by a stable sort of all candidates."""
    B, K, V = logits.shape
    out = [], [], []
    for b in range(B):
        c = np.full((K, V), -np.inf)
        for j in range(K):
            if not np.isfinite(scores[b, j]):
                continue
            if finished is not None and finished[b, j]:
                c[j, eos] = scores[b, j]
                continue
            z = logits[b, j].astype(np.float64) * float(np.float32(inv_t))
            if np.isnan(z).any() or not np.isfinite(z.max()):
                continue
            # (a sum that no order of the logits changes: beams of the same ones are equal)
            c[j] = float(scores[b, j]) + (z - z.max() - math.log(math.fsum(np.exp(z - z.max()))))
        flat = c.reshape(-1)
        at = np.argsort(-flat, kind="stable")[:n]
        out[0].append(at % V)
        out[1].append(at // V)
        out[2].append(flat[at])
    return tuple(np.array(o) for o in out)
