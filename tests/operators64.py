"""The block-scaled FP8 operators and the losses by their definitions, in 64
bits on the host: what the GPU tests compare with.  Nothing here comes from the
HIP path."""
import math

import numpy as np

import oracle


# ------------------------------------------------------------------ FP8 blocks
def e4m3_values():
    """The value of every E4M3 code (NaN codes NaN)."""
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e > 0, (1 + m / 8.0) * np.exp2(e - 7.0), m / 8.0 * 2.0 ** -6)
    v[(c & 127) == 127] = np.nan
    return np.where(c & 128, -v, v)


def quantize_blocks(bits, tile, rounding=oracle.ROUND_NEAREST_EVEN):
    """(codes, scales) of a bf16 matrix with one scale per tile x 128 block: every
    block is one row for the oracle's per-row quantizer (zeros past the matrix
    change no maximum)."""
    rows, cols = bits.shape
    pad = np.pad(bits, ((0, -rows % tile), (0, -cols % 128)))
    R, C = pad.shape[0] // tile, pad.shape[1] // 128
    flat = pad.reshape(R, tile, C, 128).transpose(0, 2, 1, 3).reshape(R * C, tile * 128)
    q, s = oracle.quantize_fp8(np.ascontiguousarray(flat), oracle.PER_ROW, rounding)
    q = q.reshape(R, C, tile, 128).transpose(0, 2, 1, 3).reshape(pad.shape)[:rows, :cols]
    return np.ascontiguousarray(q), s.reshape(R, C)


def product(xq, xs, wq, ws):
    """(y, slack) in 64 bits.  slack bounds what the matrix instruction and fp32
    accumulation may lose: it keeps a block's products to 2^-17 of the largest
    (each of the 128 may lose that; a factor 2 for the alignment of the largest
    itself), and every scaled block enters fp32 sums, half a step each for the
    factor, the product with it and the sum."""
    val = e4m3_values()
    M, K = xq.shape
    N = wq.shape[0]
    y, mag, slack = np.zeros((M, N)), np.zeros((M, N)), np.zeros((M, N))
    for b in range(xs.shape[1]):
        k = slice(128 * b, min(K, 128 * b + 128))
        x, w = val[xq[:, k]], val[wq[:, k]]
        f = xs[:, b].astype(np.float64)[:, None] * np.repeat(ws[:, b].astype(np.float64), 128)[:N][None]
        y += f * (x @ w.T)
        mag += np.abs(f) * (np.abs(x) @ np.abs(w).T)
        slack += np.abs(f) * (128 * 2.0 ** -16 * np.abs(x).max(1)[:, None] * np.abs(w).max(1)[None])
    return y, slack + (xs.shape[1] + 2) * 2.0 ** -23 * mag


# ------------------------------------------------------------------ losses
def f32(v):
    return float(np.float32(v))


def shares(B, L, mask, aggregate, groups=None, n_groups=0, norm=1.0):
    """a_t of every response (NaN for a group id out of range, 0 for an empty response)."""
    n = mask.reshape(B, L).astype(bool).sum(1)
    a = np.zeros(B)
    if aggregate == "group":
        ok = (groups >= 0) & (groups < n_groups)
        live = {g: int(((groups == g) & (n > 0)).sum()) for g in range(n_groups)}
        P = sum(v > 0 for v in live.values())
        for i in range(B):
            a[i] = np.nan if not ok[i] else 1 / (P * live[int(groups[i])] * n[i]) if n[i] else 0.0
    else:
        for i in range(B):
            if n[i]:
                a[i] = {"sequence": 1 / ((n > 0).sum() * n[i]), "token": 1 / n.sum(),
                        "constant": 1 / f32(norm)}[aggregate]
    return a


def policy_loss(B, L, mask, new, old, adv, per_token, aggregate, groups=None, n_groups=0, ref=None, weight=None, eps_low=0.2,
                eps_high=0.2, dual_clip=0.0, kl_coef=0.0, kl="k3", norm=1.0):
    """dict(loss, coef, stats, size): size = sum of the magnitudes that the loss adds up."""
    a = shares(B, L, mask, aggregate, groups, n_groups, norm)
    coef = np.zeros(B * L)
    pol = klsum = size = 0.0
    clipped = dual = moved = count = 0
    lo, hi, D, beta = 1 - f32(eps_low), 1 + f32(eps_high), f32(dual_clip), f32(kl_coef)
    for t in np.flatnonzero(mask.reshape(-1)):
        i = t // L
        if np.isnan(a[i]):
            coef[t] = np.nan
            continue
        A = float(adv[t] if per_token else adv[i])
        w = 1.0 if weight is None else float(weight[t])
        delta = float(new[t]) - float(old[t])
        r = math.exp(delta)
        u, c = r * A, min(max(r, lo), hi) * A
        m, live = (u, True) if u <= c else (c, False)
        clipped += not live
        if D > 0 and A < 0 and m < D * A:
            m, live = D * A, False
            dual += 1
        k = dk = 0.0
        if ref is not None:
            q = float(ref[t]) - float(new[t])
            k, dk = {"k1": (-q, 1.0), "k2": (q * q / 2, -q), "k3": (math.expm1(q) - q, -math.expm1(q))}[kl]
        pol += a[i] * -w * m
        klsum += a[i] * k
        size += a[i] * (abs(w * m) + (beta * abs(k) if beta else 0.0))
        moved += math.expm1(delta) - delta
        count += 1
        coef[t] = a[i] * ((-w * u if live else 0.0) + (beta * dk if beta else 0.0))
    d = max(1, count)
    return dict(loss=pol + beta * klsum if beta else pol, coef=coef, size=size,
                stats=np.array([pol, klsum, clipped / d, dual / d, moved / d, count]))


def preference_loss(B, L, mask, new, chosen, rejected, ref=None, weight=None, beta=0.1, margin=0.0, smoothing=0.0,
                    form="sigmoid", mean=False):
    """dict(loss, coef, rewards, size) as policy_loss."""
    valid = mask.reshape(B, L) != 0
    n = valid.sum(1)
    x, each = np.zeros(B), np.ones(B)
    for i in range(B):
        at = np.flatnonzero(valid[i]) + i * L
        x[i] = math.fsum(float(new[t]) - (float(ref[t]) if ref is not None else 0.0) for t in at)
        if mean:
            each[i] = 1 / max(1, n[i])
            x[i] *= each[i]
    b, e, mg, P = f32(beta), f32(smoothing), f32(margin), len(chosen)
    slope, loss, size = np.zeros(B), 0.0, 0.0
    rewards = np.full((2, P), np.nan)
    for p, (c, r) in enumerate(zip(chosen, rejected)):
        u = 1.0 if weight is None else float(weight[p])
        inside = [0 <= j < B for j in (c, r)]
        for row, (j, ok) in enumerate(zip((c, r), inside)):
            if ok:
                rewards[row, p] = b * x[j]
        if not all(inside):
            loss = math.nan
            for j, ok in zip((c, r), inside):
                if ok:
                    slope[j] = math.nan
            continue
        h = b * (x[c] - x[r]) - mg
        if form == "sigmoid":
            soft = math.log1p(math.exp(-abs(h)))
            l = (1 - e) * (soft + max(-h, 0)) + e * (soft + max(h, 0))
            s = 1 / (1 + math.exp(-h)) if h > -700 else 0.0
            s_down = 1 / (1 + math.exp(h)) if h < 700 else 0.0
            d = e * s - (1 - e) * s_down
        elif form == "hinge":
            l, d = max(0.0, 1 - h), -1.0 if h < 1 else 0.0
        else:
            l, d = ((h - 0.5) / b) ** 2, 2 * (h - 0.5) / b ** 2
        loss += u * l / P
        size += abs(u * l / P)
        slope[c] += u * d * b / P
        slope[r] -= u * d * b / P
    coef = np.where(valid, (slope * each)[:, None], 0.0).reshape(-1)
    return dict(loss=loss, coef=coef, rewards=rewards, size=size)
