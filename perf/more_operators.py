"""Calls of the operators of a decode step of the rollout policy beside the plain
FP8 product, as cases that can be timed: each in its plain form (elementary
torch operations) or, where `own` is true, through paper_2607_24062_amd.acrl.

Kinds of case:
  linear   act(x W^T + bias) + residual of block-scaled FP8 operands
  moe      a whole mixture-of-experts layer for a few tokens: router, choice of
           the experts, their gated products, the weighted sum
  beam     beam search's choice of the next tokens over beams and vocabulary
  reorder  the states of the chosen beams, gathered

Sizes: the hidden sizes 2048 / 4096 / 5120 and V = 151936 of the repository's
workloads, its small vocabulary of 2048, generic layer widths and expert counts.
"""
import math

import torch

own = False

V_FULL = 151936
E4M3_MAX = 448.0


def listed():
    return [
        # one live response through the narrowing product of a layer, added to the residual stream: latency alone counts
        {"name": "linear_one", "kind": "linear", "M": 1, "N": 2048, "K": 5120, "act": "none", "bias": "", "res": "bf16",
         "out": "bf16"},
        # a short prompt, odd in every size, all of the epilogue
        {"name": "linear_short", "kind": "linear", "M": 333, "N": 5000, "K": 2080, "act": "gelu_tanh", "bias": "f32",
         "res": "f32", "out": "bf16"},
        # a chunk of a batch through a widening layer
        {"name": "linear_chunk", "kind": "linear", "M": 8192, "N": 13824, "K": 5120, "act": "gelu", "bias": "bf16",
         "res": "", "out": "bf16"},
        # one live response decodes one token: eight experts' weights
        {"name": "moe_one", "kind": "moe", "T": 1, "d": 2048, "E": 128, "k": 8, "F": 768, "score": "softmax", "norm": True,
         "bias": False, "mask": False, "res": False, "out": "bf16"},
        # a decode step of 64 responses, some of them finished: most experts are read
        {"name": "moe_batch", "kind": "moe", "T": 64, "d": 2048, "E": 128, "k": 8, "F": 768, "score": "softmax",
         "norm": True, "bias": False, "mask": True, "res": True, "out": "bf16"},
        # few wide experts
        {"name": "moe_wide", "kind": "moe", "T": 16, "d": 4096, "E": 8, "k": 2, "F": 14336, "score": "softmax", "norm": True,
         "bias": False, "mask": False, "res": False, "out": "bf16"},
        # odd widths, experts chosen by sigmoid scores with a bias that balances their load
        {"name": "moe_odd", "kind": "moe", "T": 7, "d": 1056, "E": 60, "k": 4, "F": 1408, "score": "sigmoid", "norm": False,
         "bias": True, "mask": False, "res": True, "out": "f32"},
        # one prompt's first step: only its first beam is live
        {"name": "beam_one", "kind": "beam", "B": 1, "K": 4, "V": V_FULL, "N": 4, "type": "f32", "first": True, "done": False,
         "temperature": 1.0},
        # an evaluation batch of 64 prompts of eight beams, some of which have ended
        {"name": "beam_batch", "kind": "beam", "B": 64, "K": 8, "V": V_FULL, "N": 16, "type": "f32", "first": False,
         "done": True, "temperature": 1.0},
        # a few prompts over a small vocabulary of odd size, bf16 logits
        {"name": "beam_odd", "kind": "beam", "B": 3, "K": 5, "V": 2049, "N": 10, "type": "bf16", "first": False, "done": True,
         "temperature": 0.7},
        # the hidden states of a few beams
        {"name": "reorder_hidden", "kind": "reorder", "layers": 1, "B": 3, "K": 5, "N": 5, "tokens": 1, "live": 1,
         "width": 2048},
        # key and value caches of all layers, filled to two thirds
        {"name": "reorder_cache", "kind": "reorder", "layers": 32, "B": 16, "K": 8, "N": 8, "tokens": 192, "live": 131,
         "width": 512},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    """One more case of the ranges above: sizes over their logarithm, odd ones among them."""
    kind = rng.choice(["linear", "linear", "linear", "moe", "moe", "moe", "beam", "beam", "reorder"])
    if kind == "linear":
        K = rng.choice([32 * _log_int(rng, 4, 432), 128 * _log_int(rng, 2, 108), 2048, 4096, 5120])
        N = rng.choice([_log_int(rng, 16, 16384), 128 * _log_int(rng, 2, 128), 4096, 5120, 13824])
        M = rng.choice([_log_int(rng, 1, 64), _log_int(rng, 1, 8192), 8 * _log_int(rng, 8, 1024)])
        M = max(1, min(M, int(5.5e11 / (float(N) * K))))
        return {"kind": kind, "M": M, "N": N, "K": K, "act": rng.choice(["none", "relu", "silu", "gelu", "gelu_tanh"]),
                "bias": rng.choice(["", "f32", "bf16"]), "res": rng.choice(["", "f32", "bf16"]),
                "out": "bf16"}
    if kind == "moe":
        E = rng.choice([4, 8, 16, 32, 60, 64, 128, 160, 256])
        k = min(E, rng.choice([1, 2, 2, 4, 6, 8]))
        d = rng.choice([32 * _log_int(rng, 8, 160), 1024, 2048, 4096, 5120])
        F = 32 * _log_int(rng, 4, 448)
        F = max(32, min(F, int(1.2e9 / (3.0 * E * d)) // 32 * 32))
        return {"kind": kind, "T": rng.choice([1, _log_int(rng, 1, 16), _log_int(rng, 1, 128)]), "d": d, "E": E, "k": k,
                "F": F, "score": rng.choice(["softmax", "sigmoid"]), "norm": rng.random() < 0.6, "bias": rng.random() < 0.4,
                "mask": rng.random() < 0.3, "res": rng.random() < 0.5, "out": rng.choice(["f32", "bf16"])}
    if kind == "beam":
        K = rng.choice([1, 2, 3, 4, 5, 8, 16])
        V = rng.choice([_log_int(rng, 300, 160000), V_FULL, 2048, 32000])
        B = max(1, min(_log_int(rng, 1, 64), int(7.5e7 / (float(K) * V))))
        return {"kind": kind, "B": B, "K": K, "V": V, "N": K * rng.choice([1, 2]), "type": rng.choice(["f32", "bf16"]),
                "first": rng.random() < 0.2, "done": rng.random() < 0.5, "temperature": rng.choice([1.0, 0.7, 1.3])}
    K = rng.choice([1, 2, 3, 4, 5, 8, 16])
    tokens, width = _log_int(rng, 1, 1024), rng.choice([64, 128, 512, 1024, _log_int(rng, 8, 4096)])
    layers = max(1, min(_log_int(rng, 1, 64), int(2.5e8 / (float(K) * tokens * width))))
    B = max(1, min(_log_int(rng, 1, 64), int(2.5e8 / (float(layers) * K * tokens * width))))
    return {"kind": kind, "layers": layers, "B": B, "K": K, "N": K, "tokens": tokens, "live": rng.randint(1, tokens),
            "width": width}


# ------------------------------------------------------------------ inputs
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + stream)
    return g


def _randn(shape, seed, stream):
    return torch.randn(shape, generator=_gen(seed, stream), device="cuda", dtype=torch.float32)


def _rand(shape, seed, stream):
    return torch.rand(shape, generator=_gen(seed, stream), device="cuda", dtype=torch.float32)


def _activations(rows, cols, seed):
    """Post-norm hidden states; one column in 61 is ten times as large, as outlier channels are."""
    x = _randn((rows, cols), seed, 1)
    x[:, 7::61] *= 10.0
    return x


def _codes(shape, seed, stream):
    """E4M3 codes of normally distributed weights: matrix after matrix, one generator for all."""
    g = _gen(seed, stream)
    out = torch.empty(shape, device="cuda", dtype=torch.uint8)
    for part in out.view(-1, *shape[-2:]):
        f = torch.randn(shape[-2:], generator=g, device="cuda").mul_(100.0).clamp_(-E4M3_MAX, E4M3_MAX)
        part.copy_(f.to(torch.float8_e4m3fn).view(torch.uint8))
    return out


def _weights(shape, seed, stream):
    """(codes [.., rows, cols], scales [.., ceil(rows / 128), ceil(cols / 128)]) of weights of std 2.5 / sqrt(cols)."""
    blocks = (*shape[:-2], -(-shape[-2] // 128), -(-shape[-1] // 128))
    return _codes(shape, seed, stream), (0.5 + _rand(blocks, seed, stream + 1)).mul_(0.025 / math.sqrt(shape[-1]))


def _row_codes(x):
    """(E4M3 codes, fp32 scales) of activations, one scale per row and 128 columns (amax / 448)."""
    rows, cols = x.shape
    f = torch.nn.functional.pad(x, (0, -cols % 128)).reshape(rows, -1, 128)
    s = f.abs().amax(2, keepdim=True).clamp(min=1e-20) / E4M3_MAX
    q = (f / s).clamp(-E4M3_MAX, E4M3_MAX).reshape(rows, -1)[:, :cols].to(torch.float8_e4m3fn)
    return q.contiguous().view(torch.uint8), s[:, :, 0].contiguous()


def prepare(case, seed):
    kind, s = case["kind"], {"case": dict(case)}
    if kind == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        s["xq"], s["xs"] = _row_codes(_activations(M, K, seed))
        s["wq"], s["ws"] = _weights((N, K), seed, 2)
        s["bias"] = _randn((N,), seed, 4).to(DTYPES[case["bias"]]) if case["bias"] else None
        s["res"] = _randn((M, N), seed, 5).mul_(3.0).to(DTYPES[case["res"]]) if case["res"] else None
    elif kind == "moe":
        T, d, E, F = case["T"], case["d"], case["E"], case["F"]
        s["x"] = _activations(T, d, seed).to(torch.bfloat16)
        s["router"] = _randn((E, d), seed, 6).mul_(1.0 / math.sqrt(d)).to(torch.bfloat16)
        s["w_in"], s["s_in"] = _weights((E, 2 * F, d), seed, 7)
        s["w_out"], s["s_out"] = _weights((E, d, F), seed, 9)
        s["bias"] = _randn((E,), seed, 11).mul_(0.1) if case["bias"] else None
        s["mask"] = (_rand((T,), seed, 12) > 0.2).to(torch.uint8) if case["mask"] else None
        s["res"] = _randn((T, d), seed, 5).mul_(3.0).to(torch.bfloat16) if case["res"] else None
    elif kind == "beam":
        B, K, V = case["B"], case["K"], case["V"]
        s["logits"] = _randn((B * K, V), seed, 13).mul_(2.5).to(DTYPES[case["type"]])
        if case["first"]:
            s["scores"] = torch.full((B, K), -math.inf, device="cuda")
            s["scores"][:, 0] = 0.0
        else:
            s["scores"] = -4.0 * _rand((B, K), seed, 14) - 20.0
        s["done"] = (_rand((B, K), seed, 15) < 0.15).to(torch.uint8) if case["done"] else None
        s["eos"] = V // 3
    else:
        shape = tuple(case[n] for n in ("layers", "B", "K", "tokens", "width"))
        s["state"] = _randn((shape[0], shape[1] * shape[2], *shape[3:]), seed, 16).to(torch.bfloat16).view(shape)
        s["parents"] = torch.randint(0, case["K"], (case["B"], case["N"]), generator=_gen(seed, 17), device="cuda",
                                     dtype=torch.int32)
    return s


# ------------------------------------------------------------------ one pass, plain
def _spread(scales, rows, cols, tile):
    """The scale of every element [rows, cols]."""
    return scales.repeat_interleave(128, 1)[:, :cols].repeat_interleave(tile, 0)[:rows]


def _values(q, scales, tile):
    return q.view(torch.float8_e4m3fn).float() * _spread(scales, q.shape[0], q.shape[1], tile)


def _act(v, act):
    if act == "relu":
        return v.clamp(min=0)
    if act == "silu":
        return v / (1 + torch.exp(-v))
    if act == "gelu":
        return 0.5 * v * torch.erfc(v * -math.sqrt(0.5))
    if act == "gelu_tanh":
        return v / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v * v * v)))
    return v


def _plain_linear(s):
    case = s["case"]
    y = _values(s["xq"], s["xs"], 1) @ _values(s["wq"], s["ws"], 128).t()
    if s["bias"] is not None:
        y = y + s["bias"].float()
    y = _act(y, case["act"])
    if s["res"] is not None:
        y = y + s["res"].float()
    return y.to(DTYPES[case["out"]])


def _plain_moe(s):
    case = s["case"]
    E, k = case["E"], case["k"]
    # 64 bits: a score next to another decides which expert is chosen
    l = s["x"].double() @ s["router"].double().t()
    if case["score"] == "softmax":
        p = torch.exp(l - l.amax(1, keepdim=True))
        p = p / p.sum(1, keepdim=True)
    else:
        p = 1 / (1 + torch.exp(-l))
    by = l if s["bias"] is None else p + s["bias"].double()
    ids = torch.sort(by, dim=1, descending=True, stable=True)[1][:, :k]
    w = p.gather(1, ids)
    if case["norm"]:
        w = w / w.sum(1, keepdim=True)
    w = w.float()
    if s["mask"] is not None:
        live = s["mask"][:, None] != 0
        ids, w = torch.where(live, ids, -1), torch.where(live, w, 0.0)
    x = s["x"].float()
    y = torch.zeros_like(x)
    F = case["F"]
    for e in range(E):
        u = x @ _values(s["w_in"][e], s["s_in"][e], 128).t()
        h = _act(u[:, :F], "silu") * u[:, F:]
        v = h @ _values(s["w_out"][e], s["s_out"][e], 128).t()
        hit = ids == e
        y += torch.where(hit.any(1, keepdim=True), torch.where(hit, w, 0.0).sum(1, keepdim=True) * v, 0.0)
    if s["res"] is not None:
        y = y + s["res"].float()
    return {"y": y.to(DTYPES[case["out"]]), "ids": ids.to(torch.int32), "weights": w}


def _f32(v):
    return float(torch.tensor(v, dtype=torch.float32))  # the calls take fp32 numbers


def _plain_beam(s):
    # 64 bits: a score next to another decides which candidate is chosen
    case = s["case"]
    B, K, V, N = case["B"], case["K"], case["V"], case["N"]
    c = s["logits"].double() * _f32(1.0 / case["temperature"])
    top = c.amax(1, keepdim=True)
    c = c + (s["scores"].double().reshape(-1, 1) - top - torch.log(torch.exp(c - top).sum(1, keepdim=True)))
    if s["done"] is not None:
        # a beam that has ended goes on with its last token alone, at no cost
        at_eos = torch.arange(V, device="cuda")[None] == s["eos"]
        c = torch.where(s["done"].reshape(-1, 1) != 0, torch.where(at_eos, s["scores"].double().reshape(-1, 1), -math.inf), c)
    best, at = torch.sort(c.reshape(B, K * V), dim=1, descending=True, stable=True)
    at = at[:, :N]
    return {"ids": (at % V).to(torch.int32), "parents": (at // V).to(torch.int32), "scores": best[:, :N].float()}


def _plain_reorder(s):
    st, p, live = s["state"], s["parents"].long(), s["case"]["live"]
    rows = (torch.arange(st.shape[1], device="cuda")[:, None] * st.shape[2] + p).reshape(-1)
    return st.reshape(st.shape[0], -1, *st.shape[3:])[:, rows, :live].reshape(*st.shape[:2], p.shape[1], live, st.shape[4])


# ------------------------------------------------------------------ one pass
def _run_own(s):
    from paper_2607_24062_amd import acrl

    case = s["case"]
    kind = case["kind"]
    if kind == "linear":
        act = {"none": acrl.ACT_NONE, "relu": acrl.ACT_RELU, "silu": acrl.ACT_SILU, "gelu": acrl.ACT_GELU,
               "gelu_tanh": acrl.ACT_GELU_TANH}[case["act"]]
        return acrl.acrl_linear_fp8(s["xq"], s["xs"], s["wq"], s["ws"], bias=s["bias"], activation=act, residual=s["res"],
                                    out_dtype=DTYPES[case["out"]])
    if kind == "moe":
        score = {"softmax": acrl.MOE_SOFTMAX, "sigmoid": acrl.MOE_SIGMOID}[case["score"]]
        y, ids, w = acrl.acrl_moe_fp8(s["x"], s["w_in"], s["s_in"], s["w_out"], s["s_out"], case["k"], router=s["router"],
                                      score=score, select_bias=s["bias"], renormalize=case["norm"], mask=s["mask"],
                                      residual=s["res"], out_dtype=DTYPES[case["out"]])
        return {"y": y, "ids": ids, "weights": w}
    if kind == "beam":
        ids, parents, scores = acrl.acrl_beam_step(s["logits"], s["scores"], case["N"],
                                                   inv_temperature=1.0 / case["temperature"], finished=s["done"],
                                                   eos_id=s["eos"])
        return {"ids": ids, "parents": parents, "scores": scores}
    return acrl.acrl_beam_reorder(s["state"][:, :, :, : case["live"]], s["parents"], dim=1)


def run(s):
    if own:
        return _run_own(s)
    return {"linear": _plain_linear, "moe": _plain_moe, "beam": _plain_beam, "reorder": _plain_reorder}[s["case"]["kind"]](s)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    kind = case["kind"]
    size = {"": 0, "bf16": 2, "f32": 4}
    if kind == "linear":
        M, N, K = float(case["M"]), float(case["N"]), float(case["K"])
        kb = math.ceil(K / 128)
        return {"bytes": N * K + 4 * math.ceil(N / 128) * kb + M * K + 4 * M * kb + size[case["bias"]] * N +
                (size[case["res"]] + size[case["out"]]) * M * N, "flops": 2 * M * N * K}
    if kind == "moe":
        T, d, E, k, F = (float(case[n]) for n in ("T", "d", "E", "k", "F"))
        T_live = 0.8 * T if case["mask"] else T
        read = E * (1 - (1 - k / E) ** T_live)  # experts that a token chose
        return {"bytes": read * 3 * d * F * (1 + 4 / 16384) + 2 * E * d + T * d * (2 + 2 * case["res"] + size[case["out"]]) +
                8 * T * k, "flops": 6 * T_live * k * d * F + 2 * T_live * E * d}
    if kind == "beam":
        rows = float(case["B"] * case["K"])
        live = rows * (0.85 if case["done"] else 1.0)
        return {"bytes": live * case["V"] * size[case["type"]] + 5 * rows + 12 * case["B"] * case["N"], "flops": 0.0}
    row = 2.0 * case["live"] * case["width"]
    K, N = case["K"], case["N"]
    used = K * (1 - (1 - 1 / K) ** N)  # beams that are somebody's parent
    return {"bytes": case["layers"] * case["B"] * (used + N) * row + 4 * case["B"] * N, "flops": 0.0}


# ------------------------------------------------------------------ the same in 64 bits, from the definitions
def _exact_act(v, act):
    if act == "relu":
        return torch.relu(v)
    if act == "silu":
        return v * torch.sigmoid(v)
    if act == "gelu":
        return v * torch.special.ndtr(v)
    if act == "gelu_tanh":
        return 0.5 * v * (1 + torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)))
    return v


def _exact_product(x, wq, ws):
    """x [M, K] (64 bits) times block-scaled weights, one block of columns after another."""
    y = torch.zeros((x.shape[0], wq.shape[0]), dtype=torch.float64, device="cuda")
    for b in range(ws.shape[1]):
        k = slice(128 * b, 128 * b + 128)
        f = ws[:, b].double()[torch.arange(wq.shape[0], device="cuda") // 128]
        y += f * (x[:, k] @ wq[:, k].contiguous().view(torch.float8_e4m3fn).double().t())
    return y


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "linear":
        at = torch.arange(case["K"], device="cuda") // 128
        y = _exact_product(s["xq"].view(torch.float8_e4m3fn).double() * s["xs"].double()[:, at], s["wq"], s["ws"])
        if s["bias"] is not None:
            y += s["bias"].double()
        y = _exact_act(y, case["act"])
        return y if s["res"] is None else y + s["res"].double()
    if kind == "moe":
        return _exact_moe(case, s)
    if kind == "beam":
        return _exact_beam(case, s)
    st, p = s["state"].double()[:, :, :, : case["live"]], s["parents"].tolist()
    return torch.stack([st[:, b, p[b]] for b in range(case["B"])], 1)


def _exact_moe(case, s):
    """Token by token for the choice, expert by expert over its own tokens for the products."""
    T, E, k, F = case["T"], case["E"], case["k"], case["F"]
    x = s["x"].double()
    l = (x[:, None, :] * s["router"].double()[None]).sum(2)
    p = torch.softmax(l, 1) if case["score"] == "softmax" else torch.sigmoid(l)
    by = (l if s["bias"] is None else p + s["bias"].double()).tolist()
    ids = torch.tensor([sorted(range(E), key=lambda e: (-row[e], e))[:k] for row in by], device="cuda")
    w = p.gather(1, ids)
    if case["norm"]:
        w = w / w.sum(1, keepdim=True)
    if s["mask"] is not None:
        ids[s["mask"] == 0] = -1
        w[s["mask"] == 0] = 0.0
    y = s["res"].double() if s["res"] is not None else torch.zeros_like(x)
    for e in range(E):
        t, slot = torch.nonzero(ids == e, as_tuple=True)
        if t.numel() == 0:
            continue
        u = _exact_product(x[t], s["w_in"][e], s["s_in"][e])
        h = _exact_act(u[:, :F], "silu") * u[:, F:]
        y[t] += w[t, slot][:, None] * _exact_product(h, s["w_out"][e], s["s_out"][e])
    return {"y": y, "ids": ids.to(torch.int32), "weights": w}


def _exact_beam(case, s):
    """A beam's best by its logits alone, then the beams' bests together."""
    B, K, V, N = case["B"], case["K"], case["V"], case["N"]
    scores = s["scores"].double().tolist()
    done = s["done"].tolist() if s["done"] is not None else [[0] * K] * B
    ids, parents, best = [], [], []
    for b in range(B):
        z = s["logits"][b * K: (b + 1) * K].double()
        lse = torch.logsumexp(z * _f32(1.0 / case["temperature"]), 1).tolist()
        top, at = torch.sort(z, dim=1, descending=True, stable=True)
        top, at = (top[:, :N] * _f32(1.0 / case["temperature"])).tolist(), at[:, :N].tolist()
        found = []
        for j in range(K):
            if done[b][j]:
                rest = [v for v in range(N + 1) if v != s["eos"]][: N - 1]
                found += [(-scores[b][j], j * V + s["eos"])] + [(math.inf, j * V + v) for v in rest]
            elif scores[b][j] == -math.inf:
                found += [(math.inf, j * V + v) for v in range(min(N, V))]
            else:
                found += [(-(scores[b][j] + t - lse[j]), j * V + v) for t, v in zip(top[j], at[j])]
        found = sorted(found)[:N]
        ids.append([f % V for _, f in found])
        parents.append([f // V for _, f in found])
        best.append([-c for c, _ in found])
    as_int = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    return {"ids": as_int(ids), "parents": as_int(parents), "scores": torch.tensor(best, dtype=torch.float64, device="cuda")}
