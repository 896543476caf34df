"""The rest of a decoder's step beside its attention layer, as timed cases.

Around an attention layer a step has the norms of a block, fused with the gate and the residual stream they stand in; a
mixture of experts in the feed-forward place: the router that chooses some experts for each token, and the chosen experts' gated
products with 4-bit weights; and at the end the choice of the next token from the logits.  A case is one call of
one of them on what a program has in hand before the call: tensors on the GPU, packed weights, descriptors, a workspace.

Activations are normal, the residual stream has some channels of large magnitude; 4-bit codes and their group scales come from
normal weights by the largest magnitude of each group; logits are normal with a few tokens far above the rest, as a trained head
leaves them.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------------------------- cases
def _norm(dtype, tokens, channels, pre="rms", post="none", gate="none", residual=True, bias=False, alpha=1.0, beta=1.0, name=None):
    """sum = alpha * residual + beta * gate * post(x), y = pre(sum); gate: none, one row for all tokens, or a row each."""
    c = {"op": "norm", "dtype": dtype, "tokens": tokens, "channels": channels, "pre": pre, "post": post, "gate": gate,
         "residual": residual, "bias": bias, "alpha": alpha, "beta": beta}
    return dict(c, name=name) if name else c


def _route(dtype, tokens, channels, experts, top_k, score="softmax", bias=False, normalize=True, scale=1.0, name=None):
    c = {"op": "route", "dtype": dtype, "tokens": tokens, "channels": channels, "experts": experts, "top_k": top_k, "score": score,
         "bias": bias, "normalize": normalize, "scale": scale}
    return dict(c, name=name) if name else c


def _experts(dtype, tokens, channels, inter, experts, top_k, group, zeros=False, residual=True, act="silu", skew=0.0, name=None):
    """skew: how uneven the router is; 0: every expert alike."""
    c = {"op": "experts", "dtype": dtype, "tokens": tokens, "channels": channels, "inter": inter, "experts": experts, "top_k": top_k,
         "group": group, "zeros": zeros, "residual": residual, "act": act, "skew": skew}
    return dict(c, name=name) if name else c


def _sample(dtype, rows, vocab, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, mixed=False, name=None):
    """mixed: every row has settings of its own, as the users of one batch do (some greedy, some without any limit)."""
    c = {"op": "sample", "dtype": dtype, "rows": rows, "vocab": vocab, "temperature": temperature, "top_k": top_k, "top_p": top_p,
         "min_p": min_p, "mixed": mixed}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one user's token between two blocks: latency
        _norm("f16", 1, 4096, name="norm_f16_t1"),
        # a block with norms on both sides and a learned gate a channel, an odd width
        _norm("f16", 1003, 5003, pre="layer", post="rms", gate="row", bias=True, alpha=0.9, beta=0.5, name="norm_f16_t1003_odd"),
        # a long prompt
        _norm("bf16", 8192, 8192, name="norm_bf16_t8192"),
        # the router for one token: latency
        _route("bf16", 1, 4096, 64, 8, name="route_bf16_t1"),
        # the router for the tokens of a full batch with some drafts, chosen with a bias that evens the load
        _route("f16", 509, 4096, 128, 6, score="sigmoid", bias=True, scale=2.5, name="route_f16_t509"),
        # one user's token: eight experts' weights
        _experts("f16", 1, 4096, 1024, 64, 8, 128, name="experts_f16_t1"),
        # a handful of users, small groups with zero points, some experts liked more than others
        _experts("bf16", 7, 2000, 1408, 60, 4, 32, zeros=True, act="gelu", skew=1.0, name="experts_bf16_t7"),
        # a full batch: nearly all experts' weights
        _experts("bf16", 64, 4096, 1024, 128, 8, 128, name="experts_bf16_t64"),
        # a chunk of a prompt: some tens of rows to an expert
        _experts("f16", 500, 2048, 1408, 32, 4, 128, residual=False, skew=0.5, name="experts_f16_t500"),
        # one user's next token by the usual settings: latency
        _sample("f16", 1, 128000, 0.8, 50, 0.95, name="sample_f16_r1"),
        # a batch that cuts the tail by its mass alone, an odd vocabulary
        _sample("bf16", 48, 151643, 1.0, 0, 0.9, name="sample_bf16_r48_top_p"),
        # many users with settings of their own
        _sample("f32", 256, 50257, mixed=True, name="sample_f32_r256_mixed"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def draw(rng):
    """One more call of the same kinds: norms of 1 to 8192 tokens of 64 to 8192 channels; routers and experts for 1 to 512 tokens and
    2 to 128 experts; samples of 1 to 256 rows of 100 to 160000 logits."""
    op = rng.choice(["norm", "norm", "route", "experts", "experts", "experts", "sample", "sample"])
    if op == "norm":
        tokens, channels = _log_int(rng, 1, 8192), _log_int(rng, 64, 8192)
        if rng.random() < 0.6:
            channels = max(64, channels // 64 * 64)
        return _norm(rng.choice(["f16", "bf16", "f32"] if tokens * channels <= 1 << 25 else ["f16", "bf16"]), tokens, channels,
                     rng.choice(["rms", "rms", "layer", "none"]), rng.choice(["none", "none", "rms", "layer"]),
                     rng.choice(["none", "none", "row", "token"]) if tokens * channels <= 1 << 25 else "none", rng.random() < 0.8, rng.random() < 0.4,
                     rng.choice([1.0, 0.9, 2.0]), rng.choice([1.0, 0.22, 0.5]))
    if op == "route":
        experts = _log_int(rng, 2, 128)
        return _route(rng.choice(["f16", "bf16"]), _log_int(rng, 1, 512), 8 * _log_int(rng, 16, 512), experts, rng.randint(1, min(8, experts)),
                      rng.choice(["softmax", "sigmoid"]), rng.random() < 0.5, rng.random() < 0.7, rng.choice([1.0, 2.5]))
    if op == "experts":
        experts = _log_int(rng, 2, 128)
        channels, inter = 16 * _log_int(rng, 16, 256), 16 * _log_int(rng, 8, 128)
        while experts * channels * inter > 128 * 4096 * 1024:
            experts = max(2, experts // 2)
        tokens, top_k = _log_int(rng, 1, 512), rng.randint(1, min(8, experts))
        while tokens * top_k * channels * inter > 500 * 4 * 2048 * 1408:
            tokens = max(1, tokens // 2)
        return _experts(rng.choice(["f16", "bf16"]), tokens, channels, inter, experts, top_k, rng.choice([32, 64, 128]), rng.random() < 0.5,
                        rng.random() < 0.5, rng.choice(["silu", "gelu"]), rng.choice([0.0, 0.5, 1.5]))
    dtype, rows = rng.choice(["f16", "bf16", "f32"]), _log_int(rng, 1, 256)
    vocab = _log_int(rng, 100, min(160000, 256 * 50257 // rows))
    if rng.random() < 0.4:
        return _sample(dtype, rows, vocab, mixed=True)
    return _sample(dtype, rows, vocab, rng.choice([1.0, 0.6, 1.3]), rng.choice([0, 0, 1, 40, 1000]), rng.choice([1.0, 1.0, 0.9, 0.5]),
                   rng.choice([0.0, 0.0, 0.05]))


# ----------------------------------------------------------------------- inputs of a case
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(g, shape, std, dtype):
    return (torch.randn(shape, generator=g, device=DEV) * std).to(dtype)


def _codes(g, n, k, group, zeros, dtype):
    """4-bit weights of n units: codes uint8 [n, k/2] (the even one of a pair in the low bits), scales and zero points [n, groups]."""
    groups = (k + group - 1) // group
    codes = torch.empty((n, k // 2), dtype=torch.uint8, device=DEV)
    scales = torch.empty((n, groups), dtype=dtype, device=DEV)
    zps = torch.empty((n, groups), dtype=torch.uint8, device=DEV) if zeros else None
    rows_at_once = max(1, (1 << 26) // k)   # (the 32-bit values of a whole stack of experts are not kept)
    for r in range(0, n, rows_at_once):
        rows = min(rows_at_once, n - r)
        w = torch.randn((rows, groups * group), generator=g, device=DEV).view(rows, groups, group) / math.sqrt(k)
        if not zeros:
            sc = (w.abs().amax(-1) / 7).to(dtype)
            c = torch.round(w / sc.float()[..., None]).clamp_(-8, 7) + 8
        else:
            lo, hi = w.amin(-1).clamp_(max=0), w.amax(-1).clamp_(min=0)
            sc = ((hi - lo) / 15).to(dtype)
            z = torch.round(-lo / sc.float()).clamp_(0, 15)
            zps[r:r + rows] = z.to(torch.uint8)
            c = (torch.round(w / sc.float()[..., None]) + z[..., None]).clamp_(0, 15)
        c = c.view(rows, groups * group)[:, :k].to(torch.uint8)
        codes[r:r + rows] = c[:, 0::2] | (c[:, 1::2] << 4)
        scales[r:r + rows] = sc
    return codes, scales, zps


def _inputs(case, seed):
    g, dtype = _gen(seed), DTYPES[case["dtype"]]
    if case["op"] == "norm":
        t, c = case["tokens"], case["channels"]
        loud = torch.where(torch.rand(c, generator=g, device=DEV) < 0.01, 20.0, 1.0)
        s = {"x": _normal(g, (t, c), 1.0, dtype),
             "residual": (torch.randn((t, c), generator=g, device=DEV) * loud + 0.3).to(dtype) if case["residual"] else None,
             "gate": _normal(g, (1 if case["gate"] == "row" else t, c), 0.7, dtype) if case["gate"] != "none" else None}
        for which in ("post", "pre"):
            on = case[which] != "none"
            s[which + "_weight"] = 1.0 + 0.2 * torch.randn(c, generator=g, device=DEV) if on else None
            s[which + "_bias"] = 0.1 * torch.randn(c, generator=g, device=DEV) if on and case["bias"] else None
        s["sum"] = torch.empty((t, c), dtype=dtype, device=DEV)
        s["y"] = torch.empty((t, c), dtype=dtype, device=DEV) if case["pre"] != "none" else None
        return s
    if case["op"] == "route":
        t, c, e = case["tokens"], case["channels"], case["experts"]
        return {"x": _normal(g, (t, c), 1.0, dtype), "w": _normal(g, (e, c), 1.5 / math.sqrt(c), dtype),
                "bias": 0.1 * torch.randn(e, generator=g, device=DEV) if case["bias"] else None,
                "chosen": torch.empty((t, case["top_k"]), dtype=torch.int32, device=DEV),
                "weights": torch.empty((t, case["top_k"]), dtype=torch.float32, device=DEV)}
    if case["op"] == "experts":
        t, c, i, e = case["tokens"], case["channels"], case["inter"], case["experts"]
        liked = case["skew"] * torch.randn(e, generator=g, device=DEV)
        scores = liked + torch.randn((t, e), generator=g, device=DEV)
        top, chosen = torch.topk(scores, case["top_k"], dim=1)
        weights = torch.exp(top - top.amax(1, keepdim=True))
        s = {"x": _normal(g, (t, c), 1.0, dtype), "chosen": chosen.to(torch.int32).contiguous(),
             "weights": (weights / weights.sum(1, keepdim=True)).contiguous(),
             "residual": _normal(g, (t, c), 1.0, dtype) if case["residual"] else None, "y": torch.empty((t, c), dtype=dtype, device=DEV)}
        s["up"] = _codes(g, e * 2 * i, c, case["group"], case["zeros"], dtype)      # an expert's gates, then its other units
        s["down"] = _codes(g, e * c, i, case["group"], case["zeros"], dtype)
        return s
    r, v = case["rows"], case["vocab"]
    logits = torch.randn((r, v), generator=g, device=DEV) * 2.0
    peaks = torch.randint(0, v, (r, 24), generator=g, device=DEV)
    heights = torch.empty((r, 24), device=DEV).exponential_(0.35, generator=g) + 3.0
    logits.scatter_add_(1, peaks, heights)
    s = {"logits": logits.to(dtype), "uniform": torch.rand(r, generator=g, device=DEV),
         "tokens": torch.empty(r, dtype=torch.int32, device=DEV), "probs": torch.empty(r, dtype=torch.float32, device=DEV)}
    if case["mixed"]:
        def pick(values, dt=torch.float32):
            return torch.tensor(values, dtype=dt).to(DEV)[torch.randint(0, len(values), (r,), generator=g, device=DEV)]
        s["temperature"], s["top_k"] = pick([0.0, 0.5, 0.8, 1.0, 1.0, 1.5]), pick([0, 0, 0, 20, 100, 2000], torch.int32)
        s["top_p"], s["min_p"] = pick([1.0, 1.0, 0.99, 0.9, 0.6]), pick([0.0, 0.0, 0.0, 0.02, 0.2])
    else:
        s["temperature"] = torch.full((r,), case["temperature"], device=DEV)
        s["top_k"] = torch.full((r,), case["top_k"], dtype=torch.int32, device=DEV) if case["top_k"] else None
        s["top_p"] = torch.full((r,), case["top_p"], device=DEV) if case["top_p"] < 1 else None
        s["min_p"] = torch.full((r,), case["min_p"], device=DEV) if case["min_p"] > 0 else None
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if not own:
        return s
    # what a program keeps from call to call: descriptors, a workspace, weights in the library's own order
    from paper_1904_08368_amd import binding as B
    if case["op"] == "norm":
        kinds = {"none": B.NORM_NONE, "rms": B.NORM_RMS, "layer": B.NORM_LAYER}
        s["d"] = B.residual_norm_desc(s["x"], s["residual"], s["gate"], s["sum"], s["y"], kinds[case["post"]], kinds[case["pre"]],
                                      post_eps=1e-5, pre_eps=1e-5, branch_scale=case["beta"], residual_scale=case["alpha"])
    elif case["op"] == "route":
        s["d"] = B.route_desc(s["x"], s["w"], s["chosen"], B.SCORE_SOFTMAX if case["score"] == "softmax" else B.SCORE_SIGMOID,
                              case["normalize"], case["scale"])
        s["workspace"] = torch.zeros(B.relay_route_workspace_bytes(s["d"]), dtype=torch.uint8, device=DEV)
    elif case["op"] == "experts":
        i, c, e = case["inter"], case["channels"], case["experts"]
        for name, n, k in (("up", e * 2 * i, c), ("down", e * c, i)):
            codes, scales, zps = s[name]
            x, y = (torch.empty((0, w), dtype=scales.dtype, device=DEV) for w in (k, n))
            d = B.qdense_w4_desc(x, y, case["group"], zps)
            s[name + "_packed"] = torch.empty(B.relay_qdense_w4_packed_bytes(d), dtype=torch.uint8, device=DEV)
            B.relay_prepack_qdense_w4(d, codes, scales, zps, s[name + "_packed"])
        s["d"] = B.experts_w4_desc(s["x"], s["chosen"], s["y"], e, i, case["group"], case["zeros"],
                                   B.ACT_SILU if case["act"] == "silu" else B.ACT_GELU, s["residual"])
        s["workspace"] = torch.zeros(B.relay_experts_w4_workspace_bytes(s["d"]), dtype=torch.uint8, device=DEV)
    else:
        s["d"] = B.sample_desc(s["logits"])
        s["workspace"] = torch.zeros(B.relay_sample_workspace_bytes(s["d"]), dtype=torch.uint8, device=DEV)
    return s


# ------------------------------------------------------------------------------- one pass
def run(s):
    return _run_own(s) if own else PLAIN[s["case"]["op"]](s)


def _run_own(s):
    from paper_1904_08368_amd import binding as B
    op = s["case"]["op"]
    if op == "norm":
        B.relay_residual_norm(s["d"], s["x"], s["residual"], s["gate"], s["post_weight"], s["post_bias"], s["pre_weight"], s["pre_bias"],
                              s["sum"], s["y"])
        return (s["sum"], s["y"]) if s["y"] is not None else s["sum"]
    if op == "route":
        B.relay_route(s["d"], s["x"], s["w"], s["bias"], s["chosen"], s["weights"], s["workspace"])
        return s["chosen"], s["weights"]
    if op == "experts":
        B.relay_experts_w4(s["d"], s["x"], s["chosen"], s["weights"], s["up_packed"], s["down_packed"], s["residual"], s["y"], s["workspace"])
        return s["y"]
    B.relay_sample(s["d"], s["logits"], s["temperature"], s["top_k"], s["top_p"], s["min_p"], s["uniform"], s["tokens"], s["probs"], s["workspace"])
    return s["tokens"], s["probs"]


def _normalised(x, kind, weight, bias):
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-5) * weight
    return y if bias is None else y + bias


def _plain_norm(s):
    case, b = s["case"], s["x"].float()
    if case["post"] != "none":
        b = _normalised(b, case["post"], s["post_weight"], s["post_bias"])
    if s["gate"] is not None:
        b = b * s["gate"].float()
    b = b * case["beta"]
    if s["residual"] is not None:
        b = b + s["residual"].float() * case["alpha"]
    total = b.to(s["x"].dtype)
    if case["pre"] == "none":
        return total
    return total, _normalised(b, case["pre"], s["pre_weight"], s["pre_bias"]).to(s["x"].dtype)


def _plain_route(s):
    # (64 bits: a choice between two experts next to each other must not hang on the order of a sum)
    case = s["case"]
    logits = s["x"].double() @ s["w"].double().t()
    if case["score"] == "softmax":
        score = torch.exp(logits - logits.amax(1, keepdim=True))
        score = score / score.sum(1, keepdim=True)
    else:
        score = 1.0 / (1.0 + torch.exp(-logits))
    by = score if s["bias"] is None else score + s["bias"].double()
    chosen = torch.sort(by, dim=1, descending=True, stable=True)[1][:, :case["top_k"]]
    weights = score.gather(1, chosen)
    if case["normalize"]:
        weights = weights / weights.sum(1, keepdim=True)
    return chosen.to(torch.int32), (weights * case["scale"]).float()


def _dequantised(parts, rows, k, group):
    codes, scales, zps = parts
    c = torch.stack([codes[rows] & 15, codes[rows] >> 4], dim=-1).flatten(1).float()
    zero = 8.0 if zps is None else zps[rows].float().repeat_interleave(group, 1)[:, :k]
    return (c - zero) * scales[rows].float().repeat_interleave(group, 1)[:, :k]


def _activated(g, act):
    return g / (1.0 + torch.exp(-g)) if act == "silu" else 0.5 * g * (1.0 + torch.erf(g * math.sqrt(0.5)))


def _plain_experts(s):
    case = s["case"]
    c, i, group = case["channels"], case["inter"], case["group"]
    out = torch.zeros(s["y"].shape, device=DEV) if s["residual"] is None else s["residual"].float()
    x = s["x"].float()
    for e in range(case["experts"]):
        tok, slot = torch.where(s["chosen"] == e)
        if len(tok) == 0:
            continue
        h = x[tok] @ _dequantised(s["up"], slice(e * 2 * i, (e + 1) * 2 * i), c, group).t()
        h = _activated(h[:, :i], case["act"]) * h[:, i:] * s["weights"][tok, slot][:, None]
        out[tok] += h @ _dequantised(s["down"], slice(e * c, (e + 1) * c), i, group).t()
    return out.to(s["y"].dtype)


def _plain_sample(s):
    # (64 bits: a uniform number may fall next to the border between two tokens)
    l = s["logits"].double()
    rows, vocab = l.shape
    best = l.amax(1, keepdim=True)
    t = s["temperature"].double()[:, None]
    greedy = t <= 0
    z = (l - best) / torch.where(greedy, torch.ones_like(t), t)
    v, order = torch.sort(z, dim=1, descending=True, stable=True)
    w = torch.exp(v)
    rank = torch.arange(vocab, device=DEV)[None]
    keep = torch.ones_like(w, dtype=torch.bool)
    if s["top_k"] is not None:
        k = s["top_k"].long()[:, None]
        keep &= (rank < k) | (k <= 0)
    if s["top_p"] is not None:
        p = s["top_p"].double()[:, None]
        mass = torch.cumsum(w * keep, 1)
        # a token belongs to the shortest prefix that reaches p if what lies ahead of it does not
        ahead = torch.cat([torch.zeros((rows, 1), dtype=mass.dtype, device=DEV), mass[:, :-1]], 1)
        keep &= (ahead < p * mass[:, -1:]) | (p >= 1) | (rank == 0)
    if s["min_p"] is not None:
        keep &= w >= s["min_p"].double()[:, None]
    keep = torch.where(greedy, rank == 0, keep)
    kept = w * keep
    cum = torch.cumsum(kept, 1)
    # the uniform number names a place in the kept tokens' mass, the likeliest first
    at = (cum <= s["uniform"].double()[:, None] * cum[:, -1:]).sum(1, keepdim=True)
    return order.gather(1, at)[:, 0].to(torch.int32), (kept.gather(1, at)[:, 0] / cum[:, -1]).float()


PLAIN = {"norm": _plain_norm, "route": _plain_route, "experts": _plain_experts, "sample": _plain_sample}


# ------------------------------------------------------------------- the same in 64 bits
def _norm64(v, kind, weight, bias):
    var, mean = (torch.var_mean(v, dim=-1, unbiased=False, keepdim=True) if kind == "layer"
                 else (v.square().sum(-1, keepdim=True) / v.shape[-1], 0.0))
    out = (v - mean) / torch.sqrt(var + 1e-5) * weight.double()
    return out if bias is None else out + bias.double()


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "norm":
        v = s["x"].double()
        if case["post"] != "none":
            v = _norm64(v, case["post"], s["post_weight"], s["post_bias"])
        v = v * (case["beta"] if s["gate"] is None else case["beta"] * s["gate"].double())
        if s["residual"] is not None:
            v += case["alpha"] * s["residual"].double()
        return (v, _norm64(v, case["pre"], s["pre_weight"], s["pre_bias"])) if case["pre"] != "none" else v
    if case["op"] == "route":
        return None, _exact_route(case, s)
    if case["op"] == "experts":
        return _exact_experts(case, s)
    return None, _exact_sample(s)


def _exact_route(case, s):
    """The weights: experts found one after another, the largest that is left first."""
    logits = torch.matmul(s["x"].double(), s["w"].double().t().contiguous())
    score = torch.softmax(logits, 1) if case["score"] == "softmax" else torch.sigmoid(logits)
    by = score.clone() if s["bias"] is None else score + s["bias"].double()
    out = torch.empty((case["tokens"], case["top_k"]), dtype=torch.float64, device=DEV)
    for i in range(case["top_k"]):
        at = torch.argmax(by, 1, keepdim=True)
        out[:, i:i + 1] = torch.gather(score, 1, at)
        by.scatter_(1, at, -math.inf)
    return out * case["scale"] / (out.sum(1, keepdim=True) if case["normalize"] else 1.0)


def _exact_experts(case, s):
    """Slot by slot of the tokens, an expert's units some at a time, codes as integers and scales group by group."""
    t, c, i = case["tokens"], case["channels"], case["inter"]

    def product(x, parts, first, n):
        codes, scales, zps = parts
        rows = slice(first, first + n)
        w = torch.empty((n, x.shape[1]), dtype=torch.float64, device=DEV)
        w[:, 0::2], w[:, 1::2] = (codes[rows] % 16).double(), (codes[rows] // 16).double()
        which = torch.arange(x.shape[1], device=DEV) // case["group"]
        w -= 8.0 if zps is None else zps[rows].double()[:, which]
        return torch.matmul(x, (w * scales[rows].double()[:, which]).t())

    out = torch.zeros((t, c), dtype=torch.float64, device=DEV)
    x, chosen = s["x"].double(), s["chosen"].cpu().numpy()
    for e in np.unique(chosen):
        for slot in range(case["top_k"]):
            tok = torch.from_numpy(np.nonzero(chosen[:, slot] == e)[0]).to(DEV)
            if len(tok) == 0:
                continue
            g, u = (product(x[tok], s["up"], int(e) * 2 * i + part * i, i) for part in (0, 1))
            a = g * torch.sigmoid(g) if case["act"] == "silu" else torch.nn.functional.gelu(g)
            out[tok] += product(a * u, s["down"], int(e) * c, c) * s["weights"].double()[tok, slot, None]
    return out if s["residual"] is None else out + s["residual"].double()


def _exact_sample(s):
    """Row by row on the host: the probability of the token that the uniform number names."""
    logits, u = s["logits"].double().cpu().numpy(), s["uniform"].double().cpu().numpy()
    get = lambda name, default: np.full(len(u), default) if s[name] is None else s[name].double().cpu().numpy()
    temperature, top_k, top_p, min_p = get("temperature", 1.0), get("top_k", 0), get("top_p", 1.0), get("min_p", 0.0)
    out = np.ones(len(u))
    for r, l in enumerate(logits):
        if temperature[r] <= 0:
            continue
        order = np.argsort(-l, kind="stable")
        w = np.exp((l[order] - l[order[0]]) / temperature[r])
        n = int(top_k[r]) if 0 < top_k[r] < len(l) else len(l)
        if top_p[r] < 1:
            mass = np.cumsum(w[:n])
            n = int(np.searchsorted(mass, top_p[r] * mass[-1], side="left")) + 1
        n = max(1, min(n, int(np.count_nonzero(w >= min_p[r]))))
        cum = np.cumsum(w[:n])
        out[r] = w[int(np.searchsorted(cum, u[r] * cum[-1], side="right"))] / cum[-1]
    return torch.from_numpy(out).to(DEV)


# -------------------------------------------------------------------------- what a pass is
def _active(case):
    """How many experts some token names: of as many choices as there are, spread evenly."""
    e = case["experts"]
    return e * (1.0 - (1.0 - case["top_k"] / e) ** case["tokens"])


def work(case):
    """Each input once and each output once; of the experts only those that some token has chosen."""
    es = {"f16": 2, "bf16": 2, "f32": 4}[case["dtype"]]
    if case["op"] == "norm":
        elems = case["tokens"] * case["channels"]
        tensors = 2 + (1 if case["residual"] else 0) + (1 if case["pre"] != "none" else 0) + (1 if case["gate"] == "token" else 0)
        norms = (case["pre"] != "none") + (case["post"] != "none")
        return {"bytes": tensors * elems * es + case["channels"] * 4 * norms * (2 if case["bias"] else 1) + (case["channels"] * es if case["gate"] == "row" else 0),
                "flops": (4.0 + 6.0 * norms) * elems}
    if case["op"] == "route":
        t, c, e = case["tokens"], case["channels"], case["experts"]
        return {"bytes": (t * c + e * c) * es + t * case["top_k"] * 8, "flops": 2.0 * t * e * c}
    if case["op"] == "experts":
        t, c, i = case["tokens"], case["channels"], case["inter"]
        groups = 2 * i * ((c + case["group"] - 1) // case["group"]) + c * ((i + case["group"] - 1) // case["group"])
        expert = 3 * c * i // 2 + groups * (es + (1 if case["zeros"] else 0))
        return {"bytes": int(_active(case) * expert) + t * c * es * (3 if case["residual"] else 2) + t * case["top_k"] * 8,
                "flops": 6.0 * t * case["top_k"] * c * i}
    n = case["rows"] * case["vocab"]
    return {"bytes": n * es + case["rows"] * 28, "flops": 4.0 * n}
