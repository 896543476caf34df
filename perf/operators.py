"""The operators of an attention layer that is served from a paged cache, as timed cases.

Such a layer is four launches: a dense product with 4-bit weights that makes the queries, keys and values
of the new tokens; the rotation of queries and keys by their positions, which also stores keys and values into the
pages of the cache; the attention of the new tokens over the cache; and a dense product back to the
residual stream.  A case is one call of one of them, on what a program has in hand before the call: tensors on
the GPU, page tables, a table of cosines and sines, packed weights, descriptors, a workspace.

Activations are normal; queries and keys give scores of a standard deviation of about 2 to 3, as trained heads do;
4-bit codes and their group scales come from normal weights by the largest magnitude of each group.
Pages lie in the cache in random order, and slots that no token has reached yet hold what an earlier
sequence left there.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------------------------- cases
def _append(dtype, tokens, q_heads, kv_heads, head_dim, rotary_dim, style, page_size, first, name=None):
    """`tokens` new tokens of one sequence from position `first` on: rotate q and k, store k and v."""
    c = {"op": "append", "dtype": dtype, "tokens": tokens, "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim,
         "rotary_dim": rotary_dim, "style": style, "page_size": page_size, "first": first}
    return dict(c, name=name) if name else c


def _rope(dtype, tokens, heads, head_dim, rotary_dim, style, inverse, name=None):
    """Rotation of a tensor outside a cache; inverse: the gradient of the rotation."""
    c = {"op": "rope", "dtype": dtype, "tokens": tokens, "heads": heads, "head_dim": head_dim, "rotary_dim": rotary_dim,
         "style": style, "inverse": inverse}
    return dict(c, name=name) if name else c


def _attention(dtype, batch, new, kv, q_heads, kv_heads, head_dim, page_size, causal=True, window=0, ragged=True, name=None):
    """`batch` sequences of up to `kv` cached tokens, the last up to `new` of which are this call's."""
    c = {"op": "attention", "dtype": dtype, "batch": batch, "new": new, "kv": kv, "q_heads": q_heads, "kv_heads": kv_heads,
         "head_dim": head_dim, "page_size": page_size, "causal": causal, "window": window, "ragged": ragged}
    return dict(c, name=name) if name else c


def _w4(dtype, m, n, k, group, zeros=False, bias=False, residual=False, name=None):
    c = {"op": "w4", "dtype": dtype, "m": m, "n": n, "k": k, "group": group, "zeros": zeros, "bias": bias, "residual": residual}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one user, one token: latency of a decode step's smallest launch
        _append("f16", 1, 32, 8, 128, 128, "half", 16, 1023, name="append_f16_t1"),
        # a prompt of odd length with a partly rotated head of 80 channels in adjacent pairs, far into a long context
        _append("bf16", 5003, 24, 8, 80, 32, "interleaved", 32, 60001, name="append_bf16_t5003_partial"),
        # the gradient of the rotation in a training step, in 32 bits
        _rope("f32", 4096, 32, 128, 128, "half", True, name="rope_grad_f32_t4096"),
        # one user's next token over a short chat
        _attention("f16", 1, 1, 700, 32, 8, 128, 16, ragged=False, name="decode_f16_b1_kv700"),
        # a full batch of users of all lengths, eight query heads to a key head
        _attention("bf16", 48, 1, 8192, 64, 8, 128, 64, name="decode_bf16_b48_kv8192"),
        # one user's next token over a very long document
        _attention("f16", 1, 1, 100001, 32, 4, 128, 16, ragged=False, name="decode_f16_b1_kv100001"),
        # chunks of some prompts over what is cached of them, sliding window, heads of 64
        _attention("bf16", 3, 509, 9001, 16, 4, 64, 16, window=4096, name="chunk_bf16_b3_window"),
        # a whole long prompt at once
        _attention("f16", 1, 8192, 8192, 16, 4, 128, 64, ragged=False, name="prompt_f16_8192"),
        # the projection back to the residual stream for one token: latency
        _w4("f16", 1, 4096, 4096, 128, residual=True, name="w4_f16_m1"),
        # a handful of tokens, odd widths, groups of 64 of which the last is short, zero points
        _w4("bf16", 6, 10007, 5000, 64, zeros=True, bias=True, name="w4_bf16_m6_odd"),
        # a large matrix for one token: the weights' bytes are all there is
        _w4("bf16", 1, 32768, 8192, 128, name="w4_bf16_m1_large"),
        # a chunk of a prompt: a matrix product
        _w4("f16", 1500, 8192, 4096, 128, name="w4_f16_m1500"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def draw(rng):
    """One more call of the same kinds: 1 to 8192 rotated tokens, 1 to 48 sequences with 1 to 100001 cached tokens, products
    of 1 to 1500 rows; any of the types, head sizes, group sizes, page sizes and masks."""
    op = rng.choice(["append", "rope", "attention", "attention", "attention", "w4", "w4", "w4"])
    dtype = rng.choice(["f16", "bf16"])
    if op in ("append", "rope"):
        dtype = rng.choice(["f16", "bf16", "f32"])
        head_dim = rng.choice([64, 80, 96, 128, 256])
        rotary_dim = head_dim if rng.random() < 0.6 else rng.choice([16, 32, head_dim // 2])
        style = rng.choice(["half", "interleaved"])
        tokens = _log_int(rng, 1, 8192)
        kv_heads = rng.choice([1, 2, 4, 8])
        if op == "rope":
            return _rope(dtype, tokens, kv_heads * rng.choice([1, 3, 4]), head_dim, rotary_dim, style, rng.random() < 0.5)
        return _append(dtype, tokens, kv_heads * rng.choice([1, 3, 4, 8]), kv_heads, head_dim, rotary_dim, style,
                       rng.choice([1, 16, 24, 32, 64, 128]), _log_int(rng, 1, 100000))
    if op == "attention":
        kv_heads = rng.choice([1, 2, 4, 8])
        head_dim = rng.choice([64, 80, 96, 128, 256])
        page_size = rng.choice([1, 16, 24, 32, 64, 128])
        window = rng.choice([0, 0, 0, 1, 100, 1024])
        kind = rng.choice(["decode", "decode", "chunk", "prompt"])
        if kind == "decode":
            batch, new = _log_int(rng, 1, 48), rng.choice([1, 1, 1, 2, 5])
            kv = _log_int(rng, new, max(8, min(100001, 400000 // batch)))
        elif kind == "chunk":
            batch, new = _log_int(rng, 1, 8), _log_int(rng, 2, 700)
            kv = _log_int(rng, new, max(new, 30000 // batch))
        else:
            batch = _log_int(rng, 1, 4)
            new = kv = _log_int(rng, 16, 5000 // batch)
        return _attention(dtype, batch, new, max(kv, new), kv_heads * rng.choice([1, 3, 4, 8]), kv_heads, head_dim, page_size,
                          rng.random() < 0.85, window, rng.random() < 0.7)
    m, n, k = _log_int(rng, 1, 1500), _log_int(rng, 64, 32768), 8 * _log_int(rng, 8, 1024)
    while m * n * k > 1500 * 8192 * 4096 or n * k > 32768 * 8192:
        n = max(64, n // 2 + 1)
    return _w4(dtype, m, n, k, rng.choice([32, 64, 128]), rng.random() < 0.5, rng.random() < 0.5, rng.random() < 0.5)


# ----------------------------------------------------------------------- inputs of a case
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(g, shape, std, dtype):
    return (torch.randn(shape, generator=g, device=DEV) * std).to(dtype)


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype).to(DEV)


def _cos_sin(first, rows, rotary_dim):
    """Rows of the table from position `first` on: base 10000, the frequencies stretched by 4 as for a context four times as long."""
    f = 10000.0 ** (-torch.arange(0, rotary_dim, 2, device=DEV, dtype=torch.float64) / rotary_dim) / 4.0
    a = (first + torch.arange(rows, device=DEV, dtype=torch.float64))[:, None] * f
    return torch.stack([a.cos(), a.sin()], dim=-1).float()


def _lengths(case):
    """(new tokens, cached tokens) of every sequence: the same for every seed, so that a case is one amount of work."""
    rng = random.Random(case["batch"] * 1000003 + case["new"] * 1009 + case["kv"])
    out = []
    for b in range(case["batch"]):
        if case["ragged"] and b:
            new = rng.randint(min(case["new"], max(1, case["new"] // 2)), case["new"])
            out.append((new, max(new, rng.randint(max(1, case["kv"] // 4), case["kv"]))))
        else:
            out.append((case["new"], case["kv"]))
    return out


def _inputs(case, seed):
    g, dtype = _gen(seed), DTYPES[case["dtype"]]
    if case["op"] == "rope":
        s = {"x": _normal(g, (case["tokens"], case["heads"], case["head_dim"]), 1.0, dtype)}
        s["table"] = _cos_sin(0, case["tokens"], case["rotary_dim"])
        s["positions"] = torch.randint(0, case["tokens"], (case["tokens"],), generator=g, device=DEV, dtype=torch.int32)
        s["y"] = torch.empty_like(s["x"])
        return s
    if case["op"] == "append":
        t, d, ps = case["tokens"], case["head_dim"], case["page_size"]
        hq, hkv = case["q_heads"], case["kv_heads"]
        # q, k and v are ranges of the rows that one projection writes
        qkv = _normal(g, (t, (hq + 2 * hkv) * d), 1.0, dtype)
        q, k, v = qkv.split([hq * d, hkv * d, hkv * d], dim=1)
        pages = (case["first"] % ps + t + ps - 1) // ps + 3
        cache = _normal(g, (2, pages, ps, hkv, d), 1.0, dtype)
        order = torch.randperm(pages, generator=g, device=DEV)
        at = case["first"] % ps + torch.arange(t, device=DEV)
        slots = (order[at // ps] * ps + at % ps).to(torch.int32)
        return {"q": q.view(t, hq, d), "k": k.view(t, hkv, d), "v": v.view(t, hkv, d), "k_cache": cache[0], "v_cache": cache[1],
                "slots": slots, "slots_long": slots.long(), "table": _cos_sin(case["first"], t, case["rotary_dim"]),
                "positions": torch.arange(t, device=DEV, dtype=torch.int32),
                "q_out": torch.empty((t, hq, d), dtype=dtype, device=DEV)}
    if case["op"] == "attention":
        lens = _lengths(case)
        d, ps = case["head_dim"], case["page_size"]
        per_seq = max((kv + ps - 1) // ps for _, kv in lens)
        need = sum((kv + ps - 1) // ps for _, kv in lens)
        cache = _normal(g, (2, need + 2, ps, case["kv_heads"], d), 1.0, dtype)
        order = torch.randperm(need + 2, generator=g, device=DEV).to(torch.int32)
        table = torch.zeros((case["batch"], per_seq), dtype=torch.int32, device=DEV)
        at = 0
        for b, (_, kv) in enumerate(lens):
            n = (kv + ps - 1) // ps
            table[b, :n] = order[at:at + n]
            at += n
        starts = [0]
        for new, _ in lens:
            starts.append(starts[-1] + new)
        q = _normal(g, (starts[-1], case["q_heads"], d), 2.5, dtype)
        return {"q": q, "k_cache": cache[0], "v_cache": cache[1], "page_table": table, "q_starts": _ints(starts),
                "kv_lens": _ints([kv for _, kv in lens]), "lens": lens, "scale": 1.0 / math.sqrt(d), "out": torch.empty_like(q)}
    m, n, k, group = case["m"], case["n"], case["k"], case["group"]
    groups = (k + group - 1) // group
    # (weights a slab of rows at a time: the 32-bit values of a whole large matrix are not kept)
    codes = torch.empty((n, k), dtype=torch.uint8, device=DEV)
    scales = torch.empty((n, groups), dtype=dtype, device=DEV)
    zeros = torch.empty((n, groups), dtype=torch.uint8, device=DEV) if case["zeros"] else None
    for r in range(0, n, 8192):
        rows = min(8192, n - r)
        w = torch.randn((rows, groups * group), generator=g, device=DEV).view(rows, groups, group) / math.sqrt(k)
        if zeros is None:
            sc = (w.abs().amax(-1) / 7).to(dtype)
            c = torch.round(w / sc.float()[..., None]).clamp_(-8, 7) + 8
        else:
            lo, hi = w.amin(-1).clamp_(max=0), w.amax(-1).clamp_(min=0)
            sc = ((hi - lo) / 15).to(dtype)
            z = torch.round(-lo / sc.float()).clamp_(0, 15)
            zeros[r:r + rows] = z.to(torch.uint8)
            c = (torch.round(w / sc.float()[..., None]) + z[..., None]).clamp_(0, 15)
        codes[r:r + rows] = c.view(rows, groups * group)[:, :k].to(torch.uint8)
        scales[r:r + rows] = sc
    s = {"x": _normal(g, (m, k), 1.0, dtype), "codes": codes[:, 0::2] | (codes[:, 1::2] << 4), "scales": scales, "zeros": zeros}
    s["bias"] = _normal(g, (n,), 0.1, torch.float32) if case["bias"] else None
    s["residual"] = _normal(g, (m, n), 1.0, dtype) if case["residual"] else None
    s["y"] = torch.empty((m, n), dtype=dtype, device=DEV)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if not own:
        return s
    # what a program keeps from call to call: descriptors, a workspace, weights in the library's own order
    from paper_1904_08368_amd import binding as B
    if case["op"] in ("append", "rope"):
        style = B.ROPE_HALF if case["style"] == "half" else B.ROPE_INTERLEAVED
        if case["op"] == "rope":
            s["d"] = B.rope_desc(s["x"], s["table"], s["y"], style, case["inverse"])
        else:
            s["d"] = B.rope_append_desc(s["q"], s["k"], s["v"], s["table"], s["q_out"], s["k_cache"], style)
    elif case["op"] == "attention":
        s["d"] = B.paged_attention_desc(s["q"], s["k_cache"], s["page_table"], s["out"], max(n for n, _ in s["lens"]),
                                        max(n for _, n in s["lens"]), s["scale"], case["causal"], case["window"])
        s["workspace"] = torch.zeros(B.relay_paged_attention_workspace_bytes(s["d"]), dtype=torch.uint8, device=DEV)
    else:
        s["d"] = B.qdense_w4_desc(s["x"], s["y"], case["group"], s["zeros"], s["bias"], s["residual"])
        s["packed"] = torch.empty(B.relay_qdense_w4_packed_bytes(s["d"]), dtype=torch.uint8, device=DEV)
        B.relay_prepack_qdense_w4(s["d"], s["codes"], s["scales"], s["zeros"], s["packed"])
    return s


# ------------------------------------------------------------------------------- one pass
def run(s):
    return _run_own(s) if own else PLAIN[s["case"]["op"]](s)


def _run_own(s):
    from paper_1904_08368_amd import binding as B
    op = s["case"]["op"]
    if op == "rope":
        B.relay_rope(s["d"], s["x"], s["table"], s["positions"], s["y"])
        return s["y"]
    if op == "append":
        B.relay_rope_append(s["d"], s["q"], s["k"], s["v"], s["table"], s["positions"], s["slots"], s["q_out"], s["k_cache"], s["v_cache"])
        return s["q_out"], s["k_cache"], s["v_cache"]
    if op == "attention":
        B.relay_paged_attention(s["d"], s["q"], s["k_cache"], s["v_cache"], s["page_table"], s["q_starts"], s["kv_lens"], s["out"],
                                s["workspace"])
        return s["out"]
    B.relay_qdense_w4(s["d"], s["x"], s["packed"], s["bias"], s["residual"], s["y"])
    return s["y"]


def _rotate(x, table, positions, style, inverse):
    cs = table[positions]
    c, sn = cs[:, None, :, 0], cs[:, None, :, 1]
    if inverse:
        sn = -sn
    rd = 2 * table.shape[1]
    y = x.float()
    a, b = (y[..., :rd // 2], y[..., rd // 2:rd]) if style == "half" else (y[..., 0:rd:2], y[..., 1:rd:2])
    ra, rb = a * c - b * sn, b * c + a * sn
    turned = torch.cat([ra, rb], dim=-1) if style == "half" else torch.stack([ra, rb], dim=-1).flatten(-2)
    return torch.cat([turned, y[..., rd:]], dim=-1).to(x.dtype)


def _plain_rope(s):
    return _rotate(s["x"], s["table"], s["positions"], s["case"]["style"], s["case"]["inverse"])


def _plain_append(s):
    style = s["case"]["style"]
    q = _rotate(s["q"], s["table"], s["positions"], style, False)
    s["k_cache"].view(-1, *s["k"].shape[1:])[s["slots_long"]] = _rotate(s["k"], s["table"], s["positions"], style, False)
    s["v_cache"].view(-1, *s["v"].shape[1:])[s["slots_long"]] = s["v"]
    return q, s["k_cache"], s["v_cache"]


def _allowed(case, new, kv, rows):
    """Keys that new tokens `rows` of a sequence see."""
    p = (kv - new + rows)[:, None]
    j = torch.arange(kv, device=DEV)[None, :]
    ok = (j <= p) if case["causal"] else torch.ones_like(j <= p)
    return ok & (j > p - case["window"]) if case["window"] else ok


def _plain_attention(s):
    case = s["case"]
    group, ps = case["q_heads"] // case["kv_heads"], case["page_size"]
    out = torch.empty_like(s["q"])
    at = 0
    for b, (new, kv) in enumerate(s["lens"]):
        pages = s["page_table"][b, :(kv + ps - 1) // ps].long()
        for h in range(case["kv_heads"]):
            k = s["k_cache"][pages, :, h].flatten(0, 1)[:kv].float()
            v = s["v_cache"][pages, :, h].flatten(0, 1)[:kv].float()
            step = max(1, (1 << 27) // (kv * group))
            for r in range(0, new, step):
                rows = torch.arange(r, min(new, r + step), device=DEV)
                q = s["q"][at + r:at + r + step, h * group:(h + 1) * group][:len(rows)].float()
                x = (q.reshape(-1, q.shape[-1]) @ k.t()).view(len(rows), group, kv) * s["scale"]
                x = x.masked_fill(~_allowed(case, new, kv, rows)[:, None], -math.inf)
                x = torch.exp(x - x.amax(-1, keepdim=True))
                o = (x.view(-1, kv) @ v).view(len(rows), group, -1) / x.sum(-1, keepdim=True)
                out[at + r:at + r + len(rows), h * group:(h + 1) * group] = o.to(out.dtype)
        at += new
    return out


def _plain_w4(s):
    case = s["case"]
    codes = torch.stack([s["codes"] & 15, s["codes"] >> 4], dim=-1).flatten(1)
    n, k = codes.shape
    zero = 8.0 if s["zeros"] is None else s["zeros"].float().repeat_interleave(case["group"], 1)[:, :k]
    w = (codes.float() - zero) * s["scales"].float().repeat_interleave(case["group"], 1)[:, :k]
    y = s["x"].float() @ w.t()
    if s["bias"] is not None:
        y = y + s["bias"]
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(s["x"].dtype)


PLAIN = {"rope": _plain_rope, "append": _plain_append, "attention": _plain_attention, "w4": _plain_w4}


# ------------------------------------------------------------------- the same in 64 bits
def _turn64(x, cs, style, sign):
    """Complex product: channel pairs times cos + i sin, conjugated for the gradient."""
    rd = 2 * cs.shape[1]
    z = torch.complex(cs[..., 0].double(), sign * cs[..., 1].double())[:, None]
    y = x.double().clone()
    part = y[..., :rd]
    pairs = part.unflatten(-1, (2, rd // 2)).movedim(-2, -1) if style == "half" else part.unflatten(-1, (rd // 2, 2))
    w = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * z)
    y[..., :rd] = w.movedim(-1, -2).flatten(-2) if style == "half" else w.flatten(-2)
    return y


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "rope":
        return _turn64(s["x"], s["table"][s["positions"].long()], case["style"], -1.0 if case["inverse"] else 1.0)
    if case["op"] == "append":
        cs = s["table"][s["positions"].long()]
        kc, vc = s["k_cache"].double(), s["v_cache"].double()
        page, at = s["slots_long"] // case["page_size"], s["slots_long"] % case["page_size"]
        kc[page, at] = _turn64(s["k"], cs, case["style"], 1.0)
        vc[page, at] = s["v"].double()
        return _turn64(s["q"], cs, case["style"], 1.0), kc, vc
    if case["op"] == "attention":
        return _exact_attention(case, s)
    m, n, k = case["m"], case["n"], case["k"]
    out = torch.empty((m, n), dtype=torch.float64, device=DEV)
    which = torch.arange(k, device=DEV) // case["group"]
    x = s["x"].double()
    for r in range(0, n, 4096):
        rows = slice(r, min(n, r + 4096))
        c = torch.empty((rows.stop - r, k), dtype=torch.float64, device=DEV)
        c[:, 0::2] = (s["codes"][rows] % 16).double()
        c[:, 1::2] = (s["codes"][rows] // 16).double()
        c -= 8.0 if s["zeros"] is None else s["zeros"][rows].double()[:, which]
        c *= s["scales"][rows].double()[:, which]
        out[:, rows] = torch.matmul(x, c.t())
    if s["bias"] is not None:
        out += s["bias"].double()
    if s["residual"] is not None:
        out += s["residual"].double()
    return out


def _exact_attention(case, s):
    """Head by head of the queries, some rows at a time, keys looked up one by one through the page table."""
    ps, group = case["page_size"], case["q_heads"] // case["kv_heads"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    start = 0
    for b, (new, kv) in enumerate(s["lens"]):
        j = torch.arange(kv, device=DEV)
        page, slot = s["page_table"][b].long()[j // ps], j % ps
        for h in range(case["q_heads"]):
            k, v = s["k_cache"][page, slot, h // group].double(), s["v_cache"][page, slot, h // group].double()
            for r in range(0, new, 4096):
                i = torch.arange(r, min(r + 4096, new), device=DEV)
                pos = (kv - new + i).unsqueeze(1)
                sees = torch.ones((len(i), kv), dtype=torch.bool, device=DEV)
                if case["causal"]:
                    sees &= j <= pos
                if case["window"]:
                    sees &= pos - j < case["window"]
                x = torch.matmul(s["q"][start + r:start + r + len(i), h].double() * s["scale"], k.t())
                p = torch.softmax(torch.where(sees, x, torch.full_like(x, -math.inf)), dim=-1)
                out[start + r:start + r + len(i), h] = torch.matmul(p, v)
        start += new
    return out


# -------------------------------------------------------------------------- what a pass is
def work(case):
    """Each input once and each output once; of a cache only the keys and values that some new token sees, or the
    slots that are written."""
    es = {"f16": 2, "bf16": 2, "f32": 4}[case["dtype"]]
    if case["op"] == "rope":
        elems, pairs = case["tokens"] * case["heads"] * case["head_dim"], case["rotary_dim"] // 2
        return {"bytes": 2 * elems * es + case["tokens"] * (8 * pairs + 4), "flops": 6.0 * case["tokens"] * case["heads"] * pairs}
    if case["op"] == "append":
        t, pairs = case["tokens"], case["rotary_dim"] // 2
        elems = t * (case["q_heads"] + 2 * case["kv_heads"]) * case["head_dim"]
        return {"bytes": 2 * elems * es + t * (8 * pairs + 8), "flops": 6.0 * t * (case["q_heads"] + case["kv_heads"]) * pairs}
    if case["op"] == "attention":
        keys = seen = tokens = 0
        for new, kv in _lengths(case):
            p = np.arange(kv - new, kv, dtype=np.int64)
            hi = p + 1 if case["causal"] else np.full(new, kv, dtype=np.int64)
            lo = np.maximum(0, p + 1 - case["window"]) if case["window"] else np.zeros(new, dtype=np.int64)
            seen += int((hi - lo).sum())
            keys += int(hi.max() - lo.min())
            tokens += new
        d = case["head_dim"]
        return {"bytes": es * d * (2 * keys * case["kv_heads"] + 2 * tokens * case["q_heads"]),
                "flops": 4.0 * d * case["q_heads"] * seen}
    m, n, k = case["m"], case["n"], case["k"]
    groups = (k + case["group"] - 1) // case["group"]
    nbytes = n * k // 2 + n * groups * (es + (1 if case["zeros"] else 0)) + (m * k + m * n) * es
    nbytes += 4 * n if case["bias"] else 0
    nbytes += m * n * es if case["residual"] else 0
    return {"bytes": nbytes, "flops": 2.0 * m * n * k}
