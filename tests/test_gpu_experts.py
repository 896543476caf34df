"""The experts of a mixture with 4-bit weights against 64 bits: tokens from one to many, every group size, zero points, odd widths, choices that are uneven, out of range
or twice the same, infinite and NaN tokens, strides, one workspace under calls of all sizes."""
import numpy as np
import pytest
import torch

from oracle import decoder as O

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f16": (torch.float16, 2.0 ** -11, 2.0 ** -24), "bf16": (torch.bfloat16, 2.0 ** -8, 2.0 ** -133)}


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1904_08368_amd import binding
    binding.lib()
    return binding


@pytest.fixture(scope="module")
def scratch(B):
    """One workspace for all calls, filled with NaN: nothing is expected of what it holds."""
    return torch.full((256 << 20,), 255, dtype=torch.uint8, device=DEV)


def _np(t):
    return None if t is None else t.detach().cpu().to(torch.float64).numpy()


def _up(a):
    return None if a is None else torch.from_numpy(a).to(DEV)


class Layer:
    """Experts with random codes: scales for outputs of the size of the inputs."""

    def __init__(self, B, dtype, channels, inter, experts, group, zeros=False, seed=0):
        g = np.random.default_rng(seed + channels + 3 * inter + 7 * experts)
        self.dtype, self.channels, self.inter, self.experts, self.group, self.zeros = dtype, channels, inter, experts, group, zeros
        self.packed, self.host = [], []
        for n, k in ((2 * experts * inter, channels), (experts * channels, inter)):
            groups = -(-k // group)
            codes = g.integers(0, 256, (n, k // 2)).astype(np.uint8)
            scales = torch.from_numpy((g.uniform(0.5, 2.0, (n, groups)) / np.sqrt(k) / 5).astype(np.float32)).to(TYPES[dtype][0])
            zp = g.integers(0, 16, (n, groups)).astype(np.uint8) if zeros else None
            x, y = (torch.empty((0, e), dtype=TYPES[dtype][0], device=DEV) for e in (k, n))
            zd = _up(zp)
            d = B.qdense_w4_desc(x, y, group, zd)
            packed = torch.full((d.packed_bytes,), 255, dtype=torch.uint8, device=DEV)
            B.relay_prepack_qdense_w4(d, _up(codes), scales.to(DEV), zd, packed)
            self.packed.append(packed)
            self.host.append((codes, _np(scales), zp))

    def inputs(self, tokens, top_k, seed=0, pad=0, skew=0.0, residual=True):
        g = np.random.default_rng(seed + tokens + top_k)
        up = lambda a: torch.from_numpy(a.astype(np.float32)).to(TYPES[self.dtype][0]).to(DEV)
        order = np.argsort(g.standard_normal((tokens, self.experts)) + skew * np.linspace(-1, 1, self.experts), axis=1)[:, ::-1]
        chosen = order[:, :top_k] if top_k <= self.experts else g.integers(0, self.experts, (tokens, top_k))
        return dict(x=up(g.standard_normal((tokens, self.channels + pad)))[:, :self.channels], chosen=_up(np.ascontiguousarray(chosen).astype(np.int32)),
                    weights=_up(g.dirichlet(np.ones(top_k), tokens).astype(np.float32)), residual=up(g.standard_normal((tokens, self.channels))) if residual else None)


def _run(B, scratch, layer, s, act="silu", y=None):
    y = torch.full_like(s["x"], 77.0, memory_format=torch.contiguous_format) if y is None else y
    d = B.experts_w4_desc(s["x"], s["chosen"], y, layer.experts, layer.inter, layer.group, layer.zeros, B.ACT_SILU if act == "silu" else B.ACT_GELU, s["residual"])
    assert B.relay_experts_w4_workspace_bytes(d) <= scratch.nbytes
    B.relay_experts_w4(d, s["x"], s["chosen"], s["weights"], *layer.packed, s["residual"], y, scratch)
    torch.cuda.synchronize()
    return d, y


def _check(B, scratch, layer, s, act="silu", rows=None):
    d, y = _run(B, scratch, layer, s, act)
    _, u, tiny = TYPES[layer.dtype]
    pick = slice(None) if rows is None else rows
    want, err = O.experts(_np(s["x"])[pick], s["chosen"].cpu().numpy()[pick], _np(s["weights"])[pick], *layer.host, layer.inter, layer.group, act,
                          None if s["residual"] is None else _np(s["residual"])[pick], u, tiny)
    got, tol = _np(y)[pick], err + u * (np.abs(want) + err) + tiny
    assert not np.isnan(got).any() and (np.abs(got - want) <= tol).all(), float((np.abs(got - want) / tol).max())
    return d, y


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("channels,inter,experts,group", [(256, 128, 8, 128), (272, 176, 12, 64), (144, 80, 30, 32)])
def test_tokens(B, scratch, dtype, channels, inter, experts, group):
    layer = Layer(B, dtype, channels, inter, experts, group, zeros=group != 128)
    for tokens in (1, 2, 3, 4, 5, 8, 13, 16, 17, 31, 33, 64, 70, 129):
        for top_k in (1, 2, 4, 8):
            _check(B, scratch, layer, layer.inputs(tokens, top_k), "silu" if top_k & 1 else "gelu")


@pytest.mark.parametrize("channels,inter", [(16, 16), (16, 272), (400, 16), (128, 128), (144, 1040), (2064, 48), (1008, 1408), (4096, 256)])
@pytest.mark.parametrize("group", [32, 64, 96, 128, 256, 8192])
def test_widths_and_groups(B, scratch, channels, inter, group):
    layer = Layer(B, "f16", channels, inter, 5, group, zeros=True)
    for tokens, top_k in ((1, 2), (1, 4), (9, 3), (40, 2)):
        _check(B, scratch, layer, layer.inputs(tokens, top_k))
    layer = Layer(B, "bf16", channels, inter, 3, group)
    _check(B, scratch, layer, layer.inputs(6, 2), "gelu")


@pytest.mark.parametrize("experts", [1, 2, 40])
@pytest.mark.parametrize("channels", [2048, 4096])
def test_few_pairs_of_wide_layers(B, scratch, channels, experts):
    """Up to 8 or 16 of them the second launch adds them up itself."""
    layer = Layer(B, "bf16", channels, 64, experts, 64, zeros=True)
    for tokens, top_k in ((8, 1), (9, 1), (1, 9), (4, 4), (16, 1), (17, 1), (2, 9)):
        _check(B, scratch, layer, layer.inputs(tokens, top_k))


@pytest.mark.parametrize("experts,top_k,tokens", [(1, 1, 1), (1, 1, 50), (2, 2, 100), (4, 4, 513), (128, 8, 1), (128, 8, 16), (200, 1, 64), (1024, 64, 2), (300, 10, 30)])
def test_mixtures(B, scratch, experts, top_k, tokens):
    layer = Layer(B, "f16", 96, 64, experts, 32)
    _check(B, scratch, layer, layer.inputs(tokens, top_k))
    _check(B, scratch, layer, layer.inputs(tokens, top_k, residual=False, skew=5.0))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_all_tokens_on_one_expert(B, scratch, dtype):
    layer = Layer(B, dtype, 160, 112, 40, 32, zeros=True)
    for tokens in (1, 3, 20, 65, 300):
        s = layer.inputs(tokens, 2)
        s["chosen"][:, 0] = 17
        s["chosen"][:, 1] = -1
        _check(B, scratch, layer, s)


@pytest.mark.parametrize("tokens", [1, 4, 30, 200])
def test_choices_that_name_nothing_or_one_expert_twice(B, scratch, tokens):
    layer = Layer(B, "f16", 128, 96, 9, 64)
    g = np.random.default_rng(tokens)
    s = layer.inputs(tokens, 4)
    s["chosen"].copy_(_up(g.integers(-2, 12, (tokens, 4)).astype(np.int32)))
    s["chosen"][0] = torch.tensor([3, 3, 3, 8], dtype=torch.int32)
    s["chosen"][tokens - 1, 1] = 2 ** 31 - 1
    _check(B, scratch, layer, s)
    s["chosen"][tokens - 1] = -1                           # padding: the residual, or zeros
    _, y = _check(B, scratch, layer, s)
    assert torch.equal(y[-1], s["residual"][-1])
    s["residual"] = None
    _, y = _check(B, scratch, layer, s)
    assert (y[-1] == 0).all()
    s["chosen"].fill_(-1)
    _, y = _run(B, scratch, layer, s)
    assert (y == 0).all()


@pytest.mark.parametrize("tokens", [2, 7, 90])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_a_token_keeps_its_infinities(B, scratch, tokens, dtype):
    """An infinity or a NaN in a token changes no other's result, also where they share an expert; an infinity times the weights is what the formula says."""
    layer = Layer(B, dtype, 256, 128, 4, 64)
    s = layer.inputs(tokens, 3)
    _, want = _check(B, scratch, layer, s)
    s["x"] = s["x"].clone()
    s["x"][0, 100], s["x"][tokens - 1, 7] = float("inf"), float("nan")
    _, y = _run(B, scratch, layer, s)
    assert torch.equal(y[1:tokens - 1], want[1:tokens - 1]) and torch.isnan(y[tokens - 1]).all()
    # gates and others of an infinity are +-infinity: silu of the one that is -infinity is a NaN, and a product of the others reaches every channel
    assert not torch.isfinite(y[0]).any()


@pytest.mark.parametrize("tokens", [1, 20])
def test_intermediates_past_the_range(B, scratch, tokens):
    """h past fp16's range is infinite and reaches y with its weights' signs, not as a NaN."""
    layer = Layer(B, "f16", 64, 16, 1, 32)
    s = layer.inputs(tokens, 1, residual=False)
    codes, scales, _ = layer.host[0]
    c = np.empty((32, 64))
    c[:, 0::2], c[:, 1::2] = codes & 15, codes >> 4
    w = (c - 8) * scales.repeat(32, 1)
    x = np.sign(w[0] + w[16]) * 3000.0                 # the first gate and the unit beside it are large, and positive
    s["x"].copy_(torch.from_numpy(np.tile(x.astype(np.float32), (tokens, 1))).half())
    h = (w[:16] @ x) / (1 + np.exp(-np.clip(w[:16] @ x, -700, 700))) * (w[16:] @ x)
    over = np.abs(h) > 65520
    assert over.any() and (np.abs(np.abs(h) - 65520) > 1000).all()
    cd, sd, _ = layer.host[1]
    d = np.empty((64, 16))
    d[:, 0::2], d[:, 1::2] = cd & 15, cd >> 4
    sign = np.sign((d - 8)) * np.sign(h)
    _, y = _run(B, scratch, layer, s)
    for j in range(64):
        signs = {float(v) for v in sign[j, over] if v}
        zero = (d[j, over] == 8).any()                 # (infinity times a weight of zero)
        want = np.nan if zero or len(signs) > 1 else np.inf * signs.pop()
        got = y[:, j].float().cpu().numpy()
        assert (np.isnan(got).all() if np.isnan(want) else (got == want).all()), (j, got, want)


@pytest.mark.parametrize("tokens", [3, 25, 100])
def test_strides_and_alignments(B, scratch, tokens):
    layer = Layer(B, "bf16", 128, 64, 6, 64)
    s = layer.inputs(tokens, 2, pad=24)
    _, want = _check(B, scratch, layer, s)
    flat = torch.full((3 + tokens * 133,), 7.0, dtype=torch.bfloat16, device=DEV)
    y = flat[3:].view(tokens, 133)[:, :128]
    res = torch.zeros_like(flat)[3:].view(tokens, 133)[:, :128]
    res.copy_(s["residual"])
    _run(B, scratch, layer, {**s, "residual": res}, y=y)
    assert torch.equal(y, want) and (flat[:3] == 7).all() and (flat[3:].view(tokens, 133)[:, 128:] == 7).all()
    _run(B, scratch, layer, {**s, "residual": res}, y=res)     # in the place of the residual
    assert torch.equal(res, want)


def test_rows_do_not_hang_on_each_other(B, scratch):
    """A token's result is the same, to the last bit, beside any other tokens of the same call form."""
    layer = Layer(B, "f16", 256, 128, 6, 128)
    s = layer.inputs(120, 2)
    _, y = _run(B, scratch, layer, s)
    other = layer.inputs(120, 2, seed=5)
    for k in ("x", "chosen", "weights", "residual"):
        other[k][17] = s[k][17]
    _, z = _run(B, scratch, layer, other)
    assert torch.equal(y[17], z[17])


def test_more_pairs_than_a_launch_takes(B, scratch):
    layer = Layer(B, "bf16", 64, 32, 70, 32)
    s = layer.inputs(150, 64)
    _check(B, scratch, layer, s)
    s = layer.inputs(4500, 1)
    _check(B, scratch, layer, s)


@pytest.mark.parametrize("tokens", [1, 20])
def test_streams_and_replays(B, scratch, tokens):
    layer = Layer(B, "f16", 512, 256, 16, 128)
    s = layer.inputs(tokens, 4)
    d, want = _check(B, scratch, layer, s)
    own = torch.zeros(B.relay_experts_w4_workspace_bytes(d), dtype=torch.uint8, device=DEV)
    ys = [torch.zeros_like(want) for _ in range(2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(20):   # two at a time, each with its own scratch
        with torch.cuda.stream(side):
            B.relay_experts_w4(d, s["x"], s["chosen"], s["weights"], *layer.packed, s["residual"], ys[0], own)
        B.relay_experts_w4(d, s["x"], s["chosen"], s["weights"], *layer.packed, s["residual"], ys[1], scratch)
    torch.cuda.synchronize()
    assert torch.equal(ys[0], want) and torch.equal(ys[1], want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.relay_experts_w4(d, s["x"], s["chosen"], s["weights"], *layer.packed, s["residual"], ys[0], own)
    chosen = s["chosen"].clone()
    for i in range(3):
        ys[0].fill_(i)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(ys[0], want)
        s["chosen"].copy_((chosen + 1) % 16)                # other choices, replayed, and back
        graph.replay()
        B.relay_experts_w4(d, s["x"], s["chosen"], s["weights"], *layer.packed, s["residual"], ys[1], scratch)
        torch.cuda.synchronize()
        assert torch.equal(ys[0], ys[1]) and not torch.equal(ys[0], want)
        s["chosen"].copy_(chosen)


def test_no_tokens(B):
    layer = Layer(B, "f16", 64, 32, 2, 32)
    s = {k: v[:0] for k, v in layer.inputs(1, 1).items()}
    y = torch.empty_like(s["x"])
    d = B.experts_w4_desc(s["x"], s["chosen"], y, 2, 32, 32, residual=s["residual"])
    B.relay_experts_w4(d, s["x"], s["chosen"], s["weights"], *layer.packed, s["residual"], y, None)
