"""The router of a mixture of experts against 64 bits: choices equal, weights to one rounding; tokens from one to many, experts from one to the most, experts that tie,
NaN and infinite tokens, one workspace under calls of all sizes."""
import numpy as np
import pytest
import torch

from oracle import decoder as O

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1904_08368_amd import binding
    binding.lib()
    return binding


@pytest.fixture(scope="module")
def scratch(B):
    """One workspace for all calls, cleared once."""
    return torch.zeros(64 << 20, dtype=torch.uint8, device=DEV)


def _np(t):
    return t.detach().cpu().to(torch.float64).numpy()


def _case(dtype, tokens, channels, experts, seed=0, pad=0, std=1.5):
    g = np.random.default_rng(seed + tokens + 3 * channels + 7 * experts)
    up = lambda a: torch.from_numpy(a.astype(np.float32)).to(TYPES[dtype]).to(DEV)
    x = up(g.standard_normal((tokens, channels + pad)))[:, :channels]
    return x, up(g.standard_normal((experts, channels)) * std / channels ** 0.5), torch.from_numpy((0.2 * g.standard_normal(experts)).astype(np.float32)).to(DEV)


def _check(B, scratch, x, w, bias, top_k, score="softmax", normalize=True, scale=1.0):
    tokens = x.shape[0]
    chosen, weights = torch.full((tokens + 1, top_k), -9, dtype=torch.int32, device=DEV), torch.full((tokens + 1, top_k), -9.0, device=DEV)
    d = B.route_desc(x, w, chosen[:tokens], 0 if score == "softmax" else 1, normalize, scale)
    assert B.relay_route_workspace_bytes(d) <= scratch.nbytes
    B.relay_route(d, x, w, bias, chosen, weights, scratch)
    torch.cuda.synchronize()
    want, ref = O.route(_np(x), _np(w), top_k, score, None if bias is None else bias.cpu().numpy(), normalize, float(np.float32(scale)))
    assert np.array_equal(chosen[:tokens].cpu().numpy(), want)
    # (exact but for one rounding: 2^-24, and sums and exponentials in 64 bits, some thousand times 2^-53)
    got = _np(weights[:tokens])
    assert (np.abs(got - ref) <= 2.0 ** -24 * 1.0001 * np.abs(ref) + 2.0 ** -150).all(), np.abs(got / ref - 1).max()
    assert (chosen[tokens:] == -9).all() and (weights[tokens:] == -9).all()
    return d, chosen[:tokens], weights[:tokens]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("tokens", [1, 2, 5, 15, 16, 17, 33, 64, 65, 127, 200, 513])
@pytest.mark.parametrize("channels,experts,top_k", [(128, 8, 2), (1000, 60, 4), (4096, 64, 8), (2056, 128, 6)])
def test_sizes(B, scratch, dtype, tokens, channels, experts, top_k):
    x, w, bias = _case(dtype, tokens, channels, experts)
    _check(B, scratch, x, w, None, top_k)
    _check(B, scratch, x, w, bias, top_k, "sigmoid", scale=2.5)


@pytest.mark.parametrize("experts,top_k", [(1, 1), (2, 1), (2, 2), (3, 3), (63, 10), (64, 64), (65, 64), (256, 8), (257, 8), (1000, 30), (1024, 64)])
@pytest.mark.parametrize("tokens", [1, 20, 100])
def test_experts(B, scratch, experts, top_k, tokens):
    x, w, bias = _case("bf16", tokens, 264, experts)
    for score in ("softmax", "sigmoid"):
        for b in (None, bias):
            for normalize in (True, False):
                _check(B, scratch, x, w, b, top_k, score, normalize, 0.5)


@pytest.mark.parametrize("channels", [8, 16, 24, 2040, 2048, 2064, 8192, 20000])
@pytest.mark.parametrize("tokens", [3, 90])
def test_channels_and_strides(B, scratch, channels, tokens):
    for pad in (0, 8):
        _check(B, scratch, *_case("f16", tokens, channels, 20, pad=pad), 3)


@pytest.mark.parametrize("tokens", [4, 70])
def test_experts_that_tie(B, scratch, tokens):
    """Experts with the same weights: the one with the lower number first."""
    x, w, _ = _case("f16", tokens, 512, 40)
    w[7], w[30], w[31], w[39] = w[3], w[3], w[8], w[0]
    _check(B, scratch, x, w, None, 12)
    w[:] = w[0]
    _, chosen, weights = _check(B, scratch, x, w, None, 5)
    assert (chosen == torch.arange(5, device=DEV, dtype=torch.int32)).all() and (weights == 0.2).all()


@pytest.mark.parametrize("tokens", [6, 70])
def test_scores_at_the_ends(B, scratch, tokens):
    """Logits of thousands: scores that are 0 and 1, and sums of nothing."""
    x, w, bias = _case("bf16", tokens, 256, 16, std=3000.0)
    _check(B, scratch, x, w, None, 4)
    _check(B, scratch, x, w, bias, 4, "sigmoid")
    w[:] = -w.abs()
    x = x.abs()
    _, _, weights = _check(B, scratch, x, w, bias, 4, "sigmoid")
    assert (weights == 0).all()


@pytest.mark.parametrize("tokens", [5, 80])
def test_a_token_keeps_its_nan(B, scratch, tokens):
    x, w, bias = _case("f16", tokens, 640, 24)
    d, chosen, weights = _check(B, scratch, x, w, bias, 4)
    x = x.clone()
    x[1, 5], x[3, 600] = float("nan"), float("inf")
    again, more = torch.zeros_like(chosen), torch.zeros_like(weights)
    B.relay_route(d, x, w, bias, again, more, scratch)
    torch.cuda.synchronize()
    rows = [r for r in range(tokens) if r not in (1, 3)]
    assert torch.equal(again[rows], chosen[rows]) and torch.equal(more[rows], weights[rows])
    assert torch.isnan(more[1]).all() and again[1].tolist() == [0, 1, 2, 3]
    assert ((again >= 0) & (again < 24)).all()


def test_more_tokens_than_a_launch_takes(B, scratch):
    x, w, bias = _case("bf16", 4096 + 37, 64, 12)
    _check(B, scratch, x, w, bias, 3)
    _check(B, scratch, x[:50], w, bias, 3)


def test_streams_and_replays(B, scratch):
    x, w, bias = _case("f16", 40, 1024, 64)
    d, chosen, weights = _check(B, scratch, x, w, bias, 6)
    other = torch.zeros(B.relay_route_workspace_bytes(d), dtype=torch.uint8, device=DEV)
    outs = [(torch.zeros_like(chosen), torch.zeros_like(weights)) for _ in range(2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(20):   # two at a time, each with its own scratch
        with torch.cuda.stream(side):
            B.relay_route(d, x, w, bias, *outs[0], other)
        B.relay_route(d, x, w, bias, *outs[1], scratch)
    torch.cuda.synchronize()
    for c, v in outs:
        assert torch.equal(c, chosen) and torch.equal(v, weights)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.relay_route(d, x, w, bias, *outs[0], other)
    for i in range(3):
        outs[0][0].fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0][0], chosen) and torch.equal(outs[0][1], weights)


def test_no_tokens(B):
    x, w, _ = _case("f16", 1, 64, 4)
    chosen = torch.zeros((0, 2), dtype=torch.int32, device=DEV)
    B.relay_route(B.route_desc(x[:0], w, chosen), x[:0], w, None, chosen, torch.zeros((0, 2), device=DEV), None)
