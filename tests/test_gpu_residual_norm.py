"""Norms of a block with its gate and the residual stream against 64 bits: every kind, rows from one element to the longest, any alignment, strides,
outputs in the place of inputs, rows that are all alike or hold a NaN, captured and replayed calls."""
import numpy as np
import pytest
import torch

from oracle import decoder as O

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f16": (torch.float16, 2.0 ** -11, 2.0 ** -25), "bf16": (torch.bfloat16, 2.0 ** -8, 2.0 ** -134), "f32": (torch.float32, 2.0 ** -24, 2.0 ** -150)}
KINDS = {None: 0, "rms": 1, "layer": 2}


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1904_08368_amd import binding
    return binding


def _np(t):
    return None if t is None else t.detach().cpu().to(torch.float64).numpy()


def _close(got, want, err, dtype):
    _, u, tiny = TYPES[dtype]
    got, tol = _np(got), err + u * (np.abs(want) + err) + tiny
    assert not np.isnan(got).any() and (np.abs(got - want) <= tol).all(), float((np.abs(got - want) / tol).max())


def _inputs(dtype, tokens, channels, residual=True, gate=None, mean=0.0, pad=0, off=0, seed=0):
    """Rows `pad` elements apart, the first `off` elements behind an aligned address."""
    g = np.random.default_rng(seed + 7 * tokens + channels)
    tt = TYPES[dtype][0]

    def rows(n, scale, shift):
        flat = torch.full((off + n * (channels + pad),), 3.0, dtype=tt, device=DEV)
        t = flat[off:].view(n, channels + pad)[:, :channels]
        t.copy_(torch.from_numpy((g.standard_normal((n, channels)) * scale + shift).astype(np.float32)))
        return t
    f32 = lambda shift: torch.from_numpy((g.standard_normal(channels) * 0.3 + shift).astype(np.float32)).to(DEV)
    return dict(x=rows(tokens, 1.5, mean), residual=rows(tokens, 3.0, 0.0) if residual else None,
                gate=None if gate is None else rows(1 if gate == "row" else tokens, 0.7, 0.0),
                post_weight=f32(1.0), post_bias=f32(0.0), pre_weight=f32(1.0), pre_bias=f32(0.0),
                sum=rows(tokens, 0.0, 5.0), y=rows(tokens, 0.0, 5.0))


def _run(B, s, post, pre, weights=True, biases=True, eps=(1e-5, 1e-6), alpha=1.0, beta=1.0, with_sum=True):
    def params(which, kind):
        return (s[which + "_weight"] if kind and weights else None, s[which + "_bias"] if kind and biases else None)
    out = (s["sum"] if with_sum else None, s["y"] if pre else None)
    d = B.residual_norm_desc(s["x"], s["residual"], s["gate"], *out, KINDS[post], KINDS[pre], eps[0], eps[1], beta, alpha)
    args = (s["x"], s["residual"], s["gate"], *params("post", post), *params("pre", pre), *out)
    want = O.residual_norm(_np(s["x"]), _np(s["residual"]), _np(s["gate"]),
                           *[None if not k else (k, e, _np(p[0]), _np(p[1])) for k, e, p in
                             ((post, np.float32(eps[0]), params("post", post)), (pre, np.float32(eps[1]), params("pre", pre)))],
                           float(np.float32(beta)), float(np.float32(alpha)))
    B.relay_residual_norm(d, *args)
    torch.cuda.synchronize()
    return d, args, want


def _check(B, dtype, s, post, pre, **kw):
    d, args, (v, dv, y, dy) = _run(B, s, post, pre, **kw)
    if kw.get("with_sum", True):
        _close(s["sum"], v, dv, dtype)
    if pre:
        _close(s["y"], y, dy, dtype)
    return d, args


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("channels", [1, 3, 8, 63, 64, 65, 255, 511, 512, 513, 1000, 1024, 1025, 2047, 2048, 4096, 4099, 8192, 8200, 16384])
@pytest.mark.parametrize("tokens", [1, 5])
def test_rows(B, dtype, channels, tokens):
    s = _inputs(dtype, tokens, channels)
    _check(B, dtype, s, None, "rms")
    _check(B, dtype, s, "layer", "rms", alpha=0.5, beta=2.0)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("channels", [16385, 32767, 32768])
def test_longest_rows(B, dtype, channels):
    _check(B, dtype, _inputs(dtype, 2, channels, gate="token"), "rms", "layer")


@pytest.mark.parametrize("channels", [700, 4096, 5003, 8192])
@pytest.mark.parametrize("tokens", [511, 512, 1001])
def test_many_tokens(B, channels, tokens):
    """(From 512 on a row is shared by fewer threads.)"""
    _check(B, "bf16", _inputs("bf16", tokens, channels, gate="row"), "rms", "rms")


@pytest.mark.parametrize("channels", [1032, 1536, 1544, 2560, 5121, 6600, 7168, 7169, 8193, 9216, 12288, 12289, 20000, 28000])
@pytest.mark.parametrize("tokens", [2, 600])
def test_every_number_of_waves(B, channels, tokens):
    """Rows on 3 to 16 waves, of one to four pieces a thread."""
    _check(B, "bf16", _inputs("bf16", tokens, channels, gate="row"), "layer", "rms")


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("post", [None, "rms", "layer"])
@pytest.mark.parametrize("pre", [None, "rms", "layer"])
@pytest.mark.parametrize("residual,gate", [(True, None), (False, None), (True, "row"), (False, "token"), (True, "token")])
def test_kinds(B, dtype, post, pre, residual, gate):
    s = _inputs(dtype, 6, 200, residual, gate)
    _check(B, dtype, s, post, pre, alpha=0.75, beta=-1.5)
    _check(B, dtype, s, post, pre, weights=False, biases=True)
    _check(B, dtype, s, post, pre, weights=True, biases=False)
    if pre:
        s["sum"].fill_(5)
        _check(B, dtype, s, post, pre, with_sum=False)
        assert (s["sum"] == 5).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("channels,pad,off", [(64, 8, 0), (64, 1, 0), (200, 0, 1), (1001, 3, 5), (4096, 8, 1), (700, 333, 2)])
def test_strides_and_alignments(B, dtype, channels, pad, off):
    s = _inputs(dtype, 4, channels, gate="token", pad=pad, off=off)
    _check(B, dtype, s, "rms", "layer")
    for t in (s["sum"], s["y"]):   # what lies between the rows is left as it was
        between = torch.as_strided(t, (3, pad), (channels + pad, 1), t.storage_offset() + channels)
        assert (between == 3).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("channels", [40, 3000, 9001])
def test_in_place(B, dtype, channels):
    s = _inputs(dtype, 7, channels, gate="token")
    _check(B, dtype, s, "rms", "rms")
    want = (s["sum"].clone(), s["y"].clone())
    for places in (("residual", "x"), ("x", "residual"), ("gate", "x"), ("residual", "gate")):
        t = {k: v.clone() if torch.is_tensor(v) else v for k, v in s.items()}
        t["sum"], t["y"] = t[places[0]], t[places[1]]
        _run(B, t, "rms", "rms")
        assert torch.equal(t["sum"], want[0]) and torch.equal(t["y"], want[1]), places


def test_one_row_for_all_tokens(B):
    """x of stride 0: one row, many residuals."""
    s = _inputs("f16", 9, 300)
    s["x"] = s["x"][:1].expand(9, 300)
    _check(B, "f16", s, None, "rms")


@pytest.mark.parametrize("mean", [0.0, 50.0])
def test_rows_far_from_zero(B, mean):
    """A layer norm of rows whose mean is far larger than what varies."""
    _check(B, "f32", _inputs("f32", 3, 4096, residual=False, mean=mean), None, "layer")
    _check(B, "bf16", _inputs("bf16", 3, 4096, residual=False, mean=mean), "layer", None)


def test_rows_that_are_all_alike(B):
    s = _inputs("f16", 3, 500, residual=False)
    s["x"].copy_(torch.tensor([[0.0], [2.0], [-7.5]]).expand(3, 500))
    _check(B, "f16", s, None, "layer", weights=False, biases=False)
    assert (s["y"] == 0).all()
    _check(B, "f16", s, None, "rms", weights=False, biases=False)
    assert (s["y"][0] == 0).all()


def test_a_row_keeps_its_nan(B):
    s = _inputs("bf16", 6, 700)
    _run(B, s, "rms", "layer")
    want = s["y"].clone()
    s["x"][2, 33], s["residual"][4, 0] = float("nan"), float("inf")
    _run_args = _run(B, s, "rms", "layer")
    rows = [0, 1, 3, 5]
    assert torch.equal(s["y"][rows], want[rows]) and torch.isnan(s["y"][[2, 4]]).all()
    assert torch.isinf(s["sum"][4, 0]) and torch.isfinite(s["sum"][4, 1:]).all()


def test_no_tokens(B):
    s = _inputs("f16", 3, 64)
    s = {k: (v[:0] if torch.is_tensor(v) and v.dim() == 2 else v) for k, v in s.items()}
    B.relay_residual_norm(B.residual_norm_desc(s["x"], None, None, None, s["y"]), s["x"], None, None, None, None, None, None, None, s["y"])


def test_streams_and_replays(B):
    s = _inputs("f16", 33, 1500, gate="row")
    d, args = _check(B, "f16", s, "layer", "rms")
    want = (s["sum"].clone(), s["y"].clone())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    s["y"].zero_()
    with torch.cuda.stream(side):
        side.wait_stream(torch.cuda.default_stream())
        B.relay_residual_norm(d, *args)
    side.synchronize()
    assert torch.equal(s["y"], want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.relay_residual_norm(d, *args)
    for i in range(3):
        s["sum"].fill_(i)
        s["y"].fill_(i)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(s["sum"], want[0]) and torch.equal(s["y"], want[1])


def test_more_rows_than_a_launch_takes(B):
    """2^26 rows of one element and five: y = x / sqrt(x^2 + 1), the sum in the place of x."""
    rows = (1 << 26) + 5
    x = ((torch.arange(rows, device=DEV, dtype=torch.int32) % 2001).float() / 500 - 2).half().view(rows, 1)
    before, y = x.clone(), torch.zeros_like(x)
    B.relay_residual_norm(B.residual_norm_desc(x, before, None, x, y, 0, 1, 1e-5, 1.0, 1.0, 1.0), x, before, None, None, None, None, None, x, y)
    for part in range(0, rows, 1 << 24):
        at = slice(part, min(part + (1 << 24), rows))
        v = 2 * before[at].double()
        assert torch.equal(x[at].double(), v)                        # (twice an fp16 number below 4 is one)
        want = v / (v * v + 1).sqrt()
        # fp32 with four roundings ahead of the one to fp16
        assert bool(((y[at].double() - want).abs() <= want.abs() * (2.0 ** -11 + 2.0 ** -21) + 2.0 ** -25).all())
