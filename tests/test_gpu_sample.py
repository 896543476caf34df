"""The choice of the next token against 64 bits: every type, vocabularies from one token to the largest, settings alone and together, values that crowd into
one bin or are all alike, masked, infinite and NaN logits, settings out of range, strides, captured and replayed calls."""
import math

import numpy as np
import pytest
import torch

from oracle import decoder as O

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
TOP = 1 - 2.0 ** -24
# A probability: weights in 64 bits, their sum as integers (off by a part of 2^-40 at most), one rounding to fp32, of numbers from 2^-45 on.
PROB = 2.0 ** -24 * 1.001


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1904_08368_amd import binding
    binding.lib()
    return binding


def _logits(dtype, rows, vocab, seed, std=2.0, pad=0):
    """Normal logits, a few far above the rest, as a trained head leaves them."""
    g = np.random.default_rng(seed + vocab)
    l = g.standard_normal((rows, vocab + pad)) * std
    for r in range(rows):
        at = g.integers(0, vocab, 12)
        l[r, at] += g.exponential(3.0, 12) + 2
    return torch.from_numpy(l.astype(np.float32)).to(TYPES[dtype]).to(DEV)[:, :vocab]


def _vec(v, rows, dtype=torch.float32):
    return None if v is None else torch.tensor(v if isinstance(v, (list, tuple)) else [v] * rows, dtype=dtype, device=DEV)


def _check(B, logits, temperature=None, top_k=None, top_p=None, min_p=None, uniform=0.5, with_workspace=True):
    rows = logits.shape[0]
    t, p, m, u = (_vec(v, rows) for v in (temperature, top_p, min_p, uniform))
    k = _vec(top_k, rows, torch.int32)
    tokens, probs = torch.full((rows,), -7, dtype=torch.int32, device=DEV), torch.full((rows,), -7.0, device=DEV)
    d = B.sample_desc(logits)
    ws = torch.zeros(B.relay_sample_workspace_bytes(d), dtype=torch.uint8, device=DEV) if with_workspace else None
    args = (logits, t, k, p, m, u, tokens, probs, ws)
    B.relay_sample(d, *args)
    torch.cuda.synchronize()
    host = logits.cpu().to(torch.float64).numpy()
    get = lambda v, r, default: default if v is None else float(v[r])
    for r in range(rows):
        want = O.sample(host[r], get(t, r, 1.0), int(get(k, r, 0)), get(p, r, 1.0), get(m, r, 0.0), get(u, r, 0.0) if u is not None else 0.0)
        if u is None:
            want = O.sample(host[r], 0.0)
        assert int(tokens[r]) == want[0], (r, int(tokens[r]), want, host[r][int(tokens[r])], host[r][want[0]])
        assert abs(float(probs[r]) - want[1]) <= PROB * want[1], (r, float(probs[r]), want)
    return d, args


SETTINGS = [dict(), dict(top_k=50), dict(top_p=0.9), dict(min_p=0.05), dict(top_k=40, top_p=0.95, temperature=0.8), dict(top_k=1000, temperature=1.5),
            dict(top_k=3000, top_p=0.5, temperature=3.0), dict(top_p=0.999, min_p=0.001, temperature=1.3), dict(top_k=1), dict(temperature=0.0),
            dict(top_k=2000, min_p=1e-4, temperature=2.0), dict(temperature=0.05), dict(temperature=30.0, top_p=0.3)]


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("vocab", [1, 2, 7, 8, 9, 100, 1000, 1024, 4096, 8195, 50257])
def test_settings(B, dtype, vocab):
    g = np.random.default_rng(vocab)
    logits = _logits(dtype, 4, vocab, 1)
    for s in SETTINGS:
        _check(B, logits, uniform=[float(np.float32(v)) for v in g.random(4)], **s)


@pytest.mark.parametrize("dtype,vocab", [("f16", 131073), ("bf16", 151643), ("f32", 262144), ("bf16", 1 << 20)])
def test_large_vocabularies(B, dtype, vocab):
    logits = _logits(dtype, 2, vocab, 2)
    for s in SETTINGS:
        _check(B, logits, uniform=[0.123, 0.987], **s)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_every_place(B, dtype):
    """One row under many uniform numbers: each token as often as its share, from the first to the last."""
    rows = 300
    logits = _logits(dtype, 1, 3001, 3).expand(rows, 3001)
    u = [float(np.float32(min((i + 0.5) / rows, TOP))) for i in range(rows)]
    for s in (dict(), dict(top_k=20), dict(top_p=0.8), dict(min_p=0.02)):
        _check(B, logits, uniform=u, **s)
    for s in (dict(), dict(top_k=20), dict(top_p=0.8)):
        _check(B, logits[:4], uniform=[0.0, 2.0 ** -30, TOP, 0.9999], **s)


@pytest.mark.parametrize("rows", [1, 3, 64, 257])
def test_rows_of_their_own_settings(B, rows):
    g = np.random.default_rng(rows)
    pick = lambda values: [values[i] for i in g.integers(0, len(values), rows)]
    logits = _logits("bf16", rows, 2500, 4)
    for with_workspace in (True, False):
        _check(B, logits, pick([0.0, 0.5, 1.0, 1.5]), pick([0, 0, 1, 20, 900, 2400]), pick([1.0, 1.0, 0.9, 0.4]), pick([0.0, 0.0, 0.1]),
               [float(np.float32(v)) for v in g.random(rows)], with_workspace)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("vocab", [1, 5, 1000, 2048, 2049, 70000])
def test_logits_that_are_all_alike(B, dtype, vocab):
    """Whole numbers: place floor(u n) of the n kept, the lowest numbers first."""
    logits = torch.full((4, vocab), 3.25, dtype=TYPES[dtype], device=DEV)
    u = [0.0, 0.25, 0.7, TOP]
    for s, kept in ((dict(), vocab), (dict(top_k=700), min(700, vocab)), (dict(top_p=0.5), math.ceil(vocab / 2)), (dict(min_p=1.0), vocab),
                    (dict(top_k=3, top_p=0.25), 1), (dict(temperature=7.0), vocab)):
        _, args = _check(B, logits, uniform=u, **s)
        assert args[6].tolist() == [math.floor(float(np.float32(v)) * kept) for v in u]


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_few_values(B, dtype):
    """Tens of thousands of tokens with one of three values, and one far below that spreads the bins."""
    g = np.random.default_rng(5)
    l = g.choice([1.0, 1.5, 4.0], (3, 60000), p=[0.6, 0.3, 0.1]).astype(np.float32)
    l[0, 17] = -1000.0
    logits = torch.from_numpy(l).to(TYPES[dtype]).to(DEV)
    for s in (dict(), dict(top_k=9000), dict(top_k=30000, top_p=0.9), dict(top_p=0.7), dict(min_p=0.06), dict(top_p=0.99, min_p=0.04), dict(top_k=100)):
        for u in (0.0, 0.4, 0.8, TOP):
            _check(B, logits, uniform=u, **s)


def test_values_close_together(B):
    """Tens of thousands of different numbers within a hundredth of each other."""
    g = np.random.default_rng(6)
    l = (20 + 0.01 * g.random((2, 50000))).astype(np.float32)
    l[:, 5], l[1, 6] = -60.0, 20.5
    logits = torch.from_numpy(l).to(DEV)
    for s in (dict(), dict(top_k=20000), dict(top_k=20000, top_p=0.5), dict(top_p=0.3), dict(min_p=0.995), dict(top_p=0.9, min_p=0.993), dict(temperature=0.01), dict(temperature=0.001, top_p=0.9)):
        for u in (0.0, 0.37, 0.9):
            _check(B, logits, uniform=u, **s)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_masked_tokens(B, dtype):
    """Infinities, NaN and the type's lowest number among the logits."""
    g = np.random.default_rng(7)
    logits = _logits(dtype, 6, 3000, 8)
    off = torch.from_numpy(g.random((6, 3000)) < 0.9).to(DEV)
    for row, value in enumerate((float("-inf"), torch.finfo(TYPES[dtype]).min, float("nan"), float("-inf"))):
        logits[row] = torch.where(off[row], torch.full_like(logits[row], value), logits[row])
    logits[3, :] = float("-inf")
    logits[3, 2222] = -5.0                              # one token is left
    logits[4, :] = float("-inf")                        # none
    logits[5, :] = float("nan")
    for s in SETTINGS:
        _, args = _check(B, logits, uniform=0.6, **s)
        assert args[6].tolist()[3:] == [2222, -1, -1]
    logits[0, 100] = logits[0, 2500] = float("inf")     # they share the row
    for u, token in ((0.2, 100), (0.8, 2500)):
        for s in (dict(), dict(top_p=0.9), dict(min_p=0.5), dict(top_k=100)):
            _, args = _check(B, logits[:1], uniform=u, **s)
            assert int(args[6][0]) == token


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_masked_tokens_of_long_rows(B, dtype):
    """The same of rows that are shared out: most of them masked, fewer left than top-k asks for, one left, none."""
    g = np.random.default_rng(17)
    vocab = 70001
    logits = _logits(dtype, 7, vocab, 18)
    off = torch.from_numpy(g.random((7, vocab)) < 0.97).to(DEV)
    off[1] = torch.from_numpy(g.random(vocab) < 1 - 30 / vocab).to(DEV)
    for row, value in enumerate((float("-inf"), float("-inf"), torch.finfo(TYPES[dtype]).min, float("nan"))):
        logits[row] = torch.where(off[row], torch.full_like(logits[row], value), logits[row])
    logits[4, :] = float("-inf")
    logits[4, vocab - 1] = -5.0                         # one token is left, the last
    logits[5, :] = float("-inf")                        # none
    logits[6, :] = float("nan")
    for s in SETTINGS + [dict(top_k=128), dict(top_k=129), dict(top_k=100, temperature=8.0)]:
        for with_workspace in (True, False):
            _, args = _check(B, logits, uniform=0.6, with_workspace=with_workspace, **s)
            assert args[6].tolist()[4:] == [vocab - 1, -1, -1]
    logits[0, 100] = logits[0, 60000] = float("inf")    # they share the row
    for u, token in ((0.2, 100), (0.8, 60000)):
        for s in (dict(), dict(top_p=0.9), dict(min_p=0.5), dict(top_k=100)):
            _, args = _check(B, logits[:1], uniform=u, **s)
            assert int(args[6][0]) == token


def test_long_rows_of_their_own_settings(B):
    """Rows side by side that take every way through the launches, settings out of range among them."""
    nan = float("nan")
    logits = _logits("bf16", 12, 50257, 19)
    for u in (0.2, 0.95):
        _check(B, logits, [1.0, 0.0, nan, 0.7, 1.0, 9.0, 1.0, 1.0, 1.2, 1e-38, float("inf"), 1.0], [0, 50, 50, 128, 129, 2000, -3, 1, 0, 0, 60000, 256],
               [1.0, 0.9, 0.9, nan, 0.8, 0.99, 0.9, 0.5, 1.0, 0.9, 1.0, 1.0], [0.0, 0.0, nan, 0.1, 0.0, 0.0, 0.01, 0.0, 0.05, 0.0, 0.0, 7.0], u)


def test_more_rows_than_a_launch_takes(B):
    """2^23 rows and three: each row's settings and outputs are its own."""
    rows = (1 << 23) + 3
    i = torch.arange(rows, device=DEV, dtype=torch.int32)
    logits = torch.stack([(i % 3 == 0).half(), (i % 3 != 0).half()], 1)   # 0 and 1, the larger first in every third row
    temperature = (i % 2).float()                                          # 0: the larger; 1: with u = 0.9 the smaller (weights 1 and 0.37)
    tokens, probs = torch.full((rows,), -7, dtype=torch.int32, device=DEV), torch.zeros(rows, device=DEV)
    B.relay_sample(B.sample_desc(logits), logits, temperature, None, None, None, torch.full((rows,), 0.9, device=DEV), tokens, probs)
    larger = (i % 3 != 0).int()
    assert torch.equal(tokens, torch.where(i % 2 == 0, larger, 1 - larger))
    assert float((probs - torch.where(i % 2 == 0, 1.0, 1 / (1 + math.e))).abs().max()) <= 2.0 ** -23


def test_zeros_of_both_signs_are_one_value(B):
    l = torch.zeros(1, 4000)
    l[0, ::2] *= -1.0
    for s in (dict(), dict(top_k=1500), dict(top_p=0.25)):
        for u in (0.0, 0.5, 0.75):
            _check(B, l.to(DEV), uniform=u, **s)


def test_settings_out_of_range(B):
    nan, inf = float("nan"), float("inf")
    logits = _logits("f32", 2, 999, 9)
    for s in (dict(temperature=nan), dict(temperature=inf), dict(temperature=-1.0), dict(temperature=1e-38), dict(temperature=1e38), dict(top_k=-5), dict(top_k=5000),
              dict(top_k=999), dict(top_p=nan), dict(top_p=2.0), dict(top_p=0.0), dict(top_p=-1.0), dict(min_p=nan), dict(min_p=-1.0), dict(min_p=7.0), dict(min_p=1e-30)):
        for u in (0.3, nan, -2.0, 1.0, 5.0):
            _check(B, logits, uniform=u, **s)


@pytest.mark.parametrize("l", [[3e38, -3e38, 2.9e38], [65504.0, -65504.0, 65472.0], [1e-40, 0.0, -1e-40]])
def test_extreme_logits(B, l):
    for t in (1.0, 1e37, 100.0):
        for u in (0.1, 0.6, 0.95):
            _check(B, torch.tensor([l], device=DEV), t, uniform=u)


def test_without_uniform_numbers(B):
    _check(B, _logits("bf16", 5, 700, 10), 1.0, 50, 0.9, None, None)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("pad,off", [(1, 0), (8, 3), (5, 1)])
def test_strides_and_alignments(B, dtype, pad, off):
    vocab = 1003
    src = _logits(dtype, 5, vocab, 11)
    flat = torch.full((off + 5 * (vocab + pad),), 1000.0, dtype=TYPES[dtype], device=DEV)   # (what lies between the rows would win)
    logits = flat[off:].view(5, vocab + pad)[:, :vocab]
    logits.copy_(src)
    for s in SETTINGS[:6]:
        _check(B, logits, uniform=0.77, **s)


def test_streams_and_replays(B):
    logits = _logits("f16", 7, 40000, 12)
    d, args = _check(B, logits, 0.9, 300, 0.95, 0.01, 0.66)
    want, probs = args[6].clone(), args[7].clone()
    side = torch.cuda.Stream()
    args[6].zero_()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.relay_sample(d, *args)
    side.synchronize()
    assert torch.equal(args[6], want) and torch.equal(args[7], probs)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.relay_sample(d, *args)
    for i in range(3):
        args[6].fill_(i)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(args[6], want) and torch.equal(args[7], probs)


def test_no_rows(B):
    logits = torch.zeros((0, 50), device=DEV)
    B.relay_sample(B.sample_desc(logits), logits, None, None, None, None, None, torch.zeros(0, dtype=torch.int32, device=DEV))
