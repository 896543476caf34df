"""Attention over a paged cache where keys are shared out over workgroups: parts of tiles of many rows and their join, units of many sequences in one
line, one workspace for both, results that do not depend on who arrives last."""
import numpy as np
import pytest
import torch

from .test_gpu_paged_attention import B, DEV, _both, _case, _run, _verify  # noqa: F401  (B is the fixture)

pytestmark = pytest.mark.gpu


def _again(B, s, out, ws=None):
    B.relay_paged_attention(s["d"], s["q"], s["kc"], s["vc"], s["table"], s["starts"], s["kv"], out, s["ws"] if ws is None else ws)
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("dim,ps", [(64, 16), (72, 20), (96, 48), (128, 64), (128, 7), (200, 16), (256, 33)])
@pytest.mark.parametrize("lens,hq,hkv,causal,window", [([(40, 1500)], 2, 1, True, 0), ([(17, 900), (5, 1300), (0, 700), (3, 2)], 8, 2, True, 0),
                                                       ([(150, 1100)], 2, 2, True, 600), ([(33, 1027)], 1, 1, False, 0)])
def test_parts_of_tiles(B, dtype, dim, ps, lens, hq, hkv, causal, window):
    c = _case(dtype, lens, hq, hkv, dim, ps)
    got, s = _run(B, c, causal, window)
    assert s["ws"].numel() > 0
    first = got.clone()
    for _ in range(3):
        got.fill_(7)
        _again(B, s, got)
        assert torch.equal(got, first)
    _both(B, c, causal, window)


def test_bounds_far_above_the_lengths(B):
    """The launch is sized for 20000 keys and 64 tokens; the sequences have few: tiles of one part among tiles cut for many."""
    c = _case("f16", [(30, 60), (1, 1), (20, 2500), (0, 0)], 4, 2, 64, 16)
    c["max_q"], c["max_kv"] = 64, 20000
    per = 20000 // 16
    c["table"] = np.pad(c["table"], ((0, 0), (0, per - c["table"].shape[1])), constant_values=-1)
    _both(B, c)


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_unseen_keys_in_parts(B, value):
    """The newest key and value are not finite: the tokens before see a cache without it."""
    c = _case("f16", [(40, 1500)], 4, 2, 64, 16)
    page, slot = int(c["table"][0, 1499 // 16]), 1499 % 16
    clean = {k: (v.clone() if torch.is_tensor(v) else v) for k, v in c.items()}
    for name in ("kc", "vc"):
        c[name][page, slot] = value
        clean[name][page, slot] = 0
    got, _ = _run(B, c)
    ref, s = _run(B, clean)
    assert s["ws"].numel() > 0 and torch.equal(got[:-1], ref[:-1])
    assert not torch.isfinite(got[-1].float()).all()


@pytest.mark.parametrize("workspace", [True, False])
@pytest.mark.parametrize("ps", [16, 10])
def test_infinite_values_everywhere(B, workspace, ps):
    """One channel of all values is +inf, in more masked tiles than the kernel keeps a list of: +inf in that channel of every row, the others as without."""
    c = _case("f16", [(300, 2000)], 1, 1, 64, ps, qstd=0.1)
    c["vc"][..., 5] = float("inf")
    got, _ = _run(B, c, True, 700, workspace)
    assert (got[..., 5] == float("inf")).all()
    c["vc"][..., 5] = 0
    ref, _ = _run(B, c, True, 700, workspace)
    got[..., 5] = 0
    assert torch.equal(got, ref)


@pytest.mark.parametrize("lens,hq,hkv", [([(1, 40 + 7 * i) for i in range(70)], 4, 4),           # more tiles than workgroups
                                         ([(1, 3000)] * 2 + [(1, 5)] * 70 + [(2, 900)], 2, 1),   # more sequences than lanes
                                         ([(1, 2000), (0, 50), (1, 1), (4, 700), (1, 0)], 4, 1),
                                         ([(1, 33 * i) for i in range(1, 64)], 8, 4),
                                         ([(1, 30 + 7 * i) for i in range(70)] + [(1, 2100), (2, 64)], 4, 4),
                                         ([(1, 100)] * 40 + [(1, 2300)] + [(3, 200)] * 40, 6, 3)])
@pytest.mark.parametrize("dim", [64, 136])
def test_sequences_in_one_line(B, lens, hq, hkv, dim):
    c = _case("bf16", lens, hq, hkv, dim, 16)
    _both(B, c)
    got, s = _run(B, c)
    assert s["ws"].numel() > 0 or c["max_kv"] <= 2048   # (many short sequences are not shared out)
    first = got.clone()
    for _ in range(3):
        got.fill_(7)
        _again(B, s, got)
        assert torch.equal(got, first)


def test_one_workspace_for_one_token_and_for_many(B):
    one, many = _case("f16", [(1, 3000), (1, 900)], 4, 2, 128, 16), _case("f16", [(50, 2000)], 4, 2, 128, 16)
    runs = [(c, _run(B, c)[1]) for c in (one, many)]
    ws = torch.zeros(max(s["ws"].numel() for _, s in runs), dtype=torch.uint8, device=DEV)
    for c, s in runs * 3:
        out = torch.full_like(s["q"], float("nan"))
        _again(B, s, out, ws)
        _verify(c, out, s["scale"])


def test_parts_in_a_graph(B):
    c = _case("f16", [(40, 3000)], 8, 2, 128, 16)
    got, s = _run(B, c)
    assert s["ws"].numel() > 0
    want, out, graph = got.clone(), torch.zeros_like(got), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.relay_paged_attention(s["d"], s["q"], s["kc"], s["vc"], s["table"], s["starts"], s["kv"], out, s["ws"])
    for _ in range(4):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        got.fill_(3)
        _again(B, s, got)
        assert torch.equal(got, want)
