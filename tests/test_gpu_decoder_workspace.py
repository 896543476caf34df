"""A captured decode step whose keys are shared out, replayed after longer prompts have made the shared scratch grow, and captured before anything ran."""
import pytest
import torch

from .test_gpu_decoder import D, DEV, HKV, DIM, TYPES, _dense, HQ  # noqa: F401  (D is the fixture)

pytestmark = pytest.mark.gpu
LONG, WIDTH = 4096, 192


def _layer(D, workspace):
    from paper_1904_08368_amd import binding as B
    table = torch.empty((LONG, DIM // 2, 2), device=DEV)
    B.relay_rope_table(B.rope_table_desc(LONG, DIM), table)
    return D.AttentionLayer(_dense(D, "f16", (HQ + 2 * HKV) * DIM, WIDTH, 1)[0], _dense(D, "f16", WIDTH, HQ * DIM, 2)[0], table, HQ, HKV, DIM,
                            max_tokens=700, workspace=workspace)


def _start(D, layer, x):
    cache = D.PagedCache(1, 600, 16, HKV, DIM)
    ids = [cache.open(), cache.open()]
    first = D.Step(cache, 2, 700, 700, 700)
    first.extend(ids, [680, 20])
    layer(x, 0, first)
    return cache, ids, D.Step(cache, 2, 2, 1, LONG)


@pytest.mark.parametrize("warm", [True, False])
def test_replays_after_growth(D, warm):
    g = torch.Generator(device=DEV).manual_seed(4)
    prompt, xs = (torch.randn(s, generator=g, device=DEV).half() for s in ((700, WIDTH), (8, 2, WIDTH)))
    later = torch.randn((300, WIDTH), generator=g, device=DEV).half()
    layer = _layer(D, D.Workspace())
    cache, ids, step = _start(D, layer, prompt)
    want = []
    for x in xs:
        step.extend(ids, [1, 1])
        want.append(layer(x, 0, step).clone())

    scratch = D.Workspace()
    layer = _layer(D, scratch)
    cache, ids, step = _start(D, _layer(D, D.Workspace()), prompt)
    x_in, y = torch.zeros((2, WIDTH), dtype=torch.float16, device=DEV), torch.zeros((2, WIDTH), dtype=torch.float16, device=DEV)
    if warm:
        layer(x_in, 0, step, y)   # (no tokens yet: nothing is stored)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        layer(x_in, 0, step, y)
    before = scratch.buffer
    assert (before is not None) == warm
    other = cache.open()
    chunk = D.Step(cache, 1, 300, 300, LONG)
    bystanders = []
    for t, x in enumerate(xs):
        step.extend(ids, [1, 1])
        x_in.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[t]), t
        if t in (1, 4):   # a prompt arrives between the steps
            chunk.extend([other], [300])
            eager = layer(later, 0, chunk)
            assert scratch.buffer is not before and scratch.buffer.numel() > (before.numel() if warm else 0)
            bystanders += [torch.full((1 << 22,), 3, dtype=torch.uint8, device=DEV) for _ in range(12)]
            assert torch.isfinite(eager.float()).all()
    assert all(bool((b == 3).all()) for b in bystanders)
