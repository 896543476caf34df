"""Blocks of norms, attention, router and experts on one residual stream, the head and the choice of the next token: every operator against 64 bits from what the ones
before it left, and whole decoding loops from a graph against the same run eagerly."""
import numpy as np
import pytest
import torch

from oracle import attention as OA
from oracle import decoder as O

from .test_gpu_decoder import D, DEV, DIM, GROUP, HKV, HQ, ROWS, TYPES, _close, _dense, _np  # noqa: F401  (D is the fixture)

pytestmark = pytest.mark.gpu
WIDTH, INTER, EXPERTS, TOP_K, VOCAB = 192, 96, 6, 2, 1003


def _weights(dtype, seed, *shape, std=1.0, kind=None):
    w = torch.from_numpy((np.random.default_rng(seed).standard_normal(shape) * std).astype(np.float32)).to(DEV)
    return w if kind is None else w.to(kind)


def _model(D, dtype, layers=2, max_tokens=160):
    from paper_1904_08368_amd import binding as B
    tt = TYPES[dtype][0]
    table = torch.empty((ROWS, DIM // 2, 2), device=DEV)
    B.relay_rope_table(B.rope_table_desc(ROWS, DIM), table)
    blocks, host, scratch, products = [], [], D.Workspace(), D.Workspace()
    for i in range(layers):
        at = 100 * i
        (qkv, _), (o, _) = _dense(D, dtype, (HQ + 2 * HKV) * DIM, WIDTH, at), _dense(D, dtype, WIDTH, HQ * DIM, at + 1)
        (up, wu), (down, wd) = _dense(D, dtype, EXPERTS * 2 * INTER, WIDTH, at + 2), _dense(D, dtype, EXPERTS * WIDTH, INTER, at + 3)
        router, bias = _weights(dtype, at + 4, EXPERTS, WIDTH, std=2 / WIDTH ** 0.5, kind=tt), _weights(dtype, at + 5, EXPERTS, std=0.1)
        mid = D.ResidualNorm(pre_weight=1 + 0.1 * _weights(dtype, at + 6, WIDTH), post=B.NORM_RMS, post_weight=1 + 0.1 * _weights(dtype, at + 7, WIDTH))
        out = D.ResidualNorm(pre=B.NORM_LAYER, pre_weight=1 + 0.1 * _weights(dtype, at + 8, WIDTH), pre_bias=0.1 * _weights(dtype, at + 9, WIDTH), branch_scale=0.5,
                             gate=_weights(dtype, at + 10, 1, WIDTH, kind=tt))
        attention = D.AttentionLayer(qkv, o, table, HQ, HKV, DIM, max_tokens=max_tokens, workspace=scratch)
        blocks.append(D.Block(attention, mid, D.Experts(router, up, down, TOP_K, bias, score=B.SCORE_SIGMOID, scale=1.5, workspace=products), out))
        host.append((wu, wd))
    head, whead = _dense(D, dtype, VOCAB, WIDTH, 900)
    return D.Decoder(blocks, D.ResidualNorm(pre_weight=torch.ones(WIDTH, device=DEV)), head, max_tokens), host, whead


def _norm(layer, which):
    post_weight, post_bias, pre_weight, pre_bias = (None if t is None else t.cpu().numpy() for t in layer.params)
    kind = (None, "rms", "layer")[layer.kinds[which]]
    return None if kind is None else (kind, float(np.float32(layer.kinds[which + "_eps"])), *((post_weight, post_bias) if which == "post" else (pre_weight, pre_bias)))


def _check_norm(layer, x, residual, s, n, dtype):
    v, dv, y, dy = O.residual_norm(_np(x), None if residual is None else _np(residual), None if layer.gate is None else _np(layer.gate), _norm(layer, "post"), _norm(layer, "pre"),
                                   layer.kinds["branch_scale"], layer.kinds["residual_scale"])
    _close(s, v, dv, dtype)
    _close(n, y, dy, dtype)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_every_operator_of_a_step(D, dtype):
    decoder, host, whead = _model(D, dtype)
    _, u, tiny = TYPES[dtype]
    cache = D.PagedCache(2, 64, 16, HKV, DIM, TYPES[dtype][0])
    ids = [cache.open() for _ in range(3)]
    g = torch.Generator(device=DEV).manual_seed(3)
    for new in ([70, 5, 33], [1, 1, 1]):
        step = D.Step(cache, 3, sum(new) + 2, max(new), 200)   # (two rows of padding)
        step.extend(ids, new)
        x = torch.randn((step.tokens, WIDTH), generator=g, device=DEV).to(TYPES[dtype][0])
        s, n, branch = (t[:step.tokens] for t in (decoder._s, decoder._n, decoder._branch))
        decoder.first(x, None, s, n)
        _check_norm(decoder.first, x, None, s, n, dtype)
        for i, block in enumerate(decoder.blocks):
            before = s.clone()
            block.attention(n, i, step, branch, add=False)   # (its own parts are looked at elsewhere)
            with_input = block.attention(n, i, step)
            assert torch.equal(with_input, (branch.float() + n.float()).to(n.dtype)) or dtype == "bf16" or (with_input - (branch + n)).abs().max() < 0.02
            block.mid(branch, s, s, n)
            _check_norm(block.mid, branch, before, s, n, dtype)
            chosen, weights = torch.zeros((step.tokens, TOP_K), dtype=torch.int32, device=DEV), torch.zeros((step.tokens, TOP_K), device=DEV)
            y = block.experts(n, branch, chosen=chosen, weights=weights)
            want, ref = O.route(_np(n), _np(block.experts.router), TOP_K, "sigmoid", block.experts.bias.cpu().numpy(), True, 1.5)
            assert np.array_equal(chosen.cpu().numpy(), want) and np.abs(_np(weights) - ref).max() <= 2.0 ** -24 * 1.6
            want, err = O.experts(_np(n), chosen.cpu().numpy(), _np(weights), *host[i], INTER, GROUP, u=u, tiny=tiny)
            _close(y, want, err, dtype)
            before = s.clone()
            block.out(branch, s, s, n)
            _check_norm(block.out, branch, before, s, n, dtype)
        assert torch.equal(decoder(x, step), n)                 # the same as one call (the cache's slots are written again)
        last = (step.q_starts[1:] - 1).long()
        logits = decoder.logits(n, last)
        want, bound = OA.dense_w4(_np(n)[last.cpu().numpy()], *whead, GROUP)
        _close(logits, want, bound, dtype)
        uniform = torch.tensor([0.1, 0.5, 0.9], device=DEV)
        tokens = D.Sampler()(logits, top_k=torch.full((3,), 40, dtype=torch.int32, device=DEV), uniform=uniform)
        assert tokens.tolist() == [O.sample(_np(logits)[r], top_k=40, uniform=float(uniform[r]))[0] for r in range(3)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_decoding_from_a_graph(D, dtype):
    """Prompts, then tokens that are sampled, looked up and decoded again: one captured step, replayed while the sequences grow, against eager steps."""
    rounds, batch = 24, 3
    embedding = _weights(dtype, 77, VOCAB, WIDTH, kind=TYPES[dtype][0])
    u = torch.rand((rounds, batch), generator=torch.Generator(device=DEV).manual_seed(8), device=DEV)
    prompts = [[5, 900, 33, 7] * 9, [1, 2, 3], [400]]

    def start():
        decoder, _, _ = _model(D, dtype)
        sampler, cache = D.Sampler(), D.PagedCache(2, 64, 16, HKV, DIM, TYPES[dtype][0])
        ids = [cache.open() for _ in prompts]
        first = D.Step(cache, batch, 40, 36, 200)
        first.extend(ids, [len(p) for p in prompts])
        ids_in = torch.tensor(sum(prompts, []), device=DEV)
        n = decoder(embedding.index_select(0, ids_in), first)
        tokens = sampler(decoder.logits(n, (first.q_starts[1:] - 1).long()), uniform=torch.full((batch,), 0.3, device=DEV))
        return decoder, sampler, cache, ids, tokens, D.Step(cache, batch, batch, 1, 200)

    settings = dict(temperature=torch.tensor([0.7, 1.0, 0.0], device=DEV), top_p=torch.tensor([0.9, 1.0, 1.0], device=DEV))

    def one(decoder, sampler, tokens, step, uniform):
        n = decoder(embedding.index_select(0, tokens), step)
        return sampler(decoder.logits(n), uniform=uniform, tokens=tokens, **settings)

    decoder, sampler, _, ids, tokens, step = start()
    want = []
    for r in range(rounds):
        step.extend(ids, [1] * batch)
        want.append(one(decoder, sampler, tokens, step, u[r]).tolist())
    decoder, sampler, cache, ids, tokens, step = start()
    first, uniform = tokens.clone(), torch.zeros(batch, device=DEV)
    one(decoder, sampler, tokens, step, uniform)                # (no tokens yet: nothing is stored; scratch is there)
    tokens.copy_(first)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one(decoder, sampler, tokens, step, uniform)
    bystander = torch.full((1 << 20,), 3, dtype=torch.uint8, device=DEV)
    for r in range(rounds):
        step.extend(ids, [1] * batch)
        uniform.copy_(u[r])
        graph.replay()
        torch.cuda.synchronize()
        assert tokens.tolist() == want[r], r
        if r % 7 == 3:   # eager work of the same layers between the replays
            other = torch.randn((40, WIDTH), device=DEV).to(TYPES[dtype][0])
            y = torch.empty_like(other)
            decoder.blocks[0].experts(other, y)
            assert torch.isfinite(y.float()).all()
    assert bool((bystander == 3).all())
    assert len({t for w in want for t in w}) > 5


def test_parts_that_do_not_go_together(D):
    router = torch.zeros((EXPERTS, WIDTH), dtype=torch.float16, device=DEV)
    up, down = _dense(D, "f16", EXPERTS * 2 * INTER, WIDTH, 1)[0], _dense(D, "f16", EXPERTS * WIDTH, INTER, 2)[0]
    D.Experts(router, up, down, 2)
    for bad in (lambda: D.Experts(router[:5], up, down, 2), lambda: D.Experts(router[:, :100], up, down, 2), lambda: D.Experts(router.bfloat16(), up, down, 2),
                lambda: D.Experts(router, down, up, 2)):
        with pytest.raises(ValueError):
            bad()


def test_room_for_logits(D):
    """max_rows of them, and a call for more is refused."""
    full, _, _ = _model(D, "f16", layers=1, max_tokens=40)
    few = D.Decoder(full.blocks, full.first, full.head, 40, max_rows=3)
    n = _weights("f16", 5, 8, WIDTH, kind=torch.float16)
    rows = torch.tensor([6, 0, 3], device=DEV)
    assert torch.equal(few.logits(n, rows), full.logits(n)[rows]) and torch.equal(few.logits(n[:2]), full.logits(n)[:2])
    with pytest.raises(ValueError):
        few.logits(n)


def test_calls_on_two_streams_at_once(D):
    """Workspaces of their own, and neither sees the other: router, experts and sampler side by side, eagerly and from two graphs that are replayed together."""
    dtype = TYPES["bf16"][0]
    lanes = []
    for seed in (1, 2):
        decoder, _, _ = _model(D, "bf16", layers=1, max_tokens=64)
        x, logits = _weights("bf16", seed, 50, WIDTH, kind=dtype), _weights("bf16", 10 + seed, 3, 60001, std=2.0, kind=dtype)
        lanes.append(dict(experts=decoder.blocks[0].experts, sampler=D.Sampler(), x=x, y=torch.empty_like(x), logits=logits, tokens=torch.zeros(3, dtype=torch.int32, device=DEV),
                          uniform=torch.tensor([0.2, 0.5, 0.8], device=DEV), top_p=torch.full((3,), 0.9, device=DEV), stream=torch.cuda.Stream()))

    def step(lane):
        lane["experts"](lane["x"], lane["y"])
        lane["sampler"](lane["logits"], top_p=lane["top_p"], uniform=lane["uniform"], tokens=lane["tokens"])

    want = []
    for lane in lanes:
        step(lane)
        torch.cuda.synchronize()
        want.append((lane["y"].clone(), lane["tokens"].clone()))

    def check():
        torch.cuda.synchronize()
        for lane, (y, tokens) in zip(lanes, want):
            assert torch.equal(lane["y"], y) and torch.equal(lane["tokens"], tokens)
            lane["y"].zero_()
            lane["tokens"].zero_()
        torch.cuda.synchronize()

    check()
    for _ in range(5):
        for lane in lanes:
            with torch.cuda.stream(lane["stream"]):
                for _ in range(4):
                    step(lane)
        check()
    graphs = []
    for lane in lanes:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            step(lane)
    for _ in range(5):
        for lane, graph in zip(lanes, graphs):
            with torch.cuda.stream(lane["stream"]):
                graph.replay()
        check()
