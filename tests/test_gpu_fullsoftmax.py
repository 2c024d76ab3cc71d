"""The full-softmax operators together: a training step against 64 bits, training that learns, the link-prediction mode,
and the calls of a step in a captured graph."""
import numpy as np
import pytest
import torch

import paper_2005_13789_amd as ne
from paper_2005_13789_amd import linkpred as lp
from paper_2005_13789_amd.fullsoftmax import SoftmaxTrainer

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def say(*a):
    print(*a, flush=True)


def tables(V, d, seed):
    gen = torch.Generator().manual_seed(seed)
    return [(torch.randn(V, d, generator=gen) * d ** -0.25).to(DEV) for _ in range(2)]


def test_a_step_against_64_bits():
    """The first step of AdamW moves by lr g / (|g| + eps): where the gradient is at least a thousandth of its largest value, its own
    relative error of 1e-4 at most changes that by less than a thousandth of lr; where it is zero, nothing moves."""
    V, d, n, lr = 500, 48, 300, 1e-2
    vertex, context = tables(V, d, 1)
    X, C = vertex.double(), context.double()
    gen = torch.Generator().manual_seed(2)
    pairs = torch.randint(0, V, (n, 2), generator=gen).to(torch.int32)
    pairs[::17, 1] = -1
    trainer = SoftmaxTrainer(vertex, context, batch=512)
    loss = trainer.step(pairs.to(DEV), lr).clone()
    p = pairs.long().to(DEV)
    ok = p[:, 1] >= 0
    S = torch.mm(X[p[:, 0]], C.t().contiguous())
    z = torch.logsumexp(S, 1)
    at = p[:, 1].clamp(min=0)
    want = torch.where(ok, z - S.gather(1, at[:, None])[:, 0], torch.zeros((), dtype=torch.float64, device=DEV))
    assert float((loss.double() - want).abs().max()) <= 1e-5
    G = torch.exp(S - z[:, None])
    G[torch.arange(n, device=DEV), at] -= 1.0
    G = G * ok[:, None] / n
    dX, dC = torch.zeros_like(X), torch.mm(G.t().contiguous(), X[p[:, 0]])
    dX.index_add_(0, p[:, 0], torch.mm(G, C))
    for got, old, g in ((vertex, X, dX), (context, C, dC)):
        far = g.abs() > 1e-3 * g.abs().max()
        assert float((got.double() - (old - lr * g / (g.abs() + 1e-8)))[far].abs().max()) <= lr * 1e-3 + 1e-6
        assert bool((got.double()[g == 0] == old[g == 0]).all())


@pytest.mark.parametrize("bits,compute", [(32, torch.float32), (8, torch.float32), (32, torch.bfloat16), (8, torch.bfloat16)])
def test_training_learns(bits, compute):
    """A context that follows from the source: the loss falls from log V to almost nothing."""
    V, d, n = 400, 32, 1000
    say("training", bits, compute)
    vertex, context = (t * 0.1 for t in tables(V, d, 3))
    trainer = SoftmaxTrainer(vertex, context, batch=n, state_bits=bits, compute=compute)
    gen = torch.Generator().manual_seed(4)
    first = last = None
    for _ in range(300):
        src = torch.randint(0, V, (n,), generator=gen)
        pairs = torch.stack([src, (7 * src + 3) % V], 1).to(torch.int32).to(DEV)
        last = float(trainer.step(pairs, 2e-2).mean())
        first = last if first is None else first
    say("  loss", first, "->", last)
    assert abs(first - np.log(V)) < 0.1 and last < 0.5
    if compute == torch.bfloat16:
        assert torch.equal(trainer.rows[0], vertex.bfloat16()) and torch.equal(trainer.rows[1], context.bfloat16())


def planted_partition(V, communities, inside, outside, seed):
    rng = np.random.default_rng(seed)
    size = V // communities
    u = np.repeat(np.arange(V), inside)
    v = (u // size) * size + rng.integers(0, size, u.size)
    uo = np.repeat(np.arange(V), outside)
    return np.stack([np.concatenate([u, uo]), np.concatenate([v, rng.integers(0, V, uo.size)])], axis=1)


def test_link_prediction_with_the_full_softmax():
    """The bar that the sampled modes are held to on such networks."""
    V = 2000
    edges = planted_partition(V, communities=20, inside=10, outside=1, seed=1)
    train, test = lp.split_edges(edges, 0.10, seed=2)
    t, _ = lp.train(train, V, dim=64, epochs=2, batch=4096, lr0=5e-3, walk_length=40, window=5, seed=3, mode="softmax", device=DEV)
    auc = lp.evaluate(t, V, np.concatenate([train, test]), test, seed=4)
    say("  AUC", auc)
    assert auc > 0.85


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [40, 600, 20000])
def test_captured_calls_replay_as_eager_ones(n, dtype):
    """All calls of a step in a graph (few rows, tiles, sorted ids), replayed with eager work between: the same bits every time."""
    V, d = 3000, 64
    say("graph", n, dtype)
    gen = torch.Generator().manual_seed(5)
    vertex, context = (t.to(dtype) for t in tables(V, d, 6))
    src, ctx = (torch.randint(-1, V, (n,), generator=gen).to(torch.int32).to(DEV) for _ in range(2))
    p, g32 = torch.randn(V, d, generator=gen).to(DEV), torch.zeros(V, d, device=DEV)
    m, v = torch.zeros(V, d, device=DEV), torch.zeros(V, d, device=DEV)
    h, dh = torch.empty(n, d, dtype=dtype, device=DEV), torch.empty(n, d, dtype=dtype, device=DEV)
    dw, dt = torch.empty(V, d, dtype=dtype, device=DEV), g32 if dtype == torch.float32 else torch.zeros(V, d, dtype=dtype, device=DEV)
    loss, lse = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    w1, w2 = (torch.empty(ne.ne_xent_workspace_bytes(n, V, d, dtype, k), dtype=torch.uint8, device=DEV) for k in (False, True))
    w3 = torch.empty(ne.ne_embed_workspace_bytes(V, d, n), dtype=torch.uint8, device=DEV)
    opt = ne.ne_create_adamw([p], [dt], [m], [v], torch.empty(ne.ne_adamw_workspace_bytes([V * d]), dtype=torch.uint8, device=DEV))

    def calls():
        ne.ne_embed_lookup(vertex, src, h, scale=2.0)
        ne.ne_xent_loss(h, context, ctx, loss, lse, w1)
        ne.ne_xent_grad(h, context, ctx, lse, dh, dw, w2, scale=1.0 / n)
        ne.ne_embed_grad(src, dh, dt, w3, scale=2.0)
        ne.ne_adamw_step(opt, 3, 1e-3)

    out = (h, loss, lse, dh, dw, dt, p, m, v)
    state = [t.clone() for t in (p, m, v)]

    def reset():
        for t, s in zip((p, m, v), state):
            t.copy_(s)

    calls()
    want = [t.clone() for t in out]
    reset()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        stream.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            calls()
    torch.cuda.current_stream().wait_stream(stream)
    for _ in range(4):
        reset()
        for t in (h, loss, lse, dh, dw, dt):
            t.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b)
        torch.mm(p, p.t())      # eager work between the replays


@pytest.mark.parametrize("compute", [torch.float32, torch.bfloat16])
def test_steps_of_fewer_pairs(compute):
    """One trainer takes steps of all sizes up to its batch: as a trainer of that batch does."""
    V, d, batch = 9000, 120, 6605
    gen = torch.Generator().manual_seed(7)
    pairs = torch.randint(0, V, (batch, 2), generator=gen).to(torch.int32).to(DEV)
    for n in (1, 20, 150, 2725, 4400, batch):
        say("steps of", n, compute)
        got = []
        for size in (batch, n):
            vertex, context = tables(V, d, 8)
            trainer = SoftmaxTrainer(vertex, context, batch=size, compute=compute)
            got.append([trainer.step(pairs[:n], 1e-2).clone(), vertex, context])
        assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("compute", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [40, 600])
def test_pairs_without_a_source_do_not_count(n, compute):
    """A source outside of the tables (walks are padded with -1) leaves its pair out, as such a context does: its loss is 0, the others'
    losses and both tables are those of a step in which its context is padding; a step of such pairs alone moves nothing."""
    V, d = 700, 40
    say("padded sources", n, compute)
    gen = torch.Generator().manual_seed(9)
    pairs = torch.randint(0, V, (n, 2), generator=gen).to(torch.int32)
    out = torch.zeros(n, dtype=torch.bool)
    for first, step, src in ((1, 5, -1), (2, 11, V), (3, 13, 2 ** 31 - 1), (4, 17, -2 ** 31)):
        pairs[first::step, 0] = src
        out[first::step] = True
    both = pairs.clone()
    both[out, 1] = -1
    got = []
    for p in (pairs, both):
        vertex, context = tables(V, d, 10)
        trainer = SoftmaxTrainer(vertex, context, batch=n, compute=compute)
        got.append([trainer.step(p.to(DEV), 1e-2).clone(), vertex, context])
    assert bool((got[0][0][out.to(DEV)] == 0).all()) and bool((got[0][0][~out.to(DEV)] > 0).all())
    assert all(torch.equal(a, b) for a, b in zip(*got))
    vertex, context = tables(V, d, 11)
    before = vertex.clone(), context.clone()
    trainer = SoftmaxTrainer(vertex, context, batch=n, compute=compute)
    loss = trainer.step(pairs[out].to(DEV), 1e-2)
    assert bool((loss == 0).all()) and torch.equal(vertex, before[0]) and torch.equal(context, before[1])


def test_trainer_refusals():
    vertex, context = tables(50, 8, 12)
    with pytest.raises(ValueError):
        SoftmaxTrainer(vertex, context, batch=4, state_bits=16)
    with pytest.raises(ValueError):
        SoftmaxTrainer(vertex, context[:, :4].contiguous(), batch=4)
    trainer = SoftmaxTrainer(vertex, context, batch=4)
    before = vertex.clone(), context.clone()
    for bad in (torch.zeros(0, 2), torch.zeros(5, 2), torch.zeros(4), torch.zeros(2, 3), torch.zeros(2, 1)):
        with pytest.raises(ValueError):
            trainer.step(bad.to(torch.int32).to(DEV), 1e-3)
    for bad in (torch.zeros(3, 2, dtype=torch.int64, device=DEV), torch.zeros(3, 2, dtype=torch.int32)):
        with pytest.raises((TypeError, RuntimeError)):
            trainer.step(bad, 1e-3)
    assert trainer.steps == 0 and torch.equal(vertex, before[0]) and torch.equal(context, before[1])
