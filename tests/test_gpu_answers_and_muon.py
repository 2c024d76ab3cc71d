"""Answers, the entropy term and Muon as a program uses them together: the trainer against 64 bits, answers of a trained model, the command line."""
import json
import math

import numpy as np
import pytest
import torch

import paper_2005_13789_amd as ne
from paper_2005_13789_amd import linkpred as lp
from paper_2005_13789_amd.fullsoftmax import SoftmaxTrainer

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
A, B, C = 3.4445, -4.7750, 2.0315


def say(*a):
    print(*a, flush=True)


def tables(V, d, seed):
    gen = torch.Generator().manual_seed(seed)
    return [(torch.randn(V, d, generator=gen) * d ** -0.25).to(DEV) for _ in range(2)]


def some_pairs(V, n, seed):
    gen = torch.Generator().manual_seed(seed)
    pairs = torch.randint(0, V, (n, 2), generator=gen).to(torch.int32)
    pairs[::17, 1] = -1
    pairs[3::29, 0] = V
    return pairs.to(DEV)


def orthogonal(x):
    x = x / torch.linalg.vector_norm(x)
    for _ in range(5):
        g = x.t() @ x
        x = A * x + x @ (B * g + C * (g @ g))
    return x


@pytest.mark.parametrize("weight", [0.0, 0.2])
@pytest.mark.parametrize("compute", [torch.float32, torch.bfloat16])
def test_steps_with_muon_against_64_bits(weight, compute):
    """Three steps of the whole objective.  Gradients are off by 2^-18 of their norm at most in fp32; an update's directions are all brought to the same
    size, so its error is the gradient's over the weakest part that counts: 2^-18 over singular values that differ by less than 1000 is far below the
    eighth of a step that it is held to.  In bf16 (2^-8) no such bound is left: there the first losses and the copies are looked at."""
    V, d, n, lr = 300, 24, 700, 1e-2
    vertex, context = tables(V, d, 1)
    say("muon steps", weight, compute)
    trainer = SoftmaxTrainer(vertex, context, batch=n, optimizer="muon", entropy_weight=weight, compute=compute, weight_decay=0.1)
    tabs = [t.double().clone() for t in (vertex, context)]
    first = [t.clone() for t in tabs]
    moms = [torch.zeros_like(t) for t in tabs]
    scale = 0.2 * math.sqrt(V)
    for step in range(3):
        pairs = some_pairs(V, n, 2 + step)
        loss = trainer.step(pairs, lr).clone()
        p = pairs.long()
        ok = (p[:, 0] >= 0) & (p[:, 0] < V) & (p[:, 1] >= 0)
        rows = [t.to(compute).double() for t in tabs]
        X = rows[0][p[:, 0].clamp(0, V - 1)]
        L = torch.log_softmax(X @ rows[1].t(), dim=1)
        P, E = torch.exp(L), -(torch.exp(L) * L).sum(1)
        at = p[:, 1].clamp(min=0)
        want = torch.where(ok, -L.gather(1, at[:, None])[:, 0], 0.0)
        if step == 0:
            assert float((loss.double() - want).abs().max()) <= 1e-5
        G = P * (1.0 + weight * (L + E[:, None]))
        G[torch.arange(n, device=DEV), at] -= 1.0
        G = G * ok[:, None] / n
        grads = [torch.zeros_like(rows[0]).index_add_(0, p[:, 0].clamp(0, V - 1), (G @ rows[1]) * ok[:, None]), G.t() @ X]
        for i in range(2):
            moms[i] = 0.95 * moms[i] + grads[i]
            tabs[i] = tabs[i] * (1 - lr * 0.1) - lr * scale * orthogonal(grads[i] + 0.95 * moms[i])
    for got, want, old in zip((vertex, context), tabs, first):
        moved = float(torch.linalg.vector_norm(want - old))
        err = float(torch.linalg.vector_norm(got.double() - want))
        say("  moved", moved, "off by", err)
        assert compute == torch.bfloat16 or err <= moved / 3 / 8
    if compute == torch.bfloat16:
        assert torch.equal(trainer.rows[0], vertex.bfloat16()) and torch.equal(trainer.rows[1], context.bfloat16())


@pytest.mark.parametrize("optimizer,weight", [("muon", 0.0), ("muon", 0.05), ("adamw", 0.05)])
@pytest.mark.parametrize("compute", [torch.float32, torch.bfloat16])
def test_training_and_answers(optimizer, weight, compute):
    """All parts run together, tables stay finite, and the answers are those of 64 bits on the tables' rows."""
    V, d, n = 500, 32, 900
    say("training", optimizer, weight, compute)
    vertex, context = (t * 0.3 for t in tables(V, d, 3))
    trainer = SoftmaxTrainer(vertex, context, batch=n, compute=compute, optimizer=optimizer, entropy_weight=weight)
    gen = torch.Generator().manual_seed(4)
    for _ in range(30):
        src = torch.randint(0, V, (n,), generator=gen)
        trainer.step(torch.stack([src, (7 * src + 3) % V], 1).to(torch.int32).to(DEV), 1e-2)
    assert bool(torch.isfinite(vertex).all()) and bool(torch.isfinite(context).all())
    for count, k in ((1, 1), (40, 5), (n, 64)):
        nodes = torch.randint(-1, V + 1, (count,), generator=gen).to(torch.int32).to(DEV)
        ids, logp, entropy = trainer.predict(nodes, k)
        ok = (nodes >= 0) & (nodes < V)
        S = trainer.rows[0].double()[nodes.long().clamp(0, V - 1)] @ trainer.rows[1].double().t()
        L = torch.log_softmax(S, dim=1)
        order = torch.sort(S, dim=1, descending=True, stable=True)[1][:, :k]
        assert torch.equal(ids[ok].long(), order[ok]) and bool((ids[~ok] == -1).all())
        # a score's and its sum's roundings, as in the tests of the loss: far below 1e-4 at scores of 30
        assert float((logp[ok].double() - L.gather(1, order)[ok]).abs().max() if bool(ok.any()) else 0.0) <= 1e-4
        assert bool((logp[~ok] == -math.inf).all()) and bool((entropy[~ok] == 0).all())
        assert float(((entropy.double() + (L.exp() * L).sum(1)) * ok).abs().max()) <= 1e-3


def test_steps_without_the_new_parts_are_as_before():
    """A weight of zero takes the loss's own calls, bit for bit."""
    V, d, n = 400, 40, 300
    got = []
    for kw in ({}, dict(entropy_weight=0.0, optimizer="adamw")):
        vertex, context = tables(V, d, 5)
        trainer = SoftmaxTrainer(vertex, context, batch=n, **kw)
        losses = [trainer.step(some_pairs(V, n, 6 + s), 1e-2).clone() for s in range(3)]
        got.append([*losses, vertex, context])
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_predict_refusals():
    trainer = SoftmaxTrainer(*tables(50, 8, 7), batch=4)
    for nodes, k in ((torch.zeros(0), 3), (torch.zeros(5), 3), (torch.zeros(2), 0), (torch.zeros(2), 65)):
        with pytest.raises(ValueError):
            trainer.predict(nodes.to(torch.int32).to(DEV), k)
    with pytest.raises(TypeError):
        trainer.predict(torch.zeros(2, dtype=torch.int64, device=DEV))


def test_hits_and_the_command_line(tmp_path, capsys):
    V, size = 600, 20
    rng = np.random.default_rng(1)
    u = np.repeat(np.arange(V), 8)
    edges = np.stack([u, (u // size) * size + rng.integers(0, size, u.size)], axis=1)
    f = tmp_path / "edges.txt"
    f.write_text("\n".join(f"{a} {b}" for a, b in edges.tolist()) + "\n")
    for optimizer in ("adamw", "muon"):
        assert lp.main([str(f), "--test-fraction", "0.1", "--dim", "32", "--epochs", "1", "--batch", "2048", "--mode", "softmax", "--lr", "0.005", "--walk-length", "10",
                        "--optimizer", optimizer, "--entropy-weight", "0.01", "--hits", "20"]) == 0
        out = json.loads(capsys.readouterr().out.strip().splitlines()[-1])
        say(optimizer, out)
        assert 0.0 <= out["hits_at_20"] <= 1.0 and 0.0 <= out["auc_vertex_context"] <= 1.0
    # hits by the definition
    vertex, context = tables(V, 16, 8)
    t = ne.ne_create_tables(vertex, context, 1, init=False)
    some = edges[:37]
    S = vertex.double() @ context.double().t()
    top = torch.topk(S, 7, dim=1)[1].cpu().numpy()
    want = np.mean([b in top[a] for a, b in np.concatenate([some, some[:, ::-1]])])
    assert abs(lp.hits(t, some, k=7, batch=10) - want) < 1e-12
