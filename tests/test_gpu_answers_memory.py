"""What answers hold on to: workspaces of predict() and hits(), captured answers beside later ones, arguments that are refused before anything runs."""
import pytest
import torch

import paper_2005_13789_amd as ne
from paper_2005_13789_amd.fullsoftmax import SoftmaxTrainer

DEV = "cuda:0"


def say(*a):
    print(*a, flush=True)


def trainer_of(V, d, batch, **kw):
    gen = torch.Generator().manual_seed(V)
    return SoftmaxTrainer(*[(torch.randn(V, d, generator=gen) * d ** -0.25).to(DEV) for _ in range(2)], batch=batch, **kw)


@pytest.mark.gpu
@pytest.mark.parametrize("compute", [torch.float32, torch.bfloat16])
def test_captured_answers_beside_later_ones(compute):
    """A captured predict() keeps its workspace, whatever other calls take and give back in the meantime."""
    say("captured predict", compute)
    V, n = 3000, 70
    trainer = trainer_of(V, 48, 300, compute=compute)
    nodes = torch.arange(n, dtype=torch.int32, device=DEV)
    trainer.predict(nodes, 3)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = trainer.predict(nodes, 3)
    for turn in range(4):
        nodes.copy_(torch.arange(n, dtype=torch.int32, device=DEV) * (turn + 2) % V)
        more = trainer.predict(torch.arange(300, dtype=torch.int32, device=DEV), 20 + turn)        # larger workspaces, given back
        kept = [torch.full((1 << 18,), 7, dtype=torch.uint8, device=DEV) for _ in range(8)]        # ... to tensors of others
        want_more = [x.clone() for x in more]
        graph.replay()
        torch.cuda.synchronize()
        assert all(bool((x == 7).all()) for x in kept) and all(torch.equal(a, b) for a, b in zip(more, want_more))
        assert all(torch.equal(a, b) for a, b in zip(captured, trainer.predict(nodes, 3))), turn


@pytest.mark.gpu
def test_predict_keeps_no_workspace():
    """One node's answers take a workspace of one node, whatever the trainer's batch is, and give it back."""
    trainer = trainer_of(100_000, 32, 4096)
    node = torch.zeros(1, dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    torch.cuda.reset_peak_memory_stats()
    out = trainer.predict(node, 64)
    room = ne.ne_logprob_workspace_bytes(1, 100_000, 32, torch.float32, k=64)
    assert torch.cuda.max_memory_allocated() - before <= room + (1 << 16)
    assert torch.cuda.memory_allocated() - before <= 1 << 16 and out[0].shape == (1, 64)
