"""How many rows are answered at a time: workspaces that fit beside tables of any size."""
import pytest
import torch

import paper_2005_13789_amd as ne
from paper_2005_13789_amd.linkpred import answers_batch


@pytest.mark.parametrize("k", [1, 10, 64])
@pytest.mark.parametrize("V,d", [(1, 1), (1000, 64), (100_003, 128), (1_000_000, 128), (10_000_000, 128), (100_000_000, 128), (2_000_000_000, 8), (50_000_000, 512)])
def test_batches_of_answers(V, d, k):
    """The workspace fits into the room there is, and batches are as large as asked for where that leaves them so."""
    need = lambda n: ne.ne_logprob_workspace_bytes(n, V, d, torch.float32, k=k)  # noqa: E731
    for room in (1 << 20, 1 << 30, 4 << 30, 8 * V * d, 1 << 40):
        for most in (1, 7, 192, 300, 8192):
            n = answers_batch(V, d, k, most, room)
            assert 1 <= n <= most
            assert need(n) <= room or n == 1
            assert n == most or need(most) > room
            assert n == most or need(2 * n) > room or n > most - 64      # not much less than there is room for
    # the framework's largest tables, 100 M nodes of 128: a few thousand rows at a time beside both of them
    assert answers_batch(100_000_000, 128, 10, 8192, 8 * 100_000_000 * 128) >= 1024
