"""Calls of the answers and of their gradients at the edges of what the header allows: nothing asked for, scores of exactly 0, very large and very
small ones, more candidates than a workgroup looks at together, coefficients that add up to nothing."""
import math

import pytest
import torch

import paper_2005_13789_amd as ne

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16]


def say(*a):
    print(*a, flush=True)


def normal(n, d, dtype, seed, sd):
    return (torch.randn(n, d, generator=torch.Generator().manual_seed(seed)) * sd).to(dtype).to(DEV)


def work(n, V, d, dtype, k=0, grad=False):
    return torch.empty(ne.ne_logprob_workspace_bytes(n, V, d, dtype, k=k, grad=grad), dtype=torch.uint8, device=DEV)


# ---------------------------------------------------------------------------------------------
# gradients of nothing
# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,d,pad", [(1, 8, 0), (20, 40, 3), (300, 64, 0)])
def test_gradients_of_nothing(n, d, pad, dtype):
    """Without ids and with both scales 0 entropies may be left out, and the gradients are zeros, also behind rows that are longer than dim."""
    V = 70
    say("nothing", n, d, pad, dtype)
    h, w = normal(n, d, dtype, 1, 1.0), normal(V, d, dtype, 2, 1.0)
    lse = torch.zeros(n, device=DEV)
    for dh_too, dw_too in ((True, True), (True, False), (False, True)):
        big_h, big_w = (torch.full((r, d + pad), 3.0, dtype=dtype, device=DEV) for r in (n, V))
        dh, dw = big_h[:, :d] if dh_too else None, big_w[:, :d] if dw_too else None
        ne.ne_logprob_grad(h, w, None, lse, None, dh, dw, work(n, V, d, dtype, grad=True), logp_scale=0.0)
        for g, big in ((dh, big_h), (dw, big_w)):
            assert bool((big[:, :d] == (3.0 if g is None else 0.0)).all()) and bool((big[:, d:] == 3.0).all())


# ---------------------------------------------------------------------------------------------
# more candidates than are looked at together
# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,V,d", [(1, 5000, 16), (40, 70_003, 8), (300, 9000, 24), (600, 20_001, 16)])
def test_many_equal_rows(n, V, d, dtype):
    """Thousands of rows tie, so candidates come in several turns, each of which may be cut in halves over and over: teams of four wavefronts, of
    sixteen, and those that rows are left to.  The answers are the lowest ids, every time."""
    k = 64
    say("many equal", n, V, d, dtype)
    h, w = normal(n, d, dtype, 3, 1.0), normal(1, d, dtype, 4, 1.0).expand(V, d).contiguous()
    other = torch.arange(V, device=DEV) % 1000 == 7         # some rows differ, and are behind the others whatever h is
    w[other] = 0
    s = (h.double() @ w[:1].double().t())[:, 0]
    rows = torch.arange(V, device=DEV)
    first, zeros = rows[~other][:k], rows[other]
    lse, entropy = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    space = work(n, V, d, dtype, k)
    # positive scores: the equal rows; negative ones: the rows of zeros, then the equal rows
    want = torch.where((s > 0)[:, None], first[None], torch.cat([zeros, first])[:k][None]).to(torch.int32)
    for turn in range(8):
        ids, logp = torch.full((n, k), -7, dtype=torch.int32, device=DEV), torch.empty((n, k), device=DEV)
        ne.ne_logprob(h, w, None, lse, space, entropy=entropy, top_ids=ids, top_logp=logp)
        assert torch.equal(ids, want), turn
        if turn == 0:
            kept = logp
        assert torch.equal(logp, kept), turn


# ---------------------------------------------------------------------------------------------
# scores of exactly 0, and products below fp32's normal numbers
# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,V,k", [(40, 3000, 1), (300, 3000, 1), (300, 3000, 12), (300, 100_003, 3), (700, 70_003, 2)])
def test_rows_of_zeros_are_best(n, V, k, dtype):
    """All scores are negative but for those of single rows of zeros, wherever in a chunk of table rows these lie."""
    d = 64
    say("zeros are best", n, V, k, dtype)
    h, w = normal(n, d, dtype, 5, 1.0).abs(), -normal(V, d, dtype, 6, 1.0).abs()
    for places in ([5], [17, 1000 + 46], [63, 129, 1000 + 31], [V - 1]):
        some = w.clone()
        some[places] = 0
        lse, ids, logp = torch.empty(n, device=DEV), torch.full((n, k), -7, dtype=torch.int32, device=DEV), torch.empty((n, k), device=DEV)
        ne.ne_logprob(h, some, None, lse, work(n, V, d, dtype, k), top_ids=ids, top_logp=logp)
        S = h.double() @ some.double().t()
        S[:, places] = 0
        want = torch.sort(S, dim=1, descending=True, stable=True)[1][:, :k]
        assert torch.equal(ids.long(), want), places


@pytest.mark.parametrize("n", [40, 300])
def test_best_of_very_small_products(n):
    """Products around the smallest numbers of fp32: places in the records survive the scaling, and scores in 64 bits decide."""
    V, d, k = 1500, 64, 5
    for size in (1e-17, 1e-20, 1e-23):
        say("small products", n, size)
        h, w = normal(n, d, torch.float32, 7, size), normal(V, d, torch.float32, 8, size)
        lse, ids, logp = torch.empty(n, device=DEV), torch.full((n, k), -7, dtype=torch.int32, device=DEV), torch.empty((n, k), device=DEV)
        ne.ne_logprob(h, w, None, lse, work(n, V, d, torch.float32, k), top_ids=ids, top_logp=logp)
        want = torch.sort(h.double().cpu() @ w.double().cpu().t(), dim=1, descending=True, stable=True)[1][:, :k]
        assert torch.equal(ids.cpu().long(), want)
