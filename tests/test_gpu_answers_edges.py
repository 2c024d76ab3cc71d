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


# ---------------------------------------------------------------------------------------------
# very large scores
# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,V,k", [(3, 700, 5), (60, 1000, 40), (300, 900, 3), (300, 5000, 2), (600, 2000, 20)])
def test_large_scores(n, V, k, dtype):
    """Scores of 2^20 to 1e28: probabilities are 0 and 1 (or shares of a few rows that fp32 cannot tell apart), everything stays finite, and what the best ids are
    asked for besides changes lse by no more than its own error."""
    d, u = 40, 2.0 ** -24
    for size in (2.0 ** 20, 2.0 ** 24, 2.0 ** 25, 2.0 ** 27, 2.0 ** 30, 1e12, 1e20, 1e27):
        say("large", n, V, k, dtype, size)
        h, w = normal(n, d, dtype, 9, (size / d) ** 0.5), normal(V, d, dtype, 10, (size / d) ** 0.5 / 4)
        S, A = h.double().cpu() @ w.double().cpu().t(), h.double().cpu().abs() @ w.double().cpu().abs().t()
        z = torch.logsumexp(S, 1)
        # a score: d products and sums, of 22-bit operands; its exponent: four roundings of numbers as large as the largest scores; a sum of V terms
        tol = 2 * u * ((2 * d + 32) * A.max(1).values + 4 * (S.abs().max(1).values + z.abs() + 1)) + u * (V / 64 + 64)
        for want_k in (0, k):
            lse, entropy = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
            ids, logp = (torch.full((n, k), -7, dtype=torch.int32, device=DEV), torch.empty((n, k), device=DEV)) if want_k else (None, None)
            ne.ne_logprob(h, w, None, lse, work(n, V, d, dtype, want_k), entropy=entropy, top_ids=ids, top_logp=logp)
            err = (lse.double().cpu() - z).abs()
            assert bool((err <= tol).all()), (want_k, float((err / tol).max()))
            assert bool((entropy >= -1e-5).all()) and bool((entropy <= math.log(V) + 1e-5).all()), want_k
        values, order = torch.sort(S, dim=1, descending=True, stable=True)
        assert torch.equal(ids.cpu().long(), order[:, :k])
        lp = values[:, :k] - z[:, None]
        assert bool(((logp.double().cpu() - lp).abs() <= tol[:, None] + u * lp.abs()).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [2, 300])
def test_many_equal_large_scores_of_both_signs(n, dtype):
    """Thousands of rows far below the best ones, in whichever order they come: their shares of the entropy are 0, not infinity times 0."""
    V, d, k = 40_000, 8, 3
    h = torch.full((n, d), 3e13, dtype=dtype, device=DEV)
    sign = torch.where(torch.arange(V, device=DEV) < V // 2, -1.0, 1.0)
    for flip in (1, -1):
        say("both signs", n, dtype, flip)
        w = (sign[:, None] * flip * torch.full((V, d), 3e13, device=DEV)).to(dtype)
        for want_k in (0, k):
            lse, entropy = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
            ids, logp = (torch.full((n, k), -7, dtype=torch.int32, device=DEV), torch.empty((n, k), device=DEV)) if want_k else (None, None)
            ne.ne_logprob(h, w, None, lse, work(n, V, d, dtype, want_k), entropy=entropy, top_ids=ids, top_logp=logp)
            # log of V / 2 equal terms: sums of ones are exact, a logarithm and a product are off by 2^-23 of it each
            assert bool(((entropy - math.log(V // 2)).abs() <= 2.0 ** -22 * 10).all()) and bool(torch.isfinite(lse).all())
        first = 0 if flip < 0 else V // 2
        assert bool((ids == first + torch.arange(k, device=DEV, dtype=torch.int32)).all())


# ---------------------------------------------------------------------------------------------
# very small products
# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("n,V,d", [(40, 900, 64), (150, 900, 64), (300, 65, 40), (300, 1, 33), (600, 2049, 100)])
@pytest.mark.parametrize("sizes", [(1.0, 1e-30), (1e-30, 1.0), (1e-16, 1e-16), (1e-19, 1e-20), (1e-25, 1e-10)])
def test_small_products(n, V, d, sizes):
    """Scores next to nothing: every row of the table has the same probability, and what lies behind the table's last row has none."""
    k = 4
    say("small products", n, V, d, sizes)
    h, w = normal(n, d, torch.float32, 11, sizes[0]), normal(V, d, torch.float32, 12, sizes[1])
    z = math.log(V)             # scores are below 1e-20
    for want_k in (0, k):
        lse, entropy, given = (torch.empty(n, device=DEV) for _ in range(3))
        ids, logp = (torch.full((n, k), -7, dtype=torch.int32, device=DEV), torch.empty((n, k), device=DEV)) if want_k else (None, None)
        which = torch.arange(n, device=DEV, dtype=torch.int32) % V
        ne.ne_logprob(h, w, which, lse, work(n, V, d, torch.float32, want_k), logp=given, entropy=entropy, top_ids=ids, top_logp=logp)
        # a sum of ones is exact; its logarithm, a product and a rounding: 2^-24 of at most 8 each, and of what they are joined from
        tol = 2.0 ** -24 * (8 + 8 * z)
        assert float((lse.double() - z).abs().max()) <= tol and float((entropy.double() - z).abs().max()) <= tol and float((given.double() + z).abs().max()) <= tol
    have = min(k, V)
    want = torch.sort(h.double().cpu() @ w.double().cpu().t(), dim=1, descending=True, stable=True)[1][:, :have]
    assert torch.equal(ids.cpu().long()[:, :have], want) and float((logp[:, :have].double() + z).abs().max()) <= tol


# ---------------------------------------------------------------------------------------------
# coefficients that add up to nothing
# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("shared,scale", [(0.0, 0), (10.0, 0), (30.0, 0), (10.0, 50), (10.0, -50)])
@pytest.mark.parametrize("n,V,d", [(64, 4000, 300), (40, 3001, 296), (700, 2000, 64), (400, 9000, 512), (600, 90_000, 512), (2100, 200_003, 300), (2100, 200_003, 296)])
def test_gradients_of_tables_with_a_shared_part(n, V, d, shared, scale):
    """bf16: rows of w share a part that is larger than what tells them apart, so that a row's coefficients of the entropy, several of them large,
    cancel in dh.  Coefficients keep 11 bits (2^-11 of themselves), a score d roundings of fp32 sums, outputs 2^-8; roundings are independent, so their sums'
    squares add up: a uniform one is 3^-1/2 of its largest on average, and what many of them make is held to 1.2 (all outputs) and 2 (a row's few large
    coefficients) of what is expected.  h and w take powers of two that cancel in the
    scores (norms stay below the 2^63 from which answers are NaN: rows have about 2^6)."""
    if V > 10_000 and (shared, scale) not in ((10.0, 0), (10.0, -50)):
        return
    say("shared part", n, V, d, shared, scale)
    gen = torch.Generator().manual_seed(13)
    sd = d ** -0.25
    h = (torch.randn(n, d, generator=gen) * sd).bfloat16().to(DEV)
    w = (torch.randn(V, d, generator=gen) * sd + shared * sd * torch.randn(1, d, generator=gen)).bfloat16().to(DEV)
    ids = torch.randint(0, V, (n,), generator=gen).to(torch.int32).to(DEV)
    H, W = h.double(), w.double()
    S = H @ W.t()
    z = torch.logsumexp(S, 1)
    L = S - z[:, None]
    p = L.exp()
    E = -(p * L).sum(1)
    h, w = h * 2.0 ** -scale, w * 2.0 ** scale
    lse, entropy = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    ne.ne_logprob(h, w, ids, lse, work(n, V, d, torch.bfloat16), entropy=entropy)
    size = lambda x: float(torch.linalg.vector_norm(x))  # noqa: E731
    for l, e, given in ((0.0, 1.0, True), (0.0, 1.0, False), (1.0, 1.0, True), (1.0, 0.05, True)):
        dh, dw = torch.full_like(h, float("nan")), torch.full_like(w, float("nan"))
        ne.ne_logprob_grad(h, w, ids if given else None, lse, entropy, dh, dw, work(n, V, d, torch.bfloat16, grad=True), logp_scale=l, entropy_scale=e)
        G = -l * p - e * p * (L + E[:, None])
        G[torch.arange(n, device=DEV), ids.long()] += l
        score = 2 * d ** 0.5 * 2.0 ** -24 * float(S.abs().max() + z.abs().max())
        each = 2.0 ** -11 / 3 ** 0.5 * G.abs() + score * (G.abs() + (l + e) * p)
        for got, want, err in ((dh.double() * 2.0 ** -scale, G @ W, (each ** 2 @ (W ** 2).sum(1)).sum() ** 0.5),
                               (dw.double() * 2.0 ** scale, G.t() @ H, ((each ** 2).sum(1) @ (H ** 2).sum(1)) ** 0.5)):
            floor = 2.0 ** -38 * (l + 8 * e) * (n * V) ** 0.5 * float((W if got.shape[0] == n else H).abs().max()) * d ** 0.5
            tol = 1.2 * 2.0 ** -8 / 3 ** 0.5 * size(want) + 2 * float(err) + floor
            # (dw: c h in fp16, too)
            tol = tol if got.shape[0] == n else tol + 2 * 2.0 ** -11 / 3 ** 0.5 * size(G.abs().t() @ H.abs())
            assert size(got - want) <= tol, (l, e, given, got.shape, size(got - want) / size(want), tol / size(want))
            say("  ", l, e, given, tuple(got.shape), size(got - want) / size(want), tol / size(want))


# ---------------------------------------------------------------------------------------------
# the same bits every time
# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,V,d,k", [(1, 200_003, 64, 10), (48, 10_000, 128, 20), (300, 70_003, 24, 33), (600, 3000, 64, 16), (700, 40_001, 16, 64)])
def test_answers_are_the_same_every_time(n, V, d, k, dtype):
    """Whichever thread comes upon a row first; and an id has the same log probability as a given one and as one of the best."""
    say("same", n, V, d, k, dtype)
    h, w = normal(n, d, dtype, 14, d ** -0.25), normal(V, d, dtype, 15, d ** -0.25)
    w[V // 2:V // 2 + 300] = w[:300]                # some tie, so rows have many candidates
    given, first = torch.zeros(n, dtype=torch.int32, device=DEV), None
    for turn in range(12):
        lse, entropy, logp = (torch.empty(n, device=DEV) for _ in range(3))
        ids, best = torch.full((n, k), -7, dtype=torch.int32, device=DEV), torch.empty((n, k), device=DEV)
        space = work(n, V, d, dtype, k).fill_(17 * turn)
        ne.ne_logprob(h, w, given, lse, space, logp=logp, entropy=entropy, top_ids=ids, top_logp=best)
        if turn:                                    # the given ids were some of the best of the turn before
            assert torch.equal(logp, best[:, turn % k])
        got = [lse, entropy, ids, best]
        first = first or [x.clone() for x in got]
        assert all(torch.equal(a, b) for a, b in zip(got, first)), turn
        given = ids[:, (turn + 1) % k].contiguous()
