"""Log probabilities, entropies and best ids against a whole table, and their gradients, against 64 bits."""
import math

import pytest
import torch

import paper_2005_13789_amd as ne

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16]
U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def say(*a):
    print(*a, flush=True)


def rows(n, d, dtype, gen, sd, pad=0, shift=0):
    buf = (torch.randn(shift + n * (d + pad) + 8, generator=gen) * sd).to(dtype).to(DEV)
    return buf[shift:shift + n * (d + pad)].view(n, d + pad)[:, :d]


def make(n, V, d, dtype, seed, pad=0, shift=0, sd=None, ignored=0.2):
    gen = torch.Generator().manual_seed(seed)
    sd = d ** -0.25 if sd is None else sd
    h, w = rows(n, d, dtype, gen, sd, pad, shift), rows(V, d, dtype, gen, sd, pad, shift)
    t = torch.randint(0, V, (n,), generator=gen)
    out = torch.rand(n, generator=gen)
    t[out < ignored] = -1
    t[out < ignored / 3] = V
    return h, w, t.to(torch.int32).to(DEV)


def answers(h, w, ids, k, fill=None, rows_of_workspace=None):
    n, V, d = h.shape[0], w.shape[0], h.shape[1]
    new = lambda *s: torch.full(s, float("nan"), device=DEV)  # noqa: E731
    out = {"lse": new(n), "entropy": new(n), "logp": new(n) if ids is not None else None}
    if k:
        out["top_ids"], out["top_logp"] = torch.full((n, k), -7, dtype=torch.int32, device=DEV), new(n, k)
    work = torch.empty(ne.ne_logprob_workspace_bytes(rows_of_workspace or n, V, d, h.dtype, k=k), dtype=torch.uint8, device=DEV)
    if fill is not None:
        work.fill_(fill)
    ne.ne_logprob(h, w, ids, out["lse"], work, logp=out["logp"], entropy=out["entropy"], top_ids=out.get("top_ids"), top_logp=out.get("top_logp"))
    return out


def truth(h, w, ids):
    H, W = h.double().cpu(), w.double().cpu()
    n, V = H.shape[0], W.shape[0]
    ok = torch.ones(n, dtype=torch.bool)
    T = torch.zeros(n, dtype=torch.long)
    if ids is not None:
        T = ids.long().cpu()
        ok = (T >= 0) & (T < V)
        T = T.clamp(0, V - 1)
    H = torch.where(ok[:, None], H, torch.zeros((), dtype=torch.float64))
    kinds, which = W.unique(dim=0, return_inverse=True)      # (equal rows get equal scores, whichever way a product takes them)
    S, A = (H @ kinds.t())[:, which], H.abs() @ W.abs().t()
    return H, W, T, ok, S, A, torch.logsumexp(S, 1)


def lse_tolerance(S, A, z, d, V):
    """A score is a sum of d products in fp32 (of 22-bit operands for float32 tables): off by at most (2 d + 32) 2^-24 of its terms'
    magnitudes; the exponent and its base cost 4 2^-24 of the score's size; a sum of V terms in pieces V / 64 + 64 roundings."""
    u = 2.0 ** -24
    score_err = u * ((2 * d + 32) * A.max(1).values + 4 * (S.abs().max(1).values + z.abs() + 1))
    return score_err, 2 * score_err + u * (V / 64 + 64)


def check(h, w, ids, out, k):
    n, V, d = h.shape[0], w.shape[0], h.shape[1]
    H, W, T, ok, S, A, z = truth(h, w, ids)
    u = 2.0 ** -24
    score_err, tol = lse_tolerance(S, A, z, d, V)
    zero = torch.zeros((), dtype=torch.float64)
    L = S - z[:, None]
    p = torch.exp(L)
    E = -(p * torch.where(p > 0, L, zero)).sum(1)
    # entropy: a probability is off by 2 tol of itself, its logarithm by 2 tol; the mean magnitude of log p is at least the entropy
    tol_e = 2 * tol * (2 + (p * L.abs()).sum(1)) + u * (V / 64 + 64) * (1 + E)
    want = {"lse": (z, tol), "entropy": (E, tol_e)}
    if ids is not None:         # scores in 64 bits: what lse is off by, and a rounding
        lp = L.gather(1, T[:, None])[:, 0]
        want["logp"] = (lp, tol + u * lp.abs())
    for name, (v, t) in want.items():
        got = out[name].cpu()
        e = (got.double() - torch.where(ok, v, zero)).abs()
        assert bool((e <= t).all()), (name, float((e / t).max()))
        assert bool((got[~ok] == 0).all()), name
    if not k:
        return
    have = min(k, V)
    # the order of scores in 64 bits, the lower id first among equals
    order = torch.sort(S, dim=1, descending=True, stable=True)
    ids_, vals = out["top_ids"].cpu(), out["top_logp"].cpu()
    assert bool((ids_[~ok] == -1).all()) and bool((vals[~ok] == -math.inf).all())
    assert torch.equal(ids_[ok][:, :have].long(), order[1][ok][:, :have]), "ids"
    lp = order[0][:, :have] - z[:, None]
    e = (vals[:, :have].double() - lp).abs()[ok]
    t = (tol[:, None] + u * lp.abs())[ok]
    assert bool((e <= t).all()), "top_logp"
    assert bool((ids_[:, have:] == -1).all()) and bool((vals[:, have:] == -math.inf).all())


SHAPES = [(1, 1, 1, 1), (1, 2, 3, 5), (3, 129, 64, 64), (17, 1000, 100, 10), (33, 500, 65, 3), (64, 513, 128, 17), (65, 255, 200, 64), (127, 128, 96, 1),
          (129, 300, 33, 33), (300, 2049, 130, 10), (257, 1111, 257, 0), (1000, 700, 72, 8), (200, 130, 1030, 40), (193, 5000, 40, 50)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,V,d,k", SHAPES)
def test_answers(n, V, d, k, dtype):
    say("answers", n, V, d, k, dtype)
    h, w, ids = make(n, V, d, dtype, n + V + d)
    check(h, w, ids, answers(h, w, ids, k, fill=255), k)
    check(h, w, None, answers(h, w, None, k, fill=255), k)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,shift", [(1, 0), (0, 1), (8, 0), (24, 3)])
def test_strides_and_alignment(pad, shift, dtype):
    for n in (20, 210):
        say("strides", n, pad, shift, dtype)
        h, w, ids = make(n, 333, 64, dtype, 3, pad, shift)
        check(h, w, ids, answers(h, w, ids, 12), 12)


@pytest.mark.parametrize("dtype", TYPES)
def test_large_tiles(dtype):
    """Tiles of 256 x 256, whose wavefronts have two chunks of table rows each."""
    say("large tiles", dtype)
    h, w, ids = make(600, 100_003, 400, dtype, 5)
    check(h, w, ids, answers(h, w, ids, 20), 20)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,V,d,k", [(513, 40_000, 24, 64), (1500, 70_001, 20, 5), (700, 66_000, 33, 1), (5000, 17_000, 16, 30), (600, 131_073, 8, 12)])
def test_many_rows_of_large_tables(n, V, d, k, dtype):
    """Groups of tiles, whose best decide which records are read; splits of the table that end early."""
    say("groups", n, V, d, k, dtype)
    h, w, ids = make(n, V, d, dtype, n + k)
    check(h, w, ids, answers(h, w, ids, k, fill=255), k)
    w[:] = w[torch.arange(V, device=DEV) % 1000]       # equal rows in many groups
    check(h[:520], w, ids[:520], answers(h[:520], w, ids[:520], k, fill=127), k)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [5, 300])
def test_equal_scores(n, dtype):
    """Equal rows tie exactly: the lowest ids first, whichever tiles they are in; a table of zeros, and rows of zeros."""
    V, d, k = 3000, 48, 20
    say("equal", n, dtype)
    h, w, ids = make(n, V, d, dtype, 7)
    w[:] = w[torch.arange(V, device=DEV) % 37]           # 37 different rows, each some 80 times
    check(h, w, ids, answers(h, w, ids, k), k)
    w[:] = w[0].clone()
    out = answers(h, w, None, k)
    assert bool((out["top_ids"] == torch.arange(k, device=DEV, dtype=torch.int32)).all())
    w.zero_()
    out = answers(h, w, None, k)
    assert bool((out["top_ids"] == torch.arange(k, device=DEV, dtype=torch.int32)).all())
    assert bool((out["entropy"] - math.log(V)).abs().max() < 1e-5)
    h, w, ids = make(n, V, d, dtype, 8)
    h[::2] = 0
    check(h, w, ids, answers(h, w, ids, k), k)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [3, 200])
def test_nearly_equal_scores(n, dtype):
    """Rows that differ in their last bit only: sums in 32 bits do not tell which score is larger, the answers do."""
    V, d, k = 700, 256, 30
    say("nearly equal", n, dtype)
    h, w, ids = make(n, V, d, dtype, 9)
    gen = torch.Generator().manual_seed(10)
    base = w[0].clone()
    w[:] = base
    at = torch.randint(0, d, (V,), generator=gen).to(DEV)
    row = torch.arange(V, device=DEV)
    w[row, at] = w[row, at] * (1 + torch.finfo(dtype).eps)
    if dtype == torch.float32:
        assert (h.float() @ w.t())[0].unique().numel() < V
    check(h, w, ids, answers(h, w, ids, k), k)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [4, 150])
def test_scales(n, dtype):
    """Peaked and flat rows, and tables far from 1."""
    V, d, k = 900, 64, 9
    for sd in (1e-12, 1e-3, 1.0, 3.0):
        say("scales", n, sd, dtype)
        h, w, ids = make(n, V, d, dtype, 11, sd=sd)
        check(h, w, ids, answers(h, w, ids, k), k)
    say("scales", "squares below fp32")
    h, w, ids = make(n, V, d, torch.float32, 12)
    H, W = h.to(dtype), (w * 1e-25).to(dtype)
    check(H, W, ids, answers(H, W, ids, k), k)
    h, w, ids = make(n, V, d, dtype, 12)
    for a, b in ((1e12, 1e-12), (1e-12, 1e12)):
        say("scales", a, b)
        H, W = (h * a).to(dtype), (w * b).to(dtype)
        check(H, W, ids, answers(H, W, ids, k), k)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [6, 140])
def test_values_that_are_not_finite(n, dtype):
    V, d, k = 400, 40, 5
    h, w, ids = make(n, V, d, dtype, 13, ignored=0.0)
    good = answers(h, w, ids, k)
    h2, ids2 = h.clone(), ids.clone()
    h2[1, 3], h2[2, 0], h2[3, 39], h2[4] = float("nan"), float("inf"), -float("inf"), float("nan")
    ids2[4] = -1
    out = answers(h2, w, ids2, k)
    for name, v in out.items():
        assert torch.equal(v[5:], good[name][5:]), name
        assert torch.equal(v[0], good[name][0]), name
    for i in (1, 2, 3):
        assert all(bool(torch.isnan(out[name][i]).all()) for name in ("lse", "logp", "entropy", "top_logp")) and bool((out["top_ids"][i] == -1).all())
    assert out["lse"][4] == 0 and out["logp"][4] == 0 and out["entropy"][4] == 0 and bool((out["top_ids"][4] == -1).all())
    for bad in (float("nan"), float("inf"), -float("inf")):
        w2 = w.clone()
        w2[V - 1, 2] = bad
        out = answers(h, w2, ids, k)
        assert all(bool(torch.isnan(out[name]).all()) for name in ("lse", "logp", "entropy", "top_logp")) and bool((out["top_ids"] == -1).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_workspaces_of_more_rows_serve_fewer(dtype):
    V, d, k = 1500, 96, 7
    for n in (1, 15, 16, 17, 32, 33, 64, 65, 128, 191, 192, 193, 256, 600):
        assert ne.ne_logprob_workspace_bytes(n, V, d, dtype, k=k) <= ne.ne_logprob_workspace_bytes(n + 1, V, d, dtype, k=k)
    for n in (1, 60, 100, 199):
        h, w, ids = make(n, V, d, dtype, 14)
        check(h, w, ids, answers(h, w, ids, k, rows_of_workspace=200), k)


def test_no_rows():
    w = torch.randn(10, 8, device=DEV)
    h, none, nothing = torch.empty(0, 8, device=DEV), torch.empty(0, device=DEV), torch.empty(0, dtype=torch.uint8, device=DEV)
    ne.ne_logprob(h, w, torch.empty(0, dtype=torch.int32, device=DEV), none, nothing, logp=none)
    dw = torch.full((10, 8), 3.0, device=DEV)
    ne.ne_logprob_grad(h, w, None, none, none, None, dw, nothing, logp_scale=0.0, entropy_scale=1.0)
    assert bool((dw == 0).all())


# ---------------------------------------------------------------------------------------------
# gradients
# ---------------------------------------------------------------------------------------------
def gradients(h, w, ids, logp_grad=None, entropy_grad=None, logp_scale=1.0, entropy_scale=0.0, dh=True, dw=True, fill=None):
    n, V, d = h.shape[0], w.shape[0], h.shape[1]
    out = answers(h, w, ids, 0)
    work = torch.empty(ne.ne_logprob_workspace_bytes(n, V, d, h.dtype, grad=True), dtype=torch.uint8, device=DEV)
    if fill is not None:
        work.fill_(fill)
    dh = torch.full((n, d), float("nan"), dtype=h.dtype, device=DEV) if dh else None
    dw = torch.full((V, d), float("nan"), dtype=h.dtype, device=DEV) if dw else None
    ne.ne_logprob_grad(h, w, ids, out["lse"], out["entropy"], dh, dw, work, logp_grad=logp_grad, entropy_grad=entropy_grad,
                       logp_scale=logp_scale, entropy_scale=entropy_scale)
    return dh, dw


def check_gradients(h, w, ids, dh, dw, logp_grad=None, entropy_grad=None, logp_scale=1.0, entropy_scale=0.0):
    """G: an exponential (2 tol of itself) times a factor made of log p and the entropy (off by 2 tol + tol_e and 8 roundings of what it is the sum
    of); rounded to 22 bits, or for bf16 tables to bf16, and 2^-38 of f = |l| + 8 |e|; sums of V or n products; outputs are rounded once."""
    n, V, d = h.shape[0], w.shape[0], h.shape[1]
    u, op = 2.0 ** -24, U[h.dtype] if h.dtype == torch.bfloat16 else 2.0 ** -22
    H, W, T, ok, S, A, z = truth(h, w, ids)
    _, tol = lse_tolerance(S, A, z, d, V)
    zero = torch.zeros((), dtype=torch.float64)
    one = torch.ones(n, dtype=torch.float64)
    l = logp_scale * (one if logp_grad is None else logp_grad.double().cpu()) * ok
    e = entropy_scale * (one if entropy_grad is None else entropy_grad.double().cpu()) * ok
    L = S - z[:, None]
    p = torch.exp(L)
    E = -(p * torch.where(p > 0, L, zero)).sum(1)
    tol_e = 2 * tol * (2 + (p * L.abs()).sum(1)) + u * (V / 64 + 64) * (1 + E)
    hot = torch.zeros(n, V, dtype=torch.float64)
    if ids is not None:
        hot.scatter_(1, T[:, None], 1.0)
    G = l[:, None] * (hot - p) - e[:, None] * p * (L + E[:, None])
    G = torch.where(ok[:, None], G, zero)
    f = l.abs() + 8 * e.abs()
    parts = l.abs()[:, None] + e.abs()[:, None] * (L.abs() + E[:, None] + 10)
    err = p * ((2 * tol + 8 * u)[:, None] * parts + e.abs()[:, None] * (2 * tol + tol_e)[:, None]) + op * G.abs() + (2.0 ** -38 + 0.0) * f[:, None]
    err = torch.where(ok[:, None], err, zero)
    for got, want, size, er, k, name in (
            (dh, G @ W, G.abs() @ W.abs(), err @ W.abs(), V, "dh"),
            (dw, G.t() @ H, G.abs().t() @ H.abs(), err.t() @ H.abs(), n, "dw")):
        if got is None:
            continue
        tol_g = 1.01 * (er + ((2 * k + 64) * u + 2.0 ** -22) * size)
        tol_g = tol_g + U[h.dtype] * (want.abs() + tol_g) + 1e-30
        diff = (got.double().cpu() - want).abs()
        assert bool((diff <= tol_g).all()), (name, float((diff / tol_g).max()))
    if dh is not None:
        assert bool((dh.cpu()[~ok] == 0).all())


GRAD_SHAPES = [(1, 1, 1), (1, 2, 3), (3, 129, 64), (17, 1000, 100), (33, 500, 65), (64, 513, 128), (65, 255, 200), (129, 300, 33), (300, 2049, 130),
               (257, 1111, 257), (1000, 700, 72), (20, 130, 1030), (16, 300, 256)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,V,d", GRAD_SHAPES)
def test_gradients(n, V, d, dtype):
    say("gradients", n, V, d, dtype)
    h, w, ids = make(n, V, d, dtype, n + V + d)
    for kw in (dict(logp_scale=-1.0 / n, entropy_scale=-0.05 / n), dict(logp_scale=0.0, entropy_scale=1.0), dict(logp_scale=0.3, entropy_scale=0.0)):
        check_gradients(h, w, ids, *gradients(h, w, ids, fill=255, **kw), **kw)
    kw = dict(logp_scale=0.0, entropy_scale=-2.0)
    check_gradients(h, w, None, *gradients(h, w, None, fill=255, **kw), **kw)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [14, 150])
def test_gradients_of_rows(n, dtype):
    """Factors of rows, some of them zero, negative, or very small; one output at a time."""
    V, d = 333, 80
    h, w, ids = make(n, V, d, dtype, 8)
    a, b = torch.randn(n, device=DEV), torch.randn(n, device=DEV)
    a[::7], b[::5], b[1::9] = 0.0, 0.0, b[1::9] * 1e-6
    kw = dict(logp_grad=a, entropy_grad=b, logp_scale=0.5, entropy_scale=-0.25)
    dh, dw = gradients(h, w, ids, **kw)
    check_gradients(h, w, ids, dh, dw, **kw)
    assert torch.equal(gradients(h, w, ids, dw=False, **kw)[0], dh) and torch.equal(gradients(h, w, ids, dh=False, **kw)[1], dw)


def test_gradients_of_log_probabilities_are_the_losses():
    for dtype in TYPES:
        for n in (10, 100):
            h, w, ids = make(n, 400, 64, dtype, 15)
            lse, loss = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
            work = torch.empty(ne.ne_xent_workspace_bytes(n, 400, 64, dtype, True), dtype=torch.uint8, device=DEV)
            ne.ne_xent_loss(h, w, ids, loss, lse, work)
            dh, dw = torch.empty_like(h), torch.empty_like(w)
            ne.ne_xent_grad(h, w, ids, lse, dh, dw, work, scale=0.125)
            work = torch.empty(ne.ne_logprob_workspace_bytes(n, 400, 64, dtype, grad=True), dtype=torch.uint8, device=DEV)
            dh2, dw2 = torch.empty_like(h), torch.empty_like(w)
            ne.ne_logprob_grad(h, w, ids, lse, None, dh2, dw2, work, logp_scale=-0.125)
            assert torch.equal(dh, dh2) and torch.equal(dw, dw2)


def test_gradients_against_differences():
    """The objective's change along a direction, by central differences of ne_logprob's own answers."""
    n, V, d = 40, 300, 32
    h, w, ids = make(n, V, d, torch.float32, 16, ignored=0.1)
    gen = torch.Generator().manual_seed(17)
    kw = dict(logp_scale=0.7, entropy_scale=-0.4)
    dh, dw = gradients(h, w, ids, **kw)

    def objective(h, w):
        out = answers(h, w, ids, 0)
        return float(0.7 * out["logp"].double().sum() - 0.4 * out["entropy"].double().sum())

    for which in (0, 1):
        x = (h, w)[which]
        v = torch.randn(x.shape, generator=gen).to(DEV)
        step = 2.0 ** -8
        args = [(h + step * v, w), (h - step * v, w)] if which == 0 else [(h, w + step * v), (h, w - step * v)]
        slope = (objective(*args[0]) - objective(*args[1])) / (2 * step)
        want = float(((dh, dw)[which].double() * v.double()).sum())
        # differences: a third derivative times step^2 / 6 (scores move by |v| |x| step, about 0.02 a row), and 64 roundings of n values of size 10
        assert abs(slope - want) <= 0.01 * abs(want) + 2e-4 * n, (which, slope, want)


def test_streams_and_graphs():
    """A captured pass replays on new inputs; two streams with a workspace each do not disturb one another."""
    n, V, d, k = 70, 900, 64, 6
    h, w, ids = make(n, V, d, torch.bfloat16, 18)
    h2, w2, ids2 = make(n, V, d, torch.bfloat16, 19)
    sets = [(h.clone(), w.clone(), ids.clone()) for _ in range(2)]
    outs, works = [], []
    for _ in range(2):
        new = lambda *s, dtype=torch.float32: torch.empty(s, dtype=dtype, device=DEV)  # noqa: E731
        outs.append(dict(lse=new(n), logp=new(n), entropy=new(n), top_ids=new(n, k, dtype=torch.int32), top_logp=new(n, k), dh=torch.empty_like(h.contiguous()),
                         dw=torch.empty_like(w.contiguous())))
        works.append(new(max(ne.ne_logprob_workspace_bytes(n, V, d, torch.bfloat16, k=k), ne.ne_logprob_workspace_bytes(n, V, d, torch.bfloat16, grad=True)),
                         dtype=torch.uint8))

    def run(i):
        H, W, T = sets[i]
        o = outs[i]
        ne.ne_logprob(H, W, T, o["lse"], works[i], logp=o["logp"], entropy=o["entropy"], top_ids=o["top_ids"], top_logp=o["top_logp"])
        ne.ne_logprob_grad(H, W, T, o["lse"], o["entropy"], o["dh"], o["dw"], works[i], logp_scale=-1.0, entropy_scale=-0.1)

    run(0)
    first = {name: v.clone() for name, v in outs[0].items()}
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for i, s in enumerate(streams):
        with torch.cuda.stream(s):
            run(i)
    torch.cuda.synchronize()
    for o in outs:
        for name, v in o.items():
            assert torch.equal(v, first[name]), name
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(0)
    for source in ((h2, w2, ids2), (h, w, ids), (h2, w2, ids2)):
        for to, x in zip(sets[0], source):
            to.copy_(x)
        for to, x in zip(sets[1], source):
            to.copy_(x)
        for v in outs[0].values():
            v.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        run(1)
        torch.cuda.synchronize()
        for name, v in outs[0].items():
            assert torch.equal(v, outs[1][name]), name
