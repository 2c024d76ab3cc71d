"""Softmax cross entropy against a whole table and its gradients, against 64 bits."""
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


def call(h, w, t, loss_grad=None, scale=1.0, dh=True, dw=True, fill=None):
    n, V, d = h.shape[0], w.shape[0], h.shape[1]
    loss, lse = torch.full((n,), float("nan"), device=DEV), torch.full((n,), float("nan"), device=DEV)
    work = torch.empty(ne.ne_xent_workspace_bytes(n, V, d, h.dtype, False), dtype=torch.uint8, device=DEV)
    if fill is not None:
        work.fill_(fill)
    ne.ne_xent_loss(h, w, t, loss, lse, work)
    work = torch.empty(ne.ne_xent_workspace_bytes(n, V, d, h.dtype, True), dtype=torch.uint8, device=DEV)
    if fill is not None:
        work.fill_(fill)
    dh = torch.full((n, d), float("nan"), dtype=h.dtype, device=DEV) if dh else None
    dw = torch.full((V, d), float("nan"), dtype=h.dtype, device=DEV) if dw else None
    ne.ne_xent_grad(h, w, t, lse, dh, dw, work, loss_grad=loss_grad, scale=scale)
    return loss, lse, dh, dw


def check(h, w, t, loss, lse, dh, dw, loss_grad=None, scale=1.0):
    """Bounds from the arithmetic: a score is a sum of d products in fp32 (of 22-bit operands for float32 tables), so it is off by
    at most (2 d + 32) 2^-24 of its terms' magnitudes; the exponent and its base cost 4 2^-24 of the score's size; a sum of
    V terms in pieces V / 64 + 64 roundings.  G: rounded to bf16 or to 22 bits (and 2^-38 of 1), sums of V or n products; outputs
    are rounded once."""
    n, V, d = h.shape[0], w.shape[0], h.shape[1]
    u, op = 2.0 ** -24, U[h.dtype] if h.dtype == torch.bfloat16 else 2.0 ** -22
    H, W, T = h.double().cpu(), w.double().cpu(), t.long().cpu()
    ok = (T >= 0) & (T < V)
    H = torch.where(ok[:, None], H, torch.zeros((), dtype=torch.float64))
    S, A = H @ W.t(), H.abs() @ W.abs().t()
    z = torch.logsumexp(S, 1)
    at = T.clamp(0, V - 1)
    want_loss = torch.where(ok, z - S.gather(1, at[:, None])[:, 0], torch.zeros((), dtype=torch.float64))
    want_lse = torch.where(ok, z, torch.zeros((), dtype=torch.float64))
    score_err = u * ((2 * d + 32) * A.max(1).values + 4 * (S.abs().max(1).values + z.abs() + 1))
    tol = 2 * score_err + u * (V / 64 + 64)
    for got, want, name in ((loss, want_loss, "loss"), (lse, want_lse, "lse")):
        e = (got.double().cpu() - want).abs()
        assert bool((e <= tol).all()), (name, float((e / tol).max()))
        assert bool((got.cpu()[~ok] == 0).all())
    c = torch.ones(n, dtype=torch.float64) if loss_grad is None else loss_grad.double().cpu()
    c = c * scale
    p = torch.exp(S - z[:, None])
    hot = torch.zeros(n, V, dtype=torch.float64).scatter_(1, at[:, None], 1.0)
    G = torch.where(ok[:, None], p - hot, torch.zeros((), dtype=torch.float64)) * c[:, None]
    E = (p * (2 * tol[:, None] + 8 * u)) * c.abs()[:, None] + op * G.abs() + 2.0 ** -38 * c.abs()[:, None]
    E = torch.where(ok[:, None], E, torch.zeros((), dtype=torch.float64))
    for got, want, size, err, k, name in (
            (dh, G @ W, G.abs() @ W.abs(), E @ W.abs(), V, "dh"),
            (dw, G.t() @ H, G.abs().t() @ H.abs(), E.t() @ H.abs(), n, "dw")):
        if got is None:
            continue
        tol_g = 1.01 * (err + ((2 * k + 64) * u + 2.0 ** -22) * size)
        tol_g = tol_g + U[h.dtype] * (want.abs() + tol_g) + 1e-30
        e = (got.double().cpu() - want).abs()
        assert bool((e <= tol_g).all()), (name, float((e / tol_g).max()))
    if dh is not None:
        assert bool((dh.cpu()[~ok] == 0).all())


SHAPES = [(1, 1, 1), (1, 2, 3), (2, 127, 8), (3, 129, 64), (17, 1000, 100), (33, 500, 65), (64, 513, 128), (65, 255, 200), (127, 128, 96), (129, 300, 33),
          (300, 2049, 130), (257, 1111, 257), (1000, 700, 72), (200, 130, 1030)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,V,d", SHAPES)
def test_loss_and_gradients(n, V, d, dtype):
    say("xent", n, V, d, dtype)
    h, w, t = make(n, V, d, dtype, n + V + d)
    check(h, w, t, *call(h, w, t, scale=1.0 / n, fill=255), scale=1.0 / n)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,shift", [(1, 0), (0, 1), (8, 0), (24, 3)])
def test_strides_and_alignment(pad, shift, dtype):
    n, V, d = 70, 260, 64
    say("strides", pad, shift, dtype)
    h, w, t = make(n, V, d, dtype, 3, pad, shift)
    loss, lse, dh, dw = call(h, w, t)
    check(h, w, t, loss, lse, dh, dw)
    # gradients into slices of wider buffers: what lies between the rows stays
    big_h, big_w = torch.full((n, d + 5), 3.0, dtype=dtype, device=DEV), torch.full((V, d + 3), 3.0, dtype=dtype, device=DEV)
    work = torch.empty(ne.ne_xent_workspace_bytes(n, V, d, dtype, True), dtype=torch.uint8, device=DEV)
    ne.ne_xent_grad(h, w, t, lse, big_h[:, 2:2 + d], big_w[:, 1:1 + d], work)
    assert torch.equal(big_h[:, 2:2 + d], dh) and torch.equal(big_w[:, 1:1 + d], dw)
    for gap in (big_h[:, :2], big_h[:, 2 + d:], big_w[:, :1], big_w[:, 1 + d:]):
        assert bool((gap == 3.0).all())


def test_rows_far_apart():
    """Rows of a table that lie 8 MB or more apart: a tile's rows span more than 32 bits of bytes."""
    n, V, d, stride = 100, 700, 64, (1 << 22) + 8
    gen = torch.Generator().manual_seed(20)
    big = torch.empty(V * stride, dtype=torch.bfloat16, device=DEV)
    for step in (1 << 12, stride):
        w = big[:V * step].view(V, step)[:, :d]
        w.copy_((torch.randn(V, d, generator=gen) * 0.3).bfloat16())
        h, _, t = make(n, V, d, torch.bfloat16, 21)
        check(h, w, t, *call(h, w, t))


@pytest.mark.parametrize("dtype", TYPES)
def test_loss_gradients_of_rows(dtype):
    """A factor for every row, some of them zero, negative, or very small."""
    n, V, d = 150, 333, 80
    h, w, t = make(n, V, d, dtype, 8)
    c = torch.randn(n, device=DEV)
    c[::7] = 0.0
    c[1::9] *= 1e-6
    loss, lse, dh, dw = call(h, w, t, loss_grad=c, scale=0.25)
    check(h, w, t, loss, lse, dh, dw, loss_grad=c, scale=0.25)
    only_h = call(h, w, t, loss_grad=c, scale=0.25, dw=False)[2]
    only_w = call(h, w, t, loss_grad=c, scale=0.25, dh=False)[3]
    assert torch.equal(only_h, dh) and torch.equal(only_w, dw)


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_without_a_target_may_hold_anything(dtype):
    n, V, d = 200, 400, 64
    h, w, t = make(n, V, d, dtype, 4)
    loss, lse, dh, dw = call(h, w, t)
    out = (t < 0) | (t >= V)
    dirty = h.clone()
    dirty[out] = float("nan")
    dirty[torch.nonzero(out)[0, 0]] = float("inf")
    again = call(dirty, w, t)
    for a, b in zip((loss, lse, dh, dw), again):
        assert torch.equal(a, b)
    none = torch.full_like(t, -1)
    loss, lse, dh, dw = call(dirty, w, none)
    for x in (loss, lse, dh, dw):
        assert bool((x == 0).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_a_nan_stays_in_its_row(dtype):
    n, V, d = 140, 300, 64
    h, w, t = make(n, V, d, dtype, 6, ignored=0.0)
    loss, lse, dh, _ = call(h, w, t)
    h2 = h.clone()
    h2[5, 3] = float("nan")
    h2[77, 1] = float("inf")
    l2, z2, dh2, dw2 = call(h2, w, t)
    keep = torch.ones(n, dtype=torch.bool, device=DEV)
    keep[5] = keep[77] = False
    assert torch.equal(loss[keep], l2[keep]) and torch.equal(lse[keep], z2[keep]) and torch.equal(dh[keep], dh2[keep])
    assert bool(torch.isnan(l2[~keep]).all()) and bool(torch.isnan(dh2[~keep]).all()) and bool(torch.isnan(dw2).any())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sd", [1e-4, 3.0])
def test_small_and_large_scores(sd, dtype):
    """Nearly uniform softmaxes, and ones that are 1 at one row and 0 elsewhere (scores of hundreds)."""
    say("scores", sd, dtype)
    h, w, t = make(90, 500, 128, dtype, 10, sd=sd)
    check(h, w, t, *call(h, w, t))


def test_tables_of_very_different_sizes():
    """float32 halves follow each matrix's own largest magnitude."""
    for a, b in ((1e-20, 1e20), (1e15, 1e-15), (1e-30, 1.0)):
        h, w, t = make(60, 200, 64, torch.float32, 12)
        h, w = h * a, w * b
        check(h, w, t, *call(h, w, t))


def test_several_pieces_of_the_table():
    """More rows than the scores of a piece have room for: the pieces' gradients add up."""
    n, V, d = 9000, 9000, 16
    h, w, t = make(n, V, d, torch.float32, 14, ignored=0.05)
    loss, lse, dh, dw = call(h, w, t, scale=1.0 / n)
    H, W = h.double(), w.double()
    T = t.long()
    ok = (T >= 0) & (T < V)
    S = torch.mm(H, W.t())
    z = torch.logsumexp(S, 1)
    assert float((lse.double() - z)[ok].abs().max()) <= 1e-5
    G = torch.exp(S - z[:, None])
    G[torch.arange(n, device=DEV), T.clamp(0, V - 1)] -= 1.0
    G = G * (ok / n)[:, None]
    for got, want in ((dh, torch.mm(G, W)), (dw, torch.mm(G.t().contiguous(), H))):
        assert float((got.double() - want).norm() / want.norm()) <= 1e-5


def test_gradient_against_differences():
    """Central differences of the summed loss in 64 bits of step 2^-6 along 20 directions: the third derivative's share is
    step^2 / 6 of about 1, the losses' own error 1e-6 / step."""
    n, V, d = 40, 120, 24
    h, w, t = make(n, V, d, torch.float32, 16)
    _, _, dh, dw = call(h, w, t)
    gen = torch.Generator().manual_seed(1)
    step = 2.0 ** -6
    for _ in range(20):
        a, b = torch.randn(n, d, generator=gen).to(DEV), torch.randn(V, d, generator=gen).to(DEV)
        a, b = a / a.norm(), b / b.norm()
        up, down = (call(h + s * a, w + s * b, t)[0].double().sum() for s in (step, -step))
        slope = float((up - down) / (2 * step))
        want = float((dh.double() * a.double()).sum() + (dw.double() * b.double()).sum())
        assert abs(slope - want) <= 2e-3, (slope, want)


@pytest.mark.parametrize("dtype,n,V,d", [(torch.bfloat16, 1100, 60000, 400), (torch.bfloat16, 8300, 8200, 384), (torch.bfloat16, 600, 9000, 200),
                                         (torch.bfloat16, 3000, 20000, 100), (torch.float32, 1500, 20000, 60), (torch.float32, 2000, 9000, 120),
                                         (torch.float32, 1000, 30000, 300), (torch.bfloat16, 300, 150001, 256), (torch.float32, 16, 200003, 32)])
def test_larger_shapes(dtype, n, V, d):
    """Large and small tiles, rows of H in registers, partial sums and none, one piece and several: against 64 bits on the GPU.  Norms of
    the differences: scores are off by about 2^-22 sqrt(d), bf16 coefficients and outputs by 2^-9 each (rounding errors of independent
    elements: 2^-9 / sqrt(3) of their root mean square); twice that."""
    say("larger", dtype, n, V, d)
    h, w, t = make(n, V, d, dtype, n + d, ignored=0.1)
    loss, lse, dh, dw = call(h, w, t, scale=1.0 / n)
    H, W, T = h.double(), w.double(), t.long()
    ok = (T >= 0) & (T < V)
    S = torch.mm(H, W.t().contiguous())
    z = torch.logsumexp(S, 1)
    at = T.clamp(0, V - 1)
    want = z - S.gather(1, at[:, None])[:, 0]
    assert float((lse.double() - z)[ok].abs().max()) <= 2e-5 and float((loss.double() - want)[ok].abs().max()) <= 2e-5
    G = torch.exp(S - z[:, None])
    G[torch.arange(n, device=DEV), at] -= 1.0
    G = G * (ok / n)[:, None]
    bar = 2 * 2.0 ** -9 * (2 / 3) ** 0.5 if dtype == torch.bfloat16 else 1e-5
    for got, ref in ((dh, torch.mm(G, W)), (dw, torch.mm(G.t().contiguous(), H))):
        assert float((got.double() - ref).norm() / ref.norm()) <= bar, float((got.double() - ref).norm() / ref.norm())


@pytest.mark.parametrize("dtype,n,V,d", [(torch.bfloat16, 3000, 130000, 64), (torch.float32, 5000, 40000, 40), (torch.bfloat16, 4136, 100000, 300),
                                         (torch.bfloat16, 40, 4300000, 8), (torch.float32, 20, 4300000, 8), (torch.bfloat16, 100, 3000000, 16)])
def test_pieces_and_long_rows(dtype, n, V, d):
    """Coefficients that take several pieces of the table, and pieces of which one row of H has millions: bounds as above."""
    test_larger_shapes(dtype, n, V, d)


@pytest.mark.parametrize("dtype,n,V,d", [(torch.bfloat16, 38400, 3000, 64), (torch.float32, 40000, 2000, 40), (torch.bfloat16, 20000, 5000, 400)])
def test_many_rows(dtype, n, V, d):
    """More tiles of rows than places for workgroups, or about as many: bounds as above."""
    test_larger_shapes(dtype, n, V, d)


FEW = [(1, 3000, 1024), (16, 1000, 600), (20, 999, 500), (32, 777, 257), (5, 500, 16), (9, 17, 40), (16, 16, 128), (12, 5000, 250), (128, 300, 300),
       (33, 400, 600), (30, 300, 1000), (64, 333, 384), (64, 150, 1100), (4, 100, 1500), (31, 4000, 30)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,V,d", FEW)
def test_few_rows(n, V, d, dtype):
    """Few rows against tables of all widths, in one launch or two, with factors, in strided rows, one gradient at a time."""
    say("few", n, V, d, dtype)
    h, w, t = make(n, V, d, dtype, n + V + d, pad=3, shift=1)
    t[0] = V - 1
    c = torch.randn(n, generator=torch.Generator().manual_seed(d)).to(DEV)
    loss, lse, dh, dw = call(h, w, t, loss_grad=c, scale=0.5, fill=255)
    check(h, w, t, loss, lse, dh, dw, loss_grad=c, scale=0.5)
    assert torch.equal(call(h, w, t, loss_grad=c, scale=0.5, dw=False)[2], dh) and torch.equal(call(h, w, t, loss_grad=c, scale=0.5, dh=False)[3], dw)
    big_h, big_w = torch.full((n, d + 5), 3.0, dtype=dtype, device=DEV), torch.full((V, d + 3), 3.0, dtype=dtype, device=DEV)
    work = torch.empty(ne.ne_xent_workspace_bytes(n, V, d, dtype, True), dtype=torch.uint8, device=DEV)
    ne.ne_xent_grad(h, w, t, lse, big_h[:, 2:2 + d], big_w[:, 1:1 + d], work, loss_grad=c, scale=0.5)
    assert torch.equal(big_h[:, 2:2 + d], dh) and torch.equal(big_w[:, 1:1 + d], dw)
    for gap in (big_h[:, :2], big_h[:, 2 + d:], big_w[:, :1], big_w[:, 1 + d:]):
        assert bool((gap == 3.0).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_few_rows_that_hold_anything(dtype):
    n, V, d = 14, 700, 90
    h, w, t = make(n, V, d, dtype, 30, ignored=0.0)
    t[3], t[8] = -1, V
    first = call(h, w, t)
    dirty = h.clone()
    dirty[3], dirty[8] = float("nan"), float("inf")
    assert all(torch.equal(a, b) for a, b in zip(first, call(dirty, w, t)))
    dirty = h.clone()
    dirty[5, 7] = float("nan")
    loss, lse, dh, dw = call(dirty, w, t)
    keep = torch.arange(n, device=DEV) != 5
    assert torch.equal(loss[keep], first[0][keep]) and torch.equal(dh[keep], first[2][keep])
    assert bool(torch.isnan(loss[5])) and bool(torch.isnan(dh[5]).all()) and bool(torch.isnan(dw).all())
    none = call(h, w, torch.full_like(t, -1))
    assert all(bool((x == 0).all()) for x in none)


@pytest.mark.parametrize("dtype,n,V,d", [(torch.float32, 1, 200003, 256), (torch.float32, 32, 100003, 130), (torch.float32, 9, 50001, 1000),
                                         (torch.bfloat16, 16, 150001, 200), (torch.float32, 128, 60001, 250),
                                         (torch.float32, 170, 140001, 250), (torch.float32, 90, 45000, 790)])
def test_few_rows_of_large_tables(dtype, n, V, d):
    """Bounds as those of larger shapes."""
    test_larger_shapes(dtype, n, V, d)


def test_no_rows():
    w = torch.randn(50, 16, device=DEV)
    empty = torch.empty(0, 16, device=DEV)
    ids, f = torch.empty(0, dtype=torch.int32, device=DEV), torch.empty(0, device=DEV)
    ne.ne_xent_loss(empty, w, ids, f, f, None)
    dw = torch.ones_like(w)
    ne.ne_xent_grad(empty, w, ids, f, empty, dw, None)
    assert bool((dw == 0).all())


def test_the_same_every_time():
    for dtype in TYPES:
        h, w, t = make(500, 3000, 128, dtype, 18)
        first = call(h, w, t, fill=0)
        again = call(h, w, t, fill=255)
        assert all(torch.equal(a, b) for a, b in zip(first, again))


def halves(x, floor):
    """Largest error of x as the header states it: 2^-23 of the element, or `floor` of the matrix's largest magnitude."""
    return torch.maximum(2.0 ** -23 * x.abs(), torch.full_like(x, floor * float(x.abs().max())))


MIXED = ["plain", "outlier of w", "outlier of h", "small columns", "small rows", "small factors", "peaked"]


@pytest.mark.parametrize("kind", MIXED)
@pytest.mark.parametrize("n,V,d", [(16, 700, 96), (150, 900, 96), (200, 40000, 64)])
def test_float32_magnitudes_mixed_in_a_matrix(n, V, d, kind):
    """Bounds from the stated precision.  Halves: an element's error is 2^-23 of it, or 2^-38 of its matrix's largest magnitude, G's 2^-39 at
    least; of the four products of halves the smallest, up to 2^-22 of the whole, is left out; a sum of k terms takes 3 k roundings.  Few
    rows: no floors.  Every element is compared by itself, rows of the table that nobody's target names among them."""
    say("mixed", n, V, d, kind)
    few = n <= 32
    u, floor_m, floor_g = 2.0 ** -24, 0.0 if few else 2.0 ** -38, 0.0 if few else 2.0 ** -39
    h, w, t = make(n, V, d, torch.float32, n + V, ignored=0.1)
    h, w, c = h.contiguous(), w.contiguous(), torch.ones(n, device=DEV)
    if kind == "outlier of w":          # (a column that no row of H sees: the scores stay as they are)
        h[:, 5] = 0.0
        w[7, 5] = 2.0 ** 18
    elif kind == "outlier of h":
        w[:, 5] = 0.0
        h[3, 5] = 2.0 ** 18
        t[3] = 2
    elif kind == "small columns":
        h[:, 4:9] *= 2.0 ** -20
        w[:, 11:13] *= 2.0 ** -22
    elif kind == "small rows":
        h[::3] *= 2.0 ** -20
        w[1::3] *= 2.0 ** -22
    elif kind == "small factors":
        c[::2] = 2.0 ** -20
    elif kind == "peaked":              # coefficients from 1 down to 2^-60 and less
        h *= 6.0
    loss, lse, dh, dw = call(h, w, t, loss_grad=c, scale=0.5)
    H, W, T, C = h.double(), w.double(), t.long(), c.double()[:, None]
    ok = ((T >= 0) & (T < V))[:, None]
    H = torch.where(ok, H, 0.0)
    eh, ew = halves(H, floor_m), halves(W, floor_m)
    mm = lambda a, b: torch.mm(a.contiguous(), b.contiguous())  # noqa: E731
    S, A = mm(H, W.t()), mm(H.abs(), W.abs().t())
    z = torch.logsumexp(S, 1)[:, None]
    at = T.clamp(0, V - 1)[:, None]
    es = mm(eh, W.abs().t() + ew.t()) + mm(H.abs(), ew.t()) + (2.0 ** -22 + (3 * d + 32) * u) * A + 4 * u * (S.abs() + z.abs() + 1)
    tol = 2 * es.max(1).values[:, None] + u * (V / 64 + 64)
    for got, want, name in ((loss, z - S.gather(1, at), "loss"), (lse, z, "lse")):
        e = (got.double()[:, None] - torch.where(ok, want, 0.0)).abs()
        assert bool((e <= tol).all()), (name, float((e / tol).max()))
    p = torch.exp(S - z)
    G = torch.where(ok, p - torch.zeros_like(S).scatter_(1, at, 1.0), 0.0)
    E = torch.where(ok, p * (1.01 * (es + tol) + 8 * u) + torch.clamp(2.0 ** -23 * G.abs(), min=floor_g), 0.0)
    CH = C * H
    ech = halves(CH, floor_m) + u * CH.abs()
    for got, want, size, err, k, name in ((dh, mm(G, W) * C, mm(G.abs(), W.abs()) * C, (mm(E, W.abs() + ew) + mm(G.abs(), ew)) * C, V, "dh"),
                                          (dw, mm(G.t(), CH), mm(G.abs().t(), CH.abs()), mm(E.t(), CH.abs() + ech) + mm(G.abs().t(), ech), n, "dw")):
        bound = 0.5 * (err + (2.0 ** -22 + (3 * k + 64) * u) * size) * 1.01 + 1e-37
        e = (got.double() - 0.5 * want).abs()
        assert bool((e <= bound).all()), (name, float((e / bound).max()))
        say("  ", name, "worst share of the bound", float((e / bound).max()))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,V,d", [(1, 50, 64), (14, 700, 90), (60, 300, 128), (140, 300, 64), (140, 300, 100), (300, 3000, 200), (1100, 60000, 400)])
def test_infinities_and_nans_in_the_table(n, V, d, dtype):
    """A NaN in w, and in float32 an infinity, makes every loss of a row with a target NaN.  In bfloat16 an infinity gives a row a score
    of plus infinity (or NaN, against a zero): NaN; or of minus infinity: that table row counts as one of probability 0, or the loss
    is NaN.  Rows without a target stay 0; nothing of it is left for the next call."""
    say("infinities in w", n, V, d, dtype)
    h, w, t = make(n, V, d, dtype, n + d, ignored=0.2 if n > 1 else 0.0)
    at, col = V // 3, d - 3
    if n > 1:
        t[0] = at                   # its own score is the one that is not finite
        h[1, col] = 0.0
        t[1] = 2
    ok = (t >= 0) & (t < V)
    clean = call(h, w, t)
    side = h[:, col].double()
    rest = w.double().clone()
    rest[at] = 0.0
    S = torch.mm(h.double(), rest.t().contiguous())
    S[:, at] = -float("inf")
    z = torch.logsumexp(S, 1)
    want = z - S.gather(1, t.long().clamp(0, V - 1)[:, None])[:, 0]        # (infinite where the target is that row)
    for value in (float("inf"), -float("inf"), float("nan")):
        bad = w.clone()
        bad[at, col] = value
        loss, lse, _, _ = call(h, bad, t)
        assert bool((loss[~ok] == 0).all()) and bool((lse[~ok] == 0).all())
        may = ok & (side * value < 0) if dtype == torch.bfloat16 else torch.zeros_like(ok)
        assert bool(torch.isnan(loss[ok & ~may]).all()) and bool(torch.isnan(lse[ok & ~may]).all())
        left = may & ~torch.isnan(loss)
        say("  ", value, "rows that may go on without it", int(may.sum()), "that do", int(left.sum()))
        assert bool(((lse.double() - z)[left].abs() <= 2e-5).all())
        near = (loss.double() - want).abs() <= 2e-5
        assert bool((near | (loss.double() == want))[left].all())
    assert all(torch.equal(a, b) for a, b in zip(clean, call(h, w, t)))


@pytest.mark.parametrize("n,V,d,pad", [(100, 3000, 64, 0), (257, 1111, 257, 0), (300, 2000, 130, 3), (1100, 60000, 400, 0), (3000, 130000, 64, 0)])
def test_rows_of_a_table_with_much_in_common(n, V, d, pad):
    """bfloat16: a part that all rows of w share, ten times as large as what tells them apart, has no share in dh, as a row's coefficients
    add up to nothing; their roundings must not bring it in.  Independent rounding errors of 2^-8 / sqrt(3) at most, relative: of every
    coefficient but the target's, and of the output; twice their root mean square."""
    gen = torch.Generator().manual_seed(n + d)
    sd = d ** -0.25
    w, common, t = torch.randn(V, d + pad, generator=gen) * sd, torch.randn(d + pad, generator=gen) * 10 * sd, torch.randint(0, V, (n,), generator=gen)
    h = torch.randn(n, d + pad, generator=gen) * sd + 0.5 * w[t]
    h -= (h @ common)[:, None] / (common @ common) * common         # (no row sees the common part: scores stay moderate)
    h, w = h.bfloat16().to(DEV)[:, :d], (w + common).bfloat16().to(DEV)[:, :d]
    t[::9] = -1
    c = torch.rand(n, generator=gen).to(DEV) + 0.5
    t = t.to(torch.int32).to(DEV)
    dh = call(h, w, t, loss_grad=c, scale=1.0 / n)[2]
    H, W, T = h.double(), w.double(), t.long()
    ok, at = (T >= 0)[:, None], T.clamp(min=0)[:, None]
    S = torch.mm(H, W.t().contiguous())
    G = torch.where(ok, torch.exp(S - torch.logsumexp(S, 1)[:, None]) * c.double()[:, None] / n, 0.0)
    others = G.scatter(1, at, 0.0)
    G.scatter_add_(1, at, torch.where(ok, -c.double()[:, None] / n, 0.0))
    want = torch.mm(G, W)
    bar = 2 * 2.0 ** -8 / 3 ** 0.5 * (want.square().sum() + (others.square().sum(0) @ W.square()).sum()).sqrt()
    say("common part", n, V, d, "share of the bar", float((dh.double() - want).norm() / bar), "relative error", float((dh.double() - want).norm() / want.norm()))
    assert float((dh.double() - want).norm()) <= float(bar)


@pytest.mark.parametrize("factors", [False, True])
@pytest.mark.parametrize("n,V,d,pad", [(100, 3000, 64, 0), (257, 1111, 257, 0), (300, 2000, 130, 3), (1100, 60000, 400, 0), (3000, 130000, 64, 0), (2000, 700, 512, 0)])
def test_dw_in_bfloat16_is_nearly_the_rounded_one(n, V, d, pad, factors):
    """dw against the 64-bit one rounded to bfloat16: they differ where an error reaches across the edge of two values, which an error e does
    with probability |e| / spacing and which then makes a whole spacing, so that the squared difference is e times the spacing, 2^-7 of the
    value at most.  e is the root mean square of rounding errors of 2^-12 / sqrt(3), relative, of coefficients and, with factors, of rows times
    these; one and a half times the whole."""
    gen = torch.Generator().manual_seed(n + d)
    sd = d ** -0.25
    w, t = torch.randn(V, d + pad, generator=gen) * sd, torch.randint(0, V, (n,), generator=gen)
    h = (torch.randn(n, d + pad, generator=gen) * sd + 0.5 * w[t]).bfloat16().to(DEV)[:, :d]
    w = w.bfloat16().to(DEV)[:, :d]
    t[::9] = -1
    t = t.to(torch.int32).to(DEV)
    c = torch.rand(n, generator=gen).to(DEV) + 0.5 if factors else None
    dw = call(h, w, t, loss_grad=c, scale=1.0 / n)[3].double()
    H, T = h.double(), t.long()
    ok, at = (T >= 0)[:, None], T.clamp(min=0)[:, None]
    S = torch.mm(H, w.double().t().contiguous())
    G = torch.exp(S - torch.logsumexp(S, 1)[:, None]).scatter_add_(1, at, torch.full((n, 1), -1.0, dtype=torch.float64, device=DEV))
    G = torch.where(ok, G, 0.0).t().contiguous()
    CH = H / n if c is None else H * c.double()[:, None] / n
    want = torch.mm(G, CH)
    e = 2.0 ** -12 / 3 ** 0.5 * ((2 if factors else 1) * torch.mm(G.square(), CH.square())).sqrt()
    bar = 1.5 * (2.0 ** -7 * want.abs() * e).sum().sqrt()
    off = (dw - want.bfloat16().double()).norm()
    say("dw", n, V, d, "share of the bar", float(off / bar), "of dw", float(off / want.norm()), "error", float((dw - want).norm() / want.norm()))
    assert float(off) <= float(bar)


@pytest.mark.parametrize("dtype,n,d", [(torch.float32, 16, 1000), (torch.float32, 16, 1600), (torch.float32, 1, 1011), (torch.float32, 30, 780), (torch.bfloat16, 16, 4700),
                                       (torch.bfloat16, 30, 2300)])
def test_sums_of_few_wide_rows(dtype, n, d):
    """Root mean square of the errors of lse, which is nearly the score S of a target that a row leans to.  An addition in fp32 is off by 2^-24 / sqrt(3)
    of its result, root mean square.  S is made of C sums (4 up to 16 rows, 2 up to 32) of m of the d / 32 steps each, which grow evenly to S / C, so that
    together they are off by 2^-24 S sqrt(m / (9 C)); joining them and taking exponentials and the logarithm are six more roundings of S at most.  One
    and a half times that."""
    V, chains = 3000, 4 if n <= 16 else 2
    square = bar = 0.0
    runs = max(4, 96 // n)
    for seed in range(runs):
        gen = torch.Generator().manual_seed(seed)
        w, t = torch.randn(V, d, generator=gen) * d ** -0.25, torch.randint(0, V, (n,), generator=gen)
        h = (torch.randn(n, d, generator=gen) * d ** -0.25 + 0.5 * w[t]).to(dtype).to(DEV)
        w, t = w.to(dtype).to(DEV), t.to(torch.int32).to(DEV)
        lse = call(h, w, t, dh=False, dw=False)[1].double()
        z = torch.logsumexp(torch.mm(h.double(), w.double().t().contiguous()), 1)
        square += float((lse - z).square().mean()) / runs
        bar += float((z.square() * (-(-d // 32) / chains / (9 * chains) + 6 / 3)).mean()) * 2.0 ** -48 / runs
    say("few wide rows", dtype, n, d, "error", square ** 0.5, "share of the bar", (square / bar) ** 0.5 / 1.5)
    assert square ** 0.5 <= 1.5 * bar ** 0.5
