"""Newton-Schulz updates and Muon's step, against the same products in 64 bits."""
import math

import pytest
import torch

import paper_2005_13789_amd as ne

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16]
U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
A, B, C = 3.4445, -4.7750, 2.0315


def say(*a):
    print(*a, flush=True)


def exact(x, steps=5):
    x = x.double()
    wide = x.shape[1] > x.shape[0]
    x = x.t() if wide else x
    norm = torch.linalg.vector_norm(x)
    x = x / norm if norm > 0 else x
    for _ in range(steps):
        g = x.t() @ x
        x = A * x + x @ (B * g + C * (g @ g))
    return x.t() if wide else x


def tolerance(x, steps, small):
    """Of the result's 2-norm over all elements, relative to it.  Operands keep 22 bits and a product of halves leaves out 2^-22 of its terms: a product's
    result is off by eta = 4 2^-22 of the norms of its operands, of which a step of the small side takes up to four one after the other.  What they
    do to a direction of singular value s: G's error eta of its largest eigenvalue changes s Q(s^2) by eta (1 + s_max^2 / s^2) of itself as long as a G serves,
    three steps at most, in which s grows by 3.4445 each time, so that the later stages see what has grown; and a step after that multiplies relative errors by
    at most |s f'(s) / f(s)| = 3 (s near the ends of where they settle)."""
    s = torch.linalg.svdvals(x.double().cpu())
    s = s / torch.linalg.vector_norm(s)
    s = s[s > 0]
    eta, total, at, left = 4 * 2.0 ** -22, torch.zeros_like(s), s.clone(), steps
    first = True
    while left > 0:
        now = min(left, 3 if first else 2)
        total = total * 3.0 ** (0 if first else now) + 4 * now * eta * (1 + at.max() ** 2 / at.clamp(min=1e-12) ** 2)
        for _ in range(now):
            at = (A * at + B * at ** 3 + C * at ** 5).abs()
        first, left = False, left - now
    total = total.clamp(max=2.0)
    return float(torch.linalg.vector_norm(total * at) / torch.linalg.vector_norm(at))


def orthogonal(x, steps=5, out_type=None, fill=None, out=None):
    work = torch.empty(ne.ne_orthogonalize_workspace_bytes(*x.shape), dtype=torch.uint8, device=DEV)
    if fill is not None:
        work.fill_(fill)
    out = torch.full(x.shape, float("nan"), dtype=out_type or x.dtype, device=DEV) if out is None else out
    ne.ne_orthogonalize(x, out, work, steps=steps)
    return out


def check(x, out, steps=5):
    want = exact(x.cpu(), steps)
    tol = tolerance(x, steps, min(x.shape)) + U[out.dtype]
    err = float(torch.linalg.vector_norm(out.double().cpu() - want) / torch.linalg.vector_norm(want).clamp(min=1e-300))
    assert err <= tol, (tuple(x.shape), err, tol)


def update(rows, cols, seed, dtype=torch.float32, strong=0.3, size=1e-4):
    gen = torch.Generator().manual_seed(seed)
    r = min(8, rows, cols)
    x = strong * torch.randn(rows, r, generator=gen) @ torch.randn(r, cols, generator=gen) + torch.randn(rows, cols, generator=gen)
    return (x * size).to(dtype).to(DEV)


SHAPES = [(1, 1), (1, 7), (9, 1), (2, 2), (5, 3), (31, 33), (33, 31), (64, 64), (100, 40), (40, 100), (127, 129), (129, 127), (300, 128), (1000, 100),
          (97, 2001), (2001, 97), (4000, 65), (513, 300), (260, 1030), (700, 700), (5000, 160), (20_000, 33)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_orthogonalize(rows, cols, dtype):
    say("orthogonalize", rows, cols, dtype)
    x = update(rows, cols, rows + cols, dtype)
    kept = x.clone()
    check(x, orthogonal(x, fill=255))
    check(x, orthogonal(x, out_type=torch.float32 if dtype == torch.bfloat16 else torch.bfloat16, fill=255))
    assert torch.equal(x, kept)


@pytest.mark.parametrize("steps", range(1, ne.NE_ORTHOGONAL_MAX_STEPS + 1))
def test_numbers_of_steps(steps):
    say("steps", steps)
    for shape in ((200, 50), (50, 200), (300, 200)):
        x = update(*shape, 1)
        check(x, orthogonal(x, steps=steps), steps)


@pytest.mark.parametrize("size", [1e-30, 1e-12, 1.0, 1e6, 1e18])
def test_sizes_of_values(size):
    """The result does not depend on the update's size."""
    say("size", size)
    x = update(400, 60, 2, size=size)
    check(x, orthogonal(x))


@pytest.mark.parametrize("shape", [(600, 80), (80, 600), (500, 256)])
def test_spectra(shape):
    """Singular values that fall by a hundred or more: weak directions keep what fp32 products keep of them."""
    small = min(shape)
    gen = torch.Generator().manual_seed(3)
    u, _ = torch.linalg.qr(torch.randn(shape[0], small, generator=gen, dtype=torch.float64))
    v, _ = torch.linalg.qr(torch.randn(shape[1], small, generator=gen, dtype=torch.float64))
    j = torch.arange(1, small + 1, dtype=torch.float64)
    for name, s in (("1/j", 1 / j), ("two groups", torch.where(j <= 4, 1.0, 0.01)), ("exp", torch.exp(-6 * j / small)), ("rank 5", (j <= 5).double())):
        say("spectrum", shape, name)
        x = ((u * s) @ v.t()).float().to(DEV)
        if name == "rank 5":        # directions of rounding errors alone have no value to compare with: the five have
            want, got = exact(x.cpu()), orthogonal(x).double().cpu()
            five = (u[:, :5] * exact(torch.diag(s[:5]).float()).diagonal()) @ v[:, :5].t()
            assert float(torch.linalg.vector_norm((got - five).t() @ u[:, :5])) < 1e-4 * float(torch.linalg.vector_norm(five))
            assert bool(torch.isfinite(got).all()) and bool(torch.isfinite(want).all())
            continue
        check(x, orthogonal(x))


def test_zeros_and_values_that_are_not_finite():
    x = torch.zeros(70, 40, device=DEV)
    assert bool((orthogonal(x) == 0).all())
    for bad in (float("nan"), float("inf"), -float("inf")):
        for shape in ((70, 40), (40, 70)):
            x = update(*shape, 4)
            x[3, 5] = bad
            assert bool(torch.isnan(orthogonal(x)).all()), bad


@pytest.mark.parametrize("dtype", TYPES)
def test_strides_and_places(dtype):
    for rows, cols in ((200, 65), (65, 200)):
        big = torch.full((rows, cols + 7), 3.0, dtype=dtype, device=DEV)
        x = update(rows, cols, 5, dtype)
        want = orthogonal(x)
        big[:, 3:3 + cols] = x
        view = big[:, 3:3 + cols]
        assert torch.equal(orthogonal(view), want)
        orthogonal(view, out=view)                  # in place
        assert torch.equal(view, want)
        assert bool((big[:, :3] == 3).all()) and bool((big[:, 3 + cols:] == 3).all())


def test_wide_is_the_transposed_of_tall():
    x = update(300, 70, 6)
    assert torch.equal(orthogonal(x), orthogonal(x.t().contiguous()).t())


def muon_reference(p, g, m, lr, momentum, nesterov, weight_decay, scale, steps, grad_scale):
    """In 64 bits, and the update that was brought near 1."""
    f = lambda v: float(torch.tensor(v, dtype=torch.float32))  # noqa: E731
    g = g.double().cpu() * f(grad_scale)
    m = m.double().cpu() * f(momentum) + g
    u = g + f(momentum) * m if nesterov else m
    o = exact(u, steps)
    return p.double().cpu() * (1 - f(lr) * f(weight_decay)) - f(lr) * f(scale) * o, m, u, o


@pytest.mark.parametrize("grad_type", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 50), (300, 64), (129, 40), (1000, 100), (200, 300), (64, 1000), (700, 129)])
def test_step(rows, cols, grad_type):
    say("step", rows, cols, grad_type)
    for nesterov, copy in ((True, True), (False, False)):
        gen = torch.Generator().manual_seed(rows)
        p = (torch.randn(rows, cols, generator=gen) * 0.1).to(DEV)
        m, g = update(rows, cols, 7, size=1e-3), update(rows, cols, 8, grad_type)
        c = torch.zeros(rows, cols, dtype=torch.bfloat16, device=DEV) if copy else None
        kw = dict(lr=0.02, momentum=0.95, nesterov=nesterov, weight_decay=0.1, scale=0.2 * math.sqrt(max(rows, cols)), steps=5, grad_scale=0.5)
        want_p, want_m, u, o = muon_reference(p, g, m, **kw)
        work = torch.empty(ne.ne_orthogonalize_workspace_bytes(rows, cols), dtype=torch.uint8, device=DEV).fill_(255)
        ne.ne_muon_step(p, g, m, work, param_bf16=c, **kw)
        assert bool(((m.double().cpu() - want_m).abs() <= 2.0 ** -23 * (want_m.abs() + g.double().cpu().abs())).all())
        step = 0.02 * kw["scale"]
        # the update's error, three roundings of the parameter and the update's own (which momentum's roundings move by no more than its operands')
        err = float(torch.linalg.vector_norm(p.double().cpu() - want_p))
        tol = step * (1.5 * tolerance(u, 5, min(rows, cols)) + 2.0 ** -22) * float(torch.linalg.vector_norm(o)) + 2.0 ** -22 * float(torch.linalg.vector_norm(want_p))
        assert err <= tol, (err, tol)
        if copy:
            assert torch.equal(c, p.bfloat16())


def test_step_with_strides():
    rows, cols = 150, 33
    wide = [torch.full((rows, cols + 9), 3.0, device=DEV) for _ in range(3)]
    views = [b[:, 4:4 + cols] for b in wide]
    p, g, m = update(rows, cols, 9, size=0.1), update(rows, cols, 10), update(rows, cols, 11)
    for v, x in zip(views, (p, g, m)):
        v.copy_(x)
    work = torch.empty(ne.ne_orthogonalize_workspace_bytes(rows, cols), dtype=torch.uint8, device=DEV)
    ne.ne_muon_step(p, g, m, work, 0.01)
    ne.ne_muon_step(*views, work, 0.01)
    for v, x in zip(views, (p, g, m)):
        assert torch.equal(v, x)
    for b in wide:
        assert bool((b[:, :4] == 3).all()) and bool((b[:, 4 + cols:] == 3).all())


def test_streams_and_graphs():
    """A captured step replays on the state that it left; two streams with a workspace each do not disturb one another."""
    rows, cols = 400, 48

    def state(seed):
        return [update(rows, cols, seed, size=0.1), update(rows, cols, seed + 1), torch.zeros(rows, cols, device=DEV),
                torch.empty(ne.ne_orthogonalize_workspace_bytes(rows, cols), dtype=torch.uint8, device=DEV)]

    want = state(20)
    history = []
    for _ in range(3):
        ne.ne_muon_step(*want, 0.01, weight_decay=0.1)
        history.append((want[0].clone(), want[2].clone()))
    states, streams = [state(20), state(20)], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for s, stream in zip(states, streams):
        with torch.cuda.stream(stream):
            ne.ne_muon_step(*s, 0.01, weight_decay=0.1)
    torch.cuda.synchronize()
    for s in states:
        assert torch.equal(s[0], history[0][0]) and torch.equal(s[2], history[0][1])
    s = state(20)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ne.ne_muon_step(*s, 0.01, weight_decay=0.1)
    for t in range(3):
        graph.replay()
        torch.cuda.synchronize()
        s[3].fill_(t)
        assert torch.equal(s[0], history[t][0]) and torch.equal(s[2], history[t][1]), t
