"""Every number of Newton-Schulz steps, on matrices whose singular values lie within a factor of three: no direction is weak, so the results are bound to a
hundredth at each number, and one step more or less differs by a tenth or more."""
import pytest
import torch

import paper_2005_13789_amd as ne

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
A, B, C = 3.4445, -4.7750, 2.0315


def f(s):
    return A * s + B * s ** 3 + C * s ** 5


def growth(s):
    """By how much a step multiplies an error between directions i and j of a matrix of singular values s: the differences (f(s_i) - f(s_j)) / (s_i - s_j) of its
    symmetric part, (f(s_i) + f(s_j)) / (s_i + s_j) of the other, and f(s_i) / s_i towards directions that the matrix does not have."""
    near = (s[:, None] - s[None]).abs() < 1e-9
    mean = (s[:, None] + s[None]) / 2
    slope = A + 3 * B * mean ** 2 + 5 * C * mean ** 4
    differences = torch.where(near, slope, (f(s)[:, None] - f(s)[None]) / torch.where(near, torch.ones_like(mean), s[:, None] - s[None]))
    return [differences.abs(), ((f(s)[:, None] + f(s)[None]) / (2 * mean)).abs(), (f(s) / s).abs()[:, None].expand_as(mean)]


def tolerance(s, steps):
    """Of the result's 2-norm, relative to it.  A product of operands of 22 bits is off by eta = 4 2^-22 of their norms; a G serves three steps at first and two later,
    each takes up to four such products, and G's error counts 1 + s_max^2 / s_min^2 times.  What a stage leaves grows along the later steps as growth() says."""
    s = s / torch.linalg.vector_norm(s)
    eta, errors, left = 4 * 2.0 ** -22, [], steps
    while left > 0:
        now = min(left, 2 if errors else 3)
        size = 4 * now * eta * float(1 + s.max() ** 2 / s.min() ** 2)
        for _ in range(now):
            for e in errors:
                e[1] = [a * b for a, b in zip(e[1], growth(s))]
            s = f(s)
        errors.append([size * float(torch.linalg.vector_norm(s)), [torch.ones(len(s), len(s), dtype=torch.float64)] * 3])
        left -= now
    total = sum(size * max(float(a.max()) for a in by) for size, by in errors)
    return total / float(torch.linalg.vector_norm(s)) + 2.0 ** -24


@pytest.mark.parametrize("rows,cols", [(200, 30), (30, 200), (4000, 100), (300, 200), (200, 300), (500, 300), (1100, 1030)])
def test_every_number_of_steps(rows, cols):
    small = min(rows, cols)
    gen = torch.Generator().manual_seed(rows)
    u, v = (torch.linalg.qr(torch.randn(side, small, generator=gen, dtype=torch.float64))[0] for side in (rows, cols))
    s = torch.linspace(1, 3, small, dtype=torch.float64)
    x = ((u * s) @ v.t()).float().to(DEV)
    s = torch.linalg.svdvals(x.double().cpu())
    work = torch.empty(ne.ne_orthogonalize_workspace_bytes(rows, cols), dtype=torch.uint8, device=DEV).fill_(255)
    want = x.double() if rows >= cols else x.double().t()
    want = want / torch.linalg.vector_norm(want)
    for steps in range(1, ne.NE_ORTHOGONAL_MAX_STEPS + 1):
        print("steps", rows, cols, steps, flush=True)
        before, g = want, want.t() @ want
        want = A * want + want @ (B * g + C * (g @ g))
        tol = tolerance(s, steps)
        assert tol < 0.01 and float(torch.linalg.vector_norm(want - before) / torch.linalg.vector_norm(want)) > 0.1
        out = torch.full_like(x, float("nan"))
        ne.ne_orthogonalize(x, out, work, steps=steps)
        err = float(torch.linalg.vector_norm((out if rows >= cols else out.t()).double() - want) / torch.linalg.vector_norm(want))
        print("   off by", err, "of", tol, flush=True)
        assert err <= tol, (steps, err, tol)
