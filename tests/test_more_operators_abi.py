"""Refusals of the answers' and the Newton-Schulz operators: every call below fails on the host before anything is enqueued."""
import ctypes

import pytest
import torch

import paper_2005_13789_amd as ne
from paper_2005_13789_amd import linkpred
from paper_2005_13789_amd.fullsoftmax import SoftmaxTrainer

P = ctypes.c_void_p(0x10000)        # never dereferenced
ODD2, ODD1, ODD128 = ctypes.c_void_p(0x10002), ctypes.c_void_p(0x10001), ctypes.c_void_p(0x10080)
BIG = 1 << 50


def test_log_probability_refusals():
    L = ne.lib()

    def call(h=P, hs=8, w=P, ws=8, ty=0, ids=P, n=4, rows=10, dim=8, k=3, logp=P, lse=P, ent=P, ti=P, tl=P, work=P, size=BIG):
        return L.ne_logprob(h, hs, w, ws, ty, ids, n, rows, dim, k, logp, lse, ent, ti, tl, work, size, None)

    need = ne.ne_logprob_workspace_bytes(4, 10, 8, torch.float32, k=3)
    assert need > 0
    for bad in (dict(h=None), dict(h=ODD2), dict(w=None), dict(w=ODD1, ty=1), dict(hs=7), dict(ws=7), dict(ty=2), dict(ids=ODD2), dict(n=-1), dict(n=2**24 + 1),
                dict(rows=0), dict(rows=2**31), dict(dim=0), dict(dim=ne.NE_OP_MAX_DIM + 1), dict(k=-1), dict(k=ne.NE_TOP_MAX + 1), dict(lse=None), dict(lse=ODD2),
                dict(logp=ODD2), dict(ent=ODD1), dict(ids=None), dict(ti=None), dict(tl=None), dict(ti=ODD2), dict(tl=ODD2), dict(work=None), dict(work=ODD128),
                dict(size=need - 1)):
        assert call(**bad) == ne.NE_ERR_ARG, bad
        assert b"ne_logprob" in L.ne_last_error()
    assert call(n=0, h=None, ids=None, logp=None, lse=None, work=None) == ne.NE_OK


def test_log_probability_gradient_refusals():
    L = ne.lib()

    def call(h=P, hs=8, w=P, ws=8, ty=0, ids=P, lse=P, ent=P, a=None, b=None, ls=1.0, es=1.0, n=4, rows=10, dim=8, dh=P, dhs=8, dw=P, dws=8, work=P, size=BIG):
        return L.ne_logprob_grad(h, hs, w, ws, ty, ids, lse, ent, a, b, ls, es, n, rows, dim, dh, dhs, dw, dws, work, size, None)

    need = ne.ne_logprob_workspace_bytes(4, 10, 8, torch.float32, grad=True)
    for bad in (dict(h=None), dict(h=ODD2), dict(w=None), dict(w=ODD1, ty=1), dict(hs=7), dict(ws=7), dict(dhs=7), dict(dws=7), dict(ty=2), dict(ids=ODD2), dict(ids=None),
                dict(n=-1), dict(n=2**24 + 1), dict(rows=0), dict(rows=2**31), dict(dim=0), dict(dim=ne.NE_OP_MAX_DIM + 1), dict(lse=None), dict(lse=ODD2), dict(ent=None),
                dict(ent=ODD2), dict(a=ODD2), dict(b=ODD1), dict(ls=float("nan")), dict(es=float("inf")), dict(dh=ODD2), dict(dw=ODD2), dict(work=None),
                dict(work=ODD128), dict(size=need - 1)):
        assert call(**bad) == ne.NE_ERR_ARG, bad
        assert b"ne_logprob_grad" in L.ne_last_error()
    assert call(dh=None, dw=None) == ne.NE_OK               # nothing asked for
    assert call(n=0, h=None, ids=None, lse=None, dw=None, work=None) == ne.NE_OK
    for bad in ((-1, 10, 8), (4, 0, 8), (4, 10, 0), (0, 10, 8)):
        assert ne.ne_logprob_workspace_bytes(*bad, torch.bfloat16) == 0 and ne.ne_logprob_workspace_bytes(*bad, torch.bfloat16, grad=True) == 0
    assert ne.ne_logprob_workspace_bytes(4, 10, 8, torch.float32, k=65) == 0
    with pytest.raises(TypeError):
        ne.ne_logprob_workspace_bytes(4, 10, 8, torch.float16)


def test_orthogonalize_refusals():
    L = ne.lib()

    def call(x=P, xt=0, xs=8, rows=10, cols=8, steps=5, out=P, ot=0, os_=8, work=P, size=BIG):
        return L.ne_orthogonalize(x, xt, xs, rows, cols, steps, out, ot, os_, work, size, None)

    need = ne.ne_orthogonalize_workspace_bytes(10, 8)
    assert need > 0
    for bad in (dict(x=None), dict(x=ODD2), dict(x=ODD1, xt=1), dict(xt=2), dict(ot=-1), dict(xs=7), dict(os_=7), dict(rows=-1), dict(cols=-1), dict(rows=2**31),
                dict(rows=ne.NE_ORTHOGONAL_MAX_SIDE + 1, cols=ne.NE_ORTHOGONAL_MAX_SIDE + 1, xs=5000, os_=5000), dict(steps=0),
                dict(steps=ne.NE_ORTHOGONAL_MAX_STEPS + 1), dict(out=None), dict(out=ODD2), dict(work=None), dict(work=ODD128), dict(size=need - 1)):
        assert call(**bad) == ne.NE_ERR_ARG, bad
        assert b"ne_orthogonalize" in L.ne_last_error()
    assert call(rows=0, x=None, out=None, work=None) == ne.NE_OK and call(cols=0, x=None, out=None, work=None) == ne.NE_OK
    for bad in ((0, 8), (8, 0), (-1, 8), (5000, 5000), (2**31, 4)):
        assert ne.ne_orthogonalize_workspace_bytes(*bad) == 0


def test_muon_refusals():
    L = ne.lib()

    def call(p=P, ps=8, g=P, gt=0, gs=8, m=P, ms=8, c=None, cs=0, rows=10, cols=8, steps=5, lr=0.1, mu=0.9, nest=1, wd=0.0, scale=1.0, gscale=1.0, work=P, size=BIG):
        return L.ne_muon_step(p, ps, g, gt, gs, m, ms, c, cs, rows, cols, steps, lr, mu, nest, wd, scale, gscale, work, size, None)

    need = ne.ne_orthogonalize_workspace_bytes(10, 8)
    nan, inf = float("nan"), float("inf")
    for bad in (dict(p=None), dict(p=ODD2), dict(g=None), dict(g=ODD2), dict(g=ODD1, gt=1), dict(gt=3), dict(m=None), dict(m=ODD2), dict(c=ODD1, cs=8), dict(c=P, cs=7),
                dict(ps=7), dict(gs=7), dict(ms=7), dict(rows=-1), dict(cols=2**31), dict(steps=0), dict(steps=11), dict(lr=nan), dict(lr=-0.1), dict(mu=1.0),
                dict(mu=-0.1), dict(mu=nan), dict(wd=-1.0), dict(wd=inf), dict(scale=nan), dict(gscale=inf), dict(lr=1e30, scale=1e30), dict(work=None),
                dict(work=ODD128), dict(size=need - 1)):
        assert call(**bad) == ne.NE_ERR_ARG, bad
        assert b"ne_muon_step" in L.ne_last_error()
    assert call(rows=0, p=None, g=None, m=None, work=None) == ne.NE_OK


def test_binding_refuses_what_the_kernels_cannot_take():
    host = torch.zeros(4, 8)
    with pytest.raises(TypeError):
        ne.ne_logprob(host, host, None, host[0], None)
    with pytest.raises(TypeError):
        ne.ne_logprob_grad(host, host, None, host[0], None, None, None, None)
    with pytest.raises(TypeError):
        ne.ne_orthogonalize(host, host, None)
    with pytest.raises(TypeError):
        ne.ne_muon_step(host, host, host, None, 0.1)


@pytest.mark.parametrize("V,d", [(1, 1), (100, 8), (3000, 64), (10000, 128), (100003, 200), (50000, 300), (200003, 512), (777, 1500), (1000000, 40)])
def test_workspaces_serve_smaller_calls(V, d):
    """What a call of n rows needs is no more than what a call of more rows needs."""
    sizes = sorted(set(list(range(1, 140)) + [int(140 * 1.03 ** k) for k in range(180)]))
    for dtype in (torch.float32, torch.bfloat16):
        for k in (0, 1, 17, 64):
            need = [ne.ne_logprob_workspace_bytes(n, V, d, dtype, k=k) for n in sizes]
            assert need == sorted(need)
        need = [ne.ne_logprob_workspace_bytes(n, V, d, dtype, grad=True) for n in sizes]
        assert need == sorted(need)


def test_trainer_and_command_line_refusals():
    t = torch.zeros(5, 4)
    for kw in (dict(optimizer="sgd"), dict(optimizer="muon", state_bits=8), dict(entropy_weight=float("nan"))):
        with pytest.raises(ValueError):
            SoftmaxTrainer(t, t.clone(), 4, **kw)
    for args in (["--hits", "65"], ["--hits", "-1"], ["--optimizer", "sgd"]):
        with pytest.raises(SystemExit):
            linkpred.main(["nowhere.txt", *args])


def test_tables_of_too_long_sides_for_muon_are_refused():
    t = torch.empty(5000, ne.NE_ORTHOGONAL_MAX_SIDE + 1, device="meta")
    with pytest.raises(ValueError, match="smaller side"):
        SoftmaxTrainer(t, t, 4, optimizer="muon")
