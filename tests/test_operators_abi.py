"""Refusals of the full-softmax operators: every call below fails on the host before anything is enqueued."""
import ctypes
import gc
import weakref

import pytest
import torch

import paper_2005_13789_amd as ne

P = ctypes.c_void_p(0x10000)        # never dereferenced
ODD2, ODD1 = ctypes.c_void_p(0x10002), ctypes.c_void_p(0x10001)
BIG = 1 << 40


def test_lookup_refusals():
    L = ne.lib()

    def call(table=P, tt=0, ts=8, rows=10, dim=8, ids=P, n=4, scale=1.0, out=P, ot=0, os_=8):
        return L.ne_embed_lookup(table, tt, ts, rows, dim, ids, n, scale, out, ot, os_, None)

    for bad in (dict(rows=0), dict(rows=2**31), dict(dim=0), dict(dim=ne.NE_OP_MAX_DIM + 1), dict(n=-1), dict(n=ne.NE_EMBED_MAX_IDS + 1), dict(tt=2), dict(ot=-1),
                dict(ts=7), dict(os_=7), dict(scale=float("nan")), dict(table=None), dict(table=ODD2), dict(table=ODD1, tt=1), dict(out=None),
                dict(out=ODD2), dict(ids=None), dict(ids=ODD2)):
        assert call(**bad) == ne.NE_ERR_ARG, bad
        assert b"ne_embed_lookup" in L.ne_last_error()
    assert call(n=0, table=None, ids=None, out=None) == ne.NE_OK


def test_gradient_refusals():
    L = ne.lib()

    def call(ids=P, n=4, grad=P, gt=0, gs=8, scale=1.0, rows=10, dim=8, out=P, ot=0, os_=8, acc=0, ws=P, size=BIG):
        return L.ne_embed_grad(ids, n, grad, gt, gs, scale, rows, dim, out, ot, os_, acc, ws, size, None)

    need = ne.ne_embed_workspace_bytes(10, 8, 4)
    assert need > 0
    for bad in (dict(rows=0), dict(dim=0), dict(n=-1), dict(gt=3), dict(ot=3), dict(gs=7), dict(gs=-8), dict(os_=0), dict(scale=float("inf")), dict(ids=None),
                dict(grad=None), dict(grad=ODD2), dict(out=None), dict(ws=None), dict(ws=ctypes.c_void_p(0x10080)), dict(size=need - 1)):
        assert call(**bad) == ne.NE_ERR_ARG, bad
        assert b"ne_embed_grad" in L.ne_last_error()
    assert call(n=0, acc=1, ids=None, grad=None, ws=None, size=0) == ne.NE_OK
    assert ne.ne_embed_workspace_bytes(0, 8, 4) == 0 and ne.ne_embed_workspace_bytes(10, 8, 0) == 0


def test_cross_entropy_refusals():
    L = ne.lib()

    def loss(h=P, hs=8, w=P, ws=8, ty=0, t=P, n=4, rows=10, dim=8, lo=P, lse=P, work=P, size=BIG):
        return L.ne_xent_loss(h, hs, w, ws, ty, t, n, rows, dim, lo, lse, work, size, None)

    def grad(h=P, hs=8, w=P, ws=8, ty=0, t=P, lse=P, c=None, scale=1.0, n=4, rows=10, dim=8, dh=P, dhs=8, dw=P, dws=8, work=P, size=BIG):
        return L.ne_xent_grad(h, hs, w, ws, ty, t, lse, c, scale, n, rows, dim, dh, dhs, dw, dws, work, size, None)

    common = (dict(h=None), dict(h=ODD2), dict(w=None), dict(w=ODD1, ty=1), dict(hs=7), dict(ws=7), dict(ty=2), dict(t=None), dict(t=ODD2), dict(n=-1),
              dict(n=2**24 + 1), dict(rows=0), dict(rows=2**31), dict(dim=0), dict(dim=ne.NE_OP_MAX_DIM + 1), dict(lse=None), dict(work=None),
              dict(work=ctypes.c_void_p(0x10080)))
    for bad in common + (dict(lo=None), dict(lo=ODD2), dict(size=ne.ne_xent_workspace_bytes(4, 10, 8, torch.float32, False) - 1)):
        assert loss(**bad) == ne.NE_ERR_ARG, bad
        assert b"ne_xent_loss" in L.ne_last_error()
    for bad in common + (dict(scale=float("nan")), dict(c=ODD2), dict(dh=ODD2), dict(dw=ODD2), dict(dhs=7), dict(dws=7),
                         dict(size=ne.ne_xent_workspace_bytes(4, 10, 8, torch.float32, True) - 1)):
        assert grad(**bad) == ne.NE_ERR_ARG, bad
        assert b"ne_xent_grad" in L.ne_last_error()
    assert loss(n=0, h=None, t=None) == ne.NE_OK
    assert grad(n=0, h=None, t=None, dw=None) == ne.NE_OK
    assert grad(dh=None, dw=None) == ne.NE_OK               # nothing asked for
    for bad in ((-1, 10, 8), (4, 0, 8), (4, 10, 0), (0, 10, 8)):
        assert ne.ne_xent_workspace_bytes(*bad, torch.bfloat16, True) == 0
    with pytest.raises(TypeError):
        ne.ne_xent_workspace_bytes(4, 10, 8, torch.float16, True)


def test_adamw_refusals():
    L = ne.lib()
    out = ctypes.c_void_p()

    def create(bits=32, count=1, work=P, size=BIG, outp=ctypes.byref(out), arr="one", **kw):
        t = dict(param=P, grad=P, m=P, v=P, m_scale=P, v_scale=P, param_bf16=None, n=100, weight_decay=0.0, grad_type=0) | kw
        one = (ne.NeAdamwTensor * 1)(ne.NeAdamwTensor(**t)) if arr == "one" else arr
        return L.ne_create_adamw(outp, one, count, bits, 0, work, size, None)

    need = ne.ne_adamw_workspace_bytes([100])
    assert need > 0
    for bad in (dict(bits=16), dict(count=0), dict(count=65537), dict(outp=None), dict(arr=None), dict(work=None), dict(work=ctypes.c_void_p(0x10080)), dict(size=need - 1),
                dict(n=0), dict(n=2**33), dict(param=None), dict(param=ODD2), dict(grad=None), dict(grad=ODD2), dict(grad=ODD1, grad_type=1), dict(m=None),
                dict(v=ODD2), dict(grad_type=5), dict(param_bf16=ODD1), dict(weight_decay=-0.1), dict(weight_decay=float("nan")),
                dict(bits=8, m_scale=None), dict(bits=8, v_scale=ODD2)):
        assert create(**bad) == ne.NE_ERR_ARG, bad
        assert b"ne_create_adamw" in L.ne_last_error()
    assert ne.ne_adamw_workspace_bytes([]) == 0 and ne.ne_adamw_workspace_bytes([0]) == 0
    assert L.ne_adamw_step(None, 1, 0.1, 0.9, 0.999, 1e-8, 1.0, None) == ne.NE_ERR_ARG
    L.ne_destroy_adamw(None)


def test_binding_refuses_what_the_kernels_cannot_take():
    host = torch.zeros(4, 8)
    ids = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(TypeError):
        ne.ne_embed_lookup(host, ids, host)
    with pytest.raises(TypeError):
        ne.ne_embed_grad(ids, host, host, None)
    with pytest.raises(TypeError):
        ne.ne_xent_loss(host, host, ids, host[0], host[0], None)
    with pytest.raises(TypeError):
        ne.ne_create_adamw([host], [host], [host.half()], [host], None)


@pytest.mark.parametrize("V,d", [(1, 1), (100, 8), (3000, 64), (10000, 128), (100003, 200), (50000, 300), (200003, 512), (777, 1500), (1000000, 40)])
def test_workspaces_serve_smaller_calls(V, d):
    """What a call of n rows needs is no more than what a call of more rows needs."""
    sizes = sorted(set(list(range(1, 140)) + [int(140 * 1.03 ** k) for k in range(180)]))
    for dtype in (torch.float32, torch.bfloat16):
        for grad in (False, True):
            need = [ne.ne_xent_workspace_bytes(n, V, d, dtype, grad) for n in sizes]
            assert need == sorted(need)
    need = [ne.ne_embed_workspace_bytes(V, d, n) for n in sizes + [2 ** 18, 270000, 2 ** 20]]
    assert need == sorted(need)


def test_an_adamw_handle_keeps_its_tensors():
    """The kernels hold the tensors' addresses: what the caller does to the lists afterwards must not free them."""
    lists = [[torch.zeros(4), torch.zeros(5)] for _ in range(4)]
    refs = [weakref.ref(t) for ts in lists for t in ts]
    opt = ne.AdamW(None, (*lists, None, None, [None, torch.zeros(5)]), torch.zeros(8))
    for ts in lists:
        ts.clear()
    gc.collect()
    assert all(r() is not None for r in refs)
    del opt
    gc.collect()
    assert all(r() is None for r in refs)
