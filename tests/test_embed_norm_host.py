"""Embedding lookup and gradient, gradient norm and clipping: what they refuse, without a GPU."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2509_04084_amd import lowdiff as ld

FAKE = 0x10000  # never dereferenced: every call below fails its checks or has nothing to do
V = ctypes.c_void_p
F = ctypes.c_float
NULL, RANGE, WORKSPACE, ALIGN = -1, -2, -3, -5


def _p(a):
    return V(a.ctypes.data)


def test_norm_refusals():
    lib = ld.load()
    n = np.array([10, 20], np.int64)
    two = (V * 2)(FAKE, FAKE)
    wsb = lib.ld_grad_norm_workspace(2)
    assert wsb > 0 and lib.ld_grad_norm_workspace(-1) == 0 and lib.ld_grad_norm_workspace((1 << 20) + 1) == 0
    assert lib.ld_grad_norm_workspace(0) >= 8  # a call without tensors still has a sum

    def call(g=two, n=n, count=2, dtype=0, sumsq=FAKE, norm=FAKE, ws=FAKE, wsb=wsb):
        return lib.ld_grad_norm(g, _p(n) if n is not None else None, count, dtype, 0, V(sumsq), V(norm), V(ws), wsb, None)

    assert call(g=None) == NULL and call(n=None) == NULL and call(sumsq=0) == NULL and call(g=(V * 2)(FAKE, 0)) == NULL
    assert call(count=-1) == RANGE and call(count=(1 << 20) + 1) == RANGE and call(dtype=3) == RANGE and call(dtype=-1) == RANGE
    assert call(n=np.array([10, -1], np.int64)) == RANGE
    assert call(n=np.array([1 << 41, 1], np.int64)) == RANGE and call(n=np.array([1, 1 << 62], np.int64)) == RANGE
    assert call(g=(V * 2)(FAKE, FAKE + 2)) == ALIGN and call(dtype=1, g=(V * 2)(FAKE, FAKE + 1)) == ALIGN
    assert call(sumsq=FAKE + 4) == ALIGN and call(norm=FAKE + 2) == ALIGN
    assert call(ws=0) == WORKSPACE and call(ws=FAKE + 8) == WORKSPACE and call(wsb=wsb - 1) == WORKSPACE


def test_clip_refusals():
    lib = ld.load()
    n = np.array([10, 20], np.int64)
    two = (V * 2)(FAKE, FAKE)
    wsb = lib.ld_grad_norm_workspace(2)

    def both(g=two, o=two, n=n, count=2, dtype=0, odtype=0, limit=1.0, s=FAKE):
        a = lib.ld_clip_grads(g, o, _p(n), count, dtype, odtype, V(s), F(limit), None)
        b = lib.ld_clip_grad_norm(g, o, _p(n), count, dtype, odtype, F(limit), V(s), V(FAKE), wsb, None)
        assert a == b, (a, b)
        return a

    assert both(g=None) == NULL and both(o=None) == NULL and both(s=0) == NULL and both(o=(V * 2)(FAKE, 0)) == NULL
    assert both(limit=-1.0) == RANGE and both(limit=float("nan")) == RANGE and both(odtype=7) == RANGE and both(count=-1) == RANGE
    assert both(n=np.array([-5, 1], np.int64)) == RANGE
    assert both(odtype=1, o=(V * 2)(FAKE, FAKE + 1)) == ALIGN and both(g=(V * 2)(FAKE + 1, FAKE)) == ALIGN
    assert lib.ld_clip_grads(two, two, _p(n), 2, 0, 0, V(FAKE + 4), F(1.0), None) == ALIGN
    assert lib.ld_clip_grad_norm_workspace(2, _p(n)) == 0  # few elements are done with in one launch
    n = np.array([10, 200000], np.int64)
    assert lib.ld_clip_grad_norm_workspace(2, _p(n)) == wsb and lib.ld_clip_grad_norm_workspace(-1, _p(n)) == 0
    for bad in ((FAKE, wsb - 1), (0, wsb), (FAKE + 16, wsb)):
        assert lib.ld_clip_grad_norm(two, two, _p(n), 2, 0, 0, F(1.0), V(FAKE), V(bad[0]), bad[1], None) == WORKSPACE
    assert lib.ld_clip_grads(None, None, None, 0, 0, 0, V(FAKE), F(1.0), None) == 0  # nothing to do


def test_lookup_refusals():
    lib = ld.load()

    def call(table=FAKE, rows=100, ts=64, pos=0, P=0, ps=0, dtype=1, ids=FAKE, at=0, it=1, T=8, d=64, out=FAKE, os=64, ot=1):
        return lib.ld_embed_lookup(V(table), rows, ts, V(pos), P, ps, dtype, V(ids), V(at), it, T, d, F(1.0), V(out), os, ot, None)

    assert call(table=0) == NULL and call(ids=0) == NULL and call(out=0) == NULL and call(pos=FAKE, P=5, ps=64) == NULL
    for bad in (dict(rows=-1), dict(T=-1), dict(d=-1), dict(d=(1 << 20) + 1, ts=1 << 21, os=1 << 21), dict(ts=-1), dict(os=63), dict(dtype=3), dict(ot=-1), dict(it=2),
                dict(pos=FAKE, at=FAKE, P=-1, ps=64), dict(pos=FAKE, at=FAKE, P=5, ps=-1)):
        assert call(**bad) == RANGE, bad
    for bad in (dict(table=FAKE + 1), dict(out=FAKE + 1), dict(ids=FAKE + 4), dict(it=0, ids=FAKE + 2), dict(ot=0, out=FAKE + 2),
                dict(pos=FAKE + 1, at=FAKE, P=5, ps=64), dict(pos=FAKE, at=FAKE + 4, P=5, ps=64)):
        assert call(**bad) == ALIGN, bad
    assert call(T=0, table=0, ids=0, out=0) == 0 and call(d=0, os=0) == 0


def test_embed_grad_refusals():
    lib = ld.load()
    wsb = lib.ld_embed_grad_workspace(2000, 100, 64)
    assert wsb > 0 and lib.ld_embed_grad_workspace(8, 100, 64) == 0  # few tokens are done with in shared memory
    for bad in ((-1, 100, 64), (8, -1, 64), (8, 100, -1), (8, 100, (1 << 20) + 1), ((1 << 24) + 1, 100, 64), (8, 2 ** 31 - 1, 64)):
        assert lib.ld_embed_grad_workspace(*bad) == 0

    def call(dout=FAKE, ds=64, dtype=1, ids=FAKE, it=1, T=2000, d=64, grad=FAKE, rows=100, gs=64, gt=0, acc=0, ws=FAKE, wsb=wsb):
        return lib.ld_embed_grad(V(dout), ds, dtype, V(ids), it, T, d, F(1.0), V(grad), rows, gs, gt, acc, V(ws), wsb, None)

    assert call(dout=0) == NULL and call(ids=0) == NULL and call(grad=0) == NULL
    for bad in (dict(T=-1), dict(T=(1 << 24) + 1), dict(rows=-1), dict(rows=2 ** 31 - 1), dict(d=-1), dict(d=(1 << 20) + 1, gs=1 << 21), dict(ds=-1), dict(gs=63), dict(dtype=5),
                dict(gt=3), dict(it=-1)):
        assert call(**bad) == RANGE, bad
    for bad in (dict(dout=FAKE + 1), dict(grad=FAKE + 2), dict(ids=FAKE + 4), dict(it=0, ids=FAKE + 1)):
        assert call(**bad) == ALIGN, bad
    assert call(ws=0) == WORKSPACE and call(ws=FAKE + 128) == WORKSPACE and call(wsb=wsb - 1) == WORKSPACE
    assert call(rows=0, grad=0) == 0 and call(d=0, gs=0) == 0 and call(T=0, acc=1, dout=0, ids=0) == 0


def test_binding_refuses_before_any_launch():
    t, ids = torch.zeros(10, 8), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(TypeError):
        ld.ld_embed_lookup(t, ids)  # not on a GPU
    with pytest.raises(TypeError):
        ld.ld_embed_lookup(t.double(), ids)
    with pytest.raises(ValueError, match="go together"):
        ld.ld_embed_lookup(t, ids, pos_table=t)
    with pytest.raises(ValueError, match="as many as ids"):
        ld.ld_embed_lookup(t, ids, pos_table=t, positions=ids[:3])
    with pytest.raises(ValueError, match="width or type"):
        ld.ld_embed_lookup(t, ids, pos_table=torch.zeros(10, 7), positions=ids)
    with pytest.raises(ValueError, match="different devices"):
        ld.ld_embed_lookup(t, ids.to("meta"))
    with pytest.raises(ValueError, match="a row of grad's width"):
        ld.ld_embed_grad(torch.zeros(3, 8), ids, t)
    with pytest.raises(ValueError, match="a row of grad's width"):
        ld.ld_embed_grad(torch.zeros(4, 7), ids, t)
    with pytest.raises(TypeError):
        ld.ld_embed_grad(torch.zeros(4, 8), ids, t)
    g = [torch.zeros(5), torch.zeros(6)]
    with pytest.raises(ValueError, match="differ in length"):
        ld.ld_clip_grad_norm(g, 1.0, g[:1])
    with pytest.raises(ValueError, match="differ in size"):
        ld.ld_clip_grad_norm(g, 1.0, g[::-1])
    with pytest.raises(TypeError):
        ld.ld_clip_grad_norm([x.double() for x in g], 1.0)
    with pytest.raises(TypeError):
        ld.ld_clip_grad_norm(g, 1.0, norm=torch.zeros(1))
    with pytest.raises(TypeError):
        ld.ld_grad_norm(g, sumsq=torch.zeros(1, dtype=torch.float64), norm=torch.zeros(1))
    with pytest.raises(ValueError, match="accumulate"):
        ld.ld_grad_norm(g, accumulate=True)
