"""Tensors that stand for two matrices of a call are refused before anything is launched; those that are only read may."""
import pytest
import torch

from paper_2509_04084_amd import lowdiff as ld
from test_gpu_muon import DEV, gen, same_bits

pytestmark = pytest.mark.gpu


def some(n, shape=(70, 90)):
    g = gen(51)
    return [torch.randn(shape, generator=g, device=DEV) for _ in range(n)]


@pytest.mark.parametrize("shape", [(4, 6), (70, 90)])
def test_orthogonalize(shape):
    a, b, c = some(3, shape)
    before = [t.clone() for t in (a, b, c)]
    for mats, outs in (([a, a], [a, b]), ([a, a], [b, a]), ([a, b], [b, a]), ([a, b], [c, c]), ([a, b, a], [c, b, a])):
        with pytest.raises(ValueError, match="two matrices"):
            ld.ld_orthogonalize(mats, outs)
    assert all(same_bits(t, u) for t, u in zip((a, b, c), before))
    twice = ld.ld_orthogonalize([a, a], [b, c])
    assert same_bits(twice[0], twice[1]) and same_bits(a, before[0])
    assert same_bits(ld.ld_orthogonalize([a], [a])[0], b)
    empty = torch.empty(0, 5, device=DEV)
    ld.ld_orthogonalize([empty, empty, b], [empty, empty, b])


@pytest.mark.parametrize("shape", [(4, 6), (70, 90)])
def test_replay(shape):
    w, m, g, other = some(4, shape)
    before = [t.clone() for t in (w, m, g, other)]
    for ws, ms, grads in (([w], [m], [[w]]), ([w], [m], [[m]]), ([w], [m], [[g], [m]]), ([w, g], [m, other], [[g, g]]),
                          ([w, g], [m, other], [[m.clone(), m.clone()], [other, m.clone()]])):
        with pytest.raises(ValueError, match="two matrices"):
            ld.ld_merge_dense_muon(ws, ms, grads, 0.1)
    assert all(same_bits(t, u) for t, u in zip((w, m, g, other), before))
    ld.ld_merge_dense_muon([w, other], [m, m.clone()], [[g, g], [g, g]], 0.1)  # read in four places
    w1, m1 = before[0].clone(), before[1].clone()
    ld.ld_merge_dense_muon([w1], [m1], [[g], [g.clone()]], 0.1)
    assert same_bits(w, w1) and same_bits(m, m1)
    ld.ld_merge_dense_muon([w], [m], [], 0.1)
    empty = torch.empty(0, 5, device=DEV)
    ld.ld_merge_dense_muon([empty, empty, w], [empty, empty, m], [[empty, empty, g]], 0.1)
