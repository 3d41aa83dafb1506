"""Matrices of more than 64 rows and columns, which go through the matrix cores' halves, that are zeros, no numbers, or of any size;
and the same call again and again. One of every kind (about square, less wide, wide, and one that is transposed)."""
import math

import pytest
import torch

from paper_2509_04084_amd import lowdiff as ld
from test_gpu_muon import BF16, DEV, F16, F32, check, gen, matrix, same_bits

pytestmark = pytest.mark.gpu
KINDS = [(100, 110), (130, 200), (100, 300), (300, 100), (66, 65)]


def updates(dtype=F32, seed=31):
    return [matrix(r, c, gen(seed + r + c), "heavy").to(dtype) for r, c in KINDS]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("which", range(len(KINDS)))
def test_zeros_and_no_numbers_stay_in_their_matrix(which, dtype):
    us = updates(dtype)
    want = ld.ld_orthogonalize(us)
    rows, cols = KINDS[which]
    us[which].zero_()
    got = ld.ld_orthogonalize(us)
    assert not got[which].any()
    assert all(same_bits(a, b) for i, (a, b) in enumerate(zip(got, want)) if i != which)
    for eps in (0.0, 1.0):
        assert not ld.ld_orthogonalize(us[which:which + 1], eps=eps)[0].any()
    for bad in (math.nan, math.inf, -math.inf):
        for at in ((0, 0), (rows - 1, cols - 1), (rows // 2, 63)):
            for rest in ("numbers", "zeros"):
                us = updates(dtype)
                if rest == "zeros":
                    us[which].zero_()
                us[which][at] = bad
                got = ld.ld_orthogonalize(us)
                assert bool(got[which].isnan().all()), (bad, at, rest)
                assert all(same_bits(a, b) for i, (a, b) in enumerate(zip(got, want)) if i != which), (bad, at, rest)


@pytest.mark.parametrize("size", [1e-44, 1e-38, 1e-30, 1e-8, 1e30, 1e38])
def test_magnitudes(size):
    for r, c in KINDS:
        z = matrix(r, c, gen(r + c))
        u = (torch.sign(z) if size < 1e-40 else z.clamp(-3, 3)).mul(size).to(F32)
        for eps in (0.0, 1e-7):
            check(ld.ld_orthogonalize([u], eps=eps)[0], u, (size, eps, r, c), eps=eps)


def test_rows_of_very_different_sizes():
    """The largest and the smallest numbers there are in one matrix: what is small against the norm is lost, nothing else."""
    for r, c in KINDS:
        u = matrix(r, c, gen(c)).clamp(-3, 3)
        u *= torch.logspace(0, -60, r, device=DEV, dtype=torch.float64)[:, None]
        u = (u * 1e38).to(F32)
        check(ld.ld_orthogonalize([u], eps=0.0)[0], u, (r, c), eps=0.0)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_a_replay_of_no_numbers(bad):
    """What is no number in one gradient makes that matrix NaN from its step on, and no other."""
    g = gen(41)
    ws, ms = [torch.randn(s, generator=g, device=DEV) for s in KINDS], [torch.zeros(s, device=DEV) for s in KINDS]
    grads = [[torch.randn(s, generator=g, device=DEV).to(BF16) for s in KINDS] for _ in range(3)]
    w0, m0 = [w.clone() for w in ws], [m.clone() for m in ms]
    ld.ld_merge_dense_muon(ws, ms, grads, 0.02)
    for i, (r, c) in enumerate(KINDS):
        w1, m1 = [w.clone() for w in w0], [m.clone() for m in m0]
        broken = [list(step) for step in grads]
        broken[1][i] = broken[1][i].clone()
        broken[1][i][r - 1, c - 1] = bad
        ld.ld_merge_dense_muon(w1, m1, broken[:1], 0.02)
        assert not bool(w1[i].isnan().any())
        ld.ld_merge_dense_muon(w1, m1, broken[1:], 0.02)
        assert bool(w1[i].isnan().all()) and int((~m1[i].isfinite()).sum()) == 1
        for k in range(len(KINDS)):
            assert k == i or (same_bits(w1[k], ws[k]) and same_bits(m1[k], ms[k]))


@pytest.mark.parametrize("shapes", [[(1600, 4800), (1600, 1600), (1600, 6400), (6400, 1600)], [(768, 768)], [(1001, 333), (517, 517), (96, 1600), (1023, 1025)]])
def test_the_same_call_gives_the_same_bits(shapes):
    us = [matrix(r, c, gen(r + c), "heavy").to(F32) for r, c in shapes]
    need = ld.ld_orthogonalize_workspace(shapes)
    want = None
    for fill in (0, 255, 0x7C, 1, 0x3C):
        got = ld.ld_orthogonalize(us, out_dtype=BF16, workspace=torch.full((need,), fill, dtype=torch.uint8, device=DEV))
        want = want or got
        assert all(same_bits(a, b) for a, b in zip(got, want)), fill


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_matrices_of_flat_buffers(dtype):
    """Weights, momenta and gradients one behind the other in flat buffers, at any element's alignment, and what lies between them."""
    shapes = [(100, 301), (7, 33), (301, 100), (1, 50), (129, 129)]
    sizes, g = [r * c for r, c in shapes], gen(71)
    at = [sum(sizes[:i]) + 3 * i + 1 for i in range(len(shapes))]  # three elements between two
    flat = [torch.randn(sum(sizes) + 3 * len(sizes) + 1, generator=g, device=DEV) for _ in range(4)]
    w, m, grads = flat[0], flat[1], [f.to(dtype) for f in flat[2:]]
    cut = lambda f: [f[a:a + n].view(s) for a, n, s in zip(at, sizes, shapes)]  # noqa: E731
    own = [[t.clone() for t in cut(f)] for f in (w, m, *grads)]
    before = w.clone(), m.clone()
    ld.ld_merge_dense_muon(cut(w), cut(m), [cut(f) for f in grads], 0.02, weight_decay=0.1)
    ld.ld_merge_dense_muon(own[0], own[1], own[2:], 0.02, weight_decay=0.1)
    assert all(same_bits(a, b) for a, b in zip(cut(w) + cut(m), own[0] + own[1]))
    between = torch.ones(w.numel(), dtype=torch.bool, device=DEV)
    for a, n in zip(at, sizes):
        between[a:a + n] = False
    assert same_bits(w[between], before[0][between]) and same_bits(m[between], before[1][between])
    assert not any(same_bits(a, b) for a, b in zip(cut(w), cut(before[0])))
