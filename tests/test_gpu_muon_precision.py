"""How precise matrices of more than 64 rows are where rounding hurts most: singular values over decades, and norms far below eps."""
import pytest
import torch

import test_gpu_muon
from paper_2509_04084_amd import lowdiff as ld
from test_gpu_muon import BF16, DEV, F16, F32, check, gen, matrix, noisy, orthogonal64, same_bits

pytestmark = pytest.mark.gpu


def rows_of_sizes(r, c, seed):
    """Rows whose sizes spread over two decades, as those of an embedding or of a wide layer's gradient do."""
    g = gen(seed)
    z = torch.randn(r, c, generator=g, device=DEV)
    return z * torch.exp(1.5 * torch.randn(r, 1, generator=g, device=DEV))


any_runs = test_gpu_muon.runs_of


def runs_of_32_bits(coeffs, m, n):
    """Two steps at most: what a matrix twice as wide as high has, one that is wider has as well."""
    return any_runs(coeffs, m, min(n, 2 * m))


@pytest.mark.parametrize("r,c", [(2048, 512), (2304, 768), (4096, 1024), (5120, 2048), (768, 2304), (400, 100)])
def test_results_of_32_bits(r, c, monkeypatch):
    """Of runs of two steps at most, whose noise has operands off by up to 2^-22: two halves, the lower one rounded to nearest, are off by
    no more than 2^-23, and what is left out of a product by no more than 2^-24. So half of that noise is the most there can be (what
    sums of 32 bits add is less than operands do)."""
    print(f"[orthogonalize] {r} x {c}, rows of many sizes", flush=True)
    monkeypatch.setattr(test_gpu_muon, "runs_of", runs_of_32_bits)
    u = rows_of_sizes(r, c, r + c)
    got, want = ld.ld_orthogonalize([u])[0], orthogonal64(u)
    noise = max(float((noisy(u, seed) - want).norm()) for seed in range(3))
    assert float((got.double() - want).norm()) <= 0.5 * noise


@pytest.mark.parametrize("out_dtype", [BF16, F16])
def test_results_of_16_bits(out_dtype):
    """Longer runs, whose errors are a small part of the rounding to 16 bits."""
    for r, c in ((1024, 256), (768, 2304)):
        u = rows_of_sizes(r, c, r + c)
        got, want = ld.ld_orthogonalize([u], out_dtype=out_dtype)[0], orthogonal64(u)
        check(got, u, (r, c), out_dtype)
        assert float((got.double() - want).norm()) <= 1.05 * float((want.to(out_dtype).double() - want).norm())


@pytest.mark.parametrize("r,c", [(100, 110), (130, 200), (100, 300), (300, 100), (768, 768), (512, 2048), (1600, 400)])
@pytest.mark.parametrize("eps", [1e-7, 1.0, 1e20])
@pytest.mark.parametrize("part", [1e-4, 1e-6, 1e-9, 1e-15, 1e-25])
def test_norms_far_below_eps(part, eps, r, c):
    """X begins `part` as large as it would without eps, and five usual steps grow it by 485 in all, so that it stays small and a step is
    next to a multiplication by a: A is under (485 * 1e-4)^2. Relative to the norm, X is off by 2^-23 where it is laid out, and each of up
    to five products Q X has operands off by 2^-23 each, leaves out 2^-24, and rounds the one sum that is not next to nothing: 5 (2 +
    0.5 + 1) 2^-23, with Q's own steps' roundings, no more than those again, 5e-6 in all. Under 2^-126 the result loses what its type does."""
    u = (torch.randn(r, c, generator=gen(r + c), device=DEV, dtype=torch.float64) * (part * eps / (r * c) ** 0.5)).to(F32)
    tiny = 2.0 ** -150 * (r * c) ** 0.5
    got, want = ld.ld_orthogonalize([u], eps=eps)[0], orthogonal64(u, eps=eps)
    assert float((got.double() - want).norm()) <= 5e-6 * float(want.norm()) + tiny, (float((got.double() - want).norm() / want.norm()))


def test_norms_about_eps():
    """Below, about and above it, of every kind side by side; a matrix by itself gives the same bits."""
    shapes = [(100, 110), (130, 200), (100, 300), (300, 100), (768, 768)]
    for part in (0.3, 0.5, 0.9, 1.0, 1.5, 3.0, 1e-2, 1e-3):
        us = [(matrix(r, c, gen(r + c), "heavy") * (part / (r * c) ** 0.5)).to(F32) for r, c in shapes]
        us = [u * (part / u.norm()) for u in us]
        got = ld.ld_orthogonalize(us, eps=1.0)
        for a, u in zip(got, us):
            check(a, u, (part, u.shape), eps=1.0)
            assert same_bits(ld.ld_orthogonalize([u], eps=1.0)[0], a)


def test_a_replay_of_vanishing_gradients():
    """Momentum that has died down far below eps: the update is next to nothing, and as precise as any."""
    g, shapes = gen(61), [(100, 110), (100, 300), (300, 100)]
    us = [torch.randn(s, generator=g, device=DEV) * 2.0 ** -60 for s in shapes]
    ws, ms = [torch.zeros(s, device=DEV) for s in shapes], [torch.zeros(s, device=DEV) for s in shapes]
    ld.ld_merge_dense_muon(ws, ms, [us], 1.0, nesterov=False, scale=-1.0)
    for w, u in zip(ws, us):
        want = orthogonal64(u)
        assert float((w.double() - want).norm()) <= 5e-6 * float(want.norm())
