"""How precise matrices of more than 64 rows are where rounding hurts most: singular values over decades."""
import pytest
import torch

import test_gpu_muon
from paper_2509_04084_amd import lowdiff as ld
from test_gpu_muon import BF16, DEV, F16, F32, check, gen, noisy, orthogonal64

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
