"""Orthogonalisation of a matrix of more than 2^31 elements."""
import numpy as np
import pytest
import torch

from paper_2509_04084_amd import lowdiff as ld

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("flip", [False, True])
def test_more_than_2_31_elements(flip):
    """A matrix with one element in every row, which stays one: each singular value goes through the polynomial by itself. An element's
    relative error is its roundings', 22 bits for each of about 40 products' operands, through slopes of at most 3.45 a step: 3.45^5 2^-22 40 = 5e-3
    were they all of the first step's; that bounds it."""
    m, n = 33000, 65536
    print(f"[orthogonalize] {m} x {n}", flush=True)
    at = torch.arange(m, device=DEV)
    col = (at * 7919 + 65535) % n  # 7919 is odd: all different
    value = 1.0 + (at % 7).float()
    u = torch.zeros(n, m, device=DEV) if flip else torch.zeros(m, n, device=DEV)
    u[(col, at) if flip else (at, col)] = value
    s = value.double() / float(value.double().square().sum().sqrt())
    for _ in range(5):
        s = s * (float(np.float32(3.4445)) + s * s * (float(np.float32(-4.7750)) + s * s * float(np.float32(2.0315))))
    out = ld.ld_orthogonalize([u], [u])[0]
    got = out[(col, at) if flip else (at, col)]
    assert bool(((got.double() - s).abs() <= 5e-3 * s.abs()).all())
    out[(col, at) if flip else (at, col)] = 0.0
    assert not any(bool(part.any()) for part in out.view(-1).split(1 << 28))
