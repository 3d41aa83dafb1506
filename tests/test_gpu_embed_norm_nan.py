"""The value tests of the embedding, the norm and clipping again, with a comparison that NaN does not pass.

`close` of test_gpu_embed_norm asks whether any difference is larger than its bound, and no comparison with NaN is true: a NaN in
a result is let through there. Same inputs, same bounds; here a result passes only where the difference is known to be small.
"""
import math

import pytest
import torch

import test_gpu_embed_norm as base
from test_gpu_embed_norm import BF16, F16, F32, STEP, UNIT


def close(got, want, spread, dtype, tag):
    assert got.dtype == dtype
    got = got.detach().double().cpu()
    bound = 1.01 * (spread + UNIT[dtype] * want.abs()) + 0.5 * STEP[dtype]
    bad = ~((got - want).abs() <= bound)
    assert not bad.any(), (tag, int(bad.sum()), int(got.isnan().sum()), bad.nonzero()[0].tolist())


@pytest.fixture
def strict(monkeypatch):
    monkeypatch.setattr(base, "close", close)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("bad", [math.nan, math.inf, 1.5])
def test_the_comparison_refuses_a_single_wrong_value(dtype, bad):
    want = torch.ones(5, 7, dtype=torch.float64)
    got = want.to(dtype)
    close(got, want, 0.0 * want, dtype, "right")
    got[3, 2] = bad
    with pytest.raises(AssertionError):
        close(got, want, 0.0 * want, dtype, "wrong")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out_dtype", [(a, b) for a in (F32, BF16, F16) for b in (F32, BF16, F16)])
@pytest.mark.parametrize("T,V,d", [(1, 1, 1), (5, 100, 7), (64, 300, 8), (65, 1000, 9), (257, 513, 127), (1000, 2000, 768), (7, 40, 12289)])
def test_lookup(strict, T, V, d, dtype, out_dtype):
    base.test_lookup(T, V, d, dtype, out_dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["uniform", "outside", "one", "two", "descending", "heavy", "none"])
@pytest.mark.parametrize("T,V,d", [(1, 1, 1), (2, 2, 3), (65, 1023, 9), (257, 1024, 64), (1000, 2047, 33), (4095, 2048, 16), (4097, 5000, 12), (9001, 70, 40),
                                   # few tokens in shares and wide rows, then chunks of 4, 8, 16 and 32 tokens
                                   (255, 40, 260), (1023, 90, 515), (129, 30, 3300), (1500, 400, 600), (8200, 3000, 1030), (34000, 2000, 41), (270000, 900, 20)])
def test_embed_grad(strict, T, V, d, kind):
    base.check_grad(T, V, d, kind, BF16 if d % 4 else F32, F32, scale=0.75 if d % 2 else 1.0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,grad_dtype", [(a, b) for a in (F32, BF16, F16) for b in (F32, BF16, F16)])
@pytest.mark.parametrize("T,V,d,kind", [(300, 90, 129, "heavy"), (2500, 1000, 264, "outside"), (2500, 200, 5, "heavy"), (129, 40, 1001, "uniform")])
def test_embed_grad_types(strict, T, V, d, kind, dtype, grad_dtype):
    base.check_grad(T, V, d, kind, dtype, grad_dtype, scale=3.5, id_dtype=torch.int32)


@pytest.mark.gpu
@pytest.mark.parametrize("T,V,d,kind", [(70001, 50257, 24, "heavy"), (40000, 1024, 100, "descending"), (300000, 9, 4, "heavy"), (16385, 4_200_000, 3, "uniform"),
                                        (1_100_000, 3000, 2, "heavy")])
def test_embed_grad_of_many_tokens(strict, T, V, d, kind):
    base.check_grad(T, V, d, kind, BF16, F32, seed=5)


@pytest.mark.gpu
@pytest.mark.parametrize("test", [base.test_lookup_shapes_strides_and_what_lies_around, base.test_embed_grad_strides_and_what_lies_around,
                                  base.test_clip_of_views_at_any_alignment], ids=lambda t: t.__name__)
def test_strides(strict, test):
    test()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out_dtype", [(F32, F32), (BF16, F32), (F16, BF16)])
def test_clip_of_neighbours(strict, dtype, out_dtype):
    base.test_clip_of_neighbours(dtype, out_dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out_dtype", [(a, b) for a in (F32, BF16, F16) for b in (F32, BF16, F16)])
@pytest.mark.parametrize("sizes", base.SIZES, ids=lambda s: f"{len(s)}x{max(s, default=0)}")
def test_clip(strict, sizes, dtype, out_dtype):
    base.test_clip(sizes, dtype, out_dtype)
