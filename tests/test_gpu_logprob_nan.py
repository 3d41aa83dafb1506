"""Rows of logits that hold nothing but NaN and minus infinities: no rows in which nothing is left, but rows without numbers."""
import math

import pytest
import torch

from paper_2509_04084_amd import lowdiff as ld
from test_gpu_logprob import BF16, DEV, F16, F32, gen, make, same_bits

pytestmark = pytest.mark.gpu
SIZES = [(4, 300), (1200, 300), (4, 9001), (130, 9001), (1100, 9001), (2, 70001)]  # a wave's rows, a workgroup's, split ones


def rows_of_nan(x, V):
    """Row by row: all NaN, all of them negative, one among minus infinities (first, within, last), a stretch of them; and, if there are
    more rows, a masked one and NaN among numbers."""
    masked = lambda *at: torch.where(torch.isin(torch.arange(V), torch.tensor(at)), math.nan, -math.inf)  # noqa: E731
    rows = [torch.full((V,), math.nan), torch.full((V,), -math.nan), masked(0), masked(V // 2), masked(V - 1), masked(*range(V // 3, V // 2))]
    return [r.to(x.dtype) for r in rows]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("top", [0, 1, 6, 33])
@pytest.mark.parametrize("T,V", SIZES)
def test_rows_of_nan_are_not_masked_rows(T, V, top, dtype):
    print(f"[score] rows of NaN, T={T} V={V} top={top} {dtype}", flush=True)
    g = gen(T + V + top)
    clean = make(T, V, dtype, g)
    clean[0] = -math.inf  # nothing is left
    ids = torch.randint(0, V, (T,), generator=g)
    for first in range(0, 6, T - 1):  # as many at a time as there are rows behind the first
        x, y = clean.clone(), ids.clone()
        kinds = rows_of_nan(x, V)[first:first + T - 1]
        for i, row in enumerate(kinds):
            x[1 + i] = row
        y[1] = -1
        bad, good = slice(1, 1 + len(kinds)), [0, *range(1 + len(kinds), T)]
        got, ref = (ld.ld_token_logprob(z.to(DEV), y.to(DEV), 1.5, entropy=True, top=top) for z in (x, clean))
        assert bool(got.stats[bad].isnan().all()) and bool(got.entropy[bad].isnan().all())
        assert float(got.logprob[1]) == 0.0 and bool(got.logprob[2:1 + len(kinds)].isnan().all())
        assert got.stats[0].tolist() == [-math.inf, 0.0] and float(got.entropy[0]) == 0.0 and float(got.logprob[0]) == -math.inf
        for a, b in zip(got, ref):
            assert a is None or same_bits(a[good], b[good])
        if top:
            assert bool(got.top_logprob[bad].isnan().all()) and bool((got.top_logprob[0] == -math.inf).all())
            for i, row in enumerate(kinds):  # NaN first, then by value, the lower index first
                order = torch.sort(row.isnan().int(), descending=True, stable=True).indices[:top]
                assert torch.equal(got.top_ids[1 + i].cpu().long(), order), i
        one = torch.ones(T, device=DEV)
        for out_dtype in (F32, BF16, F16):
            for h in (None, one):
                for which in (y, ids):
                    d = ld.ld_token_logprob_grad(x.to(DEV), got.stats, which.to(DEV), one, None if h is None else got.entropy, h, 1.5, out_dtype=out_dtype)
                    assert bool(d[bad].isnan().all()) and not bool(d[good].isnan().any()) and not bool(d[0].any())


@pytest.mark.parametrize("T,V", [(4, 9001), (1, 70001), (600, 9001)])
def test_a_part_of_nan_among_numbers(T, V):
    """A part of a split row that holds nothing but NaN, or NaN and masks: the row's largest logit is still that of the others."""
    print(f"[score] a part of NaN, T={T} V={V}", flush=True)
    g = gen(V)
    for fill in (math.nan, -math.inf):
        x = make(T, V, F32, g)
        x[:, 2048:4096] = fill
        x[:, 2100] = math.nan
        got = ld.ld_token_logprob(x.to(DEV), torch.full((T,), 7, device=DEV), entropy=True, top=2)
        others = torch.where(x.isnan(), -math.inf, x)
        assert torch.equal(got.stats[:, 0].cpu(), others.max(1).values) and bool(got.stats[:, 1].isnan().all())
        assert bool(got.logprob.isnan().all()) and bool(got.entropy.isnan().all()) and bool(got.top_logprob.isnan().all())
        first = [2048, 2049] if fill != fill else [2100, int(others[0].argmax())]
        assert got.top_ids[0].tolist() == first
