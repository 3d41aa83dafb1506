"""Rows of logits around a common offset, which says nothing of their probabilities. The bounds are those of test_gpu_logprob.py, in
which no offset stands: an exponent is one fused multiply-add against the rounded product of reference and scale, which all terms of
a sum share, and what that rounding is goes out again where sums of different references meet; differences of logits are exact."""
import pytest
import torch

from test_gpu_logprob import BF16, F16, F32, check, gen, make_ids

pytestmark = pytest.mark.gpu


def offset_rows(kind, T, V, offset, g):
    j = torch.arange(V, dtype=torch.float64)
    row = {"normal": torch.randn(T, V, generator=g, dtype=torch.float64) * 2.0,
           "last part higher": (j >= V - V // 10).double() * 3.0,             # the reference moves when nearly all is added up
           "late": (j // 2048 == (V - 1) // 2048) * (j % 8 == 5) * 3.0,       # one element of every thread's last group
           "ascending": j * 2.0 ** -8,                                       # it moves again and again
           "two levels": (j % 3 == 0) * -2.5}[kind]
    return (row + offset).to(F32).expand(T, V).contiguous()


@pytest.mark.parametrize("kind", ["normal", "last part higher", "late", "ascending", "two levels"])
@pytest.mark.parametrize("offset", [1e3, 1e5, 2.8e5, 3.6e5, -1e3, -1e5, -3e5])
def test_offsets(offset, kind):
    print(f"[score] {kind} around {offset}", flush=True)
    for T, V, top in ((3, 4001, 5), (150, 4001, 0), (3, 50257, 20), (140, 6001, 0)):
        g = gen(T + V)
        x, ids = offset_rows(kind, T, V, offset, g), make_ids(T, V, g)
        for scale in (1.0, 0.75):
            check(x, ids, scale, top, tag=(kind, offset, T, V, scale))


@pytest.mark.parametrize("dtype,offset", [(BF16, 1e3), (BF16, -3e4), (F16, 1e3), (F16, -3e4), (F16, 6e4)])
def test_offsets_of_narrow_types(dtype, offset):
    """Neighbours in these types are 1/2 to 256 apart there: at a temperature that keeps several of them probable."""
    step = torch.finfo(dtype).eps * abs(offset)
    for T, V in ((3, 9001), (140, 9001), (150, 3001)):
        g = gen(V)
        x = (offset + step * torch.randint(-3, 1, (T, V), generator=g).double()).to(dtype)
        check(x, make_ids(T, V, g), 1.0 / step, 5, tag=(dtype, offset, T, V))
