"""Embedding, gradient norm and clipping at sizes where a launch, or a branch of a kernel, is another one."""
import pytest
import torch

from paper_2509_04084_amd import lowdiff as ld

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.mark.parametrize("V", [268_435_328, 268_435_457, 600_000_011])
def test_few_tokens_and_more_rows_than_workgroups_clear_at_a_time(V):
    """A clearing workgroup takes 64 rows; a launch of 1024 threads each has 4194303 of them, one of which adds."""
    print(f"[few, many rows] V={V}", flush=True)
    grad = torch.full((V, 1), 5.0, dtype=BF16, device=DEV)
    ids = torch.tensor([V - 1, 0, V // 2], device=DEV)
    ld.ld_embed_grad(torch.ones(3, 1, device=DEV), ids, grad, 3.0)
    assert int((grad != 0).sum()) == 3 and bool((grad[ids] == 3).all())
