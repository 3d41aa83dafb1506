"""What ld_token_logprob gives are tensors of their own: none keeps another alive, and none is changed where another is."""
import pytest
import torch

from paper_2509_04084_amd import lowdiff as ld
from test_gpu_logprob import DEV, F32, gen, make

pytestmark = pytest.mark.gpu


class Logprob(torch.autograd.Function):
    """As a user's program has it: the statistics are kept for the gradient."""

    @staticmethod
    def forward(ctx, logits, ids):
        r = ld.ld_token_logprob(logits, ids, entropy=True)
        ctx.save_for_backward(logits, ids, r.stats, r.entropy)
        return r.logprob, r.entropy

    @staticmethod
    def backward(ctx, g, h):
        logits, ids, stats, entropy = ctx.saved_tensors
        return ld.ld_token_logprob_grad(logits, stats, ids, g.contiguous(), entropy, h.contiguous()), None


@pytest.mark.parametrize("rows", [(6,), (2, 3), ()])
def test_outputs_share_nothing(rows):
    g = gen(43)
    x = make(6, 500, F32, g).to(DEV).view(-1, 500)[:max(1, torch.Size(rows).numel())].reshape(*rows, 500)
    ids = torch.randint(0, 500, rows, generator=g).to(DEV)
    r = ld.ld_token_logprob(x, ids, entropy=True, top=3)
    outs = list(r)
    assert len({t.untyped_storage().data_ptr() for t in outs}) == len(outs)
    for t in outs:
        assert t.is_contiguous() and t.storage_offset() == 0 and t.untyped_storage().nbytes() == t.numel() * t.element_size() and t._base is None
    before = [t._version for t in outs]
    r.logprob.mul_(2.0)
    assert [t._version for t in outs] == [v + (t is r.logprob) for t, v in zip(outs, before)]


@pytest.mark.parametrize("rows", [(6,), (2, 3)])
def test_statistics_kept_for_a_gradient_while_outputs_change(rows):
    g = gen(47)
    x = make(6, 500, F32, g).to(DEV).view(*rows, 500).requires_grad_()
    ids = torch.randint(0, 500, rows, generator=g).to(DEV)
    y, _ = Logprob.apply(x, ids)
    y.mul_(-2.0)  # weighted in place, before the gradient is asked for
    y.sum().backward()
    want = x.detach().double().requires_grad_()
    (-2.0 * torch.log_softmax(want, -1).gather(-1, ids[..., None])).sum().backward()
    # relative errors of p as in test_gpu_logprob.py: 2^-24 (28 + 8 * 20 + 280) and 2 * 2^-24 * 30 are 3.2e-5, twice that for the weight
    assert bool(((x.grad.double() - want.grad).abs() <= 7e-5 * torch.softmax(want.detach(), -1) + 1e-6).all())
