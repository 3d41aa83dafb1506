"""Token log probabilities and their gradient: what they refuse, without a GPU."""
import ctypes

import pytest
import torch

from paper_2509_04084_amd import lowdiff as ld

FAKE = 0x10000  # never dereferenced: every call below fails its checks or has nothing to do
V = ctypes.c_void_p
F = ctypes.c_float
NULL, RANGE, WORKSPACE, ALIGN = -1, -2, -3, -5


def test_logprob_refusals():
    lib = ld.load()
    assert lib.ld_token_logprob_workspace(100000, 50257, 64) == 0  # many rows are not split
    wsb = lib.ld_token_logprob_workspace(8, 50257, 5)
    assert wsb > 0
    for bad in ((-1, 100, 0), ((1 << 24) + 1, 100, 0), (8, -1, 0), (8, (1 << 24) + 1, 0), (8, 100, 65), (8, 100, -1), (8, 3, 4)):
        assert lib.ld_token_logprob_workspace(*bad) == 0, bad

    def call(logits=FAKE, T=8, vocab=50257, stride=50257, dtype=1, ids=FAKE, it=1, scale=1.0, lp=FAKE, ent=FAKE, stats=FAKE, top=5, ti=FAKE,
             tl=FAKE, ws=FAKE, wsb=wsb):
        return lib.ld_token_logprob(V(logits), T, vocab, stride, dtype, V(ids), it, F(scale), V(lp), V(ent), V(stats), top, V(ti), V(tl), V(ws),
                                    wsb, None)

    for bad in (dict(logits=0), dict(ids=0), dict(lp=0), dict(stats=0), dict(ti=0), dict(tl=0)):
        assert call(**bad) == NULL, bad
    for bad in (dict(T=-1), dict(T=(1 << 24) + 1), dict(vocab=0), dict(vocab=-5), dict(vocab=(1 << 24) + 1), dict(stride=-1), dict(dtype=3),
                dict(it=2), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=1e-40),
                dict(top=65), dict(top=-1), dict(vocab=4)):
        assert call(**bad) == RANGE, bad
    for bad in (dict(logits=FAKE + 1), dict(dtype=0, logits=FAKE + 2), dict(ids=FAKE + 4), dict(it=0, ids=FAKE + 2), dict(lp=FAKE + 2),
                dict(ent=FAKE + 1), dict(stats=FAKE + 2), dict(ti=FAKE + 1), dict(tl=FAKE + 3)):
        assert call(**bad) == ALIGN, bad
    assert call(ws=0) == WORKSPACE and call(ws=FAKE + 128) == WORKSPACE and call(wsb=wsb - 1) == WORKSPACE
    assert call(T=0, logits=0, ids=0, lp=0, stats=0, vocab=0, top=0) == 0


def test_logprob_grad_refusals():
    lib = ld.load()

    def call(logits=FAKE, T=8, vocab=100, stride=100, dtype=1, ids=FAKE, it=1, scale=1.0, stats=FAKE, g=FAKE, gs=1, ent=FAKE, h=FAKE, hs=1,
             out=FAKE + 4096, os=100, ot=1):
        return lib.ld_token_logprob_grad(V(logits), T, vocab, stride, dtype, V(ids), it, F(scale), V(stats), V(g), gs, V(ent), V(h), hs, V(out),
                                         os, ot, None)

    for bad in (dict(logits=0), dict(stats=0), dict(out=0), dict(ids=0), dict(g=0), dict(ent=0), dict(h=0)):
        assert call(**bad) == NULL, bad
    for bad in (dict(T=-1), dict(vocab=-1), dict(vocab=(1 << 24) + 1, os=1 << 25), dict(stride=-1), dict(os=99), dict(dtype=3), dict(ot=-1),
                dict(it=5), dict(scale=0.0), dict(scale=float("nan")), dict(gs=-1), dict(hs=-1),
                dict(out=FAKE, ot=0), dict(out=FAKE, os=101)):  # in place, but of another type or stride
        assert call(**bad) == RANGE, bad
    for bad in (dict(logits=FAKE + 1), dict(out=FAKE + 1), dict(ot=0, out=FAKE + 2), dict(ids=FAKE + 4), dict(stats=FAKE + 2), dict(g=FAKE + 2),
                dict(ent=FAKE + 2), dict(h=FAKE + 1)):
        assert call(**bad) == ALIGN, bad
    assert call(T=0, logits=0, stats=0, out=0) == 0 and call(vocab=0, os=0) == 0


def test_binding_refuses_before_any_launch():
    x, ids = torch.zeros(4, 10), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(TypeError):
        ld.ld_token_logprob(x, ids)  # not on a GPU
    with pytest.raises(TypeError):
        ld.ld_token_logprob(x.double(), ids)
    with pytest.raises(TypeError):
        ld.ld_token_logprob(torch.zeros(()))
    with pytest.raises(ValueError, match="one token for every row"):
        ld.ld_token_logprob(x, ids[:3])
    with pytest.raises(ValueError, match="different devices"):
        ld.ld_token_logprob(x, ids.to("meta"))
    stats = torch.zeros(4, 2)
    with pytest.raises(ValueError, match="go together"):
        ld.ld_token_logprob_grad(x, stats, ids)
    with pytest.raises(ValueError, match="go together"):
        ld.ld_token_logprob_grad(x, stats, d_entropy=torch.zeros(4))
    with pytest.raises(ValueError, match="two values"):
        ld.ld_token_logprob_grad(x, stats[:3], ids, torch.zeros(4))
    with pytest.raises(ValueError, match="one value for every row"):
        ld.ld_token_logprob_grad(x, stats, entropy=torch.zeros(3), d_entropy=torch.zeros(4))
    with pytest.raises(TypeError):
        ld.ld_token_logprob_grad(x, stats, ids, torch.zeros(4))
