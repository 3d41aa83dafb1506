"""Memory of the binding's own on another stream than the current one, whose kernels may still be using what it was given back."""
import numpy as np
import pytest
import torch

from paper_2509_04084_amd import lowdiff as ld

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture
def blocks(monkeypatch):
    """First and last byte of every tensor that the binding allocates."""
    seen, real = [], torch.empty

    def spy(*args, **kw):
        t = real(*args, **kw)
        seen.append((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()))
        return t

    monkeypatch.setattr(torch, "empty", spy)
    return seen


def calls():
    """Every entry point that allocates, on inputs that are ready, with what it returns."""
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    V, d, T = 500, 96, 3000
    table, dout = torch.randn(V, d, device=DEV, generator=g), torch.randn(T, d, device=DEV, generator=g)
    ids = torch.randint(0, V, (T,), device=DEV, generator=g)
    n = 100_000
    grad, off, k = torch.randn(n, device=DEV, generator=g), np.array([0, 40_000, n]), np.array([400, 600], np.int32)
    idx = [torch.arange(j, n, 50, device=DEV, dtype=torch.int32) for j in range(3)]
    val = [torch.randn(i.numel(), device=DEV, generator=g) for i in idx]
    hi, hv = [i.cpu().pin_memory() for i in idx], [v.cpu().pin_memory() for v in val]

    def embed_grad(s):
        out = torch.full((V, d), 7.0, device=DEV) if s is None else room[0]
        ld.ld_embed_grad(dout, ids, out, stream=s)
        return [out]

    def merge(s):
        w = torch.zeros(n, device=DEV) if s is None else room[1]
        ld.ld_merge_sparse(w, idx, val, 0.5, stream=s, strategy=ld.LD_MERGE_SWEEP)
        return [w]

    def adam(s):
        state = [torch.zeros(n, device=DEV) for _ in range(3)] if s is None else room[2:5]
        ld.ld_merge_sparse_adam(*state, idx, val, 0, 1e-3, 0.9, 0.999, 1e-8, stream=s)
        return state

    def from_host(s):
        w = torch.zeros(n, device=DEV) if s is None else room[5]
        ld.ld_merge_sparse_from_host(w, hi, hv, 0.5, group=2, copy_stream=s, merge_stream=s)
        return [w]

    def compress(s):
        residual = torch.zeros(n, device=DEV) if s is None else room[6]
        return [residual, *ld.ld_compress_topk(grad, residual, off, k, stream=s)]

    room = [torch.full((V, d), 7.0, device=DEV)] + [torch.zeros(n, device=DEV) for _ in range(6)]  # written on the side stream
    return dict(
        lookup=lambda s: [ld.ld_embed_lookup(table, ids, 2.0, stream=s)], embed_grad=embed_grad,
        norm=lambda s: list(ld.ld_grad_norm([grad, dout], stream=s)),
        clip=lambda s: [ld.ld_clip_grad_norm([grad, dout], 1e9, stream=s)],
        compress=compress, check=lambda s: [ld.ld_check_diff(idx[0], val[0], n, stream=s)],
        combine=lambda s: list(ld.ld_combine_sparse(idx, val, n, 0.5, stream=s))[:3], merge=merge, adam=adam, from_host=from_host)


@pytest.mark.parametrize("name", ["lookup", "embed_grad", "norm", "clip", "compress", "check", "combine", "merge", "adam", "from_host"])
def test_calls_on_two_streams_share_no_memory(name, blocks):
    print(f"[streams] {name}", flush=True)
    call, side = calls()[name], torch.cuda.Stream()
    want = [t.clone() for t in call(None)]   # outputs and temporaries of this call are given back here,
    torch.cuda.synchronize()
    blocks.clear()
    call(None)                               # used again by this one, and given back while it may still run
    mine = list(blocks)
    blocks.clear()
    got = call(side)                         # nothing makes the side stream wait
    theirs = list(blocks)
    torch.cuda.synchronize()
    assert mine and len(mine) == len(theirs)
    for a, b in mine:
        for c, d in theirs:
            assert b <= c or d <= a, "a block of the current stream was given to the other one"
    for a, b in zip(got, want):
        assert torch.equal(a, b)
