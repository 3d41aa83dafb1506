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


# Bounds as in test_gpu_embed_norm, with u = 2^-24 and u_o the unit roundoff of the output's type; the definitions in 64 bits on the
# GPU. A difference passes only where it is known to be small, so that NaN does not.
U = 2.0 ** -24
UNIT = {F32: U, BF16: 2.0 ** -8, F16: 2.0 ** -11}
STEP = {F32: 2.0 ** -149, BF16: 2.0 ** -133, F16: 2.0 ** -24}
CHUNK = 1 << 26


def close(got, want, spread, tag):
    bound = 1.01 * (spread + UNIT[got.dtype] * want.abs()) + 0.5 * STEP[got.dtype]
    bad = ~((got.double() - want).abs() <= bound)
    assert not bad.any(), (tag, int(bad.sum()), bad.nonzero()[0].tolist())


def normal(seed, shape, dtype, std=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEV).mul_(std).to(dtype)


@pytest.mark.parametrize("dtype,out_dtype", [(a, b) for a in (F32, BF16, F16) for b in (F32, BF16, F16)])
@pytest.mark.parametrize("T,d", [(4099, 4104), (16391, 1030)])
def test_lookup_of_a_large_output(T, d, dtype, out_dtype):
    """More than 32 MB: written around the caches, in other steps."""
    print(f"[lookup] T={T} d={d} {dtype} -> {out_dtype}", flush=True)
    V, P = 3001, 513
    table, more = normal(1, (V, d), dtype), normal(2, (P, d), dtype)
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    ids = torch.randint(-1, V + 1, (T,), device=DEV, generator=g)
    at = torch.randint(-1, P + 1, (T,), device=DEV, generator=g)
    rows = lambda tab, i: torch.where(((i >= 0) & (i < len(tab)))[:, None], tab[i.clamp(0, len(tab) - 1)].double(), 0.0)  # noqa: E731
    for pos in (False, True):
        out = ld.ld_embed_lookup(table, ids, 27.625, more if pos else None, at if pos else None, out_dtype=out_dtype)
        want = rows(table, ids) * 27.625 + (rows(more, at) if pos else 0)
        assert out.dtype == out_dtype and out.numel() * out.element_size() > 32 << 20
        close(out, want, U * want.abs(), pos)


@pytest.mark.parametrize("dtype,grad_dtype,T,d", [(F32, F32, 33001, 2052), (F32, BF16, 17001, 4099), (F16, F32, 66001, 2056), (F16, F16, 33003, 4091),
                                                  (BF16, F32, 33003, 4091)])
def test_gradient_of_a_large_batch(dtype, grad_dtype, T, d):
    """More than 256 MB of gradients come in: read around the caches."""
    print(f"[embed_grad] T={T} d={d} {dtype} -> {grad_dtype}", flush=True)
    V, scale = 2003, 0.75
    dout, before = normal(4, (T, d), dtype, 0.1), normal(5, (V, d), grad_dtype)
    assert dout.numel() * dout.element_size() > 256 << 20
    g = torch.Generator(device=DEV)
    g.manual_seed(6)
    ids = torch.randint(-100, V + 100, (T,), device=DEV, generator=g)
    ids = torch.where(torch.rand(T, device=DEV, generator=g) < 0.2, 77, ids)  # and a row that many chunks add up to
    inside = ((ids >= 0) & (ids < V)).nonzero().flatten()
    total = torch.zeros(V, d, dtype=torch.float64, device=DEV).index_add_(0, ids[inside], dout[inside].double())
    mass = torch.zeros(V, d, dtype=torch.float64, device=DEV).index_add_(0, ids[inside], dout[inside].double().abs())
    count = torch.bincount(ids[inside], minlength=V).double()[:, None]
    for accumulate in (False, True):
        grad = before.clone()
        ld.ld_embed_grad(dout, ids, grad, scale, accumulate)
        want = total * scale + (before.double() if accumulate else 0)
        close(grad, want, U * scale * count * mass + U * want.abs(), accumulate)


def sum64(parts):
    return sum(float(x[c:c + CHUNK].double().square().sum()) for x in parts for c in range(0, x.numel(), CHUNK))


def check_clip(parts, outs, factor, tag):
    """Clipping to `factor` times the norm, and under a limit that is twice it."""
    before, norm = [x.clone() for x in parts], sum64(parts) ** 0.5
    for limit in (2.0 * norm, factor * norm):
        limit = float(torch.tensor(limit))
        f = limit / norm if norm > limit else 1.0
        got = float(ld.ld_clip_grad_norm(parts, limit, outs))
        assert abs(got - norm) <= U * (1 + 2.0 ** -10) * norm, tag
        for x, y in zip(before, parts if outs is None else outs):
            for c in range(0, x.numel(), CHUNK):
                want = x[c:c + CHUNK].double() * f
                close(y[c:c + CHUNK], want, 2 * U * want.abs() if f < 1.0 else 0.0 * want, (tag, limit, c))
        if outs is not None:
            assert all(torch.equal(a, b) for a, b in zip(before, parts)), tag  # inputs are not written


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("sizes", [[16384 * 8192], [16384 * 8192 + 1], [70_000_001, 5, 66_000_007, 8192], [150_000_003, 70_000_001]], ids=str)
def test_clip_in_place_of_more_pieces_than_workgroups(sizes, dtype):
    """16384 workgroups clip in place, a piece of 4096 fp32 or 8192 16-bit values at a time."""
    print(f"[clip in place] {sizes} {dtype}", flush=True)
    check_clip([normal(7 + i, (n,), dtype, 0.3) for i, n in enumerate(sizes)], None, 0.37, (sizes, dtype))


@pytest.mark.parametrize("dtype,out_dtype", [(F32, BF16), (BF16, F32), (F16, F16), (F32, F32)])
@pytest.mark.parametrize("n", [2047 * 4096, 2048 * 4096 + 3, 2049 * 8192, 40_000_001])
def test_clip_of_more_pieces_than_partial_sums(n, dtype, out_dtype):
    """A launch leaves 2048 partial sums at most; that many are added up by a launch of their own."""
    print(f"[clip] {n} {dtype} -> {out_dtype}", flush=True)
    parts = [normal(9, (n,), dtype, 0.3), normal(10, (77,), dtype, 0.3)]
    check_clip(parts, [torch.full((x.numel(),), 9.0, dtype=out_dtype, device=DEV) for x in parts], 0.37, (n, dtype, out_dtype))


def test_clip_of_more_than_2_31_elements():
    print("[clip] more than 2^31 elements", flush=True)
    n = 2 ** 31 + 4099
    x = torch.empty(n, dtype=BF16, device=DEV)
    for c in range(0, n, CHUNK):
        x[c:c + CHUNK] = normal(11 + c, (min(CHUNK, n - c),), BF16, 0.3)
    last = x[-5:].clone()
    check_clip([x, x.new_ones(3)], None, 0.37, "in place")
    assert bool((x[-5:].float().abs() <= 0.371 * last.float().abs()).all())
    check_clip([x], [torch.zeros(n, dtype=BF16, device=DEV)], 0.5, "into another")
