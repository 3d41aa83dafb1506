"""Embedding lookup, its gradient by sorted tokens, gradient norm and clipping on the GPU, against the definitions in 64
bits on the CPU.

Bounds, with u the unit roundoff of 32 bits (2^-24) and u_o that of the output's type (2^-24, 2^-8 for bf16, 2^-11 for fp16):
  lookup     one fused multiply-add and one rounding:   u |y| + u_o |y|
  gradient   m terms added in any order in 32 bits:     m u |scale| sum|x|, then as the lookup
  norm       64-bit squares and sums, rounded once:     u (1 + 2^-10) |norm|
  clipping   factor and product rounded to 32 bits:     2 u |y| + u_o |y|
each with 1 % for second-order terms and half of the type's smallest step for results that are subnormal in it.
"""
import math

import numpy as np
import pytest
import torch

from paper_2509_04084_amd import lowdiff as ld

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
U = 2.0 ** -24
UNIT = {F32: U, BF16: 2.0 ** -8, F16: 2.0 ** -11}
STEP = {F32: 2.0 ** -149, BF16: 2.0 ** -133, F16: 2.0 ** -24}


def close(got, want, spread, dtype, tag):
    """|got - want| <= spread + u_o |want| (+ the allowances above), element by element."""
    assert got.dtype == dtype
    got = got.detach().double().cpu()
    bound = 1.01 * (spread + UNIT[dtype] * want.abs()) + 0.5 * STEP[dtype]
    bad = (got - want).abs() > bound
    assert not bad.any(), (tag, int(bad.sum()), float((got - want).abs().max()), float(bound[bad].min()))


def normal(gen, shape, std=1.0, dtype=F32):
    return (torch.randn(shape, generator=gen, dtype=torch.float64) * std).to(dtype)


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def same_bits(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


# ---------------------------------------------------------------------------------------------- lookup

def lookup64(table, ids, scale, pos_table, positions):
    def rows(tab, i):
        i = i.flatten()
        inside = (i >= 0) & (i < tab.shape[0])
        out = torch.zeros(i.numel(), tab.shape[1], dtype=torch.float64)
        out[inside] = tab[i[inside].long()].double()
        return out
    y = rows(table, ids) * scale
    return y if pos_table is None else y + rows(pos_table, positions)


@pytest.mark.parametrize("dtype,out_dtype", [(a, b) for a in (F32, BF16, F16) for b in (F32, BF16, F16)])
@pytest.mark.parametrize("T,V,d", [(1, 1, 1), (1, 50257, 1600), (3, 7, 3), (5, 100, 7), (64, 300, 8), (65, 1000, 9), (300, 77, 64),
                                   (257, 513, 127), (1000, 2000, 768), (33, 1000, 4096), (7, 40, 12289)])
def test_lookup(T, V, d, dtype, out_dtype):
    print(f"[lookup] T={T} V={V} d={d} {dtype} -> {out_dtype}", flush=True)
    g = gen(T * 7 + d)
    table, pos_table = normal(g, (V, d), 0.5, dtype), normal(g, (V // 2 + 1, d), 0.5, dtype)
    ids = torch.randint(-1, V + 1, (T,), generator=g)
    positions = torch.randint(-1, V // 2 + 2, (T,), generator=g)
    for id_dtype in (torch.int32, torch.int64):
        for scale in (1.0, 27.625):
            for pos in (False, True):
                p = (pos_table.to(DEV), positions.to(DEV, id_dtype)) if pos else (None, None)
                out = ld.ld_embed_lookup(table.to(DEV), ids.to(DEV, id_dtype), scale, *p, out_dtype=out_dtype)
                want = lookup64(table, ids, scale, pos_table if pos else None, positions)
                assert out.shape == (T, d)
                close(out, want, U * want.abs(), out_dtype, (id_dtype, scale, pos))
    if dtype == out_dtype:  # a copy
        out = ld.ld_embed_lookup(table.to(DEV), ids.to(DEV))
        inside = (ids >= 0) & (ids < V)
        assert same_bits(out.cpu()[inside], table[ids[inside]]) and not out.cpu()[~inside].any()


def test_lookup_shapes_strides_and_what_lies_around():
    g = gen(3)
    wide = normal(g, (50, 40), 1.0, BF16)
    table = wide.to(DEV)[:, 5:26]                     # rows 40 apart, beginning at an odd element
    ids = torch.randint(0, 50, (6, 11), generator=g)
    out = ld.ld_embed_lookup(table, ids.to(DEV), 2.0)
    want = lookup64(wide[:, 5:26], ids, 2.0, None, None)
    assert out.shape == (6, 11, 21) and out.is_contiguous()
    close(out.view(66, 21), want, U * want.abs(), BF16, "view")
    room = torch.full((66, 30), 7.0, device=DEV)      # into rows of something wider: the rest of it stays
    assert ld.ld_embed_lookup(table, ids.to(DEV), 2.0, out=room[:, 3:24]) is not None
    close(room[:, 3:24], want, U * want.abs(), F32, "strided out")
    assert bool((room[:, :3] == 7).all()) and bool((room[:, 24:] == 7).all())
    one_row = ld.ld_embed_lookup(table[4:5], torch.zeros(9, dtype=torch.int32, device=DEV))
    assert same_bits(one_row.cpu(), wide[4:5, 5:26].expand(9, 21))
    shared = torch.arange(21.0, device=DEV).expand(1000, 21)  # a table whose rows are one row
    assert torch.equal(ld.ld_embed_lookup(shared, ids.to(DEV)), shared[:66].reshape(6, 11, 21))


def test_lookup_of_nothing_and_of_ids_beyond_32_bits():
    table = torch.ones(5, 8, device=DEV)
    assert ld.ld_embed_lookup(table, torch.zeros(0, dtype=torch.int64, device=DEV)).shape == (0, 8)
    assert ld.ld_embed_lookup(table[:, :0], torch.zeros(3, dtype=torch.int64, device=DEV)).shape == (3, 0)
    far = torch.tensor([2 ** 32 + 1, -2 ** 32 + 1, 2 ** 62, -2 ** 63, 4, 5], device=DEV)
    out = ld.ld_embed_lookup(table, far)
    assert out.sum(1).tolist() == [0, 0, 0, 0, 8, 0]
    assert not ld.ld_embed_lookup(table[:0], far).any()           # an empty table names nothing
    inf = torch.full((2, 8), math.inf, device=DEV)
    out = ld.ld_embed_lookup(inf, torch.tensor([0, -1], device=DEV), 0.0)
    assert bool(out[0].isnan().all()) and not out[1].any()        # a row that is not named is not multiplied either


# -------------------------------------------------------------------------------------------- gradient

def grad64(dout, ids, scale, V, grad=None):
    """Gradient, and the bound on the error of its sums, in 64 bits."""
    ids = ids.flatten().long()
    inside = (ids >= 0) & (ids < V)
    x = dout[inside].double()
    total = torch.zeros(V, dout.shape[1], dtype=torch.float64).index_add_(0, ids[inside], x)
    mass = torch.zeros(V, dout.shape[1], dtype=torch.float64).index_add_(0, ids[inside], x.abs())
    count = torch.bincount(ids[inside], minlength=V)[:V].double()
    y = total * scale + (0 if grad is None else grad.double())
    return y, U * abs(scale) * count[:, None] * mass + U * y.abs()


def make_ids(kind, T, V, g):
    if kind == "uniform":
        return torch.randint(0, V, (T,), generator=g)
    if kind == "outside":
        return torch.randint(-V // 2 - 1, V + V // 2 + 1, (T,), generator=g)
    if kind == "one":
        return torch.full((T,), V // 2)
    if kind == "two":
        return torch.arange(T) % 2 * (V - 1)
    if kind == "descending":
        return (V - 1 - torch.arange(T)) % V
    if kind == "heavy":  # half of the tokens one id, the rest anywhere
        return torch.where(torch.rand(T, generator=g) < 0.5, V // 3, torch.randint(0, V, (T,), generator=g))
    return torch.full((T,), -1)


def check_grad(T, V, d, kind, dtype=F32, grad_dtype=F32, scale=1.0, id_dtype=torch.int64, seed=0, both=True):
    print(f"[embed_grad] T={T} V={V} d={d} {kind} {dtype} -> {grad_dtype}", flush=True)
    g = gen(seed + 13 * T + V + d)
    ids, dout, before = make_ids(kind, T, V, g), normal(g, (T, d), 1.0, dtype), normal(g, (V, d), 1.0, grad_dtype)
    if T:
        dout[(ids < 0) | (ids >= V)] = math.nan  # what no row is given has to stay out of all of them
    x, i = dout.to(DEV), ids.to(DEV, id_dtype)
    for accumulate in (False, True) if both else (False,):
        grad = before.to(DEV)
        ld.ld_embed_grad(x, i, grad, scale, accumulate)
        want, spread = grad64(dout, ids, scale, V, before if accumulate else None)
        close(grad, want, spread, grad_dtype, (kind, accumulate))
        if accumulate:  # what is not named is not touched
            missing = torch.ones(V, dtype=torch.bool)
            missing[ids[(ids >= 0) & (ids < V)]] = False
            assert same_bits(grad.cpu()[missing], before[missing])
        again = before.to(DEV)
        ld.ld_embed_grad(x, i, again, scale, accumulate)
        assert same_bits(grad, again), "the same input gave other bits"


@pytest.mark.parametrize("kind", ["uniform", "outside", "one", "two", "descending", "heavy", "none"])
@pytest.mark.parametrize("T,V,d", [(1, 1, 1), (1, 50257, 64), (2, 2, 3), (63, 50, 5), (64, 64, 8), (65, 1023, 9), (257, 1024, 64),
                                   (1000, 2047, 33), (4095, 2048, 16), (4096, 300, 64), (4097, 5000, 12), (9001, 70, 40)])
def test_embed_grad(T, V, d, kind):
    check_grad(T, V, d, kind, scale=0.75 if d % 2 else 1.0)


@pytest.mark.parametrize("kind", ["uniform", "outside", "one", "two", "heavy"])
@pytest.mark.parametrize("T,V,d", [(7, 200, 300), (31, 9, 129), (255, 40, 260), (256, 50257, 131), (257, 40, 130), (512, 300, 1), (700, 20, 128),
                                   (1023, 90, 515), (1024, 70, 2), (129, 30, 33000), (200, 20_000_000, 2), (1024, 20_000_000, 1)])
def test_embed_grad_of_few_tokens(T, V, d, kind):
    check_grad(T, V, d, kind, BF16 if d % 2 else F32, F32, scale=1.25, id_dtype=torch.int32, seed=3)


@pytest.mark.parametrize("dtype,grad_dtype", [(a, b) for a in (F32, BF16, F16) for b in (F32, BF16, F16)])
@pytest.mark.parametrize("T,V,d,kind", [(300, 90, 129, "heavy"), (2500, 1000, 264, "outside"), (129, 40, 1001, "uniform")])
def test_embed_grad_types(T, V, d, kind, dtype, grad_dtype):
    check_grad(T, V, d, kind, dtype, grad_dtype, scale=3.5, id_dtype=torch.int32)


@pytest.mark.parametrize("T,V,d,kind", [(70001, 50257, 24, "heavy"), (40000, 1024, 100, "descending"), (65536, 3, 32, "uniform"),
                                        (300000, 9, 4, "heavy"), (20000, 5000, 520, "one"), (16385, 4_200_000, 3, "uniform"),
                                        (1024, 300_000, 20, "outside"), (1025, 600, 20, "heavy"), (16384, 50257, 9, "outside"),
                                        (16384, 300_000, 3, "uniform"), (1_100_000, 3000, 2, "heavy"), (2_200_000, 70_000, 1, "outside")])
def test_embed_grad_of_many_tokens(T, V, d, kind):
    check_grad(T, V, d, kind, BF16, F32, seed=5)


@pytest.mark.parametrize("length", [2, 3, 15, 16, 17, 31, 32, 33, 63, 64, 65, 130])
@pytest.mark.parametrize("T,d", [(200, 5), (900, 300), (1500, 600), (5000, 1100), (20000, 1100), (70000, 2100)])
def test_embed_grad_of_runs_of_every_length(T, d, length):
    """Whole numbers, so that every order of adding gives the same: ids that are each named as often, from some offset on."""
    print(f"[embed_grad] T={T} d={d} runs of {length}", flush=True)
    g = torch.Generator(device=DEV)
    g.manual_seed(T + length)
    for offset in (0, 7):
        ids = ((torch.arange(T, device=DEV) + offset) // length)[torch.randperm(T, device=DEV, generator=g)]
        V = (T + offset) // length + 2
        x = torch.randint(-2, 3, (T, d), device=DEV, generator=g).to(BF16)
        want = torch.zeros(V, d, device=DEV).index_add_(0, ids, x.float())
        for accumulate in (False, True):
            grad = torch.full((V, d), 4.0, device=DEV)
            ld.ld_embed_grad(x, ids, grad, accumulate=accumulate)
            assert torch.equal(grad, want + 4.0 if accumulate else want), (offset, accumulate)


def test_embed_grad_of_nothing():
    grad = torch.ones(5, 7, device=DEV)
    none, x = torch.zeros(0, dtype=torch.int64, device=DEV), torch.zeros(0, 7, device=DEV)
    ld.ld_embed_grad(x, none, grad, accumulate=True)
    assert bool((grad == 1).all())
    ld.ld_embed_grad(x, none, grad)
    assert not grad.any()
    ld.ld_embed_grad(torch.zeros(3, 7, device=DEV), none.new_zeros(3), grad[:0])
    ld.ld_embed_grad(torch.zeros(3, 0, device=DEV), none.new_zeros(3), grad[:, :0])


def test_embed_grad_of_ids_beyond_32_bits():
    ids = torch.tensor([2 ** 32 + 1, -2 ** 32 + 1, 2 ** 62, -2 ** 63, 4, 5], device=DEV)
    grad = torch.full((5, 8), 9.0, device=DEV)
    ld.ld_embed_grad(torch.ones(6, 8, device=DEV), ids, grad)
    assert grad.sum(1).tolist() == [0, 0, 0, 0, 8]


def test_embed_grad_strides_and_what_lies_around():
    g = gen(8)
    for dtype, grad_dtype, d, at in ((F32, F32, 21, 1), (BF16, F32, 40, 3), (F16, BF16, 64, 4), (BF16, BF16, 33, 0)):
        wide = normal(g, (400, d + 9), 1.0, dtype)
        ids = torch.randint(0, 60, (4, 100), generator=g)
        room = torch.full((60, d + 11), 5.0, dtype=grad_dtype, device=DEV)
        ld.ld_embed_grad(wide.to(DEV)[:, at:at + d], ids.to(DEV), room[:, 2:2 + d], 2.0)
        want, spread = grad64(wide[:, at:at + d], ids, 2.0, 60)
        close(room[:, 2:2 + d], want, spread, grad_dtype, d)
        assert bool((room[:, :2] == 5).all()) and bool((room[:, 2 + d:] == 5).all())
    one = torch.arange(16.0, device=DEV).expand(8, 50, 16)   # the gradient of a sum: one row for all tokens
    ids = torch.randint(0, 6, (8, 50), generator=g)
    grad = torch.zeros(6, 16, device=DEV)
    ld.ld_embed_grad(one[0], ids[0].to(DEV), grad)
    count = torch.bincount(ids[0], minlength=6)
    assert torch.equal(grad.cpu(), count[:, None] * torch.arange(16.0))


def test_embed_grad_keeps_infinities_and_nan_in_their_rows():
    ids = torch.tensor([0, 1, 2, 1, 3, -1, 3], device=DEV)
    x = torch.ones(7, 300, device=DEV)
    x[1, 5], x[3, 5], x[4, 7], x[5] = math.inf, -math.inf, math.inf, math.nan
    grad = torch.zeros(5, 300, device=DEV)
    ld.ld_embed_grad(x, ids, grad)
    want = torch.tensor([1.0, 2.0, 1.0, 2.0, 0.0])[:, None].repeat(1, 300)
    want[1, 5], want[3, 7] = math.nan, math.inf
    assert torch.equal(grad.cpu().nan_to_num(nan=-7.0), want.nan_to_num(nan=-7.0))


def test_embed_grad_against_differences_of_the_lookup():
    """L = sum(lookup * w) is linear in the table: with whole numbers its differences are the gradient exactly."""
    g = gen(11)
    V, d, T = 13, 20, 150
    table, w = torch.randint(-8, 9, (V, d), generator=g).float(), torch.randint(-8, 9, (T, d), generator=g).float()
    ids = torch.randint(-1, V + 1, (T,), generator=g).to(DEV)
    loss = lambda t: float((ld.ld_embed_lookup(t.to(DEV), ids, 4.0).double() * w.to(DEV).double()).sum())  # noqa: E731
    grad = torch.zeros(V, d, device=DEV)
    ld.ld_embed_grad(w.to(DEV), ids, grad, 4.0)
    for v in range(V):
        for c in range(0, d, 7):
            up, down = table.clone(), table.clone()
            up[v, c] += 1
            down[v, c] -= 1
            assert (loss(up) - loss(down)) / 2 == float(grad[v, c]), (v, c)


def test_tables_and_gradients_of_more_than_2_31_elements():
    V, d, T = 70001, 32768, 300
    table = torch.zeros(V, d, dtype=BF16, device=DEV)
    row = normal(gen(4), (d,), 1.0, BF16)
    table[V - 1] = row.to(DEV)
    ids = torch.full((T,), 7, dtype=torch.int64, device=DEV)
    ids[::2] = V - 1
    out = ld.ld_embed_lookup(table, ids)
    assert bool((out[::2] == row.to(DEV)).all()) and not out[1::2].any()
    dout = torch.ones(T, d, dtype=BF16, device=DEV)
    ld.ld_embed_grad(dout, ids, table, accumulate=True)
    want = row.float() + 150
    close(table[V - 1], want.double(), U * want.double().abs(), BF16, "last row")
    assert bool((table[7] == 150).all()) and not table[8:V - 1].any() and not table[:7].any()
    ld.ld_embed_grad(dout, ids, table)
    assert bool((table[V - 1] == 150).all()) and bool((table[7] == 150).all()) and not table[8:V - 1].any() and not table[:7].any()
    del dout, out
    many = torch.ones(70001, 32768, dtype=BF16, device=DEV)  # and of as many elements of its output
    grad = torch.zeros(3, 32768, device=DEV)
    ids = torch.full((70001,), -1, dtype=torch.int32, device=DEV)
    ids[[0, 35000, 70000]] = torch.tensor([1, 2, 2], dtype=torch.int32, device=DEV)
    ld.ld_embed_grad(many, ids, grad)
    assert bool((grad[1] == 1).all()) and bool((grad[2] == 2).all()) and not grad[0].any()


def test_more_rows_than_a_launch_has_threads_for():
    V = 70_000_001
    for T in (3, 2000, 5000):
        grad = torch.full((V, 1), 5.0, dtype=BF16, device=DEV)
        ids = torch.arange(T, device=DEV) * (V // T)
        ids[-1] = V - 1
        ld.ld_embed_grad(torch.ones(T, 1, device=DEV), ids, grad, 3.0)
        assert float(grad.float().sum()) == 3.0 * T and bool((grad[ids] == 3).all())


def test_lookup_of_more_tokens_than_a_launch_takes():
    table = torch.arange(300.0, device=DEV)[:, None].to(F16)
    ids = torch.arange(2_200_000_000, device=DEV, dtype=torch.int32).remainder_(300)
    out = ld.ld_embed_lookup(table, ids, 2.0)
    for a in (0, 2_147_480_000, 2_199_990_000):
        assert torch.equal(out[a:a + 10_000, 0], 2.0 * ids[a:a + 10_000].to(F16))


# --------------------------------------------------------------------------------------- norm, clipping

def clip64(parts, max_norm, dtype):
    norm = math.sqrt(sum(float(x.double().square().sum()) for x in parts))
    f = float(np.float32(max_norm)) / norm if norm > float(np.float32(max_norm)) else 1.0
    return norm, [x.double() * f for x in parts]


SIZES = [[1], [0], [], [7], [4096], [4097, 0, 1], [8192, 8193, 3], [100003], [5, 6, 7, 8] * 30, [1] * 400, [65537] * 9 + [1, 2],
         [3_000_017, 64, 64, 1]]


@pytest.mark.parametrize("dtype,out_dtype", [(a, b) for a in (F32, BF16, F16) for b in (F32, BF16, F16)])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{max(s, default=0)}")
def test_clip(sizes, dtype, out_dtype):
    print(f"[clip] {sizes[:6]} {dtype} -> {out_dtype}", flush=True)
    g = gen(len(sizes) + sum(sizes))
    parts = [normal(g, (n,), 0.3, dtype) for n in sizes]
    full = math.sqrt(sum(float(x.double().square().sum()) for x in parts))
    for max_norm in (0.37 * full, 2.0 * full + 1.0):
        norm, want = clip64(parts, max_norm, dtype)
        src = [x.to(DEV) for x in parts]
        outs = [torch.full((n,), 9.0, dtype=out_dtype, device=DEV) for n in sizes]
        got = ld.ld_clip_grad_norm(src, max_norm, outs)
        assert got.shape == (1,) and abs(float(got) - norm) <= U * (1 + 2.0 ** -10) * norm
        for o, w, s, x in zip(outs, want, src, parts):
            close(o, w, 2 * U * w.abs(), out_dtype, max_norm)
            assert same_bits(s.cpu(), x)                           # inputs are not written
        # the same in two calls, and in place: the same bits
        sumsq, again = ld.ld_grad_norm(src)
        assert same_bits(again, got)
        two = [torch.full((n,), 9.0, dtype=out_dtype, device=DEV) for n in sizes]
        ld.ld_clip_grads(src, sumsq, max_norm, two)
        assert all(same_bits(a, b) for a, b in zip(two, outs))
        if dtype == out_dtype:
            assert same_bits(ld.ld_clip_grad_norm(src, max_norm), got)
            assert all(same_bits(a, b) for a, b in zip(src, outs))


def test_norm_accumulates_over_types():
    g = gen(2)
    a, b = [normal(g, (1000,)), normal(g, (77,))], [normal(g, (513,), 1.0, BF16)]
    sumsq, _ = ld.ld_grad_norm([x.to(DEV) for x in a])
    total, norm = ld.ld_grad_norm([x.to(DEV) for x in b], sumsq, accumulate=True)
    assert total is sumsq
    want = sum(float(x.double().square().sum()) for x in a + b)
    assert abs(float(total) - want) <= 1e-12 * want and abs(float(norm) - math.sqrt(want)) <= U * 1.01 * math.sqrt(want)
    ld.ld_grad_norm([], sumsq, accumulate=True)
    assert abs(float(sumsq) - want) <= 1e-12 * want
    assert float(ld.ld_grad_norm([])[0]) == 0.0 and float(ld.ld_clip_grad_norm([], 1.0)) == 0.0


def test_clip_of_views_at_any_alignment():
    g = gen(6)
    for dtype in (F32, BF16, F16):
        sizes = [1, 5, 4099, 8, 30001, 2, 8191, 12]
        flat = normal(g, (sum(sizes) + 3,), 1.0, dtype)
        dev, room = flat.to(DEV), torch.full((sum(sizes) + 9,), 3.0, device=DEV)
        src, dst, at = [], [], 0
        for n in sizes:
            src.append(dev[3 + at:3 + at + n])
            dst.append(room[5 + at:5 + at + n])
            at += n
        norm, want = clip64([flat[3:]], 2.5, dtype)
        got = ld.ld_clip_grad_norm(src, 2.5, dst)
        assert abs(float(got) - norm) <= U * 1.01 * norm
        close(room[5:5 + at], want[0], 2 * U * want[0].abs(), F32, dtype)
        assert bool((room[:5] == 3).all()) and bool((room[5 + at:] == 3).all())


@pytest.mark.parametrize("dtype,out_dtype", [(F32, F32), (BF16, F32), (F16, BF16)])
def test_clip_of_neighbours(dtype, out_dtype):
    """Parts of one buffer, some apart, some that go elsewhere than behind the one before, some empty."""
    g = gen(12)
    sizes = [int(n) for n in torch.randint(0, 900, (700,), generator=g)] + [40000, 3, 0, 17]
    src = normal(g, (sum(sizes) + 10 * len(sizes),), 1.0, dtype).to(DEV)
    dst = torch.full((sum(sizes) + 10 * len(sizes),), 7.0, dtype=out_dtype, device=DEV)
    parts, outs, at, to = [], [], 0, 0
    for i, n in enumerate(sizes):
        at += i % 50 == 49   # a gap on one side, on the other, or on both, now and then
        to += 3 * (i % 40 == 39)
        parts.append(src[at:at + n])
        outs.append(dst[to:to + n])
        at, to = at + n, to + n
    outs[100], outs[101] = outs[101], outs[100]
    parts[100], parts[101] = parts[101], parts[100]
    norm, want = clip64([x.cpu() for x in parts], 5.0, dtype)
    got = ld.ld_clip_grad_norm(parts, 5.0, outs)
    assert abs(float(got) - norm) <= U * (1 + 2.0 ** -10) * norm
    close(torch.cat(outs), torch.cat(want), 2 * U * torch.cat(want).abs(), out_dtype, "neighbours")
    written = torch.zeros(dst.numel(), dtype=torch.bool, device=DEV)
    for o in outs:
        first = (o.data_ptr() - dst.data_ptr()) // dst.element_size()
        written[first:first + o.numel()] = True
    assert bool((dst[~written] == 7).all())
    apart = [x.clone() for x in parts]
    assert same_bits(ld.ld_clip_grad_norm(apart, 5.0), got)  # the order of the sum is that of the sizes, wherever the tensors lie


def test_norms_that_32_bits_do_not_hold():
    big = torch.full((100,), 3e38, device=DEV)
    assert math.isinf(float(ld.ld_clip_grad_norm([big], 1e10)))     # 3e39: finite, but not in 32 bits; clipped all the same
    assert abs(float(big[0]) - 1e9) < 1e9 * 4 * U and bool((big == big[0]).all())
    tiny = torch.full((100,), 1e-40, device=DEV)
    assert abs(float(ld.ld_clip_grad_norm([tiny], 1.0)) - 1e-39) < 1e-42
    value = float(np.float32(1e-30))
    tiny = torch.full((100,), value, device=DEV)
    ld.ld_clip_grad_norm([tiny], 1e-30)
    assert abs(float(tiny[0]) - 1e-31) < 1e-31 * 4 * U


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_a_norm_that_is_not_finite_scales_nothing(bad):
    x = torch.randn(10001, device=DEV)
    x[777] = bad
    before = x.clone()
    out = torch.zeros(10001, device=DEV)
    norm = ld.ld_clip_grad_norm([x], 0.5, [out])
    assert not math.isfinite(float(norm))
    assert same_bits(out, before)
    ld.ld_clip_grad_norm([x], 0.5)
    assert same_bits(x, before)


def test_limits_of_zero_and_infinity():
    x = torch.randn(5000, device=DEV)
    before = x.clone()
    ld.ld_clip_grad_norm([x], math.inf)
    assert same_bits(x, before)
    ld.ld_clip_grad_norm([x], 0.0)
    assert not x.any()
    assert float(ld.ld_clip_grad_norm([x], 0.0)) == 0.0 and not x.any()


# ------------------------------------------------------------------------------------ streams and graphs

def test_on_another_stream_with_the_bindings_own_memory():
    g = gen(9)
    V, d, T = 500, 96, 3000
    table, dout = normal(g, (V, d)), normal(g, (T, d))
    ids = torch.randint(0, V, (T,), generator=g)
    t, x, i, side = table.to(DEV), dout.to(DEV), ids.to(DEV), torch.cuda.Stream()
    first = None
    torch.cuda.synchronize()
    for _ in range(20):
        out = ld.ld_embed_lookup(t, i, 2.0, stream=side)
        grad = torch.empty(V, d, device=DEV)
        side.wait_stream(torch.cuda.current_stream())
        ld.ld_embed_grad(x, i, grad, stream=side)
        norm = ld.ld_clip_grad_norm([grad], 1.0, stream=side)
        grad.record_stream(side)
        junk = [torch.full((1 << 18,), 7, dtype=torch.uint8, device=DEV) for _ in range(8)]  # what a block handed out too early would get
        side.synchronize()
        got = (out.clone(), grad.clone(), norm.clone())
        first = first or got
        assert all(same_bits(a, b) for a, b in zip(got, first))
        del junk
    want, _ = grad64(dout, ids, 1.0, V)
    assert abs(float(first[2]) - float(want.square().sum().sqrt())) < 1e-4 * float(first[2])


def test_what_the_binding_refuses_on_the_gpu():
    t, ids = torch.zeros(10, 8, device=DEV), torch.zeros(4, dtype=torch.int64, device=DEV)
    for bad in (lambda: ld.ld_embed_lookup(t.double(), ids), lambda: ld.ld_embed_lookup(t, ids.to(torch.int16)), lambda: ld.ld_embed_lookup(t, ids.cpu()),
                lambda: ld.ld_embed_lookup(t.view(2, 5, 8), ids), lambda: ld.ld_embed_lookup(t.t(), ids), lambda: ld.ld_embed_lookup(t, ids[::2]),
                lambda: ld.ld_embed_lookup(t, ids, out=torch.zeros(8, 4, device=DEV).t()),
                lambda: ld.ld_embed_lookup(t, ids, out=torch.zeros(4, 7, device=DEV)),
                lambda: ld.ld_embed_lookup(t, ids, out=torch.zeros(8, device=DEV).expand(4, 8)),
                lambda: ld.ld_embed_lookup(t, ids, out=torch.zeros(4, 8, device=DEV), out_dtype=BF16),
                lambda: ld.ld_embed_grad(t[:4], ids, torch.zeros(8, device=DEV).expand(10, 8)),
                lambda: ld.ld_embed_grad(t[:4], ids, torch.zeros(2, 5, 8, device=DEV)),
                lambda: ld.ld_embed_grad(torch.zeros(2, 4, 8, device=DEV)[:, :2], ids.view(2, 2), t),
                lambda: ld.ld_embed_grad(t[:4].double(), ids, t), lambda: ld.ld_embed_grad(t[:4], ids.int().short(), t),
                lambda: ld.ld_clip_grad_norm([t, t.to(BF16)], 1.0), lambda: ld.ld_clip_grad_norm([t.t()], 1.0),
                lambda: ld.ld_clip_grad_norm([t, t.cpu()], 1.0), lambda: ld.ld_clip_grad_norm([t], 1.0, [t.cpu()]),
                lambda: ld.ld_grad_norm([t], sumsq=torch.zeros(1, device=DEV)), lambda: ld.ld_grad_norm([t], sumsq=torch.zeros(0, device=DEV).double()),
                lambda: ld.ld_clip_grads([t], torch.zeros(0, device=DEV).double(), 1.0)):
        with pytest.raises((TypeError, ValueError)):
            bad()
    for bad in (lambda: ld.ld_clip_grad_norm([t], -1.0), lambda: ld.ld_clip_grad_norm([t], math.nan),
                lambda: ld.ld_embed_grad(t.new_zeros(2000, 8), ids.new_zeros(2000), t, workspace=torch.zeros(256, dtype=torch.uint8, device=DEV))):
        with pytest.raises(ld.LowDiffError):
            bad()
    assert not t.any()


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_infinities_and_nan_pass_through_rounding(dtype):
    """What is not finite stays so in every output type, and what 16 bits do not hold becomes infinite."""
    row = torch.tensor([[math.inf, -math.inf, math.nan, 1e38, -1e38, 0.0, -0.0, 3.0, 65519.0, 65520.0]])
    out = ld.ld_embed_lookup(row.to(DEV), torch.zeros(3, dtype=torch.int64, device=DEV), out_dtype=dtype)
    grad = torch.zeros(2, 10, dtype=dtype, device=DEV)
    ld.ld_embed_grad(row.to(DEV), torch.ones(1, dtype=torch.int32, device=DEV), grad)
    clipped = torch.zeros(1, 10, dtype=dtype, device=DEV)
    ld.ld_clip_grad_norm([row.to(DEV)], 1.0, [clipped])
    want = row.to(dtype)
    for got in (out[2:], grad[1:], clipped):
        assert torch.equal(got.cpu().isnan(), want.isnan()) and torch.equal(got.cpu().nan_to_num(nan=0.0), want.nan_to_num(nan=0.0))


def test_recorded_in_a_graph():
    g = gen(10)
    V, d, T = 700, 130, 9000
    table, ids = normal(g, (V, d)).to(DEV), torch.randint(-1, V, (T,), generator=g).to(DEV)
    dout, out, grad = normal(g, (T, d)).to(DEV), torch.zeros(T, d, device=DEV), torch.zeros(V, d, device=DEV)
    norm, parts = torch.zeros(1, device=DEV), [torch.zeros(n, device=DEV) for n in (V * d, 1)]
    ws = torch.empty(ld.ld_embed_grad_workspace(T, V, d), dtype=torch.uint8, device=DEV)
    ws2 = torch.empty(int(ld.load().ld_grad_norm_workspace(2)), dtype=torch.uint8, device=DEV)
    other = torch.ones(1, device=DEV)

    def step():
        ld.ld_embed_lookup(table, ids, 2.0, out=out)
        ld.ld_embed_grad(dout, ids, grad, 0.5, workspace=ws)
        ld.ld_clip_grad_norm([grad.view(-1), other], 3.0, parts, norm, ws2)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for r in range(4):
        dout.normal_()
        ids.copy_(torch.randint(-1, V, (T,), generator=g))
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (out, grad, norm, *parts)]
        for x in (out, grad, norm, *parts):
            x.fill_(-1)
        step()
        torch.cuda.synchronize()
        assert all(same_bits(a, b) for a, b in zip(got, (out, grad, norm, *parts))), r


def test_the_example_learns_and_recovers():
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "tied_embedding.py")
    spec = importlib.util.spec_from_file_location("tied_embedding", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, norms, recovered = example.train(steps=40)
    assert recovered and losses[0] > 5.0 and losses[-1] < 0.5 * losses[0]
    again = example.train(steps=3)
    assert again[1] == norms[:3]  # the same inputs, the same gradients
