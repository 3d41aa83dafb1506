"""Token log probabilities, entropies, alternatives and their gradient on the GPU, against the definitions in 64 bits on the CPU.

Bounds, with u the unit roundoff of 32 bits (2^-24), x_j = scale (logit_j - M) <= 0, A = sum p_j |x_j|. The kernel's exponential of x_j
has an argument with at most 4 roundings relative to it (scale log2 e, its own, the reference's move) and is itself off by 1 unit (2 u);
moving the reference multiplies by another such exponential, and as it lies up to four powers of two below a value, both may have
exponents that are larger by 4 ln 2, 7 roundings of that in all: 20 u. Every term of Z is so within u (28 + 8 |x_j|), Z within
  eZ = u (28 + 8 A + adds), adds = additions a term passes through: at most 256 in a thread, 24 in the joins (V where that is less),
and from there
  L         eL = eZ + 2 u |L|
  logprob   2 u |x_id| + eL + u |logprob|
  entropy   eL + A (2 eZ + 6 u) + u 8 S2 + u (|L| + |entropy|),  S2 = sum p_j x_j^2 (the terms' errors weighted by x_j once more)
  gradient  with eP = eL + 2 u |x_j| + 3 u |log p_j| + 3 u the relative error of p_j:
            scale (|g| p_j eP + |h| p_j (eP |log p_j + H| + eP + eH + 2 u (|log p_j| + |H|))) + 4 u (sum of the terms' magnitudes)
            and the rounding to its type, u_o |d|
each with 1 % for second-order terms; exponentials under 2^-126 are zero, and results that are subnormal in their type lose half a step.
"""
import math

import pytest
import torch

from paper_2509_04084_amd import lowdiff as ld

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
U = 2.0 ** -24
UNIT = {F32: U, BF16: 2.0 ** -8, F16: 2.0 ** -11}
STEP = {F32: 2.0 ** -149, BF16: 2.0 ** -133, F16: 2.0 ** -24}
TINY = 2.0 ** -126


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def same_bits(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


def close(got, want, bound, tag):
    got = got.detach().double().cpu()
    assert got.shape == want.shape, (tag, got.shape, want.shape)
    same = (got == want) | (got.isnan() & want.isnan())
    bad = ~(same | ((got - want).abs() <= 1.01 * bound + 1e-37))
    assert not bad.any(), (tag, int(bad.sum()), got[bad][:4].tolist(), want[bad][:4].tolist(), bound[bad][:4].tolist())


class Exact:
    """The definition in 64 bits, and the bounds above."""

    def __init__(self, logits, ids, scale):
        scale = float(torch.tensor(scale, dtype=F32))
        l, V = logits.double(), logits.shape[1]
        self.M = l.max(dim=1).values
        self.empty = self.M == -math.inf
        self.x = torch.where(self.empty[:, None], -math.inf, (l - self.M[:, None]) * scale)
        self.x = torch.where(self.x < -float(torch.finfo(F32).max), -math.inf, self.x)  # beyond 32 bits
        e = self.x.exp()
        z = e.sum(dim=1)
        self.L = torch.where(self.empty, 0.0, z.log())
        self.logp = self.x - self.L[:, None]
        self.p = self.logp.exp()
        fin = torch.where(self.p > 0, self.x, 0.0)
        A, S2 = (self.p * fin.abs()).sum(1), (self.p * fin * fin).sum(1)
        self.H = torch.where(self.empty, 0.0, self.L + A)
        self.inside = (ids >= 0) & (ids < V)
        x_id = self.x.gather(1, torch.where(self.inside, ids, 0).long()[:, None])[:, 0]
        self.logprob = torch.where(self.inside, torch.where(self.empty, -math.inf, x_id - self.L), 0.0)
        eZ = U * (28 + 8 * A + min(V, 280))
        self.eL = eZ + 2 * U * self.L.abs()
        lim = x_id.clamp_min(-1e30)
        self.e_logprob = 2 * U * lim.abs() + self.eL + U * (lim - self.L).abs()
        self.eH = self.eL + A * (2 * eZ + 6 * U) + 8 * U * S2 + U * (self.L.abs() + self.H.abs())
        self.scale = scale

    def top(self, logits, k):
        """By value, the lower index first, NaN the largest."""
        key = logits.float().double()
        key = torch.where(key.isnan(), math.inf, key)
        nan_first = torch.sort((~logits.isnan()).int(), dim=1, stable=True).indices
        order = nan_first.gather(1, torch.sort(torch.where(logits.isnan(), math.inf, key).gather(1, nan_first), dim=1, descending=True,
                                               stable=True).indices)
        return order[:, :k]

    def grad(self, ids, g, h):
        T, V = self.x.shape
        g = torch.where(self.inside, g.double(), 0.0)[:, None]
        delta = torch.zeros(T, V, dtype=torch.float64)
        delta[torch.arange(T), torch.where(self.inside, ids, 0).long()] = 1.0
        h = (torch.zeros(T) if h is None else h).double()[:, None]
        logp = torch.where(self.p > 0, self.logp, 0.0)
        c = torch.where(self.p > 0, logp + self.H[:, None], 0.0)
        d = self.scale * (g * (delta - self.p) - h * self.p * c)
        d = torch.where(self.empty[:, None], 0.0, d)
        eP = self.eL[:, None] + 2 * U * self.x.clamp_min(-1e4).abs() + 3 * U * logp.abs() + 3 * U
        spread = g.abs() * self.p * eP + h.abs() * self.p * (eP * c.abs() + eP + self.eH[:, None] + 2 * U * (logp.abs() + self.H[:, None].abs()))
        spread += 4 * U * (g.abs() * (delta + self.p) + (h * self.p * c).abs()) + TINY * (g.abs() + h.abs() * 200)
        return d, torch.where(self.empty[:, None], 0.0, self.scale * spread)


def make(T, V, dtype, g, masked=0.0, spread=3.0):
    x = torch.randn(T, V, generator=g, dtype=torch.float64) * spread
    x[torch.rand(T, V, generator=g) < masked] = -math.inf
    return x.to(dtype)


def make_ids(T, V, g):
    ids = torch.randint(0, V, (T,), generator=g)
    ids[torch.rand(T, generator=g) < 0.2] = -1
    ids[torch.rand(T, generator=g) < 0.05] = V
    return ids


def check(x, ids, scale, top, id_dtype=torch.int64, dev=None, tag=""):
    """Both calls against the definition; returns what the first one gave."""
    x_dev = x.to(DEV) if dev is None else dev
    want, V = Exact(x, ids, scale), x.shape[1]
    got = ld.ld_token_logprob(x_dev, ids.to(DEV, id_dtype), scale, entropy=True, top=top)
    close(got.stats[:, 0], want.M, torch.zeros_like(want.M), (tag, "M"))
    close(got.stats[:, 1], want.L, want.eL, (tag, "L"))
    close(got.logprob, want.logprob, want.e_logprob, (tag, "logprob"))
    close(got.entropy, want.H, want.eH, (tag, "entropy"))
    if top:
        order = want.top(x, top)
        assert torch.equal(got.top_ids.cpu().long(), order), (tag, "top_ids")
        xt = want.x.gather(1, order)
        lp = torch.where(want.empty[:, None], -math.inf, xt - want.L[:, None])
        lim = xt.clamp_min(-1e30)
        close(got.top_logprob, lp, 2 * U * lim.abs() + want.eL[:, None] + U * (lim - want.L[:, None]).abs(), (tag, "top_logprob"))
    bare = ld.ld_token_logprob(x_dev, scale=scale)  # nothing else asked for
    assert bare.logprob is None and bare.entropy is None and bare.top_ids is None and same_bits(bare.stats, got.stats)
    gn = gen(T := x.shape[0])
    g, h = torch.randn(T, generator=gn), torch.randn(T, generator=gn)
    for out_dtype in (F32, BF16, F16):
        for with_entropy in (False, True):
            d, spread = want.grad(ids, g, h if with_entropy else None)
            out = ld.ld_token_logprob_grad(x_dev, got.stats, ids.to(DEV, id_dtype), g.to(DEV), got.entropy if with_entropy else None,
                                           h.to(DEV) if with_entropy else None, scale, out_dtype=out_dtype)
            assert out.dtype == out_dtype
            close(out, d, spread + UNIT[out_dtype] * d.abs() + 0.5 * STEP[out_dtype], (tag, "grad", out_dtype, with_entropy))
    return got


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("T,V,top", [(1, 1, 1), (1, 7, 7), (3, 8, 2), (2, 64, 64), (5, 499, 20), (70, 2047, 5), (3, 2048, 64), (3, 2049, 64), (9, 4096, 50),
                                     (2, 4097, 1), (1, 50257, 20), (8, 32003, 64), (300, 8191, 3), (1, 65537, 10), (2, 160001, 33), (64, 50257, 11),
                                     (127, 8191, 64), (128, 9001, 5), (511, 4000, 4), (512, 4000, 4)])
def test_scores_and_gradients(T, V, top, dtype):
    print(f"[score] T={T} V={V} top={top} {dtype}", flush=True)
    g = gen(T * 31 + V)
    for scale, masked, id_dtype in ((1.0, 0.0, torch.int64), (0.7, 0.3, torch.int32)):
        x = make(T, V, dtype, g, masked)
        if masked:
            x[:, V // 2] = 1.0  # something is left in every row
        check(x, make_ids(T, V, g), scale, top, id_dtype, tag=(T, V, scale))


@pytest.mark.parametrize("T,V,top", [(1500, 513, 8), (1030, 4096, 64), (1100, 5003, 17), (1024, 40, 40)])
def test_many_rows(T, V, top):
    """Rows that are not split: a wave's, and a workgroup's."""
    print(f"[score] T={T} V={V}", flush=True)
    g = gen(V)
    check(make(T, V, BF16, g), make_ids(T, V, g), 1.3, top)


HARD = ["equal", "ascending", "descending", "two", "zeros", "one thread", "peaked", "lowest", "huge", "far mask"]


def hard_rows(kind, T, V, g):
    j = torch.arange(V, dtype=torch.float64)
    row = {"equal": torch.full((V,), -3.25, dtype=torch.float64), "ascending": j * 2.0 ** -6, "descending": -j * 2.0 ** -6,
           "two": (j % 2) * 4.0, "zeros": torch.where(j % 3 == 0, -0.0, 0.0), "one thread": (j % 2048 < 8) * 5.0 + torch.rand(V, generator=g),
           "peaked": torch.where(j == V * 4444 // 6001, 90.0, -j * 1e-3), "lowest": torch.full((V,), torch.finfo(F32).min, dtype=torch.float64),
           "huge": torch.where(j > V - 11, 3.0e38, -3.0e38), "far mask": torch.where(j % 5 == 1, torch.randn(V, generator=g).double(), -1e9)}[kind]
    x = row.to(F32).repeat(T, 1)
    x[T // 2] = x[T // 2].roll(1234)
    return x


@pytest.mark.parametrize("T", [3, 1100])
@pytest.mark.parametrize("kind", HARD)
def test_rows_that_sorting_and_exponentials_find_hard(kind, T):
    print(f"[score] {kind} T={T}", flush=True)
    g, V = gen(7), 6001
    x = hard_rows(kind, T, V, g)
    check(x, make_ids(T, V, g), 1.0, 64, tag=kind)


@pytest.mark.parametrize("T,V,top", [(3, 6001, 1), (3, 70001, 8), (600, 6001, 5), (600, 4001, 8), (600, 4001, 9), (600, 1001, 3), (200, 20011, 33)])
@pytest.mark.parametrize("kind", HARD)
def test_few_alternatives_of_hard_rows(kind, T, V, top):
    print(f"[score] {kind} T={T} V={V} top={top}", flush=True)
    g = gen(T + V)
    check(hard_rows(kind, T, V, g), make_ids(T, V, g), 1.0, top, tag=kind)


@pytest.mark.parametrize("T,V", [(4, 300), (1200, 300), (4, 9001), (1100, 9001)])
def test_rows_in_which_nothing_is_left(T, V):
    g = gen(11)
    x = make(T, V, F16, g)
    x[::2] = -math.inf
    ids = torch.randint(0, V, (T,), generator=g)
    ids[T // 2] = -1
    got = check(x, ids, 2.0, 5)
    assert torch.equal(got.top_ids[0].cpu(), torch.arange(5, dtype=torch.int32))


@pytest.mark.parametrize("T,V", [(4, 300), (1200, 300), (4, 9001), (1100, 9001)])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.nan])
def test_infinities_and_nan_stay_in_their_rows(T, V, bad):
    g = gen(13)
    clean = make(T, V, F32, g)
    x = clean.clone()
    at = torch.tensor([V - 1, 17, V // 2, 250])
    x[1, at] = bad
    ids = torch.randint(0, V, (T,), generator=g)
    got, ref = (ld.ld_token_logprob(y.to(DEV), ids.to(DEV), 1.0, entropy=True, top=6) for y in (x, clean))
    assert bool(got.logprob[1].isnan()) and bool(got.entropy[1].isnan()) and bool(got.stats[1, 1].isnan()) and bool(got.top_logprob[1].isnan().all())
    assert got.top_ids[1, :4].cpu().tolist() == sorted(at.tolist())
    rest = clean[1].clone()
    rest[at] = -math.inf
    assert torch.equal(got.top_ids[1, 4:].cpu().long(), torch.sort(rest, descending=True, stable=True).indices[:2])
    keep = [i for i in range(T) if i != 1]
    for a, b in zip(got, ref):
        assert same_bits(a[keep], b[keep])
    d = ld.ld_token_logprob_grad(x.to(DEV), got.stats, ids.to(DEV), torch.ones(T, device=DEV), got.entropy, torch.ones(T, device=DEV))
    assert bool(d[1].isnan().all()) and not bool(d[keep].isnan().any())


def test_shapes_strides_and_what_lies_around():
    g = gen(17)
    wide = make(60, 1300, BF16, g)
    x = wide[:, 3:1204]                                       # rows 1300 apart, beginning at an odd element
    ids = make_ids(60, 1201, g)
    check(x, ids, 1.0, 9, dev=wide.to(DEV)[:, 3:1204], tag="strided")
    shaped = ld.ld_token_logprob(x.contiguous().to(DEV).view(4, 15, 1201), ids.to(DEV).view(4, 15), 1.0, entropy=True, top=2)
    flat = ld.ld_token_logprob(x.contiguous().to(DEV), ids.to(DEV), 1.0, entropy=True, top=2)
    assert shaped.logprob.shape == (4, 15) and shaped.stats.shape == (4, 15, 2) and shaped.top_ids.shape == (4, 15, 2)
    for a, b in zip(shaped, flat):
        assert same_bits(a, b.view(a.shape))
    one = wide.to(DEV)[0, :1201].expand(500, 1201)            # one row for all
    got = ld.ld_token_logprob(one)
    assert same_bits(got.stats, got.stats[:1].expand(500, 2))
    alone = ld.ld_token_logprob(wide.to(DEV)[0, :1201], torch.tensor(5, device=DEV), entropy=True)
    assert alone.logprob.shape == () and alone.stats.shape == (2,)
    # into rows of something wider: the rest of it stays; and in place
    room = torch.full((60, 1300), 7.0, dtype=BF16, device=DEV)
    gd, dev = torch.randn(60, generator=g).to(DEV), wide.to(DEV)
    ref = ld.ld_token_logprob_grad(dev[:, 3:1204], flat.stats, ids.to(DEV), gd)
    ld.ld_token_logprob_grad(dev[:, 3:1204], flat.stats, ids.to(DEV), gd, out=room[:, 3:1204])
    assert same_bits(room[:, 3:1204], ref) and bool((room[:, :3] == 7).all()) and bool((room[:, 1204:] == 7).all())
    place = dev.clone()
    ld.ld_token_logprob_grad(place[:, 3:1204], flat.stats, ids.to(DEV), gd, out=place[:, 3:1204])
    assert same_bits(place[:, 3:1204], ref) and same_bits(place[:, :3], dev[:, :3]) and same_bits(place[:, 1204:], dev[:, 1204:])


def test_gradients_that_are_one_value_or_strided():
    g, T, V = gen(19), 33, 777
    x, ids = make(T, V, F32, g).to(DEV), torch.randint(0, V, (T,), generator=g).to(DEV)
    got = ld.ld_token_logprob(x, ids, entropy=True)
    one = torch.tensor(-1.0 / T, device=DEV)
    a = ld.ld_token_logprob_grad(x, got.stats, ids, one.expand(T), got.entropy, one.expand(T))
    b = ld.ld_token_logprob_grad(x, got.stats, ids, one.repeat(T), got.entropy, one.repeat(T))
    c = ld.ld_token_logprob_grad(x, got.stats, ids, one.repeat(3 * T)[::3], got.entropy, one.repeat(2 * T)[::2])
    assert same_bits(a, b) and same_bits(a, c)


def test_gradient_against_differences():
    """A central difference over +-e of a function whose third derivative is under 2 e^0 per unit (softmax of bounded logits) is off by
    e^2 / 3 and by the rounding of two 32-bit values around 10, 2 * 2^-21, over 2 e."""
    g, T, V, e = gen(23), 4, 50, 2.0 ** -7
    x, ids = make(T, V, F32, g, spread=1.0).to(DEV), torch.randint(0, V, (T,), generator=g).to(DEV)
    got = ld.ld_token_logprob(x, ids, entropy=True)
    a, b = torch.tensor([1.0, -2.0, 0.5, 3.0], device=DEV), torch.tensor([0.3, 1.0, -1.0, 2.0], device=DEV)
    d = ld.ld_token_logprob_grad(x, got.stats, ids, a, got.entropy, b)
    value = lambda y: (lambda r: (a.double() * r.logprob.double() + b.double() * r.entropy.double()))(ld.ld_token_logprob(y, ids, entropy=True))  # noqa: E731
    for j in range(V):
        up, down = x.clone(), x.clone()
        up[:, j] += e
        down[:, j] -= e
        slope = (value(up) - value(down)) / (2 * e)
        assert bool(((slope - d[:, j].double()).abs() <= (a.abs() + 4 * b.abs()) * (e * e + 2 ** -20 / e)).all()), j


def test_of_nothing():
    x = torch.zeros(0, 100, device=DEV)
    ids = torch.zeros(0, dtype=torch.int64, device=DEV)
    got = ld.ld_token_logprob(x, ids, entropy=True, top=3)
    assert got.logprob.shape == (0,) and got.top_ids.shape == (0, 3)
    assert ld.ld_token_logprob_grad(x, got.stats, ids, torch.zeros(0, device=DEV)).shape == (0, 100)
    with pytest.raises(ld.LowDiffError):
        ld.ld_token_logprob(torch.zeros(3, 0, device=DEV))


def test_ids_beyond_32_bits_name_nothing():
    x = torch.zeros(4, 10, device=DEV)
    far = torch.tensor([2 ** 32 + 1, -2 ** 32 + 1, 2 ** 62, 5], device=DEV)
    got = ld.ld_token_logprob(x, far)
    assert got.logprob[:3].tolist() == [0, 0, 0] and float(got.logprob[3]) != 0
    d = ld.ld_token_logprob_grad(x, got.stats, far, torch.ones(4, device=DEV))
    assert not d[:3].any() and float(d[3, 5]) > 0


def test_rows_beyond_2_31_elements():
    T, V = 9000, 250000  # 2.25 G bf16
    x = torch.zeros(T, V, dtype=BF16, device=DEV)
    x[T - 1, V - 1] = 3.0
    ids = torch.full((T,), V - 1, device=DEV)
    got = ld.ld_token_logprob(x, ids, top=2)
    lse = math.log(V)
    assert float((got.logprob[:-1].double() + lse).abs().max()) <= 1e-5
    assert abs(float(got.logprob[-1]) - (3.0 - math.log(V - 1 + math.exp(3.0)))) <= 1e-5
    assert got.top_ids[0].tolist() == [0, 1] and got.top_ids[-1].tolist() == [V - 1, 0]
    ld.ld_token_logprob_grad(x, got.stats, ids, torch.ones(T, device=DEV), out=x)
    assert abs(float(x[0, V - 1]) - 1.0) <= 2 ** -7 and abs(float(x[T - 1, 0].float()) + 1 / (V - 1 + math.exp(3.0))) <= 1e-7


@pytest.mark.parametrize("V,top", [(1 << 24, 64), (1 << 24, 1), ((1 << 24) - 77, 20), (3000001, 33)])
def test_the_largest_vocabularies(V, top):
    """Rows of up to 256 parts; lists that the join holds in shared memory, and more. Against 64 bits on the GPU: L within 28 + 8 A + 280
    roundings as above, A below 20 here."""
    g = torch.Generator(device=DEV).manual_seed(V + top)
    x = (torch.randn(2, V, generator=g, device=DEV) * 2).half()
    x[1, V - 1] = 11.0
    ids = torch.tensor([V - 1, 5], device=DEV)
    got = ld.ld_token_logprob(x, ids, entropy=True, top=top)
    wide = x.double()
    lse = torch.logsumexp(wide, dim=1)
    eL = U * (28 + 160 + 280 + 2 * 20)
    assert bool(((got.logprob.double() - (wide.gather(1, ids[:, None])[:, 0] - lse)).abs() <= eL + 64 * U).all())
    p = torch.softmax(wide, dim=1)
    H = -torch.special.xlogy(p, p).sum(dim=1)
    assert bool(((got.entropy.double() - H).abs() <= 60 * eL).all())
    order = torch.sort(x.float(), dim=1, descending=True, stable=True).indices[:, :top]
    assert torch.equal(got.top_ids.long(), order)


def test_another_stream_and_a_graph():
    g, T, V = gen(29), 40, 30011
    x, ids = make(T, V, BF16, g).to(DEV), torch.randint(0, V, (T,), generator=g).to(DEV)
    gd = torch.randn(T, generator=g).to(DEV)

    def both(stream=None):
        r = ld.ld_token_logprob(x, ids, entropy=True, top=8, stream=stream)
        return [*r, ld.ld_token_logprob_grad(x, r.stats, ids, gd, r.entropy, gd, stream=stream)]
    want = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = both(side)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(got, want):
        assert same_bits(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = both()
    for _ in range(3):
        x.copy_(make(T, V, BF16, g).to(DEV))
        want = both()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, want):
            assert same_bits(a, b)


def test_refusals_on_the_gpu():
    x, ids = torch.zeros(4, 10, device=DEV), torch.zeros(4, dtype=torch.int64, device=DEV)
    stats = torch.zeros(4, 2, device=DEV)
    with pytest.raises(ValueError):
        ld.ld_token_logprob(x, ids, top=11)
    with pytest.raises(ld.LowDiffError):
        ld.ld_token_logprob(torch.zeros(4, 100, device=DEV), top=65)
    with pytest.raises(ld.LowDiffError):
        ld.ld_token_logprob(x, ids, scale=0.0)
    with pytest.raises(TypeError):
        ld.ld_token_logprob(x.t(), torch.zeros(10, dtype=torch.int64, device=DEV))
    with pytest.raises(TypeError):
        ld.ld_token_logprob(x, ids.float())
    with pytest.raises(ValueError, match="rows overlap"):
        ld.ld_token_logprob_grad(x, stats, ids, torch.zeros(4, device=DEV), out=torch.zeros(10, device=DEV).expand(4, 10))
    with pytest.raises(ValueError):
        ld.ld_token_logprob_grad(x, stats, ids, torch.zeros(4, device=DEV), out=torch.zeros(4, 9, device=DEV))
    with pytest.raises(TypeError):
        ld.ld_token_logprob_grad(x, stats, ids, torch.zeros(4, device=DEV).double())
    with pytest.raises(TypeError):
        ld.ld_token_logprob_grad(x, stats.cpu().to(DEV).double(), ids, torch.zeros(4, device=DEV))
