"""Orthogonalisation and its replay: what they refuse and what they decide on the host, without a GPU."""
import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

from paper_2509_04084_amd import lowdiff as ld

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2509_04084_amd", "csrc")
FAKE = 0x10000  # never dereferenced: every call below fails its checks or has nothing to do
V = ctypes.c_void_p
F = ctypes.c_float
NULL, RANGE, WORKSPACE, ALIGN = -1, -2, -3, -5

SHIM = """
#include "ld_muon_shape.h"
extern "C" {
double largest(double a, double b, double c, double top, int32_t odd) { return ld_muon_largest(a, b, c, top, odd); }
// begin: first steps of the runs, then their end
int32_t bounds(int32_t steps, const float* coeff, int32_t kind, double* x, double* p, double* r, double* q, int32_t* begin, int32_t* runs) {
    LdMuonBounds m = {};
    if (!ld_muon_bounds(m, steps, coeff)) return 0;
    *runs = ld_muon_runs(m, steps, kind, begin);
    x[0] = m.x[0];
    for (int32_t run = 0, s = 0; s < steps; ++s) {
        if (s == begin[run + 1]) ++run;
        x[s + 1] = m.x[s + 1], p[s] = m.p[s], r[s] = m.r[s], q[s] = ld_muon_grown(m, begin[run], s);
    }
    return 1;
}
int32_t kind(int64_t m, int64_t n) { return ld_muon_kind(m, n); }
float scale(double bound) { return ld_muon_scale(bound); }
int64_t scratch(int32_t m, int32_t n) { return ld_muon_scratch(m, n); }
void tiles(int32_t down, int32_t across, int32_t band, int32_t* r, int32_t* c) {
    for (int32_t t = 0; t < down * across; ++t) ld_muon_tile(t, down, across, band, r[t], c[t]);
}
void lower_tiles(int32_t side, int32_t band, int32_t* r, int32_t* c) {
    for (int32_t t = 0; t < side * (side + 1) / 2; ++t) ld_muon_lower_tile(t, side, band, r[t], c[t]);
}
}
"""


@pytest.fixture(scope="module")
def shim(tmp_path_factory):
    d = tmp_path_factory.mktemp("muon")
    src, lib = str(d / "shim.cpp"), str(d / "shim.so")
    with open(src, "w") as f:
        f.write(SHIM)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-fPIC", "-shared", "-fsanitize=undefined", "-fno-sanitize-recover", "-I", CSRC,
                    src, "-o", lib], check=True)
    lib = ctypes.CDLL(lib)
    lib.largest.restype = ctypes.c_double
    lib.largest.argtypes = [ctypes.c_double] * 4 + [ctypes.c_int32]
    lib.scale.restype = ctypes.c_float
    lib.scale.argtypes = [ctypes.c_double]
    lib.scratch.restype = ctypes.c_int64
    return lib


def _p(a):
    return V(a.ctypes.data)


def bounds(shim, steps, coeff, kind):
    x, p, r, q = (np.zeros(17) for _ in range(4))
    begin, runs = np.zeros(18, np.int32), np.zeros(1, np.int32)
    ok = shim.bounds(steps, _p(coeff), int(kind), _p(x), _p(p), _p(r), _p(q), _p(begin), _p(runs))
    return (x, p, r, q, begin[:runs[0] + 1].tolist()) if ok else None


def usual(steps):
    return np.ascontiguousarray(np.tile(np.float32([3.4445, -4.7750, 2.0315]), (steps, 1)))


def test_runs_of_the_usual_steps(shim):
    for kind, want in ((2, {1: [0], 2: [0], 3: [0], 4: [0, 1], 5: [0, 2], 6: [0, 3], 7: [0, 1, 4], 16: [0, 1, 4, 7, 10, 13]}),
                       (1, {1: [0], 2: [0], 3: [0, 2], 4: [0, 2], 5: [0, 2, 4], 16: list(range(0, 16, 2))}),
                       (0, {1: [0], 5: [0, 1, 2, 3, 4], 16: list(range(16))})):
        for steps, begin in want.items():
            assert bounds(shim, steps, usual(steps), kind)[4] == begin + [steps], (kind, steps)
    i64 = ctypes.c_int64
    assert [shim.kind(i64(m), i64(n)) for m, n in ((1, 1), (100, 124), (100, 125), (100, 249), (100, 250), (65536, 65536), (1, 65536), (2048, 5120), (2049, 65536))] == [0, 0, 1, 1, 2, 0, 2, 2, 1]


def test_bounds_hold_for_every_singular_value(shim):
    rs = np.random.RandomState(0)
    sigma = np.linspace(0, 1, 200001)
    tried = 0
    for case in range(80):
        steps, kind = int(rs.randint(1, 17)), int(rs.randint(3))
        coeff = usual(steps) if case == 0 else (np.float32([2.0, -1.5, 0.5]) + rs.uniform(-0.3, 0.3, (steps, 3))).astype(np.float32)
        coeff[0] *= np.float32(rs.choice([1.0, 4.0]))
        got = bounds(shim, steps, coeff, kind)
        if got is None:
            continue
        tried += 1
        x, p, r, q, begin = got
        assert begin[0] == 0 and begin[-1] == steps and all(0 < b - a <= kind + 1 for a, b in zip(begin, begin[1:]))
        s, amount = sigma.copy(), np.ones_like(sigma)
        for t in range(steps):
            if t in begin:
                amount = np.ones_like(sigma)
            a, b, c = coeff[t].astype(np.float64)
            f = a + b * s * s + c * s ** 4
            assert np.abs(s).max() <= x[t] and np.abs(f).max() <= p[t] and np.abs(f * s * s).max() <= r[t]
            s, amount = s * f, amount * f
            assert np.abs(amount).max() <= q[t] and np.abs(s).max() <= x[t + 1] and (t in begin or q[t] <= 1.02 ** 3 * 48)
    assert tried > 20


def test_largest_value_on_an_interval(shim):
    rs = np.random.RandomState(1)
    for _ in range(300):
        a, b, c, top = rs.uniform(-5, 5, 3).tolist() + [rs.uniform(0.1, 2)]
        if rs.rand() < 0.2:
            c = 0.0
        for odd in (0, 1, 2):
            x = np.linspace(0, top, 100001)
            f = np.abs(x ** odd * (a + b * x ** 2 + c * x ** 4)).max()
            got = shim.largest(a, b, c, top, odd)
            assert f <= got * (1 + 1e-12) + 1e-12 and got <= f * (1 + 1e-6) + 1e-6, (a, b, c, top, odd)


def test_scales_keep_halves_in_range(shim):
    for bound in (1e-9, 0.3, 0.999, 1.0, 1.5, 2.0, 100.0, 4096.0):
        s = shim.scale(bound)
        assert np.log2(s) == int(np.log2(s)) and s * bound <= 2.0 ** 15 and (s * bound > 2.0 ** 13 or s == 2.0 ** 15)


def refused(**kw):
    lib = ld.load()
    rows, cols = np.array([64, 100], np.int64), np.array([128, 50], np.int64)
    two = (V * 2)(FAKE, FAKE)
    a = dict(src=two, ss=None, dst=two, ds=None, rows=rows, cols=cols, n=2, dtype=0, ot=0, steps=5, coeff=None, eps=1e-7, ws=FAKE,
             wsb=lib.ld_orthogonalize_workspace(_p(rows), _p(cols), 2))
    a.update(kw)
    at = lambda x: None if x is None else _p(x)  # noqa: E731
    return lib.ld_orthogonalize(a["src"], at(a["ss"]), a["dst"], at(a["ds"]), at(a["rows"]), at(a["cols"]), a["n"], a["dtype"], a["ot"], a["steps"],
                                at(a["coeff"]), F(a["eps"]), V(a["ws"]), a["wsb"], None)


def i64(*x):
    return np.array(x, np.int64)


def test_orthogonalize_refusals():
    lib = ld.load()
    wsb = ld.ld_orthogonalize_workspace([(64, 128), (100, 50)])
    assert wsb > 0 and lib.ld_orthogonalize_workspace(None, None, 0) == 0
    assert ld.ld_orthogonalize_workspace([(-1, 4)]) == 0 and ld.ld_orthogonalize_workspace([(4, 65537)]) == 0
    for bad in (dict(src=None), dict(dst=None), dict(rows=None), dict(cols=None), dict(src=(V * 2)(FAKE, 0)), dict(dst=(V * 2)(0, FAKE))):
        assert refused(**bad) == NULL, bad
    for bad in (dict(n=-1), dict(n=(1 << 20) + 1), dict(dtype=3), dict(ot=-1), dict(steps=0), dict(steps=17), dict(eps=-1.0), dict(eps=float("nan")),
                dict(rows=i64(64, -1)), dict(cols=i64(65537, 50)), dict(ss=i64(-1, 50)), dict(ds=i64(127, 50)),
                dict(coeff=np.float32([[3, 0, 0]] * 5)), dict(coeff=np.float32([[np.nan, 0, 0]] * 5)), dict(coeff=np.float32([[np.inf, 0, 0]] * 5)),
                dict(steps=3, coeff=np.float32([[1, 0, 0], [1, 0, 0], [65, 0, 0]]))):
        assert refused(**bad) == RANGE, bad
    for bad in (dict(src=(V * 2)(FAKE + 2, FAKE)), dict(dst=(V * 2)(FAKE, FAKE + 1)), dict(dtype=1, src=(V * 2)(FAKE + 1, FAKE))):
        assert refused(**bad) == ALIGN, bad
    least = max(ld.ld_orthogonalize_workspace([s]) for s in ((64, 128), (100, 50)))
    assert least < wsb and refused(ws=0) == WORKSPACE and refused(ws=FAKE + 128) == WORKSPACE and refused(wsb=least - 1) == WORKSPACE
    assert refused(n=0, src=None, dst=None, rows=None, cols=None) == 0
    assert refused(rows=i64(0, 10), cols=i64(10, 0), src=(V * 2)(0, 0), dst=(V * 2)(0, 0), ws=0, wsb=0) == 0


def test_muon_refusals():
    lib = ld.load()
    rows, cols = i64(64, 100), i64(128, 50)
    two, six = (V * 2)(FAKE, FAKE), (V * 6)(*[FAKE] * 6)
    wsb = lib.ld_merge_dense_muon_workspace(_p(rows), _p(cols), 2, 3)
    assert wsb > lib.ld_merge_dense_muon_workspace(_p(rows), _p(cols), 2, 1) > 0
    assert lib.ld_merge_dense_muon_workspace(_p(rows), _p(cols), 2, 4097) == 0 and lib.ld_merge_dense_muon_workspace(_p(rows), _p(cols), -1, 1) == 0

    def call(w=two, m=two, g=six, rows=rows, cols=cols, n=2, W=3, dtype=1, lr=0.02, mu=0.95, decay=0.0, scale=None, steps=5, coeff=None, eps=1e-7,
             ws=FAKE, wsb=wsb):
        at = lambda x: None if x is None else _p(x)  # noqa: E731
        return lib.ld_merge_dense_muon(w, m, g, at(rows), at(cols), n, W, dtype, F(lr), F(mu), 1, F(decay), at(scale), steps, at(coeff), F(eps),
                                       V(ws), wsb, None)

    for bad in (dict(w=None), dict(m=None), dict(g=None), dict(rows=None), dict(cols=None), dict(w=(V * 2)(0, FAKE)), dict(m=(V * 2)(FAKE, 0)),
                dict(g=(V * 6)(FAKE, FAKE, FAKE, FAKE, 0, FAKE))):
        assert call(**bad) == NULL, bad
    for bad in (dict(n=-1), dict(W=-1), dict(W=4097), dict(dtype=5), dict(lr=float("nan")), dict(mu=float("inf")), dict(decay=float("nan")),
                dict(scale=np.float32([1, np.nan])), dict(steps=0), dict(steps=17), dict(eps=-1.0), dict(coeff=np.float32([[3, 0, 0]] * 5)),
                dict(rows=i64(64, -1))):
        assert call(**bad) == RANGE, bad
    for bad in (dict(w=(V * 2)(FAKE + 2, FAKE)), dict(m=(V * 2)(FAKE, FAKE + 1)), dict(g=(V * 6)(FAKE, FAKE, FAKE, FAKE + 1, FAKE, FAKE))):
        assert call(**bad) == ALIGN, bad
    least = max(ld.ld_merge_dense_muon_workspace([s]) for s in ((64, 128), (100, 50)))
    assert call(ws=0) == WORKSPACE and call(ws=FAKE + 16) == WORKSPACE and call(wsb=least - 1) == WORKSPACE
    assert call(W=0, g=None) == 0 and call(n=0) == 0


def test_workspace_is_that_of_the_largest_group(shim):
    """Groups hold up to 64 problems and 8 GiB of scratch, or one problem; counted here one problem at a time."""
    rs = np.random.RandomState(3)
    pad = lambda x: (x + 255) // 256 * 256  # noqa: E731
    for case in range(60):
        n, W = int(rs.randint(1, 9)), int(rs.choice([1, 2, 3, 63, 64, 65, 200, 4096]))
        top = int(rs.choice([40, 700, 5000, 20000]))
        shapes = [(int(rs.randint(0, top)), int(rs.randint(1, top))) for _ in range(n)]
        used = count = most = 0
        for r, c in shapes:
            if r == 0:
                continue
            need = pad(shim.scratch(min(r, c), max(r, c)))
            for _ in range(W):
                if count == 64 or (count and used + need > 2 ** 33):
                    used = count = 0
                used, count = used + need, count + 1
                most = max(most, used)
        want = 0 if most == 0 else most + 64 * 256 * 8
        assert ld.ld_merge_dense_muon_workspace(shapes, W) == want, (shapes, W)
        if W == 1:
            assert ld.ld_orthogonalize_workspace(shapes) == want


def test_binding_refuses_before_any_launch():
    a, b = torch.zeros(4, 6), torch.zeros(5, 3)
    with pytest.raises(TypeError):
        ld.ld_orthogonalize([a, b])  # not on a GPU
    with pytest.raises(TypeError, match="2-D"):
        ld.ld_orthogonalize([a, torch.zeros(4)])
    with pytest.raises(TypeError, match="one type"):
        ld.ld_orthogonalize([a, b.half()])
    with pytest.raises(ValueError, match="differ in length"):
        ld.ld_orthogonalize([a, b], [a])
    with pytest.raises(ValueError, match="three numbers"):
        ld.ld_orthogonalize([a, b], coeffs=[1.0, 2.0])
    with pytest.raises(ValueError, match="different devices"):
        ld.ld_orthogonalize([a, b.to("meta")])
    assert ld.ld_orthogonalize([]) == []
    with pytest.raises(ValueError, match="differ in length"):
        ld.ld_merge_dense_muon([a], [a, b], [[a]], 0.1)
    with pytest.raises(ValueError, match="differ in length"):
        ld.ld_merge_dense_muon([a], [a], [[a], [a, b]], 0.1)
    with pytest.raises(ValueError, match="differ in shape"):
        ld.ld_merge_dense_muon([a], [a], [[b]], 0.1)
    with pytest.raises(TypeError):
        ld.ld_merge_dense_muon([a], [a.clone()], [[a.clone()]], 0.1)
    ld.ld_merge_dense_muon([], [], [], 0.1)


def test_every_tile_is_one_workgroups(shim):
    rs = np.random.RandomState(5)
    for down, across, band in [(1, 1, 8), (1, 9, 8), (9, 1, 8), (8, 8, 8), (12, 12, 8), (1024, 1024, 8)] + [tuple(rs.randint(1, (70, 70, 12))) for _ in range(60)]:
        r, c = np.empty((2, down * across), np.int32)
        shim.tiles(int(down), int(across), int(band), _p(r), _p(c))
        assert r.min() >= 0 and r.max() < down and c.min() >= 0 and c.max() < across
        assert np.unique(r.astype(np.int64) * across + c).size == down * across, (down, across, band)
        n = down * (down + 1) // 2
        r, c = np.empty((2, n), np.int32)
        shim.lower_tiles(int(down), int(band), _p(r), _p(c))
        assert c.min() >= 0 and r.max() < down and (c <= r).all()
        assert np.unique(r.astype(np.int64) * down + c).size == n, (down, band)
        if down >= 32 and band == 8:  # 64 in a row, of eight rows and eight columns
            t = 24 * 25 // 2
            assert np.unique(r[t:t + 64]).size == 8 and np.unique(c[t:t + 64]).size == 8
