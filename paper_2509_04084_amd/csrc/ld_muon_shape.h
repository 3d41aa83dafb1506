// What an orthogonalisation decides on the host, apart from the kernels so that host code can be built from it as well: how its steps
// are cut into runs, the powers of two by which each matrix is scaled, and where a matrix's scratch lies.
#pragma once

#include <math.h>
#include <stddef.h>
#include <stdint.h>

#include "ld_map.h"

constexpr int32_t kMuonMaxSteps = 16;
constexpr int32_t kMuonPad = 64;        // rows and columns are padded to whole tiles of the smallest kind
constexpr int32_t kMuonBlock = 32;      // elements of a row side by side, their upper halves before their lower
constexpr int64_t kMuonRowBytes = 2 * 2 * kMuonBlock;

// The largest value of |f| on [0, top] of f(x) = x^odd (a + b x^2 + c x^4), odd = 0, 1 or 2, from its ends and the roots of its derivative.
inline double ld_muon_largest(double a, double b, double c, double top, int32_t odd) {
    const auto f = [&](double x) { return fabs((odd == 0 ? 1.0 : odd == 1 ? x : x * x) * (a + x * x * (b + x * x * c))); };
    double most = fmax(f(0.0), f(top));
    // f' = x^(odd - 1) (odd a + (odd + 2) b y + (odd + 4) c y^2), y = x^2
    const double p = odd * a, q = (odd + 2) * b, r = (odd + 4) * c;
    double roots[2];
    int32_t n = 0;
    if (r == 0.0) {
        if (q != 0.0) roots[n++] = -p / q;
    } else if (q * q - 4.0 * p * r >= 0.0) {
        const double d = sqrt(q * q - 4.0 * p * r);
        roots[n++] = (-q - d) / (2.0 * r);
        roots[n++] = (-q + d) / (2.0 * r);
    }
    for (int32_t i = 0; i < n; ++i)
        if (roots[i] > 0.0 && roots[i] < top * top) most = fmax(most, f(sqrt(roots[i])));
    return most;
}

// Bounds of the spectral norms at every step, from |X| <= 1 at the first; no element of a matrix is larger than its norm.
constexpr double kMuonSlack = 1.0 + 1.0 / 4096;  // for roundings
struct LdMuonBounds {
    double x[kMuonMaxSteps + 1];  // X before a step
    double p[kMuonMaxSteps];      // P = a + b A + c A^2
    double r[kMuonMaxSteps];      // P A
};
// coeff: [steps][3]. Whether all bounds stay in the range that halves are precise in.
inline bool ld_muon_bounds(LdMuonBounds& m, int32_t steps, const float* coeff) {
    m.x[0] = kMuonSlack;
    for (int32_t s = 0; s < steps; ++s) {
        const double a = coeff[3 * s], b = coeff[3 * s + 1], c = coeff[3 * s + 2];
        if (!(fabs(a) <= 64.0 && fabs(b) <= 64.0 && fabs(c) <= 64.0)) return false;
        m.p[s] = kMuonSlack * ld_muon_largest(a, b, c, m.x[s], 0);
        m.r[s] = kMuonSlack * ld_muon_largest(a, b, c, m.x[s], 2);
        m.x[s + 1] = kMuonSlack * ld_muon_largest(a, b, c, m.x[s], 1);
        if (!(m.p[s] <= 64.0 && m.r[s] <= 64.0 && m.x[s + 1] <= 8.0)) return false;
    }
    return true;
}

// A run of steps works on one Gram matrix; X is multiplied by what they amount to, and its Gram matrix formed anew, between runs. The
// Gram matrix loses directions of small singular values, the more the further a run grows them (each usual step 3.4 times), and
// a matrix that is about square has more of those than a wide one. So a run of a wide matrix (kind 1) ends at two steps or 16 times,
// counted from the first, and one that is about square (0), to which a run's matrices of m x m are no smaller than X, has runs of one
// step. Only results that are rounded to 16 bits, of matrices wider still and of up to kMuonThreeSide rows (2), come by runs of three steps
// or 48 times, counted from the last on. Five usual steps as five times 1, 2 + 2 + 1 and 2 + 3 take 15 m^2 n + 5 m^3, 9 m^2 n + 11 m^3 and
// 6 m^2 n + 14 m^3 operations of products, in 15, 18 and 17 launches; 768 x 2304 272, 262 and 243 us, 1600 x 4800 849, 716 and 625,
// 4096 x 11008 by one and two 9660 and 7990. Errors against 64 bits (relative, Frobenius) of products in 32 bits in the order of the formula, and of runs
// of one, two and three: 768 x 2304 3.6e-6, 2.6e-6, 2.7e-6, 2.6e-6; 1024 x 1024 3.1e-6, and 2.0e-6 by one. Where the sizes of the
// rows spread over two decades, runs of three lose what 32 bits hold (16 bits are rounded by 2e-4 and more): 2304 x 768 1.9e-6, 1.5e-6, 2.5e-6,
// 1.6e-5; 5120 x 2048 3.0e-6, 2.1e-6, 3.5e-6, 2.5e-5; 6400 x 1600 3.7e-6, 2.3e-6, 4.2e-6, 2.5e-5. Up to kMuonFewSide rows a matrix goes
// another way, in 64 bits (kMuonFew).
constexpr int32_t kMuonKinds = 4, kMuonFew = 3, kMuonFewSide = 64, kMuonThreeSide = 2048;
// narrow: the result goes to 16 bits
inline int32_t ld_muon_kind(int64_t m, int64_t n, bool narrow = true) {
    return 2 * n >= 5 * m && m <= kMuonThreeSide && narrow ? 2 : 4 * n >= 5 * m ? 1 : 0;
}
// First steps of the runs, and behind them the number of steps; returns the number of runs.
inline int32_t ld_muon_runs(const LdMuonBounds& b, int32_t steps, int32_t kind, int32_t* begin) {
    const bool wide = kind == 2;
    const int32_t longest = kind + 1;
    const double most = wide ? 48.0 : 16.0;
    int32_t runs = 0, length = 0;
    double grown = 1.0;
    bool cut[kMuonMaxSteps] = {};  // a run begins at the step
    for (int32_t k = 0; k < steps; ++k) {
        const int32_t s = wide ? steps - 1 - k : k;
        if (length == longest || grown * b.p[s] > most) {
            if (k > 0) cut[wide ? s + 1 : s] = true;
            length = 0, grown = 1.0;
        }
        ++length, grown *= b.p[s];
    }
    for (int32_t s = 0; s < steps; ++s)
        if (s == 0 || cut[s]) begin[runs++] = s;
    begin[runs] = steps;
    return runs;
}
// Bound of the product of a run's P up to a step.
inline double ld_muon_grown(const LdMuonBounds& b, int32_t begin, int32_t step) {
    double q = b.p[begin];
    for (int32_t s = begin + 1; s <= step; ++s) q *= kMuonSlack * b.p[s];
    return q;
}

// The power of two that brings values of up to `bound` below 2^15, which halves hold with a factor of two to spare.
inline float ld_muon_scale(double bound) {
    int e = 0;
    frexp(bound, &e);  // bound < 2^e
    return static_cast<float>(ldexp(1.0, 15 - (e < 0 ? 0 : e)));
}

// Which tile a workgroup has. Consecutive ones, which an XCD has at a time, are to share rows and columns: bands of `band` rows of tiles, in each
// of them column after column.
LD_HD void ld_muon_tile(int32_t tile, int32_t down, int32_t across, int32_t band, int32_t& r, int32_t& c) {
    const int32_t first = tile / (band * across) * band, rows = down - first < band ? down - first : band;
    const int32_t t = tile - first * across;
    r = first + t % rows, c = t / rows;
}
// The same of the tiles on and below the diagonal: what a band has left of its diagonal tiles first, these then row by row.
LD_HD int32_t ld_muon_triangle_row(int32_t tile) {
    int32_t r = static_cast<int32_t>((sqrtf(8.0f * static_cast<float>(tile) + 1.0f) - 1.0f) * 0.5f);
    while (r * (r + 1) / 2 > tile) --r;
    while ((r + 1) * (r + 2) / 2 <= tile) ++r;
    return r;
}
LD_HD void ld_muon_lower_tile(int32_t tile, int32_t side, int32_t band, int32_t& r, int32_t& c) {
    const int32_t first = ld_muon_triangle_row(tile) / band * band, rows = side - first < band ? side - first : band;
    const int32_t t = tile - first * (first + 1) / 2;
    if (t < first * rows) {
        r = first + t % rows, c = t / rows;
        return;
    }
    const int32_t d = t - first * rows, down = ld_muon_triangle_row(d);
    r = first + down, c = first + d - down * (down + 1) / 2;
}

inline int64_t ld_muon_padded(int64_t n) { return (n + kMuonPad - 1) / kMuonPad * kMuonPad; }
// Bytes of a matrix of `rows` by `cols` in halves: padded, and with room for the rows that a larger tile reads behind its end.
inline int64_t ld_muon_bytes(int64_t rows, int64_t cols) { return ld_muon_padded(rows) * ld_muon_padded(cols) * 4 + 3 * kMuonPad * kMuonRowBytes; }
// A problem's scratch: X, its transposed, one more of that size, and five of m by m (m <= n).
inline int64_t ld_muon_large(int32_t m, int32_t n) { const int64_t a = ld_muon_bytes(m, n), b = ld_muon_bytes(n, m); return a > b ? a : b; }
inline int64_t ld_muon_scratch(int32_t m, int32_t n) { return 3 * ld_muon_large(m, n) + 5 * ld_muon_bytes(m, m); }
