// Orthogonalising updates by Newton-Schulz products, and the replay of dense gradients through the optimizer that does so (Muon).
//
//   X_0 = U / (|U|_F + eps);  X_{s+1} = (a I + b A + c A^2) X_s,  A = X_s X_s^T      (of U or its transposed, rows <= columns)
//   replay: m = mu m + g;  U = g + mu m (Nesterov) or m;  w = (1 - lr wd) w - lr s X_S
//
// Products are what bounds it. Results are compared, and replayed, as 32-bit values, so operands are kept as pairs of halves, h + l with
// 22 bits, and a product is three MFMA products: hh + hl + lh, summed in 32 bits. Values are scaled by powers of two that the
// coefficients bound. A run of steps works on the Gram matrix alone: with P = a I + b A + c A^2, A' = P A P and Q' = P Q, all of m by
// m, symmetric and commuting, so that half of each is computed and mirrored; X is read for its Gram matrix and multiplied by Q once a
// run (ld_muon_shape.h says when a run ends, and why): 9 m^2 n + 11 m^3 products' operations for five steps of a wide matrix instead of
// 15 m^2 n + 5 m^3 (symmetric halves there too). Matrices of up to 64 rows go a way of their own, in 64 bits.
//
// In memory a matrix lies as blocks of 32 columns, in each of them row after row: 32 upper halves, 32 lower halves, 128 bytes, whose eight
// 16-byte pieces are permuted by the row, as shared memory wants them: a tile's block is contiguous, and is copied into shared memory as it is.
// Every element's sum runs over the columns in order and depends on nothing but its own row and column: any mixture of matrices
// in a call, and any cut of a window into calls, gives the same bits.
#include <math.h>
#include <string.h>

#include <type_traits>

#include "ld_elem.h"
#include "ld_grid.h"
#include "ld_muon_shape.h"

namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x8 __attribute__((ext_vector_type(8)));

constexpr int kThreads = 256;
constexpr int kCUs = 256;
constexpr int kMost = 64;                                    // problems of a group
constexpr int64_t kGroupBytes = static_cast<int64_t>(8) << 30;  // scratch of a group, unless one problem needs more
constexpr int kSumParts = 256;                               // partial sums of squares of a problem at most
constexpr int64_t kSumElems = 4096;                          // elements of one, at least

enum Buffer { kX, kXT, kYT, kA, kP, kR, kQ0, kQ1 };

// The matrices of a group: m <= n, `flipped` where U has more rows than columns.
struct Batch {
    char* base[kMost];
    int32_t m[kMost], n[kMost];
    int32_t flipped[kMost];
    int32_t kind[kMost];       // which of a launch's plans is a problem's
    int32_t first[kMost + 1];  // tiles of a launch before a problem's
    int32_t count;
};

__device__ __forceinline__ int64_t padded(int64_t n) { return (n + kMuonPad - 1) / kMuonPad * kMuonPad; }
__device__ __forceinline__ char* buffer_of(const Batch& b, int32_t i, int32_t which) {
    const int64_t m = padded(b.m[i]), n = padded(b.n[i]), slack = 3 * kMuonPad * kMuonRowBytes;
    const int64_t large = m * n * 4 + slack, small = m * m * 4 + slack;
    return b.base[i] + (which < 3 ? which * large : 3 * large + (which - 3) * small);
}
// A matrix whose norm is far below eps begins as small as that, and halves would not hold it. So X lies in memory times 2^lift, the part of
// (norm + eps) / norm that is a power of two, or less of it where steps have grown X since (Plan::drop): 0 where eps is below the norm. It is kept behind the
// last buffer, in the room of rows that nothing writes.
constexpr int32_t kMostLift = 96;  // 2^-96 and the scales of halves are no subnormals
__device__ __forceinline__ int32_t* lift_of(const Batch& b, int32_t i) {
    const int64_t m = padded(b.m[i]);
    return reinterpret_cast<int32_t*>(buffer_of(b, i, kQ1) + m * m * 4 + 3 * kMuonPad * kMuonRowBytes) - 1;
}
__device__ __forceinline__ int32_t left_of(int32_t lift, int32_t drop) { return lift > drop ? lift - drop : 0; }
// Tiles over a side: all of its padding is written too.
__host__ __device__ __forceinline__ int32_t tiles_of(int64_t side, int32_t tile) { return static_cast<int32_t>((side + tile - 1) / tile); }
// Where the eight upper halves of row r, columns [8 c, 8 c + 8) lie, in bytes; the lower ones are 64 bytes on, permuted alike.
__device__ __forceinline__ int64_t piece_at(int64_t rows, int64_t r, int64_t c, int32_t lower) {
    return ((c >> 2) * rows + r) * kMuonRowBytes + ((((c & 3) | lower << 2) ^ (r >> 1 & 7)) << 4);
}

__device__ __forceinline__ void split(const f32x8& x, half8& h, half8& l) {
    h = __builtin_convertvector(x, half8);
    l = __builtin_convertvector(x - __builtin_convertvector(h, f32x8), half8);
}
__device__ __forceinline__ void store_split(char* to, int64_t rows, int64_t r, int64_t c, const f32x8& x) {
    half8 h, l;
    split(x, h, l);
    *reinterpret_cast<half8*>(to + piece_at(rows, r, c, 0)) = h;
    *reinterpret_cast<half8*>(to + piece_at(rows, r, c, 1)) = l;
}

// ------------------------------------------------------------------------------------------------------------------- products

// C = left right^T of every problem: rows of `left` by rows of `right`, both over the same columns.
struct Product {
    int32_t left, right;   // buffers
    int32_t out, out_t;    // of C and, where not symmetric, of its transposed
};
struct Plan {
    Product prod[2];
    int32_t products;      // 0: a problem has no part in the launch
    int32_t apply;         // X' = Q X, with `final` where it goes
    int32_t final;
    int32_t long_sum;      // the columns are n, not m
    int32_t poly;          // C is A^2: what is kept is a I + b A + c C
    float inv;             // 1 / scale of the operands' product
    float scale[2];        // of what is kept
    float ca, cb, cc;      // coefficients, cb times 1 / scale of A
    int32_t drop;          // powers of two by which X may have grown since it was laid out, of the X that is read
    int32_t out_drop;      // and of the X that is written; where it goes nothing is left of the lift: kMostLift
};
struct Plans {
    Plan of[kMuonKinds];
};
// Where X_S goes.
struct FinalArgs {
    void* out[kMost];
    int64_t stride[kMost];
};

typedef const void __attribute__((address_space(1))) * global_ptr;
typedef void __attribute__((address_space(3))) * shared_ptr;

// A tile of SIDE by SIDE sums, by DOWN x ACROSS waves. STAGES blocks of columns have room in shared memory: one that is multiplied, the others on
// their way.
// Tiles of 64 and 128 are bound by their loads into shared memory next to the products (of 128, below, 2410 us; 1480 without the loads, 1790
// with a third of the products), those of 256 by the matrix cores and their power. Five steps of 32 matrices of 768 x 768 and of four of 2048 x 2048, us: 64 by 2 x 2 waves, three
// stages 1460 and 2660, by two waves 1570 and 2890, by one 1610 and 2770; 128 by 2 x 2, two stages 1290 and 2410, by two waves 1485
// and 2640, by eight 1300 and 2510; 256 by 2 x 4, two stages 1425 and 2290, by four 1640 and 2460, by sixteen 2260 and 3690. Blocks of 16
// columns, as many bytes and more on their way, took 3 to 8 % longer in all: twice the barriers; loads among the products rather than before them
// 2 to 7 %; asking for lines four blocks early 1 to 8 %.
template <int SIDE_, int DOWN_, int ACROSS_, int STAGES_> struct Tile {
    static constexpr int SIDE = SIDE_, DOWN = DOWN_, ACROSS = ACROSS_, STAGES = STAGES_;
    static constexpr int THREADS = DOWN * ACROSS * LD_WAVE;
    static constexpr int WAVES = SIDE == 64 ? 3 : 2;             // of a SIMD
    // Consecutive tiles, which share rows and columns, that an XCD has at a time: as many as it runs, so that its cache loads them once.
    static constexpr int RUN = SIDE == 256 ? 32 : SIDE == 64 ? 96 : 64;
    static constexpr int BAND = 8;                               // rows of tiles that they are taken from (rows of all: 64 3030 us, not 2760)
    static constexpr int R = SIDE / DOWN / 32, C = SIDE / ACROSS / 32;            // MFMA tiles of a wave
    static constexpr int BLOCK_BYTES = SIDE * static_cast<int>(kMuonRowBytes);     // an operand's, of a block
    static constexpr int FETCHES = BLOCK_BYTES / 1024 / (DOWN * ACROSS);           // loads of a wave for it
    static constexpr int ROWS = 64;                                                // rows of sums laid out at a time
    static constexpr int STRIDE = SIDE + 2;                                        // floats of one: rows and columns read by eights lie in different banks
    static constexpr int OPERANDS = 2 * STAGES * BLOCK_BYTES, SUMS = ROWS * STRIDE * 4, HELD = ROWS * SIDE * 4;
    static constexpr int SHARED = OPERANDS > SUMS + HELD ? OPERANDS : SUMS + HELD;
};

// A block of an operand's rows into shared memory, 16 bytes a lane, as they lie.
template <typename T>
__device__ __forceinline__ void fetch(const char* from, char* to) {
    const int32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / LD_WAVE);
#pragma unroll
    for (int i = 0; i < T::FETCHES; ++i) {
        const int32_t at = (wave * T::FETCHES + i) * 1024;
        __builtin_amdgcn_global_load_lds((global_ptr)(from + at + ld_lane() * 16), (shared_ptr)(to + at), 16, 0, 0);
    }
}

__device__ __forceinline__ half8 fragment(const char* tile, int32_t row, int32_t piece) {
    return *reinterpret_cast<const half8*>(tile + row * kMuonRowBytes + ((piece ^ (row >> 1 & 7)) << 4));
}

template <typename T>
__device__ __forceinline__ void multiply(const char* left, int64_t left_rows, const char* right, int64_t right_rows, int32_t blocks, char* shared,
                                         f32x16 (&acc)[T::R][T::C]) {
    const int32_t lane = ld_lane(), wave = threadIdx.x / LD_WAVE;
    const int32_t row = wave / T::ACROSS * (T::SIDE / T::DOWN) + (lane & 31), col = wave % T::ACROSS * (T::SIDE / T::ACROSS) + (lane & 31);
    const int64_t left_step = left_rows * kMuonRowBytes, right_step = right_rows * kMuonRowBytes;
    constexpr int kStages = T::STAGES;
    constexpr int kLoads = 2 * T::FETCHES;                   // of a wave for a block
    const auto fetch_block = [&](int32_t k, int32_t stage) {
        char* to = shared + stage * 2 * T::BLOCK_BYTES;
        fetch<T>(left + k * left_step, to);
        fetch<T>(right + k * right_step, to + T::BLOCK_BYTES);
    };
    // The operands of 16 columns are read while those before them are multiplied (in what order, is the compiler's: 1 % faster than the
    // reads first), and waited for before the next are read: the compiler would wait for both.
    constexpr int kSharedRead = 0xC07F;  // lgkmcnt(0), nothing else
    half8 x[2][T::R][2], y[2][T::C][2];
    const auto read = [&](int s, int32_t stage) {
        const char* now = shared + stage * 2 * T::BLOCK_BYTES;
#pragma unroll
        for (int l = 1; l >= 0; --l) {
#pragma unroll
            for (int i = 0; i < T::R; ++i) x[s][i][l] = fragment(now, row + 32 * i, 4 * l + 2 * s + (lane >> 5));
#pragma unroll
            for (int j = 0; j < T::C; ++j) y[s][j][1 - l] = fragment(now + T::BLOCK_BYTES, col + 32 * j, 4 * (1 - l) + 2 * s + (lane >> 5));
        }
    };
    const auto use = [&](int s) {  // lower halves first; one after another for every sum, whatever the tile
#pragma unroll
        for (int l = 0; l < 3; ++l)
#pragma unroll
            for (int i = 0; i < T::R; ++i)
#pragma unroll
                for (int j = 0; j < T::C; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[s][i][l == 0], y[s][j][l == 1], acc[i][j], 0, 0, 0);
    };
    for (int32_t k = 0; k < kStages && k < blocks; ++k) fetch_block(k, k);
    if (blocks >= kStages) asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((kStages - 1) * kLoads) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
    read(0, 0);
    int32_t stage = 0;
    for (int32_t k = 0; k < blocks; ++k) {
        const int32_t next = stage + 1 == kStages ? 0 : stage + 1;
        __builtin_amdgcn_s_waitcnt(kSharedRead);
        read(1, stage);
        use(0);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(kSharedRead);
        if (k + 1 < blocks) {
            // This wave's loads of the next block have arrived when no more are left than those of the blocks behind it; the barrier then
            // says it of all waves, and that all have read this block, whose room is filled anew.
            if (k + kStages <= blocks) asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((kStages - 2) * kLoads) : "memory");
            else asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
            if (k + kStages < blocks) fetch_block(k + kStages, stage);
            read(0, next);
        }
        use(1);
        __builtin_amdgcn_sched_barrier(0);
        stage = next;
    }
    __syncthreads();
}

// A barrier for what goes through shared memory alone: what is on its way to memory is not waited for, as __syncthreads does. With
// `loads` what the wave loads into shared memory is.
template <bool LOADS = false>
__device__ __forceinline__ void shared_barrier() {
    if (LOADS) asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    else asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// The sums of the `part`-th T::ROWS rows, times `inv`, as rows of 32-bit values in shared memory.
template <typename T>
__device__ __forceinline__ void lay_out(const f32x16 (&acc)[T::R][T::C], int32_t part, float inv, float* sums, int32_t stride, bool loads) {
    const int32_t lane = ld_lane(), wave = threadIdx.x / LD_WAVE, first = wave / T::ACROSS * (T::SIDE / T::DOWN);
    if (part > 0) shared_barrier();
#pragma unroll
    for (int i = 0; i < T::R; ++i) {
        if ((first + 32 * i) / T::ROWS != part) continue;
#pragma unroll
        for (int j = 0; j < T::C; ++j)
#pragma unroll
            for (int q = 0; q < 16; ++q) {
                const int32_t r = (first + 32 * i) % T::ROWS + (q & 3) + 8 * (q >> 2) + 4 * (lane >> 5);
                const int32_t c = wave % T::ACROSS * (T::SIDE / T::ACROSS) + 32 * j + (lane & 31);
                sums[r * stride + c] = acc[i][j][q] * inv;
            }
    }
    if (loads) shared_barrier<true>();
    else shared_barrier();
}

// A value's two halves side by side, as shared memory holds them between a row's way out and a column's.
typedef uint32_t u32x8 __attribute__((ext_vector_type(8)));
__device__ __forceinline__ u32x8 pack(const half8& h, const half8& l) {
    return __builtin_bit_cast(u32x8, __builtin_shufflevector(h, l, 0, 8, 1, 9, 2, 10, 3, 11, 4, 12, 5, 13, 6, 14, 7, 15));
}
__device__ __forceinline__ void store_packed(char* upper, char* lower, const u32x8& x) {
    ld_u32x4 h, l;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        h[e] = __builtin_amdgcn_perm(x[2 * e + 1], x[2 * e], 0x05040100u);
        l[e] = __builtin_amdgcn_perm(x[2 * e + 1], x[2 * e], 0x07060302u);
    }
    *reinterpret_cast<ld_u32x4*>(upper) = h;
    *reinterpret_cast<ld_u32x4*>(lower) = l;
}

// A tile's way out as halves. Four lanes write those of 32 columns of a row, which lie side by side, the next four those of the row behind
// it. A thread's pieces all have the same permutation.
template <typename T>
struct WayOut {
    static constexpr int EACH = T::ROWS * T::SIDE / 8 / T::THREADS, STEP = T::THREADS / 4;
    int32_t piece, along;
    __device__ __forceinline__ WayOut() : piece(threadIdx.x & 3), along(threadIdx.x >> 2) {}
    // of the part, row r and the first of eight columns c
    __device__ __forceinline__ void straight(int p, int32_t& r, int32_t& c) const {
        const int32_t n = along + p * STEP;
        r = n % T::ROWS, c = n / T::ROWS * 32 + piece * 8;
    }
    // the first of eight rows r, and column c
    __device__ __forceinline__ void turned(int p, int32_t& r, int32_t& c) const {
        const int32_t n = along + p * STEP;
        r = n / T::SIDE * 32 + piece * 8, c = n % T::SIDE;
    }
};

// Which problem a tile is of, and its number there.
__device__ __forceinline__ int32_t problem_of(const Batch& b, int32_t& tile) {
    int32_t lo = 0, hi = b.count - 1;
    while (lo < hi) {
        const int32_t mid = (lo + hi + 1) >> 1;
        if (b.first[mid] <= tile) lo = mid;
        else hi = mid - 1;
    }
    tile -= b.first[lo];
    return lo;
}

template <typename T>
__global__ __launch_bounds__(T::THREADS, T::WAVES) void k_symmetric(Batch batch, Plans plans) {
    __shared__ __attribute__((aligned(16))) char shared[T::SHARED];
    int32_t tile = static_cast<int32_t>(ld_xcd_piece<T::RUN>(blockIdx.x, gridDim.x));
    if (tile >= batch.first[batch.count]) return;
    const int32_t i = problem_of(batch, tile);
    const Plan a = plans.of[batch.kind[i]];
    const int32_t side = tiles_of(padded(batch.m[i]), T::SIDE), tiles = side * (side + 1) / 2, second = tile >= tiles;
    if (second) tile -= tiles;
    const Product prod = a.prod[second];
    const float scale = a.scale[second];
    int32_t tr, tc;
    ld_muon_lower_tile(tile, side, T::BAND, tr, tc);
    const int32_t m = batch.m[i], r0 = tr * T::SIDE, c0 = tc * T::SIDE;
    const int64_t rows = padded(m);
    const float inv = a.long_sum ? ldexpf(a.inv, -2 * left_of(*lift_of(batch, i), a.drop)) : a.inv;
    f32x16 acc[T::R][T::C] = {};
    multiply<T>(buffer_of(batch, i, prod.left) + r0 * kMuonRowBytes, rows, buffer_of(batch, i, prod.right) + c0 * kMuonRowBytes, rows,
                static_cast<int32_t>((a.long_sum ? padded(batch.n[i]) : rows) / kMuonBlock), shared, acc);
    float* sums = reinterpret_cast<float*>(shared);
    constexpr int S = T::STRIDE;
    char* out = buffer_of(batch, i, prod.out);
    const char* gram = buffer_of(batch, i, prod.left);
    // Only sums on and below the diagonal are kept, and mirrored, in squares of eight by eight. What is needed of A comes into shared memory
    // behind the sums.
    const WayOut<T> way;
    char* held = shared + T::SUMS;
    for (int32_t h = 0; h < T::SIDE / T::ROWS; ++h) {
        const int32_t h0 = r0 + T::ROWS * h;
        if (a.poly) {
            const int32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / LD_WAVE);
            if (h > 0) shared_barrier();
            for (int32_t k = wave; k < T::SIDE / kMuonBlock && c0 + k * kMuonBlock < rows; k += T::THREADS / LD_WAVE)
#pragma unroll
                for (int n = 0; n < T::ROWS / 8; ++n)
                    __builtin_amdgcn_global_load_lds((global_ptr)(gram + ((c0 / kMuonBlock + k) * rows + h0 + 8 * n) * kMuonRowBytes + ld_lane() * 16),
                                                     (shared_ptr)(held + (k * T::ROWS + 8 * n) * kMuonRowBytes), 16, 0, 0);
        }
        lay_out<T>(acc, h, inv, sums, S, a.poly != 0);
#pragma unroll 2
        for (int p = 0; p < WayOut<T>::EACH; ++p) {
            int32_t r, c;
            way.straight(p, r, c);
            const int32_t row = h0 + r, col = c0 + c;
            if (row >= rows || col >= rows || col > row) continue;
            float* from = sums + r * S + c;
            f32x8 x;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = from[e];
            const bool diagonal = tr == tc && row / 8 == col / 8;
            if (diagonal) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (col + e > row) x[e] = sums[(col + e - h0) * S + row - c0];
            }
            if (a.poly) {
                const char* block = held + (c >> 5) * T::ROWS * kMuonRowBytes;
                const f32x8 g = __builtin_convertvector(fragment(block, r, way.piece), f32x8) + __builtin_convertvector(fragment(block, r, way.piece | 4), f32x8);
                // the terms nearly cancel at singular values of 1: one rounding each, the smaller sums first
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = __fmaf_rn(a.cc, x[e], __fmaf_rn(a.cb, g[e], diagonal && row == col + e && row < m ? a.ca : 0.0f));
            }
            half8 upper, lower;
            split(x * scale, upper, lower);
            *reinterpret_cast<half8*>(out + piece_at(rows, row, col >> 3, 0)) = upper;
            *reinterpret_cast<half8*>(out + piece_at(rows, row, col >> 3, 1)) = lower;
            if (!diagonal) {  // to be mirrored; the squares on the diagonal are read by one another's rows
                const u32x8 both = pack(upper, lower);
#pragma unroll
                for (int e = 0; e < 8; ++e) reinterpret_cast<uint32_t*>(from)[e] = both[e];
            }
        }
        shared_barrier();
#pragma unroll 2
        for (int p = 0; p < WayOut<T>::EACH; ++p) {
            int32_t r, c;
            way.turned(p, r, c);
            if (h0 + r >= rows || c0 + c >= rows || (h0 + r) / 8 <= (c0 + c) / 8) continue;
            u32x8 x;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = reinterpret_cast<const uint32_t*>(sums)[(r + e) * S + c];
            store_packed(out + piece_at(rows, c0 + c, (h0 + r) >> 3, 0), out + piece_at(rows, c0 + c, (h0 + r) >> 3, 1), x);
        }
    }
}

// X' = Q X: kept both ways, or, the last, written where it goes. left: Q (m rows); right: X transposed (n rows).
template <typename T, bool FINAL, int OT>
__global__ __launch_bounds__(T::THREADS, T::WAVES) void k_apply(Batch batch, Plans plans, FinalArgs f) {
    __shared__ __attribute__((aligned(16))) char shared[T::SHARED];
    int32_t tile = static_cast<int32_t>(ld_xcd_piece<T::RUN>(blockIdx.x, gridDim.x));
    if (tile >= batch.first[batch.count]) return;
    const int32_t i = problem_of(batch, tile);
    const Plan a = plans.of[batch.kind[i]];
    const int32_t m = batch.m[i], n = batch.n[i], down = tiles_of(padded(m), T::SIDE);
    int32_t tr, tc;
    ld_muon_tile(tile, down, tiles_of(padded(n), T::SIDE), T::BAND, tr, tc);
    const int32_t r0 = tr * T::SIDE, c0 = tc * T::SIDE;
    const int64_t rows = padded(m), cols = padded(n);
    const int32_t lift = *lift_of(batch, i);
    const float inv = ldexpf(FINAL ? a.inv : a.inv * a.scale[0], left_of(lift, a.out_drop) - left_of(lift, a.drop));
    f32x16 acc[T::R][T::C] = {};
    multiply<T>(buffer_of(batch, i, a.prod[0].left) + r0 * kMuonRowBytes, rows, buffer_of(batch, i, a.prod[0].right) + c0 * kMuonRowBytes, cols,
                static_cast<int32_t>(rows / kMuonBlock), shared, acc);
    float* sums = reinterpret_cast<float*>(shared);
    constexpr int S = T::STRIDE, kPieces = T::SIDE / 8;
    typedef typename LdElem<OT>::type elem;
    char* straight = FINAL ? nullptr : buffer_of(batch, i, a.prod[0].out);
    char* turned = FINAL ? nullptr : buffer_of(batch, i, a.prod[0].out_t);
    elem* final_out = FINAL ? static_cast<elem*>(f.out[i]) : nullptr;
    const int64_t stride = FINAL ? f.stride[i] : 0;
    const auto write = [&](const f32x8& x, int32_t r, int32_t c, int32_t width) {
        elem* to = final_out + r * stride + c;
        if (c + 8 <= width) {
            if constexpr (OT == LD_F32) {
                typedef typename LdVec<LD_F32, 4>::type half;
                *reinterpret_cast<half*>(to) = __builtin_shufflevector(x, x, 0, 1, 2, 3);
                *reinterpret_cast<half*>(to + 4) = __builtin_shufflevector(x, x, 4, 5, 6, 7);
            } else {
                typedef LdVec<OT, 8> V;
                *reinterpret_cast<typename V::type*>(to) = V::narrow(x);
            }
            return;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (c + e < width) to[e] = static_cast<elem>(x[e]);
    };
    for (int32_t h = 0; h < T::SIDE / T::ROWS; ++h) {
        if (FINAL && batch.flipped[i]) {
            // an odd stride, and the lanes along the columns that are rows of the update: what they write lies side by side
            constexpr int kOdd = T::SIDE + 1, kDeep = T::ROWS / 8;
            lay_out<T>(acc, h, inv, sums, kOdd, false);
            for (int32_t p = threadIdx.x; p < kDeep * T::SIDE; p += T::THREADS) {
                const int32_t c = p / kDeep, r = p % kDeep * 8, ri = r0 + T::ROWS * h + r, ci = c0 + c;
                f32x8 x;
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = sums[(r + e) * kOdd + c];
                if (ci < n) write(x, ci, ri, m);
            }
            continue;
        }
        lay_out<T>(acc, h, inv, sums, S, false);
        if (FINAL) {
            for (int32_t p = threadIdx.x; p < T::ROWS * kPieces; p += T::THREADS) {
                const int32_t r = p / kPieces, c = p % kPieces * 8, ri = r0 + T::ROWS * h + r, ci = c0 + c;
                f32x8 x;
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = sums[r * S + c + e];
                if (ri < m) write(x, ri, ci, n);
            }
            continue;
        }
        const WayOut<T> way;
#pragma unroll 2
        for (int p = 0; p < WayOut<T>::EACH; ++p) {
            int32_t r, c;
            way.straight(p, r, c);
            const int32_t row = r0 + T::ROWS * h + r, col = c0 + c;
            if (row >= rows || col >= cols) continue;
            float* from = sums + r * S + c;
            f32x8 x;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = from[e];
            half8 upper, lower;
            split(x, upper, lower);
            *reinterpret_cast<half8*>(straight + piece_at(rows, row, col >> 3, 0)) = upper;
            *reinterpret_cast<half8*>(straight + piece_at(rows, row, col >> 3, 1)) = lower;
            const u32x8 both = pack(upper, lower);
#pragma unroll
            for (int e = 0; e < 8; ++e) reinterpret_cast<uint32_t*>(from)[e] = both[e];
        }
        shared_barrier();
#pragma unroll 2
        for (int p = 0; p < WayOut<T>::EACH; ++p) {
            int32_t r, c;
            way.turned(p, r, c);
            const int32_t row = r0 + T::ROWS * h + r, col = c0 + c;
            if (row >= rows || col >= cols) continue;
            u32x8 x;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = reinterpret_cast<const uint32_t*>(sums)[(r + e) * S + c];
            store_packed(turned + piece_at(cols, col, row >> 3, 0), turned + piece_at(cols, col, row >> 3, 1), x);
        }
    }
}

// ------------------------------------------------------------------------------------------------------------- before and after

__device__ __forceinline__ double block_sum(double x, double* sh) {
    for (int d = LD_WAVE / 2; d > 0; d >>= 1) x += __shfl_xor(x, d);
    __syncthreads();
    if (ld_lane() == 0) sh[threadIdx.x / LD_WAVE] = x;
    __syncthreads();
    double sum = 0.0;
    for (int w = 0; w < kThreads / LD_WAVE; ++w) sum += sh[w];
    return sum;
}

// Updates to orthogonalise: user rows and columns are those of the update, not of X.
struct Source {
    const void* src[kMost];
    int64_t stride[kMost];
    double* sums;              // [problem][kSumParts]
    float eps;
};
__device__ __forceinline__ int32_t user_rows(const Batch& b, int32_t i) { return b.flipped[i] ? b.n[i] : b.m[i]; }
__device__ __forceinline__ int32_t user_cols(const Batch& b, int32_t i) { return b.flipped[i] ? b.m[i] : b.n[i]; }
// How many partial sums the squares of a matrix have, by its size alone.
__host__ __device__ __forceinline__ int32_t sum_parts(int64_t elems) {
    const int64_t parts = (elems + kSumElems - 1) / kSumElems;
    return static_cast<int32_t>(parts < kSumParts ? parts : kSumParts);
}

// Threads of a row, a power of two, when each takes eight elements side by side at a time.
__device__ __forceinline__ int32_t lanes_log2_of(int32_t cols) {
    int32_t lanes_log2 = 0;
    while (lanes_log2 < 8 && (8 << lanes_log2) < cols) ++lanes_log2;
    return lanes_log2;
}
// Up to eight elements from p on, zeros behind them.
template <int DT>
__device__ __forceinline__ f32x8 load_eight(const typename LdElem<DT>::type* p, int32_t n) {
    f32x8 x;
    if (n >= 8) {
        if constexpr (DT == LD_F32) {
            typedef typename LdVec<LD_F32, 4>::type half;
            const half lo = *reinterpret_cast<const half*>(p), hi = *reinterpret_cast<const half*>(p + 4);
            x = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        } else {
            typedef LdVec<DT, 8> V;
            x = V::widen(*reinterpret_cast<const typename V::type*>(p));
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = e < n ? static_cast<float>(p[e]) : 0.0f;
    }
    return x;
}

template <int DT>
__global__ __launch_bounds__(kThreads) void k_squares(Batch b, Source s) {
    __shared__ double sh[kThreads / LD_WAVE];
    typedef typename LdElem<DT>::type elem;
    const int32_t i = blockIdx.y, rows = user_rows(b, i), cols = user_cols(b, i);
    const int32_t parts = sum_parts(static_cast<int64_t>(rows) * cols);
    if (static_cast<int32_t>(blockIdx.x) >= parts || b.kind[i] == kMuonFew) return;
    const elem* src = static_cast<const elem*>(s.src[i]);
    const int64_t stride = s.stride[i];
    const int32_t lanes_log2 = lanes_log2_of(cols), lanes = 1 << lanes_log2, at_once = kThreads >> lanes_log2;
    double sum = 0.0;
    for (int64_t r = static_cast<int64_t>(blockIdx.x) * at_once + (threadIdx.x >> lanes_log2); r < rows; r += static_cast<int64_t>(parts) * at_once)
        for (int32_t c = (threadIdx.x & (lanes - 1)) * 8; c < cols; c += lanes * 8) {
            const f32x8 x = load_eight<DT>(src + r * stride + c, cols - c);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum = fma(static_cast<double>(x[e]), static_cast<double>(x[e]), sum);
        }
    sum = block_sum(sum, sh);
    if (threadIdx.x == 0) s.sums[i * kSumParts + blockIdx.x] = sum;
}

// X and its transposed from the update: 64 by 64 elements a workgroup, zeros behind its edges. Rows are written as they are loaded,
// columns by way of shared memory; the elements are on their way while the partial sums are added up.
template <int DT>
__global__ __launch_bounds__(kThreads) void k_lay_out(Batch b, Source s, float scale) {
    constexpr int kStride = kMuonPad + 2, kEach = kMuonPad * kMuonPad / 8 / kThreads;
    __shared__ float tile[kMuonPad * kStride];
    __shared__ double sh[kThreads / LD_WAVE];
    typedef typename LdElem<DT>::type elem;
    const int32_t i = blockIdx.y, rows = user_rows(b, i), cols = user_cols(b, i);
    const int32_t across = (cols + kMuonPad - 1) / kMuonPad, r0 = static_cast<int32_t>(blockIdx.x) / across * kMuonPad, c0 = static_cast<int32_t>(blockIdx.x) % across * kMuonPad;
    if (r0 >= rows || b.kind[i] == kMuonFew) return;
    const elem* src = static_cast<const elem*>(s.src[i]);
    const int64_t stride = s.stride[i];
    f32x8 x[kEach];
#pragma unroll
    for (int p = 0; p < kEach; ++p) {
        const int32_t n = p * kThreads + threadIdx.x, r = r0 + n / 8, c = c0 + n % 8 * 8;
        x[p] = r < rows && c < cols ? load_eight<DT>(src + r * stride + c, cols - c) : f32x8(0.0f);
    }
    const int32_t parts = sum_parts(static_cast<int64_t>(rows) * cols);
    const double total = block_sum(static_cast<int32_t>(threadIdx.x) < parts ? s.sums[i * kSumParts + threadIdx.x] : 0.0, sh);
    const double norm = sqrt(total);
    const double eps = static_cast<double>(s.eps), ratio = (norm + eps) / norm;
    const int32_t lift = ratio >= 2.0 && norm > 0.0 ? min(ilogb(ratio), kMostLift) : 0;
    if (blockIdx.x == 0 && threadIdx.x == 0) *lift_of(b, i) = lift;
    const double f = norm == 0.0 ? 0.0 : ldexp(static_cast<double>(scale), lift) / (norm + eps);
    char* straight = buffer_of(b, i, b.flipped[i] ? kXT : kX);
    char* turned = buffer_of(b, i, b.flipped[i] ? kX : kXT);
    const int64_t all_rows = padded(rows), all_cols = padded(cols);
#pragma unroll
    for (int p = 0; p < kEach; ++p) {
        const int32_t n = p * kThreads + threadIdx.x, r = n / 8, c = n % 8 * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[p][e] = static_cast<float>(static_cast<double>(x[p][e]) * f);
            tile[r * kStride + c + e] = x[p][e];
        }
        store_split(straight, all_rows, r0 + r, (c0 + c) >> 3, x[p]);
    }
    __syncthreads();
#pragma unroll
    for (int p = 0; p < kEach; ++p) {
        const int32_t n = p * (kThreads / 4) + (threadIdx.x >> 2), c = n % kMuonPad, r = n / kMuonPad * 32 + (threadIdx.x & 3) * 8;
        f32x8 y;
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = tile[(r + e) * kStride + c];
        store_split(turned, all_cols, c0 + c, (r0 + r) >> 3, y);
    }
}

// -------------------------------------------------------------------------------------------------------------------- few rows

// Matrices of at most kMuonFewSide rows, in 64 bits. All steps work on the Gram matrix, which one workgroup holds: a launch for the parts of
// X X^T, one for all P and Q (the norm is the root of the trace), and one for Q U. In so few rows roundings do not average out before
// the steps grow them: halves left 4 x 600 up to 5.5e-6 off (relative, Frobenius; products in 32 bits 7.5e-7), this 5e-8, the rounding of
// the result. Latency is what bounds it, of 3 launches and some 17 products in turn rather than of 17 launches. By halves and so, us:
// 1 x 768 109 and 31, 32 x 1024 113 and 29, 64 x 64 81 and 65, 64 x 2048 129 and 71, 64 x 65536 1160 and 128, 32 of 64 x 2048 173
// and 133 (the steps 50 of those of 64 rows, 12 of 16). 128 rows would take eight times the products, and do not fit.
// An MFMA of 16 by 16 by 4: lane l has row (or column) l & 15 of both operands at column l >> 4, and of the sums column l & 15 and rows
// (l >> 4) + 4 q.
typedef double f64x4 __attribute__((ext_vector_type(4)));
constexpr int kFewThreads = 512;
constexpr int kFewBand = 16, kFewBands = kMuonFewSide / kFewBand, kFewTiles = kFewBands * (kFewBands + 1) / 2;  // tiles on and above the diagonal
constexpr int kFewTile = kFewBand * kFewBand;

// Columns of X that a part of its Gram matrix is of, by its columns alone: what is added up then does not depend on the rest of a call.
__host__ __device__ __forceinline__ int32_t few_columns(int32_t n) { return n <= 64 * 128 ? 128 : (n + 64 * 128 - 1) / (64 * 128) * 128; }
__device__ __forceinline__ char* few_parts(const Batch& b, int32_t i) { return buffer_of(b, i, kXT); }
__device__ __forceinline__ char* few_q(const Batch& b, int32_t i) { return buffer_of(b, i, kA); }
// Both fit what a matrix's scratch has for X transposed and for A.
static_assert(kMuonFewSide == kMuonPad && kFewTiles * kFewTile * 8 <= 128 * kMuonFewSide * 4 && kFewTiles * kFewTile * 8 <= kMuonPad * kMuonPad * 4 + 3 * kMuonPad * kMuonRowBytes &&
              kMuonFewSide * kMuonFewSide * 8 <= kMuonPad * kMuonPad * 4 + 3 * kMuonPad * kMuonRowBytes, "scratch");

// Eight columns of X from c on, of row r.
template <int DT>
__device__ __forceinline__ f32x8 few_load(const typename LdElem<DT>::type* src, int64_t stride, int32_t flipped, int32_t m, int32_t n, int32_t r, int32_t c) {
    f32x8 x(0.0f);
    if (r >= m || c >= n) return x;
    if (!flipped) return load_eight<DT>(src + r * stride + c, n - c);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (c + e < n) x[e] = static_cast<float>(src[(c + e) * stride + r]);
    return x;
}

template <int DT>
__global__ __launch_bounds__(kThreads) void k_few_gram(Batch b, Source s) {
    constexpr int kWaves = kThreads / LD_WAVE;
    __shared__ double sums[kWaves][kFewTiles * kFewTile];
    typedef typename LdElem<DT>::type elem;
    const int32_t i = blockIdx.y, m = b.m[i], n = b.n[i], lane = ld_lane(), wave = threadIdx.x / LD_WAVE;
    if (b.kind[i] != kMuonFew) return;
    const int32_t columns = few_columns(n), from = blockIdx.x * columns, to = n - from < columns ? n : from + columns;
    if (from >= n) return;
    const int32_t bands = (m + kFewBand - 1) / kFewBand;
    f64x4 acc[kFewTiles] = {};
    for (int32_t c0 = from + wave * 32; c0 < to; c0 += kWaves * 32) {
        f32x8 x[kFewBands];
#pragma unroll
        for (int t = 0; t < kFewBands; ++t)
            if (t < bands) x[t] = few_load<DT>(static_cast<const elem*>(s.src[i]), s.stride[i], b.flipped[i], m, n, kFewBand * t + (lane & 15), c0 + 8 * (lane >> 4));
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int t = 0, k = 0; t < kFewBands; ++t)
#pragma unroll
                for (int u = 0; u <= t; ++u, ++k)
                    if (t < bands) acc[k] = __builtin_amdgcn_mfma_f64_16x16x4f64(static_cast<double>(x[u][e]), static_cast<double>(x[t][e]), acc[k], 0, 0, 0);
    }
#pragma unroll
    for (int k = 0; k < kFewTiles; ++k)
#pragma unroll
        for (int q = 0; q < 4; ++q) sums[wave][k * kFewTile + q * LD_WAVE + lane] = acc[k][q];
    __syncthreads();
    double* out = reinterpret_cast<double*>(few_parts(b, i)) + static_cast<int64_t>(blockIdx.x) * kFewTiles * kFewTile;
    for (int32_t e = threadIdx.x; e < bands * (bands + 1) / 2 * kFewTile; e += kThreads) {
        double sum = 0.0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) sum += sums[w][e];
        out[e] = sum;
    }
}

struct FewArgs {
    int32_t steps;
    float eps;
    float coeff[3 * kMuonMaxSteps];
};
// Matrices are symmetric: an operand's column is read for its row, so that lanes read side by side, and rows two apart use the same banks.
__device__ __forceinline__ int32_t few_at(int32_t r, int32_t c) { return r * kMuonFewSide + (c ^ ((r & 1) << 4)); }
__global__ __launch_bounds__(kFewThreads) void k_few_steps(Batch b, FewArgs a) {
    constexpr int kWaves = kFewThreads / LD_WAVE, kMine = (2 * kFewTiles + kWaves - 1) / kWaves;
    __shared__ double A[kMuonFewSide * kMuonFewSide], P[kMuonFewSide * kMuonFewSide], Q[kMuonFewSide * kMuonFewSide], R[kMuonFewSide * kMuonFewSide];
    const int32_t i = blockIdx.x, m = b.m[i], n = b.n[i], lane = ld_lane(), wave = threadIdx.x / LD_WAVE;
    if (b.kind[i] != kMuonFew) return;
    const int32_t bands = (m + kFewBand - 1) / kFewBand, tiles = bands * (bands + 1) / 2;
    const auto place = [](int32_t k, int32_t& u, int32_t& t) {  // tile k's bands, u <= t
        t = k < 1 ? 0 : k < 3 ? 1 : k < 6 ? 2 : 3;
        u = k - t * (t + 1) / 2;
    };
    const auto product = [&](const double* left, const double* right, int32_t k) {
        int32_t u, t;
        place(k, u, t);
        f64x4 acc = {};
        for (int32_t band = 0; band < bands; ++band) {
            double x[4], y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int32_t c = kFewBand * band + 4 * e + (lane >> 4);
                x[e] = left[few_at(c, kFewBand * u + (lane & 15))], y[e] = right[few_at(c, kFewBand * t + (lane & 15))];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f64_16x16x4f64(x[e], y[e], acc, 0, 0, 0);
        }
        return acc;
    };
    // f(value, row, column) of a tile's elements, to both sides of the diagonal
    const auto keep = [&](double* to, int32_t k, const f64x4& x, auto f) {
        int32_t u, t;
        place(k, u, t);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int32_t r = kFewBand * u + (lane >> 4) + 4 * q, c = kFewBand * t + (lane & 15);
            const double y = f(x[q], r, c);
            to[few_at(r, c)] = y;
            if (u != t) to[few_at(c, r)] = y;
        }
    };
    const auto same = [](double x, int32_t, int32_t) { return x; };

    const int32_t columns = few_columns(n), parts = (n + columns - 1) / columns;
    const double* sums = reinterpret_cast<const double*>(few_parts(b, i));
    for (int32_t k = wave; k < tiles; k += kWaves) {
        f64x4 x = {};
#pragma unroll 4
        for (int32_t p = 0; p < parts; ++p)
#pragma unroll
            for (int q = 0; q < 4; ++q) x[q] += sums[(static_cast<int64_t>(p) * kFewTiles + k) * kFewTile + q * LD_WAVE + lane];
        keep(A, k, x, same);
    }
    __syncthreads();
    double trace = lane < m ? A[few_at(lane, lane)] : 0.0;
    for (int d = LD_WAVE / 2; d > 0; d >>= 1) trace += __shfl_xor(trace, d);
    const double norm = sqrt(trace), f = norm == 0.0 ? 0.0 : 1.0 / (norm + static_cast<double>(a.eps));
    __syncthreads();
    for (int32_t e = threadIdx.x; e < bands * kFewBand * kMuonFewSide; e += kFewThreads) A[e] *= f * f;
    __syncthreads();
    for (int32_t step = 0; step < a.steps; ++step) {
        const bool first = step == 0, last = step + 1 == a.steps;
        const double ca = a.coeff[3 * step], cb = a.coeff[3 * step + 1], cc = a.coeff[3 * step + 2];
        for (int32_t k = wave; k < tiles; k += kWaves) {
            const auto poly = [&](double x, int32_t r, int32_t c) { return fma(cc, x, fma(cb, A[few_at(r, c)], r == c ? ca : 0.0)); };
            const f64x4 x = product(A, A, k);
            keep(P, k, x, poly);
            if (first) keep(Q, k, x, poly);
        }
        __syncthreads();
        f64x4 x[kMine];  // P A, then P Q, which takes Q's place when all have read it
#pragma unroll
        for (int j = 0; j < kMine; ++j) {
            const int32_t k = wave + j * kWaves;
            if (k < tiles && !last) x[j] = product(P, A, k);
            else if (k >= tiles && k < 2 * tiles && !first) x[j] = product(P, Q, k - tiles);
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kMine; ++j) {
            const int32_t k = wave + j * kWaves;
            if (k < tiles && !last) keep(R, k, x[j], same);
            else if (k >= tiles && k < 2 * tiles && !first) keep(Q, k - tiles, x[j], same);
        }
        __syncthreads();
        if (last) break;
        for (int32_t k = wave; k < tiles; k += kWaves) keep(A, k, product(P, R, k), same);
        __syncthreads();
    }
    double* out = reinterpret_cast<double*>(few_q(b, i));
    for (int32_t e = threadIdx.x; e < bands * kFewBand * kMuonFewSide; e += kFewThreads) out[e] = Q[few_at(e / kMuonFewSide, e % kMuonFewSide)] * f;
}

// Q U, which holds the norm: a wave takes 16 columns, a lane's at the eight rows that few_load takes side by side where U is transposed.
constexpr int kFewColumns = kThreads / LD_WAVE * kFewBand;
template <int DT, int OT>
__global__ __launch_bounds__(kThreads) void k_few_apply(Batch b, Source s, FinalArgs out) {
    __shared__ double Q[kMuonFewSide * kMuonFewSide];
    typedef typename LdElem<DT>::type elem;
    typedef typename LdElem<OT>::type out_elem;
    const int32_t i = blockIdx.y, m = b.m[i], n = b.n[i], lane = ld_lane(), wave = threadIdx.x / LD_WAVE;
    if (b.kind[i] != kMuonFew || static_cast<int32_t>(blockIdx.x) * kFewColumns >= n) return;
    const int32_t bands = (m + kFewBand - 1) / kFewBand;
    const double* q = reinterpret_cast<const double*>(few_q(b, i));
    const int32_t c = blockIdx.x * kFewColumns + wave * kFewBand + (lane & 15), flipped = b.flipped[i];
    const elem* src = static_cast<const elem*>(s.src[i]);
    const int64_t stride = s.stride[i];
    // rows 32 h + 8 (lane >> 4) + e of column c
    float x[kMuonFewSide / 32][8];
#pragma unroll
    for (int h = 0; h < kMuonFewSide / 32; ++h) {
        const int32_t k = 32 * h + 8 * (lane >> 4);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[h][e] = k + e < m && c < n ? static_cast<float>(flipped ? src[c * stride + k + e] : src[(k + e) * stride + c]) : 0.0f;
    }
    constexpr int kRowsAtOnce = kThreads / kMuonFewSide;
    for (int32_t band = 0; band < bands; ++band) {  // a band's loads side by side
        double y[kFewBand / kRowsAtOnce];
#pragma unroll
        for (int e = 0; e < kFewBand / kRowsAtOnce; ++e) y[e] = q[band * kFewBand * kMuonFewSide + e * kThreads + threadIdx.x];
#pragma unroll
        for (int e = 0; e < kFewBand / kRowsAtOnce; ++e)
            Q[few_at(band * kFewBand + e * kRowsAtOnce + threadIdx.x / kMuonFewSide, threadIdx.x % kMuonFewSide)] = y[e];
    }
    __syncthreads();
    out_elem* to = static_cast<out_elem*>(out.out[i]);
    const int64_t to_stride = out.stride[i];
#pragma unroll
    for (int t = 0; t < kFewBands; ++t) {
        if (t >= bands) break;
        f64x4 acc = {};
#pragma unroll
        for (int h = 0; h < kMuonFewSide / 32; ++h) {
            if (32 * h >= m) break;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int32_t k = 32 * h + 8 * (lane >> 4) + e;
                const double y = k < bands * kFewBand ? Q[few_at(k, kFewBand * t + (lane & 15))] : 0.0, z = static_cast<double>(x[h][e]);
                acc = flipped ? __builtin_amdgcn_mfma_f64_16x16x4f64(z, y, acc, 0, 0, 0) : __builtin_amdgcn_mfma_f64_16x16x4f64(y, z, acc, 0, 0, 0);
            }
        }
        // lanes along the rows of what is written
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const int32_t across = lane & 15, down = (lane >> 4) + 4 * w;
            const int32_t r = kFewBand * t + (flipped ? across : down), col = blockIdx.x * kFewColumns + wave * kFewBand + (flipped ? down : across);
            if (r < m && col < n) to[flipped ? col * to_stride + r : r * to_stride + col] = static_cast<out_elem>(static_cast<float>(acc[w]));
        }
    }
}

__device__ __forceinline__ void store_eight(float* p, const f32x8& x, int32_t n) {
    typedef typename LdVec<LD_F32, 4>::type half;
    if (n >= 8) {
        *reinterpret_cast<half*>(p) = __builtin_shufflevector(x, x, 0, 1, 2, 3);
        *reinterpret_cast<half*>(p + 4) = __builtin_shufflevector(x, x, 4, 5, 6, 7);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) p[e] = x[e];
    }
}

// Momentum of a window's steps, one after another, and every step's update and the sum of its squares.
struct MomentumArgs {
    float* momentum[kMost];
    const void* grad[kMost];   // of every problem
    int32_t problem[kMost];    // a matrix's first
    int32_t steps[kMost];      // and how many it has
    double* sums;
    float mu;
    int32_t nesterov;
};
constexpr int kTogether = 4;  // steps between which the momentum stays in registers
template <int DT>
__global__ __launch_bounds__(kThreads) void k_momentum(Batch b, MomentumArgs a) {
    __shared__ double sh[kThreads / LD_WAVE];
    typedef typename LdElem<DT>::type elem;
    const int32_t p0 = a.problem[blockIdx.y], steps = a.steps[blockIdx.y];
    const int64_t elems = static_cast<int64_t>(b.m[p0]) * b.n[p0];
    const int32_t parts = sum_parts(elems);
    if (static_cast<int32_t>(blockIdx.x) >= parts) return;
    float* momentum = a.momentum[blockIdx.y];
    const int64_t from = (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) * 8, step = static_cast<int64_t>(parts) * kThreads * 8;
    for (int32_t t0 = 0; t0 < steps; t0 += kTogether) {
        double sum[kTogether] = {};
        for (int64_t e = from; e < elems; e += step) {
            const int32_t n = elems - e < 8 ? static_cast<int32_t>(elems - e) : 8;
            f32x8 m = load_eight<LD_F32>(momentum + e, n), g[kTogether];
#pragma unroll
            for (int k = 0; k < kTogether; ++k)
                if (t0 + k < steps) g[k] = load_eight<DT>(static_cast<const elem*>(a.grad[p0 + t0 + k]) + e, n);
#pragma unroll
            for (int k = 0; k < kTogether; ++k) {
                if (t0 + k >= steps) break;
                f32x8 u;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    m[i] = __fmaf_rn(a.mu, m[i], g[k][i]);
                    u[i] = a.nesterov ? __fmaf_rn(a.mu, m[i], g[k][i]) : m[i];
                    if (i < n) sum[k] = fma(static_cast<double>(u[i]), static_cast<double>(u[i]), sum[k]);
                }
                store_eight(reinterpret_cast<float*>(buffer_of(b, p0 + t0 + k, kYT)) + e, u, n);
            }
            store_eight(momentum + e, m, n);
        }
#pragma unroll
        for (int k = 0; k < kTogether; ++k) {
            if (t0 + k >= steps) break;
            const double all = block_sum(sum[k], sh);
            if (threadIdx.x == 0) a.sums[(p0 + t0 + k) * kSumParts + blockIdx.x] = all;
        }
    }
}

struct UpdateArgs {
    float* w[kMost];
    int32_t problem[kMost], steps[kMost];
    float rate[kMost];         // lr times the matrix's scale
    float keep;                // 1 - lr wd
};
__global__ __launch_bounds__(kThreads) void k_update(Batch b, UpdateArgs a) {
    const int32_t p0 = a.problem[blockIdx.y], steps = a.steps[blockIdx.y];
    const int64_t elems = static_cast<int64_t>(b.m[p0]) * b.n[p0];
    float* w = a.w[blockIdx.y];
    for (int64_t e = (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) * 8; e < elems; e += static_cast<int64_t>(gridDim.x) * kThreads * 8) {
        const int32_t n = elems - e < 8 ? static_cast<int32_t>(elems - e) : 8;
        f32x8 x = load_eight<LD_F32>(w + e, n);
        for (int32_t t = 0; t < steps; ++t) {
            const f32x8 o = load_eight<LD_F32>(reinterpret_cast<const float*>(buffer_of(b, p0 + t, kX)) + e, n);
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = __fmaf_rn(-a.rate[blockIdx.y], o[k], x[k] * a.keep);
        }
        store_eight(w + e, x, n);
    }
}

// ------------------------------------------------------------------------------------------------------------------------ host

struct Polynomial {
    int32_t steps;
    float coeff[3 * kMuonMaxSteps];
    LdMuonBounds bounds;
};

// What a kind of matrices goes through, launch by launch.
struct Program {
    int32_t count;
    Plan plan[6 * kMuonMaxSteps];
};

bool polynomial(Polynomial& p, int32_t steps, const float* coeff) {
    if (steps < 0 || steps > kMuonMaxSteps) return false;
    p.steps = steps;
    for (int32_t s = 0; s < steps; ++s) {
        const float usual[3] = {3.4445f, -4.7750f, 2.0315f};
        for (int32_t k = 0; k < 3; ++k) p.coeff[3 * s + k] = coeff ? coeff[3 * s + k] : usual[k];
    }
    return ld_muon_bounds(p.bounds, steps, p.coeff);
}

bool known_sides(int64_t rows, int64_t cols) { return rows >= 0 && cols >= 0 && rows <= LD_MAX_SIDE && cols <= LD_MAX_SIDE; }

// Bytes that a group's partial sums take before its scratch.
constexpr int64_t kSumBytes = static_cast<int64_t>(kMost) * kSumParts * sizeof(double);

int64_t scratch_of(int64_t rows, int64_t cols) {
    const int64_t m = rows < cols ? rows : cols, n = rows < cols ? cols : rows;
    return (ld_muon_scratch(static_cast<int32_t>(m), static_cast<int32_t>(n)) + 255) / 256 * 256;
}

// Appends a problem, whose result goes to out_type; whether it still has room. The first always has.
bool append(Batch& b, int64_t& used, char* scratch, int64_t room, int64_t rows, int64_t cols, int32_t out_type) {
    const int64_t need = scratch_of(rows, cols);
    if (b.count == kMost || (b.count > 0 && used + need > room)) return false;
    const int32_t i = b.count++;
    b.base[i] = scratch + used;
    b.flipped[i] = rows > cols;
    b.m[i] = static_cast<int32_t>(rows > cols ? cols : rows);
    b.n[i] = static_cast<int32_t>(rows > cols ? rows : cols);
    b.kind[i] = b.m[i] <= kMuonFewSide ? kMuonFew : ld_muon_kind(b.m[i], b.n[i], out_type != LD_F32);
    used += need;
    return true;
}

// Bytes of the largest group of `repeats` problems of every matrix in turn; a group begins anew wherever one is full.
size_t workspace_of(const int64_t* rows, const int64_t* cols, int32_t n, int64_t repeats, size_t* least = nullptr) {
    if (least) *least = 0;
    int64_t most = 0, used = 0, count = 0;  // of the group that is filled
    for (int32_t i = 0; i < n; ++i) {
        if (rows[i] == 0 || cols[i] == 0) continue;
        const int64_t need = scratch_of(rows[i], cols[i]);
        if (least && repeats > 0 && static_cast<size_t>(kSumBytes + need) > *least) *least = static_cast<size_t>(kSumBytes + need);
        const auto room = [&]() {
            const int64_t fit = (kGroupBytes - used) / need;
            return count == 0 && fit < 1 ? 1 : fit < kMost - count ? fit : kMost - count;
        };
        int64_t left = repeats;
        while (left > 0) {
            int64_t fit = room();
            if (fit < 1) used = count = 0, fit = room();
            if (left > fit && count == 0) {  // whole groups of this matrix alone
                left -= (left - 1) / fit * fit;
                if (fit * need > most) most = fit * need;
            }
            const int64_t taken = left < fit ? left : fit;
            used += taken * need, count += taken, left -= taken;
            if (used > most) most = used;
        }
    }
    return most == 0 ? 0 : static_cast<size_t>(kSumBytes + most);
}

typedef Tile<64, 2, 2, 3> Small;
typedef Tile<128, 2, 2, 2> Middle;
typedef Tile<256, 2, 4, 2> Large;

void program_of(const Polynomial& p, int32_t kind, Program& out) {
    const auto scale = [](double bound) { return ld_muon_scale(bound); };
    const LdMuonBounds& b = p.bounds;
    int32_t begin[kMuonMaxSteps + 1];
    const int32_t runs = ld_muon_runs(b, p.steps, kind, begin);
    int32_t xt = kXT, other = kYT;
    out.count = 0;
    // X before a step is no larger than its bound, and than its first norm times what the steps before may have grown it by.
    const auto drop_of = [&](int32_t step) {
        const double grown = step == 0 ? 1.0 : ld_muon_grown(b, 0, step - 1);
        return step == 0 || grown <= b.x[step] ? 0 : static_cast<int32_t>(fmin(ceil(log2(grown / b.x[step])), kMostLift));
    };
    for (int32_t run = 0; run < runs; ++run) {
        const int32_t from = begin[run], to = begin[run + 1];
        const float sx = scale(b.x[from]);
        float sa = scale(b.x[from] * b.x[from]), sq = 0.0f;
        Plan gram = {};
        gram.prod[0] = {kX, kX, kA, 0};
        gram.products = 1, gram.long_sum = 1, gram.inv = 1.0f / (sx * sx), gram.scale[0] = sa, gram.drop = drop_of(from);
        out.plan[out.count++] = gram;
        int32_t q = kP, free_q = kQ0;
        for (int32_t step = from; step < to; ++step) {
            const bool first = step == from, last = step + 1 == to;
            const float sp = scale(b.p[step]), sr = scale(b.r[step]), new_sq = scale(ld_muon_grown(b, from, step));
            const int32_t poly = first && !last ? kQ1 : kP;  // the first P is the first Q, and is kept
            Plan a = {};
            a.prod[0] = {kA, kA, poly, 0};
            a.products = 1, a.poly = 1, a.inv = 1.0f / (sa * sa), a.scale[0] = sp;
            a.ca = p.coeff[3 * step], a.cb = p.coeff[3 * step + 1] / sa, a.cc = p.coeff[3 * step + 2];
            out.plan[out.count++] = a;
            // P A and P Q at once: their operands' scales differ, which the scale of what is kept takes up
            Plan next = {};
            next.inv = 1.0f;
            if (!last) {
                next.prod[next.products] = {poly, kA, kR, 0};
                next.scale[next.products++] = sr / (sp * sa);
            }
            if (!first) {
                next.prod[next.products] = {poly, q, free_q, 0};
                next.scale[next.products++] = new_sq / (sp * sq);
            }
            if (next.products > 0) out.plan[out.count++] = next;
            if (first) {
                q = poly, sq = sp;
            } else {
                const int32_t was = q;
                q = free_q, free_q = was, sq = new_sq;
            }
            if (last) continue;
            const float new_sa = scale(b.x[step + 1] * b.x[step + 1]);
            Plan g = {};
            g.prod[0] = {poly, kR, kA, 0};
            g.products = 1, g.inv = 1.0f / (sp * sr), g.scale[0] = new_sa;
            out.plan[out.count++] = g;
            sa = new_sa;
        }
        Plan a = {};
        a.prod[0] = {q, xt, kX, other};
        a.products = 1, a.apply = 1, a.inv = 1.0f / (sq * sx), a.drop = drop_of(from);
        if (run + 1 == runs) a.final = 1, a.out_drop = kMostLift;
        else a.scale[0] = scale(b.x[to]), a.out_drop = drop_of(to);
        out.plan[out.count++] = a;
        const int32_t was = xt;
        xt = other, other = was;
    }
}

// All steps of a group whose X is laid out. Matrices of different kinds go through their programs side by side, a launch for all whose next is of
// a sort: first those that multiply X, then those that are symmetric; who comes to the last first waits.
ld_status run_steps(Batch& b, const Polynomial& p, const FinalArgs& out, int32_t out_type, hipStream_t s) {
    Program prog[kMuonKinds];
    int32_t at[kMuonKinds] = {};
    for (int32_t k = 0; k < kMuonKinds; ++k) prog[k].count = 0;
    for (int32_t i = 0; i < b.count; ++i)
        if (b.kind[i] != kMuonFew && prog[b.kind[i]].count == 0) program_of(p, b.kind[i], prog[b.kind[i]]);
    const auto launch_as = [&](auto tile, const Plans& a) {
        typedef decltype(tile) T;
        bool apply = false, final = false;
        for (const Plan& plan : a.of) apply |= plan.apply != 0, final |= plan.final != 0;
        int32_t tiles = 0;
        for (int32_t i = 0; i < b.count; ++i) {
            b.first[i] = tiles;
            const int32_t down = tiles_of(ld_muon_padded(b.m[i]), T::SIDE), across = tiles_of(ld_muon_padded(b.n[i]), T::SIDE);
            tiles += a.of[b.kind[i]].products * (apply ? down * across : down * (down + 1) / 2);
        }
        for (int32_t i = b.count; i <= kMost; ++i) b.first[i] = tiles;
        const dim3 grid((tiles + 7) / 8 * 8), threads(T::THREADS);
        if (!apply) k_symmetric<T><<<grid, threads, 0, s>>>(b, a);
        else if (final) ld_with_type(out_type, [&](auto type) { k_apply<T, true, type><<<grid, threads, 0, s>>>(b, a, out); });
        else k_apply<T, false, LD_F32><<<grid, threads, 0, s>>>(b, a, out);
        return ld_launch_status();
    };
    // Which tile: the one that is done first, by fits to what launches of 1 to 64 square matrices of 64 to 4096 took (us; within some 10 %).
    // x: tiles a CU has; a block: 32 columns. A CU works on one tile of 256, two of 128, three of 64. (4096 x 4096, one and four of
    // them, A^2: 320 and 1200 by 64, 271 and 837 by 128, 298 and 920 by 256; six: 1841, 1256, 1280. 768 x 768, one and 32: 13 and 71, 26 and
    // 73, 64 and 79. Tiles of 32, each wave for itself, were no faster than 64 for any.)
    const auto launch = [&](const Plans& a) {
        bool apply = false;
        for (const Plan& plan : a.of) apply |= plan.apply != 0;
        const int32_t sides[3] = {64, 128, 256};
        double best = 0.0;
        int32_t side = 0;
        for (int32_t k = 0; k < 3; ++k) {
            double tiles = 0.0, all_blocks = 0.0;
            for (int32_t i = 0; i < b.count; ++i) {
                const Plan& plan = a.of[b.kind[i]];
                const int32_t down = tiles_of(ld_muon_padded(b.m[i]), sides[k]), across = tiles_of(ld_muon_padded(b.n[i]), sides[k]);
                const double mine = static_cast<double>(plan.products) * (apply ? static_cast<double>(down) * across : 0.5 * down * (down + 1.0));
                tiles += mine, all_blocks += mine * (ld_muon_padded(plan.long_sum ? b.n[i] : b.m[i]) / kMuonBlock);
            }
            const double blocks = all_blocks / tiles, x = tiles / kCUs, rounds = ceil(x);
            const double time = sides[k] == 256 ? 10.0 + rounds * (6.0 + 2.4 * blocks)
                                : sides[k] == 128 ? 8.0 + blocks * fmax(0.87, 0.73 * x + 0.45) : 5.0 + blocks * fmax(0.34, 0.28 * x + 0.1);
            if (k == 0 || time < best) best = time, side = sides[k];
        }
        return side == 256 ? launch_as(Large(), a) : side == 128 ? launch_as(Middle(), a) : launch_as(Small(), a);
    };
    for (;;) {
        const auto sort_of = [](const Plan& plan) { return plan.final ? 0 : plan.apply ? 2 : 1; };
        int32_t sort = -1;
        for (int32_t k = 0; k < kMuonKinds; ++k)
            if (at[k] < prog[k].count && sort_of(prog[k].plan[at[k]]) > sort) sort = sort_of(prog[k].plan[at[k]]);
        if (sort < 0) return LD_OK;
        Plans plans = {};
        for (int32_t k = 0; k < kMuonKinds; ++k)
            if (at[k] < prog[k].count && sort_of(prog[k].plan[at[k]]) == sort) plans.of[k] = prog[k].plan[at[k]++];
        if (launch(plans) != LD_OK) return LD_ERR_HIP;
    }
}

bool has(const Batch& b, bool few) {
    for (int32_t i = 0; i < b.count; ++i)
        if ((b.kind[i] == kMuonFew) == few) return true;
    return false;
}

int32_t most_parts(const Batch& b) {
    int32_t most = 1;
    for (int32_t i = 0; i < b.count; ++i) {
        const int32_t parts = sum_parts(static_cast<int64_t>(b.m[i]) * b.n[i]);
        if (parts > most) most = parts;
    }
    return most;
}

// All of a group but its updates' squares, which `source` has the sums of.
ld_status orthogonalize_group(Batch& b, const Source& src, int32_t dtype, const Polynomial& p, const FinalArgs& out, int32_t out_type, hipStream_t s) {
    int32_t tiles = 1, parts = 1, columns = 1;
    for (int32_t i = 0; i < b.count; ++i) {
        const auto most = [](int32_t& x, int32_t y) { x = y > x ? y : x; };
        if (b.kind[i] == kMuonFew) most(parts, tiles_of(b.n[i], few_columns(b.n[i]))), most(columns, tiles_of(b.n[i], kFewColumns));
        else most(tiles, tiles_of(b.m[i], kMuonPad) * tiles_of(b.n[i], kMuonPad));
    }
    if (has(b, true)) {
        FewArgs a = {};
        a.steps = p.steps, a.eps = src.eps;
        memcpy(a.coeff, p.coeff, sizeof(a.coeff));
        ld_with_type(dtype, [&](auto type) { k_few_gram<type><<<dim3(parts, b.count), dim3(kThreads), 0, s>>>(b, src); });
        k_few_steps<<<dim3(b.count), dim3(kFewThreads), 0, s>>>(b, a);
        ld_with_type(dtype, [&](auto type) {
            ld_with_type(out_type, [&](auto to) { k_few_apply<type, to><<<dim3(columns, b.count), dim3(kThreads), 0, s>>>(b, src, out); });
        });
        if (ld_launch_status() != LD_OK) return LD_ERR_HIP;
    }
    if (!has(b, false)) return LD_OK;
    ld_with_type(dtype, [&](auto type) { k_lay_out<type><<<dim3(tiles, b.count), dim3(kThreads), 0, s>>>(b, src, ld_muon_scale(p.bounds.x[0])); });
    if (ld_launch_status() != LD_OK) return LD_ERR_HIP;
    return run_steps(b, p, out, out_type, s);
}

}  // namespace

extern "C" size_t ld_orthogonalize_workspace(const int64_t* rows, const int64_t* cols, int32_t n_mats) {
    if (!rows || !cols || n_mats < 0 || n_mats > LD_MAX_TENSORS) return 0;
    for (int32_t i = 0; i < n_mats; ++i)
        if (!known_sides(rows[i], cols[i])) return 0;
    return workspace_of(rows, cols, n_mats, 1);
}

extern "C" ld_status ld_orthogonalize(const void* const* src, const int64_t* src_stride, void* const* dst, const int64_t* dst_stride, const int64_t* rows,
                                      const int64_t* cols, int32_t n_mats, int32_t dtype, int32_t out_dtype, int32_t steps, const float* coeff,
                                      float eps, void* workspace, size_t workspace_bytes, ld_stream stream) {
    if (n_mats < 0 || n_mats > LD_MAX_TENSORS || !ld_known_type(dtype) || !ld_known_type(out_dtype) || steps < 1 || !(eps >= 0.0f && eps <= 1e30f))
        return LD_ERR_RANGE;
    if (n_mats > 0 && (!src || !dst || !rows || !cols)) return LD_ERR_NULL;
    Polynomial p;
    if (!polynomial(p, steps, coeff)) return LD_ERR_RANGE;
    for (int32_t i = 0; i < n_mats; ++i) {
        if (!known_sides(rows[i], cols[i])) return LD_ERR_RANGE;
        if (rows[i] == 0 || cols[i] == 0) continue;
        if ((src_stride && src_stride[i] < 0) || (dst_stride && dst_stride[i] < cols[i])) return LD_ERR_RANGE;
        if (!src[i] || !dst[i]) return LD_ERR_NULL;
        if (!ld_aligned(src[i], ld_type_bytes(dtype)) || !ld_aligned(dst[i], ld_type_bytes(out_dtype))) return LD_ERR_ALIGN;
    }
    size_t need;  // of one problem at a time
    if (workspace_of(rows, cols, n_mats, 1, &need) == 0) return LD_OK;
    if (!workspace || !ld_aligned(workspace, 256) || workspace_bytes < need) return LD_ERR_WORKSPACE;
    ld_begin_call();
    hipStream_t s = static_cast<hipStream_t>(stream);
    char* scratch = static_cast<char*>(workspace) + kSumBytes;
    const int64_t room_bytes = static_cast<int64_t>(workspace_bytes < (static_cast<size_t>(1) << 62) ? workspace_bytes : static_cast<size_t>(1) << 62) - kSumBytes;
    for (int32_t i = 0; i < n_mats;) {
        Batch b = {};
        Source source = {};
        FinalArgs out = {};
        int64_t used = 0;
        for (; i < n_mats; ++i) {
            if (rows[i] == 0 || cols[i] == 0) continue;
            if (!append(b, used, scratch, room_bytes, rows[i], cols[i], out_dtype)) break;
            source.src[b.count - 1] = src[i], source.stride[b.count - 1] = src_stride ? src_stride[i] : cols[i];
            out.out[b.count - 1] = dst[i], out.stride[b.count - 1] = dst_stride ? dst_stride[i] : cols[i];
        }
        if (b.count == 0) break;
        source.sums = static_cast<double*>(workspace), source.eps = eps;
        if (has(b, false)) ld_with_type(dtype, [&](auto type) { k_squares<type><<<dim3(most_parts(b), b.count), dim3(kThreads), 0, s>>>(b, source); });
        if (ld_launch_status() != LD_OK || orthogonalize_group(b, source, dtype, p, out, out_dtype, s) != LD_OK) return LD_ERR_HIP;
    }
    return LD_OK;
}

extern "C" size_t ld_merge_dense_muon_workspace(const int64_t* rows, const int64_t* cols, int32_t n_mats, int32_t W) {
    if (!rows || !cols || n_mats < 0 || n_mats > LD_MAX_TENSORS || W < 0 || W > LD_MAX_WINDOW) return 0;
    for (int32_t i = 0; i < n_mats; ++i)
        if (!known_sides(rows[i], cols[i])) return 0;
    return workspace_of(rows, cols, n_mats, W);
}

extern "C" ld_status ld_merge_dense_muon(float* const* w, float* const* m, const void* const* grad, const int64_t* rows, const int64_t* cols, int32_t n_mats,
                                         int32_t W, int32_t dtype, float lr, float mu, int32_t nesterov, float weight_decay, const float* scale,
                                         int32_t steps, const float* coeff, float eps, void* workspace, size_t workspace_bytes, ld_stream stream) {
    if (n_mats < 0 || n_mats > LD_MAX_TENSORS || W < 0 || W > LD_MAX_WINDOW || !ld_known_type(dtype) || steps < 1 || !(eps >= 0.0f && eps <= 1e30f) ||
        !(fabsf(lr) <= 1e30f) || !(fabsf(mu) <= 1e30f) || !(fabsf(weight_decay) <= 1e30f))
        return LD_ERR_RANGE;
    if (n_mats > 0 && W > 0 && (!w || !m || !grad || !rows || !cols)) return LD_ERR_NULL;
    Polynomial p;
    if (!polynomial(p, steps, coeff)) return LD_ERR_RANGE;
    if (n_mats == 0 || W == 0) return LD_OK;
    for (int32_t i = 0; i < n_mats; ++i) {
        if (!known_sides(rows[i], cols[i]) || (scale && !(fabsf(scale[i]) <= 1e30f))) return LD_ERR_RANGE;
        if (rows[i] == 0 || cols[i] == 0) continue;
        if (!w[i] || !m[i]) return LD_ERR_NULL;
        if (!ld_aligned(w[i], 4) || !ld_aligned(m[i], 4)) return LD_ERR_ALIGN;
        for (int32_t t = 0; t < W; ++t) {
            const void* g = grad[static_cast<int64_t>(t) * n_mats + i];
            if (!g) return LD_ERR_NULL;
            if (!ld_aligned(g, ld_type_bytes(dtype))) return LD_ERR_ALIGN;
        }
    }
    size_t need;  // of one problem at a time
    if (workspace_of(rows, cols, n_mats, W, &need) == 0) return LD_OK;
    if (!workspace || !ld_aligned(workspace, 256) || workspace_bytes < need) return LD_ERR_WORKSPACE;
    ld_begin_call();
    hipStream_t s = static_cast<hipStream_t>(stream);
    char* scratch = static_cast<char*>(workspace) + kSumBytes;
    const int64_t room_bytes = static_cast<int64_t>(workspace_bytes < (static_cast<size_t>(1) << 62) ? workspace_bytes : static_cast<size_t>(1) << 62) - kSumBytes;
    int32_t i = 0, t = 0;  // the next problem
    while (i < n_mats) {
        Batch b = {};
        MomentumArgs mom = {};
        UpdateArgs up = {};
        Source source = {};
        FinalArgs out = {};
        int64_t used = 0;
        int32_t mats = 0;
        for (bool room = true; room && i < n_mats;) {
            if (rows[i] == 0 || cols[i] == 0) {
                ++i;
                continue;
            }
            const int32_t from = t;
            for (; t < W && (room = append(b, used, scratch, room_bytes, rows[i], cols[i], LD_F32)); ++t) {
                const int32_t k = b.count - 1;
                mom.grad[k] = grad[static_cast<int64_t>(t) * n_mats + i];
                source.stride[k] = out.stride[k] = cols[i];
            }
            if (t > from) {
                mom.momentum[mats] = m[i], up.w[mats] = w[i];
                mom.problem[mats] = up.problem[mats] = b.count - (t - from);
                mom.steps[mats] = up.steps[mats] = t - from;
                const double s = scale ? static_cast<double>(scale[i]) : rows[i] > cols[i] ? sqrt(static_cast<double>(rows[i]) / cols[i]) : 1.0;
                up.rate[mats++] = static_cast<float>(static_cast<double>(lr) * s);
            }
            if (t == W) ++i, t = 0;
        }
        if (mats == 0) break;
        for (int32_t k = 0; k < b.count; ++k) {
            const int64_t large = ld_muon_large(b.m[k], b.n[k]);
            source.src[k] = b.base[k] + kYT * large;  // the update lies there until X is laid out
            out.out[k] = b.base[k] + kX * large;
        }
        source.sums = mom.sums = static_cast<double*>(workspace), source.eps = eps;
        mom.mu = mu, mom.nesterov = nesterov;
        up.keep = static_cast<float>(1.0 - static_cast<double>(lr) * static_cast<double>(weight_decay));
        const dim3 grid(most_parts(b), mats);
        ld_with_type(dtype, [&](auto type) { k_momentum<type><<<grid, dim3(kThreads), 0, s>>>(b, mom); });
        if (ld_launch_status() != LD_OK || orthogonalize_group(b, source, LD_F32, p, out, LD_F32, s) != LD_OK) return LD_ERR_HIP;
        k_update<<<dim3(4 * most_parts(b), mats), dim3(kThreads), 0, s>>>(b, up);
        if (ld_launch_status() != LD_OK) return LD_ERR_HIP;
    }
    return LD_OK;
}
