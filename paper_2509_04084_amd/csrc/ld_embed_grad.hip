// The embedding's gradient from the gradient of its rows: the lookup's backward pass.
//
//   grad[v, c] = round(beta * grad[v, c] + scale * sum of dout[t, c] over the tokens t with id_t = v),  beta = 0 or 1
//
// The tokens are sorted by their id first (stable), so that a row's are next to one another and in order: every sum is made in an
// order that the ids and sizes alone decide, without float atomics. What the same batch gives is the same bit for bit, as error
// feedback and a recovery that replays differentials need it.
//
// Bound by memory where there are many tokens or rows to clear (16384 tokens of GPT-2 XL, 375 MB, 81 us; 65536 at Llama's width, 800 MB,
// 191 us, of which the sum of the rows 156 at 5.2 TB/s), else by what waits on one another: the sort's launches of 4 to 11 us each (16384
// tokens of GPT-2 XL's positions, 59 MB, 27 us), the two or three reads between an id and its row.
#include <type_traits>

#include "ld_elem.h"
#include "ld_grid.h"

namespace {

// A lane's value, in every lane.
__device__ __forceinline__ uint32_t lane_of(uint32_t x, int32_t lane) {
    return static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(x), lane));
}

// The columns of a lane: N from `column` on, of which the last `own` are its own. In the row's last vector, which ends with the
// row, the first are the lane's before (their sums are made twice and written once). Rows have N columns at least, but where they are
// only cleared.
struct Columns {
    int32_t column, own;
};

template <int N>
__device__ __forceinline__ Columns columns_of(int32_t vector, int32_t d) {
    const int32_t begin = vector * N, left = d - begin;
    return {left >= N ? begin : d - N, left >= N ? N : left > 0 ? left : 0};
}

template <int DT, int N, bool STREAM>
__device__ __forceinline__ typename LdVec<DT, N>::type load_columns(const typename LdElem<DT>::type* row, Columns c) {
    const typename LdVec<DT, N>::type* p = reinterpret_cast<const typename LdVec<DT, N>::type*>(row + c.column);
    return STREAM ? __builtin_nontemporal_load(p) : *p;
}

template <int DT, int N, bool STREAM>
__device__ __forceinline__ void store_columns(typename LdElem<DT>::type* row, Columns c, typename LdVec<DT, N>::type x) {
    if (c.own == N) {
        if (STREAM) __builtin_nontemporal_store(x, reinterpret_cast<typename LdVec<DT, N>::type*>(row + c.column));
        else *reinterpret_cast<typename LdVec<DT, N>::type*>(row + c.column) = x;
    } else {
#pragma unroll
        for (int e = 1; e < N; ++e)
            if (e >= N - c.own) row[c.column + e] = x[e];
    }
}

// Rows cleared by workgroups that a launch of the sort has besides its own: what the chip has to spare there.
struct Clearing {
    void* grad;
    int64_t stride;
    int32_t d, wide;     // wide: elements of four bytes, else two
    int32_t from, rows;  // rows [from, from + rows)
};

template <int DT>
__device__ __forceinline__ void clear_span(const Clearing& c, int32_t wave, int32_t waves) {
    constexpr int N = DT == LD_F32 ? 4 : 8;
    for (int32_t r = wave; r < c.rows; r += waves) {
        typename LdElem<DT>::type* row = static_cast<typename LdElem<DT>::type*>(c.grad) + static_cast<int64_t>(c.from + r) * c.stride;
        for (int32_t l = ld_lane(); l * N < c.d; l += LD_WAVE)
            store_columns<DT, N, true>(row, columns_of<N>(l, c.d), typename LdVec<DT, N>::type(0));
    }
}

// Bytes that a launch of the sort clears: about what is written in its time. GPT-2 XL's 16 K tokens without it 97.7 us, with 16 MB 89.5,
// 32 MB 86.8, 48 MB 88.8. Rows that tokens name are written twice so: at Llama's width 65 K tokens of 32 K rows 182 and 192 us; it is done
// where there are fewer tokens than rows. The launch that sorts 2049 to 4096 tokens alone takes as long as two: 4096 tokens of GPT-2 XL with 32 MB
// 78 us, with 64 MB 72 (2048 tokens 70 either way).
constexpr int64_t kHidden = 32 << 20;

// Whether a workgroup is one of those, its work then done.
__device__ __forceinline__ bool cleared(const Clearing& c, int32_t own_blocks) {
    const int32_t block = static_cast<int32_t>(blockIdx.x) - own_blocks;
    if (block < 0) return false;
    const int32_t per = blockDim.x / LD_WAVE, wave = block * per + threadIdx.x / LD_WAVE;
    const int32_t waves = (static_cast<int32_t>(gridDim.x) - own_blocks) * per;
    if (c.wide) clear_span<LD_F32>(c, wave, waves);
    else clear_span<LD_BF16>(c, wave, waves);
    return true;
}

// ------------------------------------------------------------------ sort

// Least significant digit first, and stable. A workgroup finds the rank of its tokens among those of the same digit: a wave takes 64
// consecutive tokens a round, the lanes of equal digits found by a vote on each bit, and counts what it has had of a digit in shared
// memory; then the waves' counts are added up.
constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / LD_WAVE;

struct SortArgs {
    const void* ids;         // the first digit's input, else NULL
    int32_t wide_ids;
    const uint32_t* keys_in;
    const uint32_t* at_in;
    uint32_t* keys_out;
    uint32_t* at_out;
    uint32_t* counts;        // [tiles][1 << bits]
    int64_t V;
    int32_t T, tiles, per_tile, shift, bits;
};

// A token's key: its id, or V for one that names no row.
__device__ __forceinline__ uint32_t key_of(const SortArgs& a, int32_t i) {
    if (!a.ids) return a.keys_in[i];
    const int64_t id = a.wide_ids ? static_cast<const int64_t*>(a.ids)[i] : static_cast<const int32_t*>(a.ids)[i];
    return static_cast<uint32_t>(id >= 0 && id < a.V ? id : a.V);
}

// A wave's counts cleared, 16 bytes a lane.
__device__ __forceinline__ void clear_counts(uint16_t* seen, int32_t bins) {
    for (int32_t i = 8 * ld_lane(); i < bins; i += 8 * LD_WAVE) __builtin_memset(__builtin_assume_aligned(seen + i, 16), 0, 16);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// The token's place among those of its digit that its wave has had, `seen` (a count for each digit) being moved on.
__device__ __forceinline__ uint32_t rank_in_wave(uint32_t digit, bool in, int32_t bits, uint16_t* seen) {
    const uint64_t valid = __ballot(in);
    uint32_t lo = static_cast<uint32_t>(valid), hi = static_cast<uint32_t>(valid >> 32);
    for (int32_t b = 0; b < bits; ++b) {
        const uint32_t mine = static_cast<uint32_t>(static_cast<int32_t>(digit << (31 - b)) >> 31);  // the bit, in every place
        const uint64_t set = __ballot(mine != 0);
        lo &= ~(static_cast<uint32_t>(set) ^ mine);
        hi &= ~(static_cast<uint32_t>(set >> 32) ^ mine);
    }
    const uint64_t same = static_cast<uint64_t>(hi) << 32 | lo;
    const uint32_t below = ld_mbcnt(same);
    uint32_t before = 0;
    if (in) before = seen[digit];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (in && below == 0) seen[digit] = static_cast<uint16_t>(before + __popcll(same));
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    return before + below;
}

// A workgroup's exclusive scan of a value a thread; `sh` holds a word for each wave.
__device__ __forceinline__ uint32_t block_escan(uint32_t x, uint32_t* sh) {
    const uint32_t upto = ld_wave_iscan(x);
    const int32_t wave = threadIdx.x / LD_WAVE;
    if (ld_lane() == LD_WAVE - 1) sh[wave] = upto;
    __syncthreads();
    uint32_t from = upto - x;
    for (int w = 0; w < wave; ++w) from += sh[w];
    return from;
}

// Up to 1024 * ROUNDS tokens: all digits by one workgroup, the tokens staying in registers and shared memory. 1024 tokens 5.3 us, 4096 9.8
// (as tiles 17 to 21); 8192 would be 23 (as tiles 19), the vector units of the one compute unit being busy with the votes.
constexpr int kAloneBits = 9;                 // most bits of a digit
constexpr int kAloneBins = 1 << kAloneBits;
constexpr int kAloneMost = 4 * kSortThreads;

template <int ROUNDS>
struct SortShared {
    uint32_t keys[ROUNDS * kSortThreads];
    uint16_t tokens[ROUNDS * kSortThreads];
    __attribute__((aligned(16))) uint16_t seen[kSortWaves][kAloneBins];
    uint32_t first[kAloneBins], sh[kSortWaves];
};

// Leaves the sorted keys and tokens in shared memory.
template <int ROUNDS>
__device__ __forceinline__ void sort_in_shared(const SortArgs& a, int32_t passes, SortShared<ROUNDS>& m) {
    const int32_t bins = 1 << a.bits, wave = threadIdx.x / LD_WAVE, base = wave * (LD_WAVE * ROUNDS) + ld_lane();
    uint32_t key[ROUNDS], at[ROUNDS], rank[ROUNDS];
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const int32_t i = base + r * LD_WAVE;
        key[r] = i < a.T ? key_of(a, i) : 0;
        at[r] = i;
    }
    for (int32_t p = 0; p < passes; ++p) {
        const int32_t shift = p * a.bits;
        clear_counts(m.seen[wave], bins);
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r)
            rank[r] = rank_in_wave((key[r] >> shift) & (bins - 1), base + r * LD_WAVE < a.T, a.bits, m.seen[wave]);
        __syncthreads();
        uint32_t total = 0;
        const int32_t b = threadIdx.x;
        if (b < bins) {
#pragma unroll
            for (int w = 0; w < kSortWaves; ++w) {
                const uint32_t c = m.seen[w][b];
                m.seen[w][b] = static_cast<uint16_t>(total);
                total += c;
            }
        }
        const uint32_t from = block_escan(total, m.sh);
        if (b < bins) m.first[b] = from;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            if (base + r * LD_WAVE < a.T) {
                const uint32_t digit = (key[r] >> shift) & (bins - 1), to = m.first[digit] + m.seen[wave][digit] + rank[r];
                m.keys[to] = key[r];
                m.tokens[to] = static_cast<uint16_t>(at[r]);
            }
        }
        __syncthreads();
        if (p + 1 == passes) break;
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            const int32_t i = base + r * LD_WAVE;
            if (i < a.T) {
                key[r] = m.keys[i];
                at[r] = m.tokens[i];
            }
        }
    }
}

template <int ROUNDS>
__global__ __launch_bounds__(kSortThreads) void k_sort_alone(SortArgs a, int32_t passes, Clearing c) {
    __shared__ SortShared<ROUNDS> m;
    if (cleared(c, 1)) return;
    sort_in_shared<ROUNDS>(a, passes, m);
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const int32_t i = r * kSortThreads + threadIdx.x;
        if (i < a.T) {
            a.keys_out[i] = m.keys[i];
            a.at_out[i] = m.tokens[i];
        }
    }
}

// More tokens, two launches a digit: every tile counts its digits, then finds from all tiles' counts where each of its digits goes
// and moves its tokens there. A tile is 2048 tokens, or as many times that as keep the tiles at 256. (16384 tokens of 16 bits 21.7 us, in
// tiles of 4096 27.4, of 1024 19.6; 262,144 35.7, 35.5 and 45.2. Tiles that count all tokens themselves, without the launch before: no
// faster at 16384, slower beyond.)
constexpr int kSortRounds = 2;
constexpr int kTile = kSortThreads * kSortRounds;
constexpr int kMostTiles = 256;
constexpr int kDigitBits = 11;
constexpr int kBins = 1 << kDigitBits;

__global__ __launch_bounds__(kSortThreads) void k_sort_count(SortArgs a, Clearing c) {
    __shared__ uint32_t count[kBins];
    const int32_t bins = 1 << a.bits, base = blockIdx.x * a.per_tile;
    if (cleared(c, a.tiles)) return;
    for (int32_t i = threadIdx.x; i < bins; i += kSortThreads) count[i] = 0;
    __syncthreads();
    for (int32_t j = 0; j < a.per_tile && base + j < a.T; j += kTile) {
#pragma unroll
        for (int r = 0; r < kSortRounds; ++r) {
            const int32_t i = base + j + r * kSortThreads + threadIdx.x;
            if (i < a.T) atomicAdd(&count[(key_of(a, i) >> a.shift) & (bins - 1)], 1u);
        }
    }
    __syncthreads();
    for (int32_t i = threadIdx.x; i < bins; i += kSortThreads) a.counts[static_cast<size_t>(blockIdx.x) * bins + i] = count[i];
}

__global__ __launch_bounds__(kSortThreads) void k_sort_move(SortArgs a, Clearing c) {
    constexpr int kPer = kBins / kSortThreads, kLoads = 8;
    __shared__ uint32_t first[kBins];                // where this tile's next tokens of a digit go
    __shared__ __attribute__((aligned(16))) uint16_t seen[kSortWaves][kBins];
    __shared__ uint32_t part_before[kBins], part_all[kBins], sh[kSortWaves];
    const int32_t bins = 1 << a.bits, wave = threadIdx.x / LD_WAVE;
    const uint32_t mask = bins - 1;

    if (cleared(c, a.tiles)) return;
    // a digit's tokens in the tiles before this one, and in all of them: with fewer digits than threads the tiles are shared out
    const int32_t parts = bins < kSortThreads ? kSortThreads / bins : 1;
    for (int32_t i = threadIdx.x; i < bins * parts; i += kSortThreads) {
        const int32_t b = i & mask, part = i >> a.bits;
        uint32_t before = 0, all = 0;
        for (int32_t t0 = part; t0 < a.tiles; t0 += parts * kLoads) {
            uint32_t c[kLoads];
#pragma unroll
            for (int u = 0; u < kLoads; ++u) {
                const int32_t t = t0 + u * parts;
                c[u] = t < a.tiles ? a.counts[static_cast<size_t>(t) * bins + b] : 0;
            }
#pragma unroll
            for (int u = 0; u < kLoads; ++u) {
                all += c[u];
                if (t0 + u * parts < static_cast<int32_t>(blockIdx.x)) before += c[u];
            }
        }
        part_before[i] = before;
        part_all[i] = all;
    }
    __syncthreads();
    uint32_t before[kPer], all[kPer], sum = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int32_t b = threadIdx.x * kPer + j;
        before[j] = all[j] = 0;
        if (b < bins) {
            for (int32_t p = 0; p < parts; ++p) {
                before[j] += part_before[(p << a.bits) + b];
                all[j] += part_all[(p << a.bits) + b];
            }
        }
        sum += all[j];
    }
    uint32_t from = block_escan(sum, sh);
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int32_t b = threadIdx.x * kPer + j;
        if (b < bins) first[b] = from + before[j];
        from += all[j];
    }

    for (int32_t j = 0; j < a.per_tile; j += kTile) {
        const int32_t begin = blockIdx.x * a.per_tile + j;
        if (begin >= a.T) return;
        const int32_t base = begin + wave * (LD_WAVE * kSortRounds) + ld_lane();
        uint32_t key[kSortRounds], at[kSortRounds], rank[kSortRounds];
#pragma unroll
        for (int r = 0; r < kSortRounds; ++r) {
            const int32_t i = base + r * LD_WAVE;
            key[r] = i < a.T ? key_of(a, i) : 0;
            at[r] = i < a.T && a.at_in ? a.at_in[i] : static_cast<uint32_t>(i);
        }
        clear_counts(seen[wave], bins);
#pragma unroll
        for (int r = 0; r < kSortRounds; ++r) rank[r] = rank_in_wave((key[r] >> a.shift) & mask, base + r * LD_WAVE < a.T, a.bits, seen[wave]);
        __syncthreads();
        uint32_t moved[kPer];
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            const int32_t b = threadIdx.x + k * kSortThreads;
            moved[k] = 0;
            if (b < bins) {
#pragma unroll
                for (int w = 0; w < kSortWaves; ++w) {
                    const uint32_t c = seen[w][b];
                    seen[w][b] = static_cast<uint16_t>(moved[k]);
                    moved[k] += c;
                }
            }
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kSortRounds; ++r) {
            if (base + r * LD_WAVE < a.T) {
                const uint32_t digit = (key[r] >> a.shift) & mask, to = first[digit] + seen[wave][digit] + rank[r];
                a.keys_out[to] = key[r];
                a.at_out[to] = at[r];
            }
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            const int32_t b = threadIdx.x + k * kSortThreads;
            if (b < bins) first[b] += moved[k];
        }
        // the next round's counts are cleared and made by their own waves; its barrier is before `first` is read
    }
}

// ------------------------------------------------------------------- rows

// The sorted tokens are cut into chunks of 4 to 32, a wave for each chunk and block of columns. It adds up, one after the other,
// the runs of equal ids that begin in its chunk, to their ends where it can see them (in a window of 16 to 64 tokens from the
// chunk's first on), and writes their rows. A run that goes on further is long: every chunk that it touches leaves a partial sum,
// and k_join adds those up. Rows that no token names are cleared by workgroups of the same launch.
constexpr int kRowThreads = 256;
constexpr int kRowWaves = kRowThreads / LD_WAVE;
// Tokens whose rows a wave loads before it adds the first; where sums are added to what is there, the rows of grad that they end in with
// them. (Read when a run is done instead, one after the other: 16 K tokens of GPT-2 XL added 63 us instead of 58. 12 or 16 tokens: 85 -> 92 us
// without adding.)
constexpr int kAhead = 8;
constexpr int kClearRows = 4;     // rows that a clearing workgroup looks after (16: GPT-2 XL 102 us instead of 97)
// dout past the 256 MB that the last cache holds is read around it. GPT-2 XL's 52 MB (three batches in turn) 108 us from the cache, 124
// around it; 537 MB of bf16 at Llama's width 217 and 210, all of one id 269 and 222. Finished rows are always written around it, partial
// sums never (one id 285 us).
constexpr int64_t kStreamed = 256 << 20;
constexpr int kJoinWaves = 8;     // chunks of a joining workgroup
constexpr int kJoinAlone = 8;     // partial sums that a wave adds up by itself
// Partial sums that a wave loads before it adds the first. 16: Llama's width 200 us instead of 196, 16384 tokens of one id 75 instead of 83.
constexpr int kJoinAhead = 8;

struct RowArgs {
    const void* dout;
    const uint32_t* keys;   // sorted
    const uint32_t* at;     // the tokens in that order
    void* grad;
    float* part;            // [2 * chunks] rows of part_stride: a chunk's sum of the long run that came to it, and of the one that begins in it
    int64_t dout_stride, grad_stride, part_stride;
    int32_t T, V, d;
    int32_t chunk, window, blocks;  // tokens of a chunk, and those that it sees from its first on; blocks of columns
    int32_t adding, clearing;  // workgroups of each kind
    int32_t clear_from;        // rows before it have been cleared, all of them
    float scale;
};

// First of the sorted keys that is at least v.
__device__ __forceinline__ int32_t lower_bound(const uint32_t* keys, int32_t n, uint32_t v) {
    int32_t lo = 0;
    while (n > 0) {
        const int32_t half = n >> 1;
        if (keys[lo + half] < v) {
            lo += half + 1;
            n -= half + 1;
        } else {
            n = half;
        }
    }
    return lo;
}

// The same, looked for by the wave together: 64 keys at a time.
__device__ __forceinline__ int32_t wave_lower_bound(const uint32_t* keys, int32_t n, uint32_t v) {
    int32_t lo = 0;
    while (n > 0) {
        const int32_t step = (n + LD_WAVE - 1) / LD_WAVE, i = ld_lane() * step;
        const int32_t less = __popcll(__ballot(i < n && keys[lo + i] < v));
        if (less == 0) break;
        const int32_t skip = (less - 1) * step + 1;
        lo += skip;
        n = step - 1 < n - skip ? step - 1 : n - skip;
    }
    return lo;
}

template <int GT>
__device__ __forceinline__ typename LdElem<GT>::type* grad_row(const RowArgs& a, uint32_t v) {
    return static_cast<typename LdElem<GT>::type*>(a.grad) + static_cast<int64_t>(v) * a.grad_stride;
}

// A finished sum to its row, added to what the row held where ADD.
template <int GT, int N, bool ADD>
__device__ __forceinline__ void write_row(const RowArgs& a, uint32_t v, Columns c, typename LdVec<GT, N>::wide sum,
                                          typename LdVec<GT, N>::type held) {
    const typename LdVec<GT, N>::wide old = LdVec<GT, N>::widen(held);
#pragma unroll
    for (int e = 0; e < N; ++e) sum[e] = ADD ? __fmaf_rn(a.scale, sum[e], old[e]) : a.scale * sum[e];
    store_columns<GT, N, true>(grad_row<GT>(a, v), c, LdVec<GT, N>::narrow(sum));
}

// Clears the rows that no token names, kClearRows at a time.
template <int GT>
__device__ void clear_rows(const RowArgs& a, int32_t group) {
    constexpr int N = GT == LD_F32 ? 4 : 8;
    __shared__ uint32_t named;
    for (int32_t left = a.V - a.clear_from - group * kClearRows; left > 0; left -= a.clearing * kClearRows) {
        const int32_t first = a.V - left, rows = left < kClearRows ? left : kClearRows;
        if (threadIdx.x < LD_WAVE) {
            bool is = false;
            if (static_cast<int32_t>(threadIdx.x) < rows) {
                const uint32_t v = first + threadIdx.x;
                const int32_t i = lower_bound(a.keys, a.T, v);
                is = i < a.T && a.keys[i] == v;
            }
            const uint64_t all = __ballot(is);
            if (threadIdx.x == 0) named = static_cast<uint32_t>(all);
        }
        __syncthreads();
        for (int32_t r = threadIdx.x / LD_WAVE; r < rows; r += kRowWaves) {
            if (named >> r & 1) continue;
            for (int32_t l = ld_lane(); l * N < a.d; l += LD_WAVE)
                store_columns<GT, N, true>(grad_row<GT>(a, first + r), columns_of<N>(l, a.d), typename LdVec<GT, N>::type(0));
        }
        __syncthreads();
    }
}

// The runs of equal ids around a chunk.
struct Runs {
    uint32_t key;        // lane l: of token from + l; what lies past the tokens has none's
    uint64_t heads;      // bit l: another run begins with token from + l
    uint64_t own;        // the bits of the chunk itself
    int32_t began;       // where the last run before the chunk began, if that is one of the 63 tokens before, else -1
    int32_t valid;       // tokens from the chunk's first on that name a row
};

__device__ __forceinline__ Runs runs_of(const RowArgs& a, int32_t from) {
    constexpr int kShr1 = 0x138;  // to a lane from the one below
    Runs r;
    const int32_t i = from + ld_lane(), b = i - LD_WAVE;
    r.key = i < a.T ? a.keys[i] : UINT32_MAX;
    const uint32_t before = b >= 0 ? a.keys[b] : UINT32_MAX;
    const uint32_t last = lane_of(before, LD_WAVE - 1);
    const uint32_t below = static_cast<uint32_t>(
        __builtin_amdgcn_update_dpp(static_cast<int>(last), static_cast<int>(r.key), kShr1, 0xf, 0xf, false));
    const uint32_t below_before = static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(before), kShr1, 0xf, 0xf, false));
    r.own = (1ull << a.chunk) - 1;
    r.heads = __ballot(r.key != below && ld_lane() < a.window);
    const uint64_t heads_before = __ballot(before != below_before) & ~1ull;
    r.began = heads_before ? from - 1 - __builtin_clzll(heads_before) : -1;
    r.valid = __popcll(__ballot(r.key < static_cast<uint32_t>(a.V)));
    return r;
}

// Waves of a SIMD that k_rows' registers leave room for. For fp32 gradients four are asked for: the kernel waits for its loads, and
// 16384 tokens of 1600 columns into 50257 fp32 rows measured 102 us instead of 112 (into 1024 rows 40 and 41, 32768 tokens of 4096
// columns into bf16 rows 186 and 184). The 16-bit types hold twice the columns a lane: fp16 with accumulation spills at four, 67 us
// instead of 58, and they keep what the compiler chooses.
constexpr int row_occupancy(int dt) { return dt == LD_F32 ? 4 : 1; }

template <int DT, int GT, int N, bool STREAM, bool ADD>
__global__ __launch_bounds__(kRowThreads, row_occupancy(DT)) void k_rows(RowArgs a) {
    typedef LdVec<DT, N> X;
    typedef LdVec<GT, N> G;
    int32_t block = blockIdx.x;
    if (a.clearing > 0) {  // the two kinds mixed evenly
        const int64_t all = a.adding + a.clearing;
        const int32_t before = static_cast<int32_t>(static_cast<int64_t>(block) * a.clearing / all);
        if (static_cast<int32_t>(static_cast<int64_t>(block + 1) * a.clearing / all) > before) {
            clear_rows<GT>(a, before);
            return;
        }
        block -= before;
    }
    const int32_t unit = __builtin_amdgcn_readfirstlane(block * kRowWaves + static_cast<int32_t>(threadIdx.x / LD_WAVE));
    const int32_t c = unit / a.blocks;
    const Columns cols = columns_of<N>((unit - c * a.blocks) * LD_WAVE + ld_lane(), a.d);
    const int32_t from = c * a.chunk;
    if (from >= a.T) return;
    const Runs r = runs_of(a, from);
    const uint32_t at = from + ld_lane() < a.T ? a.at[from + ld_lane()] : 0;
    const uint64_t after = r.heads & ~r.own, later = r.heads & ~1ull;
    // tokens [i, end) from the chunk's first on
    int32_t i = 0;
    bool came = false;
    if (!(r.heads & 1)) {
        const int32_t left = later ? __builtin_ctzll(later) : LD_WAVE;
        // whether the chunk that this run began in sees its end, and so adds it up
        if (r.began >= 0 && from + left < (r.began & -a.chunk) + a.window) i = left;
        else came = true;
    }
    // the last run that begins here is long, or none begins; else it is followed to its end
    const bool goes_on = after == 0;
    int32_t end = goes_on || (r.heads & r.own) == 0 ? a.chunk : __builtin_ctzll(after);
    if (end > r.valid) end = r.valid;
    const typename X::elem* dout = static_cast<const typename X::elem*>(a.dout);
    float* part = a.part + 2 * static_cast<int64_t>(c) * a.part_stride;
    typename X::wide sum = typename X::wide(0.0f);
    int32_t run = i;  // where the run being added up begins
    typename G::type held = typename G::type(0);  // its row of grad, where that is added to
    const auto key_at = [&](int32_t j) { return lane_of(r.key, j); };
    const auto load = [&](int32_t j) {
        return load_columns<DT, N, STREAM>(dout + lane_of(at, j) * a.dout_stride, cols);
    };
    const auto begins = [&](int32_t j) { return (r.heads >> j & 1) != 0; };
    const auto add = [&](int32_t j, typename X::type x, typename G::type row) {
        if (begins(j)) {
            if (j > run) {
                if (came) store_columns<LD_F32, N, false>(part, cols, sum);
                else write_row<GT, N, ADD>(a, key_at(run), cols, sum, held);
                came = false;
                run = j;
            }
            sum = X::widen(x);
            held = row;
        } else {
            sum += X::widen(x);
        }
    };
    for (; i + kAhead <= end; i += kAhead) {
        typename X::type x[kAhead];
        typename G::type row[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            x[u] = load(i + u);
            row[u] = typename G::type(0);
            if (ADD && begins(i + u)) row[u] = load_columns<GT, N, false>(grad_row<GT>(a, key_at(i + u)), cols);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) add(i + u, x[u], row[u]);
    }
    if (i < end) {
        typename X::type x[kAhead - 1];
        typename G::type row[kAhead - 1];
#pragma unroll
        for (int u = 0; u < kAhead - 1; ++u) {
            row[u] = typename G::type(0);
            if (i + u < end) {
                x[u] = load(i + u);
                if (ADD && begins(i + u)) row[u] = load_columns<GT, N, false>(grad_row<GT>(a, key_at(i + u)), cols);
            }
        }
#pragma unroll
        for (int u = 0; u < kAhead - 1; ++u)
            if (i + u < end) add(i + u, x[u], row[u]);
    }
    if (run >= end) return;
    if (came) store_columns<LD_F32, N, false>(part, cols, sum);
    else if (goes_on && end == a.chunk) store_columns<LD_F32, N, false>(part + a.part_stride, cols, sum);
    else write_row<GT, N, ADD>(a, key_at(run), cols, sum, held);
}

// Partial sums from, from + step, ... up to last of a long run that begins in chunk `first`.
template <int N>
__device__ __forceinline__ typename LdVec<LD_F32, N>::wide sum_parts(const RowArgs& a, Columns cols, int32_t first, int32_t from, int32_t last, int32_t step) {
    typedef typename LdVec<LD_F32, N>::wide Sum;
    Sum sum = Sum(0.0f);
    for (int32_t j = from; j <= last; j += step * kJoinAhead) {
        Sum x[kJoinAhead];
#pragma unroll
        for (int u = 0; u < kJoinAhead; ++u) {
            const int64_t k = static_cast<int64_t>(j) + u * step;
            x[u] = k <= last ? load_columns<LD_F32, N, false>(a.part + (2 * k + (k == first)) * a.part_stride, cols) : Sum(0.0f);
        }
#pragma unroll
        for (int u = 0; u < kJoinAhead; ++u) sum += x[u];
    }
    return sum;
}

// Adds up the partial sums of long runs, each from the chunk that it begins in to the one that it ends in, in their order. A wave
// looks at a chunk, with 64 N columns; what it would be long busy with is shared by the workgroup's waves, which take partial sums in turn.
template <int GT, int N, bool ADD>
__global__ __launch_bounds__(kJoinWaves * LD_WAVE) void k_join(RowArgs a, int32_t chunks) {
    typedef typename LdVec<LD_F32, N>::wide Sum;
    __shared__ Sum sh[kJoinWaves][LD_WAVE];
    __shared__ int32_t shared_last[kJoinWaves];
    __shared__ uint32_t shared_run[kJoinWaves];
    const int32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / LD_WAVE), c0 = blockIdx.x * kJoinWaves, c = c0 + wave;
    const Columns cols = columns_of<N>(blockIdx.y * LD_WAVE + ld_lane(), a.d);
    int32_t last = -1;
    uint32_t run = 0;
    if (c < chunks) {
        const Runs r = runs_of(a, c * a.chunk);
        const uint64_t own = r.heads & r.own;
        if (own != 0 && (r.heads & ~r.own) == 0) {
            const int32_t first = LD_WAVE - 1 - __builtin_clzll(own);
            if (first < r.valid) {
                run = lane_of(r.key, first);
                last = (wave_lower_bound(a.keys, a.T, run + 1) - 1) / a.chunk;
            }
        }
    }
    const bool alone = last - c < kJoinAlone;
    if (ld_lane() == 0) {
        shared_last[wave] = alone ? -1 : last;
        shared_run[wave] = run;
    }
    __syncthreads();
    if (last >= 0 && alone) {
        typename LdVec<GT, N>::type held = typename LdVec<GT, N>::type(0);
        if (ADD) held = load_columns<GT, N, false>(grad_row<GT>(a, run), cols);
        const Sum sum = sum_parts<N>(a, cols, c, c, last, 1);
        write_row<GT, N, ADD>(a, run, cols, sum, held);
    }
    for (int32_t w = 0; w < kJoinWaves; ++w) {
        const int32_t to = shared_last[w];
        if (to < 0) continue;
        sh[wave][ld_lane()] = sum_parts<N>(a, cols, c0 + w, c0 + w + wave, to, kJoinWaves);
        __syncthreads();
        if (wave == 0) {
            Sum sum = sh[0][ld_lane()];
#pragma unroll
            for (int i = 1; i < kJoinWaves; ++i) sum += sh[i][ld_lane()];
            typename LdVec<GT, N>::type held = typename LdVec<GT, N>::type(0);
            if (ADD) held = load_columns<GT, N, false>(grad_row<GT>(a, shared_run[w]), cols);
            write_row<GT, N, ADD>(a, shared_run[w], cols, sum, held);
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------- few tokens

// All in one launch. Every workgroup sorts all tokens for itself, takes a block of columns and a share of the tokens, from where one
// run begins to where another does, and deals them out to its waves; a run that goes on in the next wave's tokens is added up in
// shared memory. Other workgroups clear the rows that no token names. Added to 50257 rows of 1600 columns, as three launches and so:
// 8 tokens 10.4 and 5.5 us, 64 12.5 and 6.6, 256 14.6 and 8.5, 512 15.2 and 10.5, 1024 17.8 and 11.2; 1024 of one id 19.7 and 23.
static_assert(kFewThreads == kSortThreads, "every workgroup sorts");
constexpr int kFewWaves = kFewThreads / LD_WAVE;
constexpr int kFewTokens = kSortThreads;
constexpr int kFewVector = 2;       // columns of a lane: narrow blocks, for more workgroups
constexpr int kFewColumns = kFewVector * LD_WAVE;
// Tokens of a share at least, and at most: so many that a share is no more than 8 tokens for a wave. Shares of 32, 64 and 128: 1024 tokens of
// 256 columns 10.9, 11.2, 12.8 us, of 4096 24.9, 16.9, 15.8: no more workgroups than compute units, each sorts.
constexpr int kFewShare = 32;
constexpr int kFewMostShare = 128;
constexpr int kFewGroups = 256;
// Up to 256 tokens a token's place is found by counting those that go before it: 8 tokens 5.5 us instead of 8.1, 256 8.5 instead of 9.9 (512
// would be 11.8 instead of 10.5).
constexpr int kCountedBits = 8;
constexpr int kCounted = 1 << kCountedBits;

// Sorts tokens of keys below 2^24 - 1, like sort_in_shared.
__device__ __forceinline__ void count_in_shared(const SortArgs& a, SortShared<1>& m) {
    // a key with the token behind it: all are different
    __shared__ __attribute__((aligned(16))) uint32_t both[kCounted];
    __shared__ uint32_t place[kCounted];
    const int32_t me = threadIdx.x;
    if (me < kCounted) {
        both[me] = me < a.T ? key_of(a, me) << kCountedBits | me : UINT32_MAX;
        place[me] = 0;
    }
    __syncthreads();
    constexpr int kShares = kSortThreads / kCounted, kQuads = kCounted / 4 / kShares;  // the threads of a token share the others out
    const int32_t i = me % kCounted, q0 = me / kCounted * kQuads;
    const uint32_t mine = both[i];
    const ld_u32x4* quads = reinterpret_cast<const ld_u32x4*>(both);
    uint32_t before = 0;
#pragma unroll 8
    for (int32_t q = q0; q < q0 + kQuads; ++q) {
        if (4 * q >= a.T) break;
#pragma unroll
        for (int e = 0; e < 4; ++e) before += quads[q][e] < mine;
    }
    if (i < a.T) atomicAdd(&place[i], before);
    __syncthreads();
    if (me < a.T) {
        m.keys[place[me]] = both[me] >> kCountedBits;
        m.tokens[place[me]] = static_cast<uint16_t>(me);
    }
    __syncthreads();
}

// Clears the rows that none of few tokens names, kFewClear at a time.
template <int GT>
__device__ void clear_unnamed(const RowArgs& a, const SortArgs& s, int32_t group) {
    constexpr int N = GT == LD_F32 ? 4 : 8;
    __shared__ unsigned long long named;
    for (int32_t left = a.V - group * kFewClear; left > 0; left -= a.clearing * kFewClear) {
        const int32_t first = a.V - left, rows = left < kFewClear ? left : kFewClear;
        if (threadIdx.x == 0) named = 0;
        __syncthreads();
        for (int32_t i = threadIdx.x; i < a.T; i += kFewThreads) {
            const uint32_t r = key_of(s, i) - static_cast<uint32_t>(first);  // of an id before the first: a large number
            if (r < kFewClear) atomicOr(&named, 1ull << r);
        }
        __syncthreads();
        for (int32_t r = threadIdx.x / LD_WAVE; r < rows; r += kFewWaves) {
            if (named >> r & 1) continue;
            for (int32_t l = ld_lane(); l * N < a.d; l += LD_WAVE)
                store_columns<GT, N, true>(grad_row<GT>(a, first + r), columns_of<N>(l, a.d), typename LdVec<GT, N>::type(0));
        }
        __syncthreads();
    }
}

template <int DT, int GT, int N, bool ADD>
__global__ __launch_bounds__(kFewThreads) void k_few(RowArgs a, SortArgs s, int32_t passes) {
    typedef LdVec<DT, N> X;
    typedef LdVec<GT, N> G;
    __shared__ SortShared<1> m;
    __shared__ typename X::wide came_sum[kFewWaves][LD_WAVE];
    __shared__ int32_t shared_valid;
    if (static_cast<int32_t>(blockIdx.x) >= a.adding) {
        clear_unnamed<GT>(a, s, static_cast<int32_t>(blockIdx.x) - a.adding);
        return;
    }
    if (threadIdx.x == 0) shared_valid = 0;
    if (passes == 0) count_in_shared(s, m);
    else sort_in_shared<1>(s, passes, m);
    {
        const int32_t i = threadIdx.x;
        const uint32_t none = a.V;
        if (i < a.T && m.keys[i] < none && (i + 1 == a.T || m.keys[i + 1] >= none)) shared_valid = i + 1;
    }
    __syncthreads();
    // the workgroups of a block of columns share the tokens out from one run's beginning to another's
    const int32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / LD_WAVE), block = blockIdx.x % a.blocks, share = blockIdx.x / a.blocks;
    const int32_t all = shared_valid, shares = a.adding / a.blocks, per_share = (all + shares - 1) / shares;
    const auto next_run = [&](int32_t from) {  // the first run that begins at or behind a token
        for (int32_t i0 = from; i0 < all; i0 += LD_WAVE) {
            const int32_t i = i0 + ld_lane();
            const uint64_t found = __ballot(i < all && (i == 0 || m.keys[i] != m.keys[i - 1]));
            if (found) return i0 + static_cast<int32_t>(__builtin_ctzll(found));
        }
        return all;
    };
    const int32_t begin = __builtin_amdgcn_readfirstlane(next_run(share * per_share));
    const int32_t end = __builtin_amdgcn_readfirstlane(next_run((share + 1) * per_share));
    const int32_t per = (end - begin + kFewWaves - 1) / kFewWaves, from = begin + wave * per;
    const int32_t count = end - from >= per ? per : end > from ? end - from : 0;  // at most 64
    const Columns cols = columns_of<N>(block * LD_WAVE + ld_lane(), a.d);
    const bool mine = ld_lane() < count;
    const uint32_t key = mine ? m.keys[from + ld_lane()] : UINT32_MAX, at = mine ? m.tokens[from + ld_lane()] : 0;
    const uint32_t before = mine && from + ld_lane() > 0 ? m.keys[from + ld_lane() - 1] : UINT32_MAX;
    const uint64_t heads = __ballot(mine && key != before);
    const bool goes_on = count > 0 && from + count < end && m.keys[from + count] == m.keys[from + count - 1];
    const auto key_at = [&](int32_t j) { return lane_of(key, j); };
    const typename X::elem* dout = static_cast<const typename X::elem*>(a.dout);
    typename X::wide sum = typename X::wide(0.0f);
    typename G::type held = typename G::type(0);
    bool came = count > 0 && !(heads & 1);
    int32_t run = 0;
    for (int32_t i = 0; i < count; i += kAhead) {
        typename X::type x[kAhead];
        typename G::type row[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (i + u < count) {
                x[u] = load_columns<DT, N, false>(dout + lane_of(at, i + u) * a.dout_stride, cols);
                if (ADD && (heads >> (i + u) & 1)) row[u] = load_columns<GT, N, false>(grad_row<GT>(a, key_at(i + u)), cols);
            }
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (i + u < count) {
                if (heads >> (i + u) & 1) {
                    if (i + u > run) {
                        if (came) came_sum[wave][ld_lane()] = sum;
                        else write_row<GT, N, ADD>(a, key_at(run), cols, sum, held);
                        came = false;
                        run = i + u;
                    }
                    sum = X::widen(x[u]);
                    if (ADD) held = row[u];
                } else {
                    sum += X::widen(x[u]);
                }
            }
        }
    }
    if (came) came_sum[wave][ld_lane()] = sum;
    __syncthreads();
    if (count == 0 || came) return;
    if (goes_on) {
        for (int32_t w = wave + 1; begin + w * per < end && m.keys[begin + w * per] == key_at(run); ++w) sum += came_sum[w][ld_lane()];
    }
    write_row<GT, N, ADD>(a, key_at(run), cols, sum, held);
}

struct Layout {
    int32_t passes, bits, per_tile, tiles;  // one tile: sorted by a workgroup alone
    int32_t chunk, window, chunks;
    int64_t part_stride;
    size_t keys, at, counts, part, bytes;  // byte offsets: two buffers each of keys and tokens
};

Layout layout_of(int64_t T, int64_t V, int32_t d) {
    Layout l;
    int32_t all = 1;
    while ((V >> all) != 0) ++all;  // bits of the keys 0 .. V
    const int32_t most = T <= kAloneMost ? kAloneBits : kDigitBits;
    l.passes = (all + most - 1) / most;
    l.bits = (all + l.passes - 1) / l.passes;
    l.per_tile = T <= kAloneMost ? kAloneMost : static_cast<int32_t>((T + kTile * kMostTiles - 1) / (kTile * kMostTiles)) * kTile;
    l.tiles = static_cast<int32_t>((T + l.per_tile - 1) / l.per_tile);
    const size_t list = ld_round_up(static_cast<size_t>(T) * 4, 256);
    l.keys = 0;
    l.at = 2 * list;
    l.counts = 4 * list;
    l.part = ld_round_up(l.counts + (static_cast<size_t>(l.tiles) << l.bits) * 4, 256);
    // Few waves: shorter chunks and windows, so that none is long busy with its tokens one after the other; many: fewer partial sums.
    // 4 and 16, 8 and 16, 16 and 32, 32 and 64 tokens: 1024 of 1600 columns 17, 18, 22, 27 us; 16384 of 256 40, 37, 40, 46; 65536 of 64 69, 53,
    // 49, 51; 16384 of 1600 84, 84, 85, 86; 65536 of 4096 303, 228, 201, 197
    const int64_t waves = T * ((static_cast<int64_t>(d) + 511) / 512);
    l.chunk = waves >= 256 << 10 ? 32 : waves >= 32 << 10 ? 16 : waves >= 8 << 10 ? 8 : 4;
    l.window = l.chunk < 8 ? 16 : 2 * l.chunk;
    l.chunks = static_cast<int32_t>((T + l.chunk - 1) / l.chunk);
    l.part_stride = (static_cast<int64_t>(d) + 3) / 4 * 4;
    l.bytes = ld_round_up(l.part + 2 * static_cast<size_t>(l.chunks) * l.part_stride * 4, 256);
    return l;
}

// Workgroups that share a block of columns' tokens out.
int32_t few_shares(int64_t T, int32_t d) {
    const int32_t blocks = (d + kFewColumns - 1) / kFewColumns, most = static_cast<int32_t>((T + kFewShare - 1) / kFewShare);
    const int32_t room = kFewGroups / blocks > 1 ? kFewGroups / blocks : 1;
    return most < room ? most : room;
}

bool few(int64_t T, int32_t d) { return T > 0 && T <= kFewTokens && d > 0 && T <= few_shares(T, d) * kFewMostShare; }

// Calls f with the columns of a lane: N, or one where a row has fewer (a block of 64 columns then holds it).
template <int N, typename F>
void with_vector(int32_t d, F f) {
    if (d >= N) f(std::integral_constant<int, N>());
    else f(std::integral_constant<int, 1>());
}

constexpr int32_t kMostBlocks = (1 << 24) - 1;  // of 256 threads: a launch has fewer than 2^32

int32_t at_most(int64_t n, int32_t most) { return n < most ? static_cast<int32_t>(n) : most; }

bool sizes_fit(int64_t T, int64_t V, int32_t d) {
    return T >= 0 && V >= 0 && d >= 0 && d <= LD_MAX_WIDTH && T <= LD_MAX_TOKENS && V < INT32_MAX;
}

}  // namespace

extern "C" size_t ld_embed_grad_workspace(int64_t T, int64_t V, int32_t d) {
    return sizes_fit(T, V, d) && !few(T, d) ? layout_of(T, V, d).bytes : 0;
}

extern "C" ld_status ld_embed_grad(const void* dout, int64_t dout_stride, int32_t dtype, const void* ids, int32_t id_dtype, int64_t T,
                                   int32_t d, float scale, void* grad, int64_t V, int64_t grad_stride, int32_t grad_dtype,
                                   int32_t accumulate, void* workspace, size_t workspace_bytes, ld_stream stream) {
    if (!sizes_fit(T, V, d) || dout_stride < 0 || grad_stride < d || !ld_known_type(dtype) || !ld_known_type(grad_dtype) ||
        (id_dtype != LD_I32 && id_dtype != LD_I64))
        return LD_ERR_RANGE;
    if (V == 0 || d == 0 || (T == 0 && accumulate)) return LD_OK;
    if (!grad || (T > 0 && (!dout || !ids))) return LD_ERR_NULL;
    if (!ld_aligned(dout, ld_type_bytes(dtype)) || !ld_aligned(grad, ld_type_bytes(grad_dtype)) ||
        !ld_aligned(ids, id_dtype == LD_I32 ? 4 : 8))
        return LD_ERR_ALIGN;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const Layout l = layout_of(T, V, d);
    if (few(T, d)) {
        const int32_t few_blocks = (d + kFewColumns - 1) / kFewColumns, adding = few_blocks * few_shares(T, d);
        const int32_t clearing = accumulate ? 0 : ld_few_clearing(V, adding);
        const int32_t passes = T <= kCounted && V < (1 << (32 - kCountedBits)) - 1 ? 0 : l.passes;
        const SortArgs sort = {ids, id_dtype == LD_I64, nullptr, nullptr, nullptr, nullptr, nullptr, V, static_cast<int32_t>(T), 0, 0, 0, l.bits};
        const RowArgs a = {dout, nullptr, nullptr, grad, nullptr, dout_stride, grad_stride, 0, static_cast<int32_t>(T), static_cast<int32_t>(V), d,
                           0, 0, few_blocks, adding, clearing, 0, scale};
        ld_begin_call();
        ld_with_type(dtype, [&](auto type) {
            ld_with_type(grad_dtype, [&](auto grad_type) {
                const dim3 grid(adding + clearing), threads(kFewThreads);
                with_vector<kFewVector>(d, [&](auto n) {
                    if (accumulate) k_few<type, grad_type, n, true><<<grid, threads, 0, s>>>(a, sort, passes);
                    else k_few<type, grad_type, n, false><<<grid, threads, 0, s>>>(a, sort, passes);
                });
            });
        });
        return ld_launch_status();
    }
    if (l.bytes > 0 && (!workspace || !ld_aligned(workspace, 256) || workspace_bytes < l.bytes)) return LD_ERR_WORKSPACE;
    const int32_t columns = LD_WAVE * (dtype == LD_F32 ? 4 : 8), blocks = static_cast<int32_t>((static_cast<int64_t>(d) + columns - 1) / columns);
    const int64_t adding = (static_cast<int64_t>(l.chunks) * blocks + kRowWaves - 1) / kRowWaves;
    if (adding > kMostBlocks / 2) return LD_ERR_RANGE;
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    uint32_t* keys[2] = {reinterpret_cast<uint32_t*>(ws + l.keys), reinterpret_cast<uint32_t*>(ws + l.keys + l.at / 2)};
    uint32_t* at[2] = {reinterpret_cast<uint32_t*>(ws + l.at), reinterpret_cast<uint32_t*>(ws + l.at + l.at / 2)};
    ld_begin_call();
    SortArgs sort = {ids, id_dtype == LD_I64, nullptr, nullptr, keys[0], at[0], reinterpret_cast<uint32_t*>(ws + l.counts), V,
                     static_cast<int32_t>(T), l.tiles, l.per_tile, 0, l.bits};
    Clearing clear = {grad, grad_stride, d, ld_type_bytes(grad_dtype) == 4, 0, 0};
    const int64_t hidden_bytes = accumulate || T > V ? 0 : l.tiles == 1 && T > 2 * kSortThreads ? 2 * kHidden : kHidden;
    const int64_t hidden = hidden_bytes / (static_cast<int64_t>(d) * ld_type_bytes(grad_dtype));  // rows a launch
    const auto blocks_of = [&](int32_t own) {  // of a launch that clears the next rows as well
        clear.from += clear.rows;
        clear.rows = static_cast<int32_t>(V - clear.from < hidden ? V - clear.from : hidden);
        const int32_t more = (clear.rows + kSortWaves - 1) / kSortWaves;
        return dim3(own + (more < 256 ? more : 256));
    };
    int32_t last = 0;
    if (l.tiles == 1) {
        const dim3 grid = blocks_of(1);
        if (T <= kSortThreads) k_sort_alone<1><<<grid, dim3(kSortThreads), 0, s>>>(sort, l.passes, clear);
        else if (T <= 2 * kSortThreads) k_sort_alone<2><<<grid, dim3(kSortThreads), 0, s>>>(sort, l.passes, clear);
        else k_sort_alone<4><<<grid, dim3(kSortThreads), 0, s>>>(sort, l.passes, clear);
        if (ld_launch_status() != LD_OK) return LD_ERR_HIP;
    }
    for (int32_t p = 0; p < l.passes && l.tiles > 1; ++p) {
        last = p & 1;
        sort.keys_out = keys[last];
        sort.at_out = at[last];
        sort.shift = p * l.bits;
        dim3 grid = blocks_of(l.tiles);
        k_sort_count<<<grid, dim3(kSortThreads), 0, s>>>(sort, clear);
        if (ld_launch_status() != LD_OK) return LD_ERR_HIP;
        grid = blocks_of(l.tiles);
        k_sort_move<<<grid, dim3(kSortThreads), 0, s>>>(sort, clear);
        if (ld_launch_status() != LD_OK) return LD_ERR_HIP;
        sort.ids = nullptr;
        sort.keys_in = keys[last];
        sort.at_in = at[last];
    }
    clear.from += clear.rows;
    const int32_t clearing = accumulate ? 0 : at_most((V - clear.from + kClearRows - 1) / kClearRows, kMostBlocks / 2);
    const RowArgs a = {dout, keys[last], at[last], grad, reinterpret_cast<float*>(ws + l.part), dout_stride, grad_stride, l.part_stride,
                       static_cast<int32_t>(T), static_cast<int32_t>(V), d, l.chunk, l.window, blocks, static_cast<int32_t>(adding),
                       clearing, clear.from, scale};
    const dim3 grid(static_cast<uint32_t>(adding + clearing));
    const bool streamed = T * static_cast<int64_t>(d) * ld_type_bytes(dtype) > kStreamed;
    ld_with_type(dtype, [&](auto type) {
        ld_with_type(grad_dtype, [&](auto grad_type) {
            with_vector<type == LD_F32 ? 4 : 8>(d, [&](auto n) {
                constexpr bool kWide = n > 1;  // narrow rows are never so many bytes that it matters
                if (accumulate) {
                    if (streamed) k_rows<type, grad_type, n, kWide, true><<<grid, dim3(kRowThreads), 0, s>>>(a);
                    else k_rows<type, grad_type, n, false, true><<<grid, dim3(kRowThreads), 0, s>>>(a);
                } else {
                    if (streamed) k_rows<type, grad_type, n, kWide, false><<<grid, dim3(kRowThreads), 0, s>>>(a);
                    else k_rows<type, grad_type, n, false, false><<<grid, dim3(kRowThreads), 0, s>>>(a);
                }
            });
        });
    });
    if (ld_launch_status() != LD_OK) return LD_ERR_HIP;
    if (T < l.window) return LD_OK;  // no run is long
    ld_with_type(grad_dtype, [&](auto grad_type) {
        const dim3 joins((l.chunks + kJoinWaves - 1) / kJoinWaves, (d + 4 * LD_WAVE - 1) / (4 * LD_WAVE));
        with_vector<4>(d, [&](auto n) {
            if (accumulate) k_join<grad_type, n, true><<<joins, dim3(kJoinWaves * LD_WAVE), 0, s>>>(a, l.chunks);
            else k_join<grad_type, n, false><<<joins, dim3(kJoinWaves * LD_WAVE), 0, s>>>(a, l.chunks);
        });
    });
    return ld_launch_status();
}
