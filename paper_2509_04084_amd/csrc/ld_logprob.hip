// Log probabilities of given tokens with entropy and top alternatives, and their gradient by the logits: where a training
// step's gradient begins, and how a recovered model is compared with the one that it replaces.
//
//   M = max_j logits[t, j];  x_j = scale (logits[t, j] - M);  Z = sum_j exp(x_j);  L = log Z
//   logprob[t] = x_id - L                 entropy[t] = L - sum_j exp(x_j) x_j / Z
//   dlogits[t, j] = scale (g (delta_j,id - p_j) - h p_j (log p_j + entropy[t])),  p_j = exp(x_j - L)
//
// One reading of a row: sums are kept against a reference that is moved only where a value passes it by far, so that most values cost
// a conversion, a fused multiply-add, an exponential and an addition; statistics are 32 bits wide. Bound by memory.
#include <type_traits>

#include "ld_elem.h"
#include "ld_grid.h"

namespace {

constexpr int kGroup = 8;                      // elements side by side that a thread takes at a time
constexpr int kWide = 256, kNarrow = 64;       // threads of a workgroup: one row, or a part of one
// Up to here a row that is not split is one wave's: it meets no barrier (five alternatives of 16384 x 1000 in bf16 19 us, by workgroups of
// 256 threads 76; 16384 x 4096 38 and 60, 1000 x 4096 7.8 and 8.3, 256 x 4096 7.2 and 6.6; 16384 x 8000 71 and 82, but in fp32 98
// and 90, and 1000 x 8000 11.4 and 10.4).
constexpr int32_t kNarrowElems = 4096;
constexpr int32_t kMostPart = 65536;           // elements of a part: 32 KB of group maxima for the alternatives
constexpr int32_t kPartStep = kWide * kGroup;
// Rows are split until there are as many, where they are fewer than half: by 256, 512 and 1024, us with five alternatives of 50257: 8 rows 10.2,
// 10.1, 9.9; 64 rows 12.0, 12.5, 12.7; 255 rows 13.2, 15.8, 16.4; 511 rows 17.8, 17.8, 22.3.
constexpr int64_t kWorkgroups = 256;
constexpr int kMostTop = LD_MAX_TOP;
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
// Powers of two by which a value may pass the reference before that is moved: an exponent is rounded in proportion to it.
constexpr float kFar = 4.0f;
// Powers of two that a logit stands for, at which the reference begins. Below, and at four times less above, rounding the product of a
// reference with the scale says too little of the exponent: rows whose largest logit lies there are added up another way.
constexpr float kLowest = 0x1p20f, kSteady = 0x1p19f;

struct ScoreArgs {
    const void* logits;
    const void* ids;           // NULL: no log probabilities
    float* logprob;
    float* entropy;            // NULL: none
    float* stats;
    int32_t* top_ids;
    float* top_logprob;
    float4* sums;              // of every part: largest logit, Z and S against it; NULL: rows are not split
    uint64_t* best;            // the best `top` of every part
    int64_t stride;
    int64_t row0;              // rows before this launch's
    int32_t V, part, parts, top;
    float scale;
    int32_t wide_ids;
    int32_t listed;            // groups that shared memory has room for behind the maxima
};

__device__ __forceinline__ int64_t id_at(const void* ids, int64_t t, int32_t wide) {
    return wide ? static_cast<const int64_t*>(ids)[t] : static_cast<const int32_t*>(ids)[t];
}

// A float as a whole number in the same order: -0 counts as 0, a NaN as the largest of all. Never 0.
__device__ __forceinline__ uint32_t order_of(float x) {
    if (x != x) return 0xFFFFFFFFu;
    const uint32_t b = __float_as_uint(x + 0.0f);
    return b ^ (static_cast<uint32_t>(static_cast<int32_t>(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t o) {
    return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}
// Where something of that order lies breaks ties: the lower index is the larger key.
__device__ __forceinline__ uint64_t key_of(uint32_t order, uint32_t index) {
    return static_cast<uint64_t>(order) << 32 | ~index;
}

template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp_or(float x, float other) {  // lanes without a source: `other`
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(other), __float_as_int(x), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float last_lane(float x) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), LD_WAVE - 1)); }

__device__ __forceinline__ float wave_sum(float x) {
    x += dpp_or<kDppShr + 1, 0xf>(x, 0.0f);
    x += dpp_or<kDppShr + 2, 0xf>(x, 0.0f);
    x += dpp_or<kDppShr + 4, 0xf>(x, 0.0f);
    x += dpp_or<kDppShr + 8, 0xf>(x, 0.0f);
    x += dpp_or<kDppLast16, 0xa>(x, 0.0f);
    x += dpp_or<kDppLast32, 0xc>(x, 0.0f);
    return last_lane(x);
}
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
    return static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(ld_wave_imax(x)), LD_WAVE - 1));
}

// Sums of exponentials of (logit - high): z, and s = sum of e * (logit - high) * scale in powers of two.
struct Sums {
    float high, z, s;
};
// The same against another reference, by d <= 0 powers of two. A sum of nothing stays one, also where that lies an infinity higher.
__device__ __forceinline__ Sums moved_by(Sums a, float high, float d) {
    const float f = __builtin_amdgcn_exp2f(d);
    return {high, a.z == 0.0f ? 0.0f : a.z * f, a.z == 0.0f || f == 0.0f ? 0.0f : f * __fmaf_rn(d, a.z, a.s)};
}
__device__ __forceinline__ Sums moved(Sums a, float high, float c) { return moved_by(a, high, (a.high - high) * c); }

// A row's sums, of all its parts. Maxima pass NaN over, sums do not: a row of nothing but NaN and minus infinities has a sum that is NaN and is
// no row in which nothing is left (whose sum is 0), and so that none takes it for one, its largest logit is NaN as well.
__device__ __forceinline__ Sums whole_row(Sums r) { return {r.z != r.z && r.high == -__builtin_huge_valf() ? r.z : r.high, r.z, r.s}; }

// What a row's sums say, written by one thread.
__device__ __forceinline__ float finish(const ScoreArgs& a, int64_t t, Sums r, float picked, bool inside) {
    const bool empty = r.high == -__builtin_huge_valf();
    const float log_z = empty ? 0.0f : logf(r.z);
    a.stats[2 * t] = r.high;
    a.stats[2 * t + 1] = log_z;
    if (a.logprob) a.logprob[t] = !inside ? 0.0f : empty ? r.high : __fmul_rn(picked - r.high, a.scale) - log_z;
    if (a.entropy) a.entropy[t] = empty ? 0.0f : log_z - kLn2 * (r.s / r.z);
    return log_z;
}

template <int DT>
__device__ __forceinline__ float picked_of(const ScoreArgs& a, int64_t t, bool& inside) {
    typedef typename LdElem<DT>::type elem;
    inside = false;
    if (!a.logprob) return 0.0f;
    const int64_t id = id_at(a.ids, t, a.wide_ids);
    inside = id >= 0 && id < a.V;
    return inside ? static_cast<float>(static_cast<const elem*>(a.logits)[t * a.stride + id]) : 0.0f;
}

__device__ __forceinline__ void write_top(const ScoreArgs& a, int64_t t, int32_t at, uint64_t key, float high, float log_z) {
    const float x = value_of(static_cast<uint32_t>(key >> 32));
    a.top_ids[t * a.top + at] = static_cast<int32_t>(~static_cast<uint32_t>(key));
    a.top_logprob[t * a.top + at] = high == -__builtin_huge_valf() ? high : __fmul_rn(x - high, a.scale) - log_z;
}

typedef float f32x8 __attribute__((ext_vector_type(8)));

// N elements that lie on a 16-byte boundary, or on that of all of them, as loaded.
template <int DT, int N> struct Raw {
    typedef typename LdElem<DT>::type elem;
    typedef elem type __attribute__((ext_vector_type(N)));
    static __device__ __forceinline__ type load(const elem* p) {
        if constexpr (DT == LD_F32 && N == 8) {
            typedef float half __attribute__((ext_vector_type(4)));
            const half lo = *reinterpret_cast<const half*>(p), hi = *reinterpret_cast<const half*>(p + 4);
            return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        } else {
            return *reinterpret_cast<const type*>(p);
        }
    }
    // n < N of them, minus infinity behind
    static __device__ __forceinline__ type load_some(const elem* p, int32_t n) {
        type x;
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = e < n ? p[e] : static_cast<elem>(-__builtin_huge_valf());
        return x;
    }
};
// The largest of eight; a NaN only where all are.
template <int DT>
__device__ __forceinline__ float largest(const typename Raw<DT, kGroup>::type& x) {
    if constexpr (DT == LD_F16) {  // two at a time
        typedef _Float16 half4 __attribute__((ext_vector_type(4)));
        typedef _Float16 half2 __attribute__((ext_vector_type(2)));
        const half4 a = __builtin_elementwise_max(__builtin_shufflevector(x, x, 0, 1, 2, 3), __builtin_shufflevector(x, x, 4, 5, 6, 7));
        const half2 b = __builtin_elementwise_max(__builtin_shufflevector(a, a, 0, 1), __builtin_shufflevector(a, a, 2, 3));
        return fmaxf(static_cast<float>(b[0]), static_cast<float>(b[1]));
    } else {
        const f32x8 y = __builtin_convertvector(x, f32x8);
        return fmaxf(fmaxf(fmaxf(fmaxf(y[0], y[1]), y[2]), fmaxf(fmaxf(y[3], y[4]), y[5])), fmaxf(y[6], y[7]));
    }
}
// Elements from p on up to the first on a boundary of N.
template <typename E>
__device__ __forceinline__ int32_t to_boundary(const E* p, int32_t N) {
    return static_cast<int32_t>(-static_cast<int64_t>(reinterpret_cast<uintptr_t>(p) / sizeof(E)) & (N - 1));
}

// The rank of every lane's key among the wave's, 0 for the largest. Equal keys are 0 and nothing.
__device__ __forceinline__ int32_t rank_in_wave(uint64_t key) {
    int32_t rank = 0;
    for (int j = 0; j < LD_WAVE; ++j) {
        const uint32_t lo = __builtin_amdgcn_readlane(static_cast<int>(key), j), hi = __builtin_amdgcn_readlane(static_cast<int>(key >> 32), j);
        rank += (static_cast<uint64_t>(hi) << 32 | lo) > key;
    }
    return rank;
}
// The K-th largest of all threads' keys (0: nothing), in every thread. Up to kFewTop the K largest of every wave one after
// another, and of those by counting; else every key's rank. `keys`: 256 of them.
constexpr int32_t kFewTop = 8;
template <int THREADS>
__device__ __forceinline__ uint64_t kth_of_few(uint64_t key, int32_t K, uint64_t* keys) {
    constexpr int kWaves = THREADS / LD_WAVE;
    uint64_t kept = 0;  // of lane k the wave's k-th largest
    for (int32_t k = 0; k < K; ++k) {
        const uint32_t hi = wave_max(static_cast<uint32_t>(key >> 32));
        const uint32_t lo = wave_max(static_cast<uint32_t>(key >> 32) == hi ? static_cast<uint32_t>(key) : 0u);
        const uint64_t best = static_cast<uint64_t>(hi) << 32 | lo;
        if (ld_lane() == k) kept = best;
        if (key == best) key = 0;
    }
    if (kWaves == 1) return static_cast<uint64_t>(__builtin_amdgcn_readlane(static_cast<int>(kept >> 32), K - 1)) << 32 |
                            static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(kept), K - 1));
    if (ld_lane() < K) keys[threadIdx.x / LD_WAVE * K + ld_lane()] = kept;
    __syncthreads();
    // Each wave for itself: lane i holds the i-th of the kWaves K candidates.
    const int32_t n = kWaves * K;
    const uint64_t mine = ld_lane() < n ? keys[ld_lane()] : 0;
    int32_t rank = 0;
    for (int32_t j = 0; j < n; ++j) rank += keys[j] > mine;
    const uint64_t found = __ballot(mine != 0 && rank == K - 1);
    if (!found) return 0;
    const int32_t lane = __builtin_ctzll(found);
    return static_cast<uint64_t>(__builtin_amdgcn_readlane(static_cast<int>(mine >> 32), lane)) << 32 |
           static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(mine), lane));
}

// How many of 64 keys in falling order are larger than `key`.
__device__ __forceinline__ int32_t larger_among(const uint64_t* sorted, uint64_t key) {
    int32_t n = 0;
#pragma unroll
    for (int step = 32; step > 0; step >>= 1)
        if (sorted[n + step - 1] > key) n += step;
    return n + (n == 63 && sorted[63] > key);
}

// A part of a row: its sums, and with TOP its best elements. Groups of eight begin at 16-byte boundaries (odd rows of 16-bit logits
// loaded as they lie took a fifth longer: 16384 x 50257 338 us, now 280): up to seven elements before the first are one too,
// and those behind the last. `groups`: every group's largest element.
template <int DT, int THREADS, bool ENTROPY, bool TOP>
__global__ __launch_bounds__(THREADS) void k_score(ScoreArgs a) {
    typedef typename LdElem<DT>::type elem;
    typedef Raw<DT, kGroup> R;
    constexpr int kWaves = THREADS / LD_WAVE, kOfSet = THREADS / 16;
    extern __shared__ float groups[];
    __shared__ Sums wave_sums[kWaves];
    __shared__ float wave_high[kWaves];
    __shared__ uint64_t keys[TOP ? kMostTop * kGroup : 1];
    __shared__ uint32_t counts[3], picked_groups[TOP ? kMostTop : 1];
    __shared__ uint64_t kth;
    const int64_t t = a.row0 + blockIdx.x / a.parts;
    const int32_t p = blockIdx.x % a.parts, begin = p * a.part, n = min(a.V - begin, a.part), tid = threadIdx.x;
    const elem* row = static_cast<const elem*>(a.logits) + t * a.stride + begin;
    const int32_t head = min(to_boundary(row, kGroup), n), headed = head > 0;
    const elem* body = row + head;
    const int32_t whole = (n - head) / kGroup, rest = (n - head) % kGroup, n_body = whole + (rest > 0), n_groups = headed + n_body;
    const float c = a.scale * kLog2e, infinity = __builtin_huge_valf();

    // Sums against a reference, which moves to a value that lies beyond `limit`.
    const float lowest = -kLowest / c, far = kFar / c;
    float ref = lowest, ref_c = -kLowest, limit = lowest + far, z = 0.0f, s = 0.0f;
    float high = -infinity;  // this thread's largest element, and its group
    int32_t at = tid == 0 ? 0 : tid + headed;
    const auto take = [&](const typename R::type& x, int32_t g) {
        const float m = largest<DT>(x);
        if (TOP) {
            groups[g] = m;
            if (m > high) at = g;
        }
        high = fmaxf(high, m);
        if (m > limit) {
            // by what the exponents were taken against, each rounded once: rows around 1e5 were 1e-4 off where the difference of the
            // references themselves moved them, those around 3e5 2e-3
            const float now = m * c;
            const Sums r = moved_by({ref, z, s}, m, ref_c - now);
            ref = m, ref_c = now, limit = m + far, z = r.z, s = r.s;
        }
#pragma unroll
        for (int e = 0; e < kGroup; ++e) {
            const float d = __fmaf_rn(static_cast<float>(x[e]), c, -ref_c), y = __builtin_amdgcn_exp2f(d);
            z += y;
            if (ENTROPY) s = __fmaf_rn(y, fmaxf(d, -200.0f), s);
        }
    };
    if (headed && tid == 0) take(R::load_some(row, head), 0);
    constexpr int kUnroll = 4;
    int32_t g = tid;
    for (; g + (kUnroll - 1) * THREADS < whole; g += kUnroll * THREADS) {
        typename R::type x[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) x[u] = R::load(body + (g + u * THREADS) * kGroup);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) take(x[u], headed + g + u * THREADS);
    }
    for (; g < whole; g += THREADS) take(R::load(body + g * kGroup), headed + g);
    if (g < n_body) take(R::load_some(body + g * kGroup, rest), headed + g);

    // What rounding the last ref_c has moved all exponents by.
    if (ref != lowest) {
        const float off = -__fmaf_rn(ref, c, -ref_c), f = __builtin_amdgcn_exp2f(off);
        s = f * __fmaf_rn(off, z, s);
        z *= f;
    }
    const int32_t wave = tid / LD_WAVE;
    float most = value_of(wave_max(order_of(high)));
    if (kWaves > 1) {
        if (ld_lane() == 0) wave_high[wave] = most;
        __syncthreads();
        for (int w = 0; w < kWaves; ++w) most = fmaxf(most, wave_high[w]);
    }
    Sums r = moved({ref, z, s}, most, c);
    if (most != -infinity && !(fabsf(most) * c < kSteady)) {
        r.z = r.s = 0.0f;
        for (int32_t i = tid; i < n; i += THREADS) {
            const float d = (static_cast<float>(row[i]) - most) * c, y = __builtin_amdgcn_exp2f(d);
            r.z += y;
            if (ENTROPY) r.s = __fmaf_rn(y, fmaxf(d, -200.0f), r.s);
        }
    }
    r.z = wave_sum(r.z);
    if (ENTROPY) r.s = wave_sum(r.s);
    if (kWaves > 1) {
        if (ld_lane() == 0) wave_sums[wave] = r;
        __syncthreads();
        r.z = r.s = 0.0f;
        for (int w = 0; w < kWaves; ++w) r.z += wave_sums[w].z, r.s += wave_sums[w].s;
    }
    const Sums row_sums = whole_row(r);
    float log_z = 0.0f;
    if (a.sums) {
        if (tid == 0) a.sums[blockIdx.x + a.row0 * a.parts] = make_float4(r.high, r.z, r.s, 0.0f);
    } else if (tid == 0) {
        bool inside;
        const float x = picked_of<DT>(a, t, inside);
        log_z = finish(a, t, row_sums, x, inside);
    }
    if (!TOP) return;

    const auto first_of = [&](int32_t q) { return headed && q == 0 ? 0 : head + (q - headed) * kGroup; };  // a group's elements
    const auto end_of = [&](int32_t q) { return headed && q == 0 ? head : min(head + (q - headed + 1) * kGroup, n); };
    const auto own_groups = [&](auto f) {  // of this thread, in order
        if (headed && tid == 0) f(0);
        for (int32_t q = tid; q < n_body; q += THREADS) f(headed + q);
    };
    // The maxima above passed NaN over: where there is one, or an infinity, all groups are ordered once more, one element at a time.
    uint32_t order = order_of(high);
    if (r.z != r.z) {
        order = 0;
        own_groups([&](int32_t q) {
            uint32_t o = 0;
            for (int32_t e = first_of(q); e < end_of(q); ++e) o = max(o, order_of(static_cast<float>(row[e])));
            groups[q] = value_of(o);
            if (o > order) order = o, at = q;
        });
    }
    const int32_t K = a.top;
    uint64_t* list = reinterpret_cast<uint64_t*>(groups + (n_groups + 1) / 2 * 2);  // behind the maxima
    uint64_t* best = a.best ? a.best + (a.row0 * a.parts + blockIdx.x) * K : nullptr;
    const auto rank_and_write = [&](int32_t many) {  // the best of the keys
        for (int32_t i = tid; i < many; i += THREADS) {
            const uint64_t k = keys[i];
            int32_t better = 0;
            for (int32_t j = 0; j < many; ++j) better += keys[j] > k;
            if (better >= K) continue;
            if (best) best[better] = k;
            else write_top(a, t, better, k, row_sums.high, log_z);
        }
        if (best)  // a part of fewer elements
            for (int32_t i = n + tid; i < K; i += THREADS) best[i] = 0;
    };
    const uint64_t mine = tid < n_body || (headed && tid == 0) ? key_of(order, at) : 0;
    // Few alternatives: no better bar than the K-th of what 16 sets of threads have best is passed by at least K elements, and usually by few
    // more, which are ranked (five of 16384 x 32000 212 -> 204 us, eight of 1023 x 32003 28.3 -> 27.0; with 64 sets fifty take 33.4, not 31.7).
    if (K <= kFewTop) {
        uint32_t set = static_cast<uint32_t>(mine >> 32);
        set = max(set, ld_dpp0<0xB1>(set));  // of two, of four lanes
        set = max(set, ld_dpp0<0x4E>(set));
        if (kWaves > 1) {                    // of sixteen, in the last
            set = max(set, ld_dpp0<kDppShr + 4>(set));
            set = max(set, ld_dpp0<kDppShr + 8>(set));
        }
        if (tid == 0) counts[0] = counts[1] = 0;
        if (tid % kOfSet == kOfSet - 1) picked_groups[tid / kOfSet] = set;
        __syncthreads();
        set = ld_lane() < 16 ? picked_groups[ld_lane()] : 0;
        int32_t rank = 0;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const uint32_t other = __builtin_amdgcn_readlane(set, j);
            rank += other > set || (other == set && j < ld_lane());
        }
        const uint32_t bar = __builtin_amdgcn_readlane(set, __builtin_ctzll(__ballot(rank == K - 1)));
        if (mine >> 32 >= bar && mine)
            own_groups([&](int32_t q) {
                if (order_of(groups[q]) < bar) return;
                const int32_t i = atomicAdd(&counts[0], 1u);
                if (i < a.listed) list[i] = q;
            });
        if (tid == 0) wave_sums[0] = {r.high, log_z, 0.0f};
        __syncthreads();
        const int32_t listed = counts[0];
        if (listed <= a.listed) {
            log_z = wave_sums[0].z;
            for (int32_t i = tid; i < listed * kGroup; i += THREADS) {
                const int32_t q = static_cast<int32_t>(list[i / kGroup]), e = first_of(q) + i % kGroup;
                if (e >= end_of(q)) continue;
                const uint32_t o = order_of(static_cast<float>(row[e]));
                if (o < bar) continue;
                const int32_t place = atomicAdd(&counts[1], 1u);
                if (place < kMostTop * kGroup) keys[place] = key_of(o, begin + e);
            }
            __syncthreads();
            if (counts[1] <= kMostTop * kGroup) {
                rank_and_write(counts[1]);
                return;
            }
        }
        __syncthreads();
    }
    // The best K elements lie in the K groups whose largest elements are the best K (of equal ones the lower), and those in the K
    // threads of which the same holds. First the K-th of those threads' best.
    if (tid == 0) counts[0] = counts[1] = counts[2] = 0, kth = 0;
    const bool single = n_groups <= THREADS && !headed;  // a thread has one group at most: its rank is the group's
    uint64_t least;
    if (K <= kFewTop && !single) {
        __syncthreads();
        least = kth_of_few<THREADS>(mine, K, keys);
    } else {
        int32_t rank = rank_in_wave(mine);
        __syncthreads();
        if (kWaves > 1) {
            if (mine) keys[wave * LD_WAVE + rank] = mine;
            else keys[tid] = 0;  // lanes without a group are a wave's last
            __syncthreads();
            rank = 0;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) rank += larger_among(keys + w * LD_WAVE, mine);
        }
        if (single && rank < K && mine) picked_groups[rank] = at;
        if (rank == K - 1 && mine) kth = mine;
        __syncthreads();
        least = kth;
    }
    if (tid == 0) wave_sums[0] = {r.high, log_z, 0.0f};
    // Groups of those threads that are no worse, behind the maxima. Usually few of their elements are no worse than the K-th thread's best,
    // and those are ranked at once; where many are, as in rows of equal ones, first the K best groups are found.
    int32_t kept = min(n_groups, K);
    if (!single) {
        if (mine >= least && mine)
            own_groups([&](int32_t q) {
                const uint64_t k = key_of(order_of(groups[q]), q);
                if (k >= least) list[atomicAdd(&counts[0], 1u)] = k;
            });
        __syncthreads();
        const int32_t listed = counts[0];
        log_z = wave_sums[0].z;
        for (int32_t i = tid; i < listed * kGroup; i += THREADS) {
            const int32_t q = ~static_cast<uint32_t>(list[i / kGroup]), e = first_of(q) + i % kGroup;
            if (e >= end_of(q)) continue;
            const uint32_t o = order_of(static_cast<float>(row[e]));
            if (o < least >> 32) continue;
            const int32_t at = atomicAdd(&counts[2], 1u);
            if (at < kMostTop * kGroup) keys[at] = key_of(o, begin + e);
        }
        __syncthreads();
        if (counts[2] <= kMostTop * kGroup) {
            rank_and_write(counts[2]);
            return;
        }
        kept = min(listed, K);
        for (int32_t i = tid; i < listed; i += THREADS) {
            const uint64_t k = list[i];
            int32_t better = 0;
            for (int32_t j = 0; j < listed; ++j) better += list[j] > k;
            if (better < K) picked_groups[better] = ~static_cast<uint32_t>(k);
        }
    }
    __syncthreads();
    log_z = wave_sums[0].z;
    // Their elements that are no worse than the K-th group's largest, wherever that lies in it; of those the K best.
    const int32_t last = picked_groups[kept - 1];
    const uint64_t bar = kept < K ? 1 : key_of(order_of(groups[last]), begin + end_of(last) - 1);
    for (int32_t i = tid; i < kept * kGroup; i += THREADS) {
        const int32_t q = picked_groups[i / kGroup], e = first_of(q) + i % kGroup;
        if (e >= end_of(q)) continue;
        const uint64_t k = key_of(order_of(static_cast<float>(row[e])), begin + e);
        if (k >= bar) keys[atomicAdd(&counts[1], 1u)] = k;
    }
    __syncthreads();
    rank_and_write(counts[1]);
}

// A wave joins the parts of a row, their lists in shared memory unless there are too many.
constexpr int32_t kJoinHeld = 8192;
static_assert(kMostTop <= LD_WAVE, "a lane writes an alternative");
template <int DT>
__global__ __launch_bounds__(LD_WAVE) void k_score_join(ScoreArgs a) {
    constexpr int kEach = (LD_MAX_VOCAB / kMostPart + LD_WAVE - 1) / LD_WAVE;
    const int64_t t = a.row0 + blockIdx.x;
    const float4* sums = a.sums + t * a.parts;
    const int32_t lane = threadIdx.x, all = a.parts * a.top;
    const float c = a.scale * kLog2e;
    // All that is read is on its way before any of it is used.
    extern __shared__ uint64_t lists[];
    const uint64_t* best = a.best + t * all;
    const bool held = all <= kJoinHeld;
    constexpr int kHeldEach = 8;
    uint64_t some[kHeldEach];
    if (held)
#pragma unroll
        for (int i = 0; i < kHeldEach; ++i) some[i] = lane + i * LD_WAVE < all ? best[lane + i * LD_WAVE] : 0;
    float4 part[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int32_t p = lane + i * LD_WAVE;
        part[i] = p < a.parts ? sums[p] : make_float4(-__builtin_huge_valf(), 0.0f, 0.0f, 0.0f);
    }
    bool inside;
    const float picked = picked_of<DT>(a, t, inside);
    if (held) {
#pragma unroll
        for (int i = 0; i < kHeldEach; ++i)
            if (lane + i * LD_WAVE < all) lists[lane + i * LD_WAVE] = some[i];
        for (int32_t i = lane + kHeldEach * LD_WAVE; i < all; i += LD_WAVE) lists[i] = best[i];
    }
    uint32_t high = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) high = max(high, order_of(part[i].x));
    const float most = value_of(wave_max(high));
    float z = 0.0f, s = 0.0f;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const Sums r = moved({part[i].x, part[i].y, part[i].z}, most, c);
        z += r.z, s += r.s;
    }
    const Sums r = whole_row({most, wave_sum(z), wave_sum(s)});
    float log_z = 0.0f;
    if (lane == 0) log_z = finish(a, t, r, picked, inside);
    if (a.top == 0) return;
    log_z = __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(log_z)));
    // Every lane holds the next of up to kEach parts' lists; the best of all is written, and its list moves on.
    __syncthreads();
    const auto entry = [&](int32_t i) { return held ? lists[i] : best[i]; };
    uint64_t next[kEach];
    int32_t used[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int32_t p = lane + i * LD_WAVE;
        used[i] = 0;
        next[i] = p < a.parts ? entry(p * a.top) : 0;
    }
    uint64_t kept = 0;
    for (int32_t k = 0; k < a.top; ++k) {
        uint64_t mine = next[0];
#pragma unroll
        for (int i = 1; i < kEach; ++i) mine = max(mine, next[i]);
        const uint32_t hi = wave_max(static_cast<uint32_t>(mine >> 32));
        const uint32_t lo = wave_max(static_cast<uint32_t>(mine >> 32) == hi ? static_cast<uint32_t>(mine) : 0u);
        const uint64_t winner = static_cast<uint64_t>(hi) << 32 | lo;
        if (lane == k) kept = winner;
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (next[i] == winner) {
                const int32_t p = lane + i * LD_WAVE;
                next[i] = ++used[i] < a.top ? entry(p * a.top + used[i]) : 0;
            }
    }
    if (lane < a.top) write_top(a, t, lane, kept, r.high, log_z);
}

struct GradArgs {
    const void* logits;
    const void* ids;           // NULL: no gradient by log probabilities
    const float* stats;
    const float* d_logprob;
    const float* entropy;      // NULL: no gradient by entropies
    const float* d_entropy;
    void* out;
    int64_t stride, out_stride, d_logprob_stride, d_entropy_stride;
    int64_t row0;
    uint32_t pieces, chunks;   // of the launch, and of a row
    int32_t V;
    float scale;
    int32_t wide_ids;
};

// A thread's elements side by side: 16 bytes of the gradient, so that a wave writes whole lines.
template <int OT> constexpr int grad_group() { return OT == LD_F32 ? 4 : 8; }
// Elements of a thread: few, of many threads (16384 x 50257 in bf16 529 us with 16, 576 with 32, 605 with 64, 647 with 8; fp32 to fp32 1138
// with 16, 1045 with 8).
template <int DT, int OT> constexpr int grad_elems() { return DT == LD_F32 && OT == LD_F32 ? 8 : 16; }
// Consecutive chunks that an XCD takes: 517 us in runs of 16 and 64, 527 of 4, 534 one by one.
constexpr uint32_t kGradRun = 16;
constexpr int32_t kLine = 128;

template <int OT>
__device__ __forceinline__ void store_streamed(typename LdElem<OT>::type* p, const float (&y)[grad_group<OT>()]) {
    typedef float wide __attribute__((ext_vector_type(grad_group<OT>())));
    typedef typename LdElem<OT>::type narrow __attribute__((ext_vector_type(grad_group<OT>())));
    wide x;
#pragma unroll
    for (int e = 0; e < grad_group<OT>(); ++e) x[e] = y[e];
    __builtin_nontemporal_store(__builtin_convertvector(x, narrow), reinterpret_cast<narrow*>(p));
}

// A chunk of a row. Every element is read and written by one thread, so that the gradient may take the logits' place. Groups begin where
// the gradient's lines do: those elements before the first and behind the last that are fewer go one by one.
template <int DT, int OT, int THREADS, bool ENTROPY>
__global__ __launch_bounds__(THREADS) void k_score_grad(GradArgs a) {
    typedef typename LdElem<DT>::type elem;
    typedef typename LdElem<OT>::type out_elem;
    constexpr int N = grad_group<OT>(), kUnroll = grad_elems<DT, OT>() / N, kChunk = THREADS * grad_elems<DT, OT>();
    typedef LdVec<DT, N> V;
    const uint32_t piece = ld_xcd_piece<kGradRun>(blockIdx.x, gridDim.x);
    if (piece >= a.pieces) return;
    const int64_t t = a.row0 + piece / a.chunks;
    out_elem* out = static_cast<out_elem*>(a.out) + t * a.out_stride;
    const elem* row = static_cast<const elem*>(a.logits) + t * a.stride;
    const int32_t head = min(to_boundary(out, kLine / static_cast<int32_t>(sizeof(out_elem))), a.V), chunk = piece % a.chunks, begin = head + chunk * kChunk;
    const float high = a.stats[2 * t], log_z = a.stats[2 * t + 1];  // the largest logit, L
    const int64_t id = a.ids ? id_at(a.ids, t, a.wide_ids) : -1;
    const bool inside = id >= 0 && id < a.V;
    const float g = inside ? a.scale * a.d_logprob[t * a.d_logprob_stride] : 0.0f;
    const int32_t named = inside ? static_cast<int32_t>(id) : -1;
    const float h = ENTROPY ? a.scale * a.d_entropy[t * a.d_entropy_stride] : 0.0f, entropy = ENTROPY ? a.entropy[t] : 0.0f;
    const auto at = [&](float x) {  // without what the token named gets
        const float logp = __fmaf_rn(x - high, a.scale, -log_z), p = __builtin_amdgcn_exp2f(logp * kLog2e);
        if (ENTROPY) return p > 0.0f ? -p * __fmaf_rn(h, logp + entropy, g) : -p * g;
        return -p * g;
    };
    const auto one = [&](int32_t i) {
        float y = at(static_cast<float>(row[i]));
        if (i == named) y += g;
        out[i] = static_cast<out_elem>(y);
    };
    if (high == -__builtin_huge_valf()) {  // nothing is left
        for (int32_t i = (chunk == 0 ? 0 : begin) + threadIdx.x; i < min(a.V, begin + kChunk); i += THREADS) out[i] = static_cast<out_elem>(0.0f);
        return;
    }
    if (chunk == 0 && static_cast<int32_t>(threadIdx.x) < head) one(threadIdx.x);
    const int32_t whole = min(a.V - begin, kChunk) / N;
    typename V::type x[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        const int32_t q = threadIdx.x + u * THREADS;
        if (q < whole) x[u] = *reinterpret_cast<const typename V::type*>(row + begin + q * N);
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        const int32_t q = threadIdx.x + u * THREADS, first = begin + q * N;
        if (q >= whole) continue;
        float y[N];
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] = at(static_cast<float>(x[u][e]));
        const int32_t own = named - first;
        if (static_cast<uint32_t>(own) < static_cast<uint32_t>(N)) {
#pragma unroll
            for (int e = 0; e < N; ++e) y[e] = e == own ? y[e] + g : y[e];
        }
        store_streamed<OT>(out + first, y);
    }
    const int32_t end = begin + whole * N + static_cast<int32_t>(threadIdx.x);
    if (whole < kChunk / N && end < a.V) one(end);
}

// How a call splits its rows.
struct Split {
    int32_t part, parts;
    bool narrow;
};
Split split_of(int64_t T, int32_t V) {
    const int32_t most = (V + kPartStep - 1) / kPartStep, least = (V + kMostPart - 1) / kMostPart;
    int64_t parts = T > 0 && T < kWorkgroups / 2 ? (kWorkgroups + T - 1) / T : 1;
    parts = parts > most ? most : parts < least ? least : parts;
    if (parts > LD_MAX_VOCAB / kMostPart) parts = LD_MAX_VOCAB / kMostPart;  // few rows of very many columns
    const int32_t part = static_cast<int32_t>((most + parts - 1) / parts) * kPartStep;
    const int32_t count = (V + part - 1) / part;
    return {count == 1 ? V : part, count, count == 1 && V <= kNarrowElems};
}

bool known_shape(int64_t T, int32_t V, int32_t top) {
    return T >= 0 && T <= LD_MAX_TOKENS && V >= 0 && V <= LD_MAX_VOCAB && top >= 0 && top <= kMostTop && (top <= V || T == 0);
}

}  // namespace

extern "C" size_t ld_token_logprob_workspace(int64_t T, int32_t V, int32_t top) {
    if (!known_shape(T, V, top) || T == 0 || V == 0) return 0;
    const Split sp = split_of(T, V);
    if (sp.parts == 1) return 0;
    return ld_round_up(static_cast<size_t>(T) * sp.parts * (sizeof(float4) + sizeof(uint64_t) * top), 256);
}

extern "C" ld_status ld_token_logprob(const void* logits, int64_t T, int32_t V, int64_t stride, int32_t dtype, const void* ids,
                                      int32_t id_dtype, float scale, float* logprob, float* entropy, float* stats, int32_t top,
                                      int32_t* top_ids, float* top_logprob, void* workspace, size_t workspace_bytes, ld_stream stream) {
    if (!known_shape(T, V, top) || stride < 0 || !ld_known_type(dtype) || (id_dtype != LD_I32 && id_dtype != LD_I64) ||
        !(scale >= 1e-30f && scale <= 1e30f))
        return LD_ERR_RANGE;
    if (T == 0) return LD_OK;
    if (V == 0) return LD_ERR_RANGE;
    if (!logits || !stats || (ids == nullptr) != (logprob == nullptr) || (top > 0 && (!top_ids || !top_logprob))) return LD_ERR_NULL;
    const int32_t in = ld_type_bytes(dtype), id_bytes = id_dtype == LD_I32 ? 4 : 8;
    if (!ld_aligned(logits, in) || !ld_aligned(ids, id_bytes) || !ld_aligned(logprob, 4) || !ld_aligned(entropy, 4) || !ld_aligned(stats, 4) ||
        !ld_aligned(top_ids, 4) || !ld_aligned(top_logprob, 4))
        return LD_ERR_ALIGN;
    const Split sp = split_of(T, V);
    const size_t need = ld_token_logprob_workspace(T, V, top);
    if (need > 0 && (!workspace || !ld_aligned(workspace, 256) || workspace_bytes < need)) return LD_ERR_WORKSPACE;
    ld_begin_call();
    hipStream_t st = static_cast<hipStream_t>(stream);
    float4* sums = sp.parts > 1 ? static_cast<float4*>(workspace) : nullptr;
    uint64_t* best = sums && top ? reinterpret_cast<uint64_t*>(sums + T * sp.parts) : nullptr;
    const int32_t threads = sp.narrow ? kNarrow : kWide;
    // maxima of the groups, with one more where rows do not begin at a boundary, and the list of those that `top` threads hold
    const int32_t n_groups = sp.part / kGroup + 2, of_thread = (n_groups + threads - 1) / threads + 1;
    const int32_t listed = n_groups < top * of_thread ? n_groups : top * of_thread;
    const size_t shared = top ? (n_groups + 1) / 2 * 2 * sizeof(float) + listed * sizeof(uint64_t) : 0;
    const size_t join_shared = sp.parts * top <= kJoinHeld ? static_cast<size_t>(sp.parts) * top * sizeof(uint64_t) : 0;
    const int64_t most = ld_workgroups(static_cast<int64_t>(1) << 40, threads) / sp.parts;  // rows of a launch
    for (int64_t t = 0; t < T; t += most) {
        const int64_t rows = T - t < most ? T - t : most;
        const ScoreArgs a = {logits, ids, logprob, entropy, stats, top_ids, top_logprob, sums, best, stride, t,
                             V, sp.part, sp.parts, top, scale, id_dtype == LD_I64, listed};
        const dim3 grid(static_cast<uint32_t>(rows * sp.parts));
        ld_with_type(dtype, [&](auto type) {
            const auto launch = [&](auto wide, auto with_entropy, auto with_top) {
                k_score<type, decltype(wide)::value, decltype(with_entropy)::value, decltype(with_top)::value>
                    <<<grid, dim3(decltype(wide)::value), shared, st>>>(a);
            };
            const auto by_flags = [&](auto wide) {
                if (entropy && top) launch(wide, std::true_type(), std::true_type());
                else if (entropy) launch(wide, std::true_type(), std::false_type());
                else if (top) launch(wide, std::false_type(), std::true_type());
                else launch(wide, std::false_type(), std::false_type());
            };
            if (sp.narrow) by_flags(std::integral_constant<int, kNarrow>());
            else by_flags(std::integral_constant<int, kWide>());
        });
        if (ld_launch_status() != LD_OK) return LD_ERR_HIP;
        if (sp.parts == 1) continue;
        ld_with_type(dtype, [&](auto type) { k_score_join<type><<<dim3(static_cast<uint32_t>(rows)), dim3(LD_WAVE), join_shared, st>>>(a); });
        if (ld_launch_status() != LD_OK) return LD_ERR_HIP;
    }
    return LD_OK;
}

extern "C" ld_status ld_token_logprob_grad(const void* logits, int64_t T, int32_t V, int64_t stride, int32_t dtype, const void* ids,
                                           int32_t id_dtype, float scale, const float* stats, const float* d_logprob,
                                           int64_t d_logprob_stride, const float* entropy, const float* d_entropy, int64_t d_entropy_stride,
                                           void* d_logits, int64_t out_stride, int32_t out_dtype, ld_stream stream) {
    if (!known_shape(T, V, 0) || stride < 0 || out_stride < V || !ld_known_type(dtype) || !ld_known_type(out_dtype) ||
        (id_dtype != LD_I32 && id_dtype != LD_I64) || !(scale >= 1e-30f && scale <= 1e30f) || d_logprob_stride < 0 || d_entropy_stride < 0)
        return LD_ERR_RANGE;
    if (T == 0 || V == 0) return LD_OK;
    if (!logits || !stats || !d_logits || (ids == nullptr) != (d_logprob == nullptr) || (entropy == nullptr) != (d_entropy == nullptr))
        return LD_ERR_NULL;
    if (d_logits == logits && (out_dtype != dtype || out_stride != stride)) return LD_ERR_RANGE;
    const int32_t in = ld_type_bytes(dtype), id_bytes = id_dtype == LD_I32 ? 4 : 8;
    if (!ld_aligned(logits, in) || !ld_aligned(ids, id_bytes) || !ld_aligned(stats, 4) || !ld_aligned(d_logprob, 4) || !ld_aligned(entropy, 4) ||
        !ld_aligned(d_entropy, 4) || !ld_aligned(d_logits, ld_type_bytes(out_dtype)))
        return LD_ERR_ALIGN;
    ld_begin_call();
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int32_t elems = dtype == LD_F32 && out_dtype == LD_F32 ? grad_elems<LD_F32, LD_F32>() : grad_elems<LD_BF16, LD_BF16>();
    const bool narrow = V <= kNarrow * elems;  // a wave's: 16384 x 1000 in bf16 11 us, by 256 threads 17
    const int32_t threads = narrow ? kNarrow : kWide, chunk = threads * elems, chunks = (V + chunk - 1) / chunk;
    const int64_t most = (ld_workgroups(static_cast<int64_t>(1) << 40, threads) - 7) / chunks;
    for (int64_t t = 0; t < T; t += most) {
        const int64_t rows = T - t < most ? T - t : most;
        const uint32_t pieces = static_cast<uint32_t>(rows * chunks);
        const GradArgs a = {logits, ids, stats, d_logprob, entropy, d_entropy, d_logits, stride, out_stride, d_logprob_stride,
                            d_entropy_stride, t, pieces, static_cast<uint32_t>(chunks), V, scale, id_dtype == LD_I64};
        const dim3 grid((pieces + 7) / 8 * 8);
        ld_with_type(dtype, [&](auto type) {
            ld_with_type(out_dtype, [&](auto out_type) {
                if (narrow && entropy) k_score_grad<type, out_type, kNarrow, true><<<grid, dim3(kNarrow), 0, st>>>(a);
                else if (narrow) k_score_grad<type, out_type, kNarrow, false><<<grid, dim3(kNarrow), 0, st>>>(a);
                else if (entropy) k_score_grad<type, out_type, kWide, true><<<grid, dim3(kWide), 0, st>>>(a);
                else k_score_grad<type, out_type, kWide, false><<<grid, dim3(kWide), 0, st>>>(a);
            });
        });
        if (ld_launch_status() != LD_OK) return LD_ERR_HIP;
    }
    return LD_OK;
}
