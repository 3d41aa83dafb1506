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
constexpr int32_t kNarrowElems = 4096;         // up to here a row is one wave's
constexpr int32_t kMostPart = 65536;           // elements of a part: 32 KB of group maxima for the alternatives
constexpr int32_t kPartStep = kWide * kGroup;
constexpr int64_t kWorkgroups = 1024;          // rows are split until there are as many
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
// The same against another, not lower, reference. A sum of nothing stays one, also where that lies an infinity higher.
__device__ __forceinline__ Sums moved(Sums a, float high, float c) {
    const float d = (a.high - high) * c, f = __builtin_amdgcn_exp2f(d);
    return {high, a.z == 0.0f ? 0.0f : a.z * f, a.z == 0.0f || f == 0.0f ? 0.0f : f * __fmaf_rn(d, a.z, a.s)};
}

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

template <int DT>
__device__ __forceinline__ f32x8 load_group(const typename LdElem<DT>::type* p) {
    if constexpr (DT == LD_F32) {
        typedef typename LdVec<LD_F32, 4>::type half;
        const half lo = *reinterpret_cast<const half*>(p), hi = *reinterpret_cast<const half*>(p + 4);
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
        typedef LdVec<DT, 8> V;
        return V::widen(*reinterpret_cast<const typename V::type*>(p));
    }
}
// The same at the end of a row, minus infinity behind it.
template <int DT>
__device__ __forceinline__ f32x8 load_ragged(const typename LdElem<DT>::type* p, int32_t n) {
    f32x8 x;
#pragma unroll
    for (int e = 0; e < kGroup; ++e) x[e] = e < n ? static_cast<float>(p[e]) : -__builtin_huge_valf();
    return x;
}

// A part of a row: its sums, and with TOP its best elements. `groups`: the order of every group's largest element.
template <int DT, int THREADS, bool ENTROPY, bool TOP>
__global__ __launch_bounds__(THREADS) void k_score(ScoreArgs a) {
    typedef typename LdElem<DT>::type elem;
    constexpr int kWaves = THREADS / LD_WAVE;
    extern __shared__ uint32_t groups[];
    __shared__ Sums wave_sums[kWaves];
    __shared__ uint32_t wave_high[kWaves];
    __shared__ uint64_t keys[TOP ? kMostTop * kGroup : 1];
    __shared__ uint32_t list_count, picked_groups[TOP ? kMostTop : 1];
    __shared__ uint64_t kth;
    const int64_t t = a.row0 + blockIdx.x / a.parts;
    const int32_t p = blockIdx.x % a.parts, begin = p * a.part, n = min(a.V - begin, a.part);
    const int32_t n_groups = (n + kGroup - 1) / kGroup, whole = n / kGroup, tid = threadIdx.x;
    const elem* row = static_cast<const elem*>(a.logits) + t * a.stride + begin;
    const float c = a.scale * kLog2e;

    const float lowest = -kLowest / c;
    float ref = lowest, ref_c = -kLowest, z = 0.0f, s = 0.0f;
    uint32_t high = 0, at = 0;  // order of this thread's largest element, and its group
    const auto take = [&](const f32x8& x, int32_t g) {
        float m = fmaxf(fmaxf(fmaxf(fmaxf(x[0], x[1]), x[2]), fmaxf(fmaxf(x[3], x[4]), x[5])), fmaxf(x[6], x[7]));
        const uint32_t o = order_of(m);
        if (o > high) high = o, at = g;
        if (TOP) groups[g] = o;
        if (m * c > ref_c + kFar) {
            const Sums r = moved({ref, z, s}, m, c);
            ref = m, ref_c = m * c, z = r.z, s = r.s;
        }
#pragma unroll
        for (int e = 0; e < kGroup; ++e) {
            const float d = __fmaf_rn(x[e], c, -ref_c), y = __builtin_amdgcn_exp2f(d);
            z += y;
            if (ENTROPY) s = __fmaf_rn(y, fmaxf(d, -200.0f), s);
        }
    };
    constexpr int kUnroll = 4;
    int32_t g = tid;
    for (; g + (kUnroll - 1) * THREADS < whole; g += kUnroll * THREADS) {
        f32x8 x[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) x[u] = load_group<DT>(row + static_cast<int64_t>(g + u * THREADS) * kGroup);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) take(x[u], g + u * THREADS);
    }
    for (; g < whole; g += THREADS) take(load_group<DT>(row + static_cast<int64_t>(g) * kGroup), g);
    if (g < n_groups) take(load_ragged<DT>(row + static_cast<int64_t>(g) * kGroup, n - whole * kGroup), g);

    // What rounding ref_c has moved all exponents by.
    if (ref != lowest) {
        const float off = -__fmaf_rn(ref, c, -ref_c), f = __builtin_amdgcn_exp2f(off);
        s = f * __fmaf_rn(off, z, s);
        z *= f;
    }
    const int32_t wave = tid / LD_WAVE;
    uint32_t top_order = wave_max(high);
    if (kWaves > 1) {
        if (ld_lane() == 0) wave_high[wave] = top_order;
        __syncthreads();
        for (int w = 0; w < kWaves; ++w) top_order = max(top_order, wave_high[w]);
    }
    const float most = value_of(top_order);
    Sums r = moved({ref, z, s}, most, c);
    if (most != -__builtin_huge_valf() && !(fabsf(most) * c < kSteady)) {
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
    float log_z = 0.0f;
    if (a.sums) {
        if (tid == 0) a.sums[blockIdx.x + a.row0 * a.parts] = make_float4(r.high, r.z, r.s, 0.0f);
    } else if (tid == 0) {
        bool inside;
        const float x = picked_of<DT>(a, t, inside);
        log_z = finish(a, t, r, x, inside);
    }
    if (!TOP) return;

    // The maxima above passed NaN over: where there is one, or an infinity, all groups are ordered once more, one element at a time.
    if (r.z != r.z) {
        high = 0;
        for (int32_t q = tid; q < n_groups; q += THREADS) {
            uint32_t o = 0;
            for (int32_t e = q * kGroup; e < min(q * kGroup + kGroup, n); ++e) o = max(o, order_of(static_cast<float>(row[e])));
            groups[q] = o;
            if (o > high) high = o, at = q;
        }
    }
    // The best K elements lie in the K groups whose largest elements are the best K (of equal ones the lower), and those in the K
    // threads of which the same holds.
    const int32_t K = a.top;
    __syncthreads();
    const uint64_t mine = high ? key_of(high, at) : 0;
    keys[tid] = mine;
    if (tid == 0) list_count = 0, kth = 0;
    __syncthreads();
    int32_t rank = 0;
    for (int j = 0; j < THREADS; ++j) rank += keys[j] > mine;
    if (rank == K - 1 && mine) kth = mine;
    __syncthreads();
    // Groups of those threads that are no worse than the K-th thread's best, behind the maxima.
    const uint64_t least = kth;
    uint32_t* list = groups + n_groups;
    if (mine >= least)
        for (int32_t q = tid; q < n_groups; q += THREADS)
            if (key_of(groups[q], q) >= least) list[atomicAdd(&list_count, 1u)] = q;
    __syncthreads();
    const int32_t listed = list_count, kept = min(listed, K);
    for (int32_t i = tid; i < listed; i += THREADS) {
        const uint64_t k = key_of(groups[list[i]], list[i]);
        int32_t better = 0;
        for (int32_t j = 0; j < listed; ++j) better += key_of(groups[list[j]], list[j]) > k;
        if (better < K) picked_groups[better] = list[i];
    }
    __syncthreads();
    for (int32_t i = tid; i < kept * kGroup; i += THREADS) {
        const int32_t e = static_cast<int32_t>(picked_groups[i / kGroup]) * kGroup + i % kGroup;
        keys[i] = e < n ? key_of(order_of(static_cast<float>(row[e])), begin + e) : 0;
    }
    if (tid == 0) wave_sums[0] = {r.high, log_z, 0.0f};
    __syncthreads();
    log_z = wave_sums[0].z;
    uint64_t* best = a.best ? a.best + (a.row0 * a.parts + blockIdx.x) * K : nullptr;
    for (int32_t i = tid; i < kept * kGroup; i += THREADS) {
        const uint64_t k = keys[i];
        int32_t better = 0;
        for (int32_t j = 0; j < kept * kGroup; ++j) better += keys[j] > k;
        if (better >= K || !k) continue;
        if (best) best[better] = k;
        else write_top(a, t, better, k, r.high, log_z);
    }
    if (best)  // a part of fewer elements
        for (int32_t i = n + tid; i < K; i += THREADS) best[i] = 0;
}

// A wave joins the parts of a row.
template <int DT>
__global__ __launch_bounds__(LD_WAVE) void k_score_join(ScoreArgs a) {
    constexpr int kEach = (LD_MAX_VOCAB / kMostPart + LD_WAVE - 1) / LD_WAVE;
    const int64_t t = a.row0 + blockIdx.x;
    const float4* sums = a.sums + t * a.parts;
    const int32_t lane = threadIdx.x;
    const float c = a.scale * kLog2e;
    uint32_t high = 0;
    for (int32_t p = lane; p < a.parts; p += LD_WAVE) high = max(high, order_of(sums[p].x));
    const float most = value_of(wave_max(high));
    float z = 0.0f, s = 0.0f;
    for (int32_t p = lane; p < a.parts; p += LD_WAVE) {
        const float4 x = sums[p];
        const Sums r = moved({x.x, x.y, x.z}, most, c);
        z += r.z, s += r.s;
    }
    const Sums r = {most, wave_sum(z), wave_sum(s)};
    float log_z = 0.0f;
    if (lane == 0) {
        bool inside;
        const float x = picked_of<DT>(a, t, inside);
        log_z = finish(a, t, r, x, inside);
    }
    if (a.top == 0) return;
    log_z = __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(log_z)));
    // Every lane holds the next of up to kEach parts' lists; the best of all is written, and its list moves on.
    const uint64_t* best = a.best + t * a.parts * a.top;
    uint64_t next[kEach];
    int32_t used[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int32_t p = lane + i * LD_WAVE;
        used[i] = 0;
        next[i] = p < a.parts ? best[static_cast<int64_t>(p) * a.top] : 0;
    }
    for (int32_t k = 0; k < a.top; ++k) {
        uint64_t mine = next[0];
#pragma unroll
        for (int i = 1; i < kEach; ++i) mine = max(mine, next[i]);
        const uint32_t hi = wave_max(static_cast<uint32_t>(mine >> 32));
        const uint32_t lo = wave_max(static_cast<uint32_t>(mine >> 32) == hi ? static_cast<uint32_t>(mine) : 0u);
        const uint64_t winner = static_cast<uint64_t>(hi) << 32 | lo;
        if (lane == 0) write_top(a, t, k, winner, most, log_z);
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (next[i] == winner && winner) {
                const int32_t p = lane + i * LD_WAVE;
                next[i] = ++used[i] < a.top ? best[static_cast<int64_t>(p) * a.top + used[i]] : 0;
            }
    }
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
    int32_t V, chunks;
    float scale;
    int32_t wide_ids;
};

constexpr int kGradUnroll = 4;

template <int OT>
__device__ __forceinline__ void store_group(typename LdElem<OT>::type* p, const f32x8& y) {
    if constexpr (OT == LD_F32) {
        typedef LdVec<LD_F32, 4> V;
        __builtin_nontemporal_store(typename V::type(__builtin_shufflevector(y, y, 0, 1, 2, 3)), reinterpret_cast<typename V::type*>(p));
        __builtin_nontemporal_store(typename V::type(__builtin_shufflevector(y, y, 4, 5, 6, 7)), reinterpret_cast<typename V::type*>(p + 4));
    } else {
        typedef LdVec<OT, 8> V;
        __builtin_nontemporal_store(V::narrow(y), reinterpret_cast<typename V::type*>(p));
    }
}

// A chunk of a row. Every element is read and written by one thread, so that the gradient may take the logits' place.
template <int DT, int OT, int THREADS, bool ENTROPY>
__global__ __launch_bounds__(THREADS) void k_score_grad(GradArgs a) {
    typedef typename LdElem<DT>::type elem;
    typedef typename LdElem<OT>::type out_elem;
    constexpr int32_t kChunk = THREADS * kGroup * kGradUnroll;
    const int64_t t = a.row0 + blockIdx.x / a.chunks;
    const int32_t begin = blockIdx.x % a.chunks * kChunk, n = min(a.V - begin, kChunk);
    const elem* row = static_cast<const elem*>(a.logits) + t * a.stride + begin;
    out_elem* out = static_cast<out_elem*>(a.out) + t * a.out_stride + begin;
    const float high = a.stats[2 * t], log_z = a.stats[2 * t + 1];  // the largest logit, L
    const bool empty = high == -__builtin_huge_valf();
    int64_t id = a.ids ? id_at(a.ids, t, a.wide_ids) : -1;
    const bool inside = id >= 0 && id < a.V;
    const float g = inside ? a.scale * a.d_logprob[t * a.d_logprob_stride] : 0.0f;
    const int32_t named = inside && id >= begin && id < begin + n ? static_cast<int32_t>(id - begin) : -1;
    const float h = ENTROPY ? a.scale * a.d_entropy[t * a.d_entropy_stride] : 0.0f, entropy = ENTROPY ? a.entropy[t] : 0.0f;
    const auto at = [&](float x, int32_t i) {
        const float logp = __fmaf_rn(x - high, a.scale, -log_z), p = __builtin_amdgcn_exp2f(logp * kLog2e);
        float d = (i == named ? g : 0.0f) - p * g;
        if (ENTROPY) d -= p > 0.0f ? h * (p * (logp + entropy)) : 0.0f;
        return empty ? 0.0f : d;
    };
    const int32_t whole = n / kGroup;
    f32x8 x[kGradUnroll];
#pragma unroll
    for (int u = 0; u < kGradUnroll; ++u) {
        const int32_t q = threadIdx.x + u * THREADS;
        if (q < whole) x[u] = load_group<DT>(row + q * kGroup);
    }
#pragma unroll
    for (int u = 0; u < kGradUnroll; ++u) {
        const int32_t q = threadIdx.x + u * THREADS;
        if (q >= whole) continue;
        f32x8 y;
#pragma unroll
        for (int e = 0; e < kGroup; ++e) y[e] = at(x[u][e], q * kGroup + e);
        store_group<OT>(out + q * kGroup, y);
    }
    const int32_t rest = whole * kGroup + static_cast<int32_t>(threadIdx.x);
    if (rest < n) out[rest] = static_cast<out_elem>(at(static_cast<float>(row[rest]), rest));
}

// How a call splits its rows.
struct Split {
    int32_t part, parts;
    bool narrow;
};
Split split_of(int64_t T, int32_t V) {
    if (V <= kNarrowElems && T >= kWorkgroups) return {V, 1, true};
    const int32_t most = (V + kPartStep - 1) / kPartStep, least = (V + kMostPart - 1) / kMostPart;
    int64_t parts = T > 0 ? (kWorkgroups + T - 1) / T : 1;
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
    // maxima of the groups, and the list of those that `top` threads hold
    const int32_t n_groups = (sp.part + kGroup - 1) / kGroup, of_thread = (n_groups + threads - 1) / threads;
    const size_t shared = top ? (n_groups + static_cast<size_t>(n_groups < top * of_thread ? n_groups : top * of_thread)) * sizeof(uint32_t) : 0;
    const int64_t most = ld_workgroups(static_cast<int64_t>(1) << 40, threads) / sp.parts;  // rows of a launch
    for (int64_t t = 0; t < T; t += most) {
        const int64_t rows = T - t < most ? T - t : most;
        const ScoreArgs a = {logits, ids, logprob, entropy, stats, top_ids, top_logprob, sums, best, stride, t,
                             V, sp.part, sp.parts, top, scale, id_dtype == LD_I64};
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
        ld_with_type(dtype, [&](auto type) { k_score_join<type><<<dim3(static_cast<uint32_t>(rows)), dim3(LD_WAVE), 0, st>>>(a); });
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
    const bool narrow = V <= kNarrow * kGroup * kGradUnroll;
    const int32_t threads = narrow ? kNarrow : kWide, chunk = threads * kGroup * kGradUnroll, chunks = (V + chunk - 1) / chunk;
    const int64_t most = ld_workgroups(static_cast<int64_t>(1) << 40, threads) / chunks;
    for (int64_t t = 0; t < T; t += most) {
        const int64_t rows = T - t < most ? T - t : most;
        const GradArgs a = {logits, ids, stats, d_logprob, entropy, d_entropy, d_logits, stride, out_stride, d_logprob_stride,
                            d_entropy_stride, t, V, chunks, scale, id_dtype == LD_I64};
        const dim3 grid(static_cast<uint32_t>(rows * chunks));
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
