// The embedding's gradient from the gradient of its rows: the lookup's backward pass.
//
//   grad[v, c] = round(beta * grad[v, c] + scale * sum of dout[t, c] over the tokens t with id_t = v),  beta = 0 or 1
//
// The tokens are sorted by their id first (stable), so that a row's are next to one another and in order: every sum is made in an
// order that the sizes alone decide, without float atomics. What the same batch gives is the same bit for bit, as error feedback
// and a recovery that replays differentials need it.
#include <type_traits>

#include "ld_elem.h"

namespace {

// ------------------------------------------------------------------ sort

// Least significant digit first, two launches a digit: every tile counts its digits, then finds from all tiles' counts where
// each of its digits goes and moves its tokens there.
constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / LD_WAVE;
constexpr int kSortRounds = 4;                             // tokens of a lane
constexpr int kTile = kSortThreads * kSortRounds;          // tokens of a workgroup
constexpr int kWaveTokens = LD_WAVE * kSortRounds;         // consecutive tokens of a wave
constexpr int kDigitBits = 11;                             // most bits of a digit
constexpr int kBins = 1 << kDigitBits;

struct SortArgs {
    const void* ids;         // the first digit's input, else NULL
    int32_t wide_ids;
    const uint32_t* keys_in;
    const uint32_t* at_in;
    uint32_t* keys_out;
    uint32_t* at_out;
    uint32_t* counts;        // [tiles][1 << bits]
    int64_t V;
    int32_t T, tiles, shift, bits;
};

// A token's key: its id, or V for one that names no row.
__device__ __forceinline__ uint32_t key_of(const SortArgs& a, int32_t i) {
    if (!a.ids) return a.keys_in[i];
    const int64_t id = a.wide_ids ? static_cast<const int64_t*>(a.ids)[i] : static_cast<const int32_t*>(a.ids)[i];
    return static_cast<uint32_t>(id >= 0 && id < a.V ? id : a.V);
}

__global__ __launch_bounds__(kSortThreads) void k_sort_count(SortArgs a) {
    __shared__ uint32_t count[kBins];
    const int32_t bins = 1 << a.bits;
    for (int32_t i = threadIdx.x; i < bins; i += kSortThreads) count[i] = 0;
    __syncthreads();
    const int32_t base = blockIdx.x * kTile;
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) {
        const int32_t i = base + r * kSortThreads + threadIdx.x;
        if (i < a.T) atomicAdd(&count[(key_of(a, i) >> a.shift) & (bins - 1)], 1u);
    }
    __syncthreads();
    for (int32_t i = threadIdx.x; i < bins; i += kSortThreads) a.counts[static_cast<size_t>(blockIdx.x) * bins + i] = count[i];
}

__global__ __launch_bounds__(kSortThreads) void k_sort_move(SortArgs a) {
    __shared__ uint32_t first[kBins];                 // where this tile's tokens of a digit begin in the output
    __shared__ uint16_t before[kSortWaves][kBins];    // of a digit, in the waves before (while counting: in this wave so far)
    __shared__ uint32_t wave_total[kSortWaves];
    const int32_t bins = 1 << a.bits, wave = threadIdx.x / LD_WAVE;
    const uint32_t mask = bins - 1;

    // a digit's tokens in the tiles before this one, and in all of them
    constexpr int kPer = kBins / kSortThreads;
    uint32_t mine[kPer], all[kPer], sum = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int32_t b = threadIdx.x * kPer + j;
        mine[j] = all[j] = 0;
        if (b < bins) {
            for (int32_t t = 0; t < a.tiles; ++t) {
                const uint32_t c = a.counts[static_cast<size_t>(t) * bins + b];
                all[j] += c;
                if (t < static_cast<int32_t>(blockIdx.x)) mine[j] += c;
            }
        }
        sum += all[j];
    }
    const uint32_t upto = ld_wave_iscan(sum);
    if (ld_lane() == LD_WAVE - 1) wave_total[wave] = upto;
    for (int32_t i = threadIdx.x; i < bins; i += kSortThreads)
        for (int w = 0; w < kSortWaves; ++w) before[w][i] = 0;
    __syncthreads();
    uint32_t from = upto - sum;
    for (int w = 0; w < wave; ++w) from += wave_total[w];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int32_t b = threadIdx.x * kPer + j;
        if (b < bins) first[b] = from + mine[j];
        from += all[j];
    }

    // a token's rank among those of its digit in its wave: earlier rounds, and the lanes below in its own
    uint32_t key[kSortRounds], at[kSortRounds], rank[kSortRounds];
    const int32_t base = blockIdx.x * kTile + wave * kWaveTokens + ld_lane();
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) {
        const int32_t i = base + r * LD_WAVE;
        const bool in = i < a.T;
        key[r] = in ? key_of(a, i) : 0;
        at[r] = in && a.at_in ? a.at_in[i] : static_cast<uint32_t>(i);
        const uint32_t digit = (key[r] >> a.shift) & mask;
        uint64_t same = __ballot(in);
        for (int32_t b = 0; b < a.bits; ++b) {
            const uint64_t set = __ballot((digit >> b) & 1);
            same &= (digit >> b) & 1 ? set : ~set;
        }
        const uint32_t below = ld_mbcnt(same);
        uint32_t so_far = 0;
        if (in) so_far = before[wave][digit];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (in && below == 0) before[wave][digit] = static_cast<uint16_t>(so_far + __popcll(same));
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        rank[r] = so_far + below;
    }
    __syncthreads();
    for (int32_t i = threadIdx.x; i < bins; i += kSortThreads) {
        uint32_t total = 0;
        for (int w = 0; w < kSortWaves; ++w) {
            const uint32_t c = before[w][i];
            before[w][i] = static_cast<uint16_t>(total);
            total += c;
        }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) {
        if (base + r * LD_WAVE < a.T) {
            const uint32_t digit = (key[r] >> a.shift) & mask;
            const uint32_t to = first[digit] + before[wave][digit] + rank[r];
            a.keys_out[to] = key[r];
            a.at_out[to] = at[r];
        }
    }
}

// ------------------------------------------------------------------- rows

struct RowArgs {
    const void* dout;
    const uint32_t* keys;   // sorted
    const uint32_t* at;     // the tokens in that order
    void* grad;
    int64_t dout_stride, grad_stride;
    int32_t T, V, d;
    float scale;
    int32_t accumulate;
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

// A workgroup per row of the table.
template <int DT, int GT>
__global__ __launch_bounds__(256) void k_rows(RowArgs a) {
    const uint32_t v = blockIdx.x;
    const int32_t from = lower_bound(a.keys, a.T, v), to = lower_bound(a.keys, a.T, v + 1);
    if (from == to && a.accumulate) return;
    const typename LdElem<DT>::type* dout = static_cast<const typename LdElem<DT>::type*>(a.dout);
    typename LdElem<GT>::type* grad = static_cast<typename LdElem<GT>::type*>(a.grad) + static_cast<int64_t>(v) * a.grad_stride;
    for (int32_t c = threadIdx.x; c < a.d; c += 256) {
        float sum = 0.0f;
        for (int32_t i = from; i < to; ++i) sum += static_cast<float>(dout[a.at[i] * a.dout_stride + c]);
        grad[c] = static_cast<typename LdElem<GT>::type>(a.accumulate ? __fmaf_rn(a.scale, sum, static_cast<float>(grad[c])) : a.scale * sum);
    }
}

struct Layout {
    int32_t passes, bits, tiles;
    size_t keys, at, counts, bytes;  // byte offsets: two buffers each of keys and tokens
};

Layout layout_of(int64_t T, int64_t V) {
    Layout l;
    int32_t all = 1;
    while ((V >> all) != 0) ++all;  // bits of the keys 0 .. V
    l.passes = (all + kDigitBits - 1) / kDigitBits;
    l.bits = (all + l.passes - 1) / l.passes;
    l.tiles = static_cast<int32_t>((T + kTile - 1) / kTile);
    const size_t list = ld_round_up(static_cast<size_t>(T) * 4, 256);
    l.keys = 0;
    l.at = 2 * list;
    l.counts = 4 * list;
    l.bytes = ld_round_up(l.counts + (static_cast<size_t>(l.tiles) << l.bits) * 4, 256);
    return l;
}

bool sizes_fit(int64_t T, int64_t V, int32_t d) {
    return T >= 0 && V >= 0 && d >= 0 && T <= LD_MAX_TOKENS && V < INT32_MAX;
}

}  // namespace

extern "C" size_t ld_embed_grad_workspace(int64_t T, int64_t V, int32_t d) {
    return sizes_fit(T, V, d) ? layout_of(T, V).bytes : 0;
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
    const Layout l = layout_of(T, V);
    if (l.bytes > 0 && (!workspace || !ld_aligned(workspace, 256) || workspace_bytes < l.bytes)) return LD_ERR_WORKSPACE;
    hipStream_t s = static_cast<hipStream_t>(stream);
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    uint32_t* keys[2] = {reinterpret_cast<uint32_t*>(ws + l.keys), reinterpret_cast<uint32_t*>(ws + l.keys + l.at / 2)};
    uint32_t* at[2] = {reinterpret_cast<uint32_t*>(ws + l.at), reinterpret_cast<uint32_t*>(ws + l.at + l.at / 2)};
    ld_begin_call();
    for (int32_t p = 0; p < l.passes && T > 0; ++p) {
        const SortArgs a = {p == 0 ? ids : nullptr, id_dtype == LD_I64, keys[(p + 1) & 1], p == 0 ? nullptr : at[(p + 1) & 1], keys[p & 1],
                            at[p & 1], reinterpret_cast<uint32_t*>(ws + l.counts), V, static_cast<int32_t>(T), l.tiles, p * l.bits, l.bits};
        k_sort_count<<<dim3(l.tiles), dim3(kSortThreads), 0, s>>>(a);
        if (ld_launch_status() != LD_OK) return LD_ERR_HIP;
        k_sort_move<<<dim3(l.tiles), dim3(kSortThreads), 0, s>>>(a);
        if (ld_launch_status() != LD_OK) return LD_ERR_HIP;
    }
    const int32_t last = (l.passes + 1) & 1;
    const RowArgs a = {dout, keys[last], at[last], grad, dout_stride, grad_stride, static_cast<int32_t>(T), static_cast<int32_t>(V), d, scale,
                       accumulate};
    ld_with_type(dtype, [&](auto type) {
        ld_with_type(grad_dtype, [&](auto grad_type) {
            k_rows<type, grad_type><<<dim3(static_cast<uint32_t>(V)), dim3(256), 0, s>>>(a);
        });
    });
    return ld_launch_status();
}
