// Embedding lookup with scaling: where a training step's or a request's tokens become the model's first activations.
//
//   out[t, c] = round(scale * table[id_t, c] + pos_table[position_t, c])
//
// A row outside its table counts as zeros (padding, say as id -1). One fused multiply-add in 32 bits, rounded once.
// Bound by memory: the named rows read, T rows written. 32768 tokens of 4096 bf16 columns 60 us (5.6 TB/s), 16384 of 1600 with
// positions 16.
#include <type_traits>

#include "ld_elem.h"

namespace {

constexpr int kThreads = 256;
// An output past what the second-level caches hold is written around them, and in shorter steps (vectors of a row that a thread loads
// before it stores the first): 268 MB 79 us kept, 61 streamed, 64 in steps of 4; a smaller one stays for the layer that reads it next (8191
// rows of 768 8.5 us in steps of 4, 9.3 of 2).
constexpr int64_t kStreamed = 32 << 20;
template <bool STREAM> constexpr int steps() { return STREAM ? 2 : 4; }

struct LookupArgs {
    const void* table;
    const void* pos_table;  // NULL: none
    const void* ids;
    const void* positions;
    void* out;
    int64_t V, P, T;
    int64_t table_stride, pos_stride, out_stride;  // elements from a row to the next
    int32_t d;
    float scale;
    int32_t lanes_log2;     // threads of a row
    int32_t wide_ids;       // 64-bit ids and positions
};

__device__ __forceinline__ int64_t id_at(const void* ids, int64_t t, int32_t wide) {
    return wide ? static_cast<const int64_t*>(ids)[t] : static_cast<const int32_t*>(ids)[t];
}

// Threads in groups of 2^lanes_log2, a token each. A row's last vector begins where it ends with the row and so may name
// elements of the one before once more, the same values.
template <int DT, int OT, bool STREAM>
__global__ __launch_bounds__(kThreads) void k_lookup(LookupArgs a) {
    constexpr int N = DT == LD_F32 || OT == LD_F32 ? 4 : 8, kUnroll = steps<STREAM>();
    typedef LdVec<DT, N> V;
    typedef LdVec<OT, N> O;
    const int32_t lanes = 1 << a.lanes_log2;
    const int64_t t = static_cast<int64_t>(blockIdx.x) * (kThreads >> a.lanes_log2) + (threadIdx.x >> a.lanes_log2);
    if (t >= a.T) return;
    const int64_t id = id_at(a.ids, t, a.wide_ids), at = a.pos_table ? id_at(a.positions, t, a.wide_ids) : -1;
    const bool named = id >= 0 && id < a.V, placed = at >= 0 && at < a.P;
    const typename V::elem* row = static_cast<const typename V::elem*>(a.table) + (named ? id : 0) * a.table_stride;
    const typename V::elem* pos = static_cast<const typename V::elem*>(a.pos_table) + (placed ? at : 0) * a.pos_stride;
    typename O::elem* out = static_cast<typename O::elem*>(a.out) + t * a.out_stride;
    const int32_t lane = threadIdx.x & (lanes - 1);
    if (a.d < N) {
        for (int32_t c = lane; c < a.d; c += lanes) {
            const float x = named ? static_cast<float>(row[c]) : 0.0f, p = placed ? static_cast<float>(pos[c]) : 0.0f;
            out[c] = static_cast<typename O::elem>(a.pos_table ? __fmaf_rn(a.scale, x, p) : a.scale * x);
        }
        return;
    }
    const int32_t vectors = (a.d + N - 1) / N, end = a.d - N;
    for (int32_t v0 = lane; v0 < vectors; v0 += lanes * kUnroll) {
        typename V::type x[kUnroll], p[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int32_t v = v0 + u * lanes, c = v * N < end ? v * N : end;
            x[u] = typename V::type(0);
            p[u] = typename V::type(0);
            if (v < vectors && named) x[u] = *reinterpret_cast<const typename V::type*>(row + c);
            if (v < vectors && placed) p[u] = *reinterpret_cast<const typename V::type*>(pos + c);
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int32_t v = v0 + u * lanes, c = v * N < end ? v * N : end;
            const typename V::wide xw = V::widen(x[u]), pw = V::widen(p[u]);
            typename V::wide y;
#pragma unroll
            for (int e = 0; e < N; ++e) y[e] = a.pos_table ? __fmaf_rn(a.scale, xw[e], pw[e]) : a.scale * xw[e];
            if (v < vectors) {
                typename O::type* to = reinterpret_cast<typename O::type*>(out + c);
                if (STREAM) __builtin_nontemporal_store(O::narrow(y), to);
                else *to = O::narrow(y);
            }
        }
    }
}

}  // namespace

extern "C" ld_status ld_embed_lookup(const void* table, int64_t V, int64_t table_stride, const void* pos_table, int64_t P,
                                     int64_t pos_stride, int32_t dtype, const void* ids, const void* positions, int32_t id_dtype,
                                     int64_t T, int32_t d, float scale, void* out, int64_t out_stride, int32_t out_dtype,
                                     ld_stream stream) {
    if (V < 0 || T < 0 || d < 0 || d > LD_MAX_WIDTH || table_stride < 0 || out_stride < d || !ld_known_type(dtype) || !ld_known_type(out_dtype) ||
        (id_dtype != LD_I32 && id_dtype != LD_I64))
        return LD_ERR_RANGE;
    if (pos_table && (P < 0 || pos_stride < 0)) return LD_ERR_RANGE;
    if (T == 0 || d == 0) return LD_OK;
    if ((V > 0 && !table) || !ids || !out || (pos_table && !positions)) return LD_ERR_NULL;
    const int32_t in = ld_type_bytes(dtype), id_bytes = id_dtype == LD_I32 ? 4 : 8;
    if (!ld_aligned(table, in) || !ld_aligned(pos_table, in) || !ld_aligned(out, ld_type_bytes(out_dtype)) ||
        !ld_aligned(ids, id_bytes) || !ld_aligned(positions, id_bytes))
        return LD_ERR_ALIGN;
    const int32_t n = dtype == LD_F32 || out_dtype == LD_F32 ? 4 : 8, vectors = (d + n - 1) / n;
    const bool streamed = T * static_cast<int64_t>(d) * ld_type_bytes(out_dtype) > kStreamed;
    const int32_t unroll = streamed ? steps<true>() : steps<false>();
    int32_t lanes_log2 = 0;
    while (lanes_log2 < 8 && (unroll << lanes_log2) < vectors) ++lanes_log2;
    // few tokens: fewer vectors a thread, so that more of the chip loads at once
    while (lanes_log2 < 8 && (1 << lanes_log2) < vectors && (T << lanes_log2) < 256 * 1024) ++lanes_log2;
    const int64_t per = kThreads >> lanes_log2, most = per << 23;  // tokens of a launch, which has fewer than 2^32 threads
    hipStream_t st = static_cast<hipStream_t>(stream);
    ld_begin_call();
    for (int64_t t = 0; t < T; t += most) {
        const int64_t tokens = T - t < most ? T - t : most;
        const LookupArgs a = {table, pos_table, static_cast<const char*>(ids) + t * id_bytes,
                              positions ? static_cast<const char*>(positions) + t * id_bytes : nullptr,
                              static_cast<char*>(out) + t * out_stride * ld_type_bytes(out_dtype), V, P, tokens, table_stride, pos_stride,
                              out_stride, d, scale, lanes_log2, id_dtype == LD_I64};
        const dim3 grid(static_cast<uint32_t>((tokens + per - 1) / per));
        ld_with_type(dtype, [&](auto type) {
            ld_with_type(out_dtype, [&](auto out_type) {
                if (streamed) k_lookup<type, out_type, true><<<grid, dim3(kThreads), 0, st>>>(a);
                else k_lookup<type, out_type, false><<<grid, dim3(kThreads), 0, st>>>(a);
            });
        });
        if (ld_launch_status() != LD_OK) return LD_ERR_HIP;
    }
    return LD_OK;
}
