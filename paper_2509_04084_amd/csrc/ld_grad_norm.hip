// The norm of a step's whole gradient, over many tensors, and clipping by it: what a training loop does between the
// backward pass and ld_compress_topk / ld_snapshot_layers.
//
//   S = sum over all elements of x^2;  norm = sqrt(S);  factor = norm > max_norm ? max_norm / norm : 1
//   out = round(x * factor)
//
// Squares and sums are 64 bits wide: the square of a 32-bit value is exact there and can neither overflow nor vanish, and the
// conversion and the addition cost nothing beside the memory (6.7 TB/s of bf16). Bound by memory: n elements read for S, read
// again and written for the clipped values; a gradient in place under the limit is not touched a second time. GPT-2 XL's 580
// bf16 gradients (3.1 GB) 462 us for the norm, 1002 for the clipped copy (6.2 TB/s); that the second reading begins where the
// first one ended, in what the last cache still holds, changed nothing.
#include <math.h>

#include <type_traits>

#include "ld_elem.h"
#include "ld_grid.h"

namespace {

constexpr int kThreads = kClipThreads;
constexpr int kUnroll = 4;                 // vectors per thread and piece
constexpr int kTensorGroup = 16;
constexpr int kNormGrid = 2048;            // workgroups of a launch, each with a partial sum
// Consecutive pieces that an XCD clips at a time, as for the snapshot: 3.1 GB of one tensor 1491 us in runs of 64, 1494 of 16, 1688 of 4, 1569
// piece by piece. The sum, in rounds of the same workgroups, is no faster so (490 us; 102 MB 25 instead of 23).
constexpr uint32_t kXcdRun = 64;
constexpr int64_t kAloneElems = 32768;     // up to here one workgroup does the whole call
constexpr int kAloneThreads = 1024;

// The tensors of a launch, in its arguments: up to GROUPS groups of 16, with DST where each goes to. A tensor is cut into pieces, the
// last one ragged.
template <int GROUPS, bool DST>
struct TensorBatch {
    static constexpr int kMost = GROUPS * kTensorGroup;
    static constexpr bool kDst = DST;
    int32_t first_of_group[kTensorGroup];  // [0]: all pieces; then every 16th of first_piece
    int32_t first_piece[kMost + 1];        // entries past the last tensor: all pieces
    const void* src[kMost];
    void* dst[DST ? kMost : 1];
    int16_t last[kMost];                   // elements of a tensor's last piece
};
typedef TensorBatch<16, false> SummedTensors;
typedef TensorBatch<11, true> ClippedTensors;
// Host time of a launch with 4 KB of arguments 4.6 us, with 400 bytes 4.2
typedef TensorBatch<1, false> FewSummed;
typedef TensorBatch<1, true> FewClipped;
static_assert(sizeof(SummedTensors) <= 4000 && sizeof(ClippedTensors) <= 4000, "the arguments of a kernel must fit 4 KB");

// The tensor that a piece belongs to: two reads of 16 consecutive entries each.
template <int GROUPS, bool DST>
__device__ __forceinline__ int tensor_of(const TensorBatch<GROUPS, DST>& b, int32_t piece) {
    int group = 0, t = 0;
    if (GROUPS > 1) {
#pragma unroll
        for (int i = 1; i < kTensorGroup; ++i) group += b.first_of_group[i] <= piece;
    }
    const int32_t* first = b.first_piece + group * kTensorGroup;
#pragma unroll
    for (int i = 1; i < kTensorGroup; ++i) t += first[i] <= piece;
    return group * kTensorGroup + t;
}

template <int N> constexpr int piece_elems() { return kThreads * kUnroll * N; }

// Sum over a workgroup, the same order every time; in every thread of it.
__device__ __forceinline__ double block_sum(double x, double* sh) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
    const int waves = blockDim.x / LD_WAVE;
    if (ld_lane() == 0) sh[threadIdx.x / LD_WAVE] = x;
    __syncthreads();
    double total = 0.0;
    for (int w = 0; w < waves; ++w) total += sh[w];
    return total;
}

// Where a piece lies, and its elements.
struct Piece {
    int tensor;
    int64_t first;
    int32_t have;
};

template <int N, typename B>
__device__ __forceinline__ Piece piece_of(const B& b, int32_t p) {
    const int t = tensor_of(b, p);
    return {t, static_cast<int64_t>(p - b.first_piece[t]) * piece_elems<N>(),
            p + 1 == b.first_piece[t + 1] ? b.last[t] : piece_elems<N>()};
}

// The squares of a thread's part of a piece, which THREADS share, this one being the `me`-th. Read around the caches: 81 us instead of 90
// for 498 MB of fp32.
template <int DT, int N, int THREADS, typename B>
__device__ __forceinline__ double squares(const B& b, int32_t p, int32_t me, double sum) {
    typedef LdVec<DT, N> V;
    const Piece at = piece_of<N>(b, p);
    const typename V::elem* src = static_cast<const typename V::elem*>(b.src[at.tensor]) + at.first;
#pragma unroll
    for (int u = 0; u < piece_elems<N>() / N / THREADS; ++u) {
        const int32_t i = (u * THREADS + me) * N;
        if (i + N <= at.have) {
            const typename V::wide x = V::widen(__builtin_nontemporal_load(reinterpret_cast<const typename V::type*>(src + i)));
#pragma unroll
            for (int e = 0; e < N; ++e) sum = fma(static_cast<double>(x[e]), static_cast<double>(x[e]), sum);
        } else {
            for (int32_t e = i; e < at.have && e < i + N; ++e) {
                const double x = static_cast<double>(static_cast<float>(src[e]));
                sum = fma(x, x, sum);
            }
        }
    }
    return sum;
}

// A thread's part of a piece scaled.
template <int DT, int OT, int N, int THREADS, typename B>
__device__ __forceinline__ void scale_piece(const B& b, int32_t p, int32_t me, float factor) {
    constexpr int kVectors = piece_elems<N>() / N / THREADS;
    typedef LdVec<DT, N> V;
    typedef LdVec<OT, N> O;
    const Piece at = piece_of<N>(b, p);
    const typename V::elem* src = static_cast<const typename V::elem*>(b.src[at.tensor]) + at.first;
    typename O::elem* dst = static_cast<typename O::elem*>(b.dst[at.tensor]) + at.first;
    if (at.have == piece_elems<N>()) {
        const typename V::type* v = reinterpret_cast<const typename V::type*>(src) + me;
        typename O::type* o = reinterpret_cast<typename O::type*>(dst) + me;
#pragma unroll 1
        for (int u0 = 0; u0 < kVectors; u0 += kUnroll) {
            typename V::type x[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) x[u] = __builtin_nontemporal_load(v + (u0 + u) * THREADS);
#pragma unroll
            for (int u = 0; u < kUnroll; ++u)
                __builtin_nontemporal_store(O::narrow(V::widen(x[u]) * factor), o + (u0 + u) * THREADS);
        }
        return;
    }
#pragma unroll kUnroll
    for (int u = 0; u < kVectors; ++u) {
        const int32_t i = (u * THREADS + me) * N;
        if (i + N <= at.have) {
            const typename V::type x = *reinterpret_cast<const typename V::type*>(src + i);
            *reinterpret_cast<typename O::type*>(dst + i) = O::narrow(V::widen(x) * factor);
        } else {
            for (int32_t e = i; e < at.have && e < i + N; ++e)
                dst[e] = static_cast<typename O::elem>(static_cast<float>(src[e]) * factor);
        }
    }
}

// A norm that is not finite clips nothing: the caller sees it in the norm.
__device__ __forceinline__ float factor_of(double sumsq, float max_norm) {
    const double norm = sqrt(sumsq);
    return norm > max_norm && norm < __builtin_huge_val() ? static_cast<float>(max_norm / norm) : 1.0f;
}

template <int DT, typename B>
__global__ __launch_bounds__(kThreads) void k_sum_squares(B b, double* __restrict__ part) {
    __shared__ double sh[kThreads / LD_WAVE];
    double sum = 0.0;
    for (int32_t p = blockIdx.x; p < b.first_of_group[0]; p += gridDim.x) sum = squares<DT, DT == LD_F32 ? 4 : 8, kThreads>(b, p, threadIdx.x, sum);
    sum = block_sum(sum, sh);
    if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

// The sum of `count` partial sums, by a workgroup; the same in every workgroup of THREADS threads.
__device__ __forceinline__ double sum_of(const double* __restrict__ part, int32_t count, double* sh) {
    if (count == 1) return *part;
    double sum = 0.0;
    for (int32_t i = threadIdx.x; i < count; i += blockDim.x) sum += part[i];
    return block_sum(sum, sh);
}

__global__ __launch_bounds__(kAloneThreads) void k_norm_finish(const double* __restrict__ part, int32_t count, int32_t accumulate,
                                                               double* __restrict__ sumsq, float* __restrict__ norm) {
    __shared__ double sh[kAloneThreads / LD_WAVE];
    double sum = sum_of(part, count, sh);
    if (threadIdx.x == 0) {
        if (accumulate) sum += *sumsq;
        *sumsq = sum;
        if (norm) *norm = static_cast<float>(sqrt(sum));
    }
}

// Every workgroup adds up the partial sums itself (`count` of them; one: the sum is known). norm: written where it is not yet.
template <int DT, int OT, typename B>
__global__ __launch_bounds__(kThreads) void k_clip(B b, const double* __restrict__ part, int32_t count, float max_norm, int32_t in_place,
                                                   float* __restrict__ norm) {
    __shared__ double sh[kThreads / LD_WAVE];
    const double sum = sum_of(part, count, sh);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = static_cast<float>(sqrt(sum));
    const float factor = factor_of(sum, max_norm);
    if (in_place && factor == 1.0f) return;
    const int32_t pieces = b.first_of_group[0], places = (pieces + 7) / 8 * 8;
    for (int32_t q = blockIdx.x; q < places; q += gridDim.x) {
        const int32_t p = static_cast<int32_t>(ld_xcd_piece<kXcdRun>(q, places));
        if (p < pieces) scale_piece<DT, OT, DT == LD_F32 || OT == LD_F32 ? 4 : 8, kThreads>(b, p, threadIdx.x, factor);
    }
}

// A small call by one workgroup, its waves taking pieces in turn (there may be many, of an element each).
template <int DT, int OT, typename B>
__global__ __launch_bounds__(kAloneThreads) void k_clip_alone(B b, float max_norm, int32_t in_place, float* __restrict__ norm) {
    constexpr int N = DT == LD_F32 || OT == LD_F32 ? 4 : 8;
    __shared__ double sh[kAloneThreads / LD_WAVE];
    double sum = 0.0;
    const int32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / LD_WAVE), waves = kAloneThreads / LD_WAVE;
    for (int32_t p = wave; p < b.first_of_group[0]; p += waves) sum = squares<DT, N, LD_WAVE>(b, p, ld_lane(), sum);
    sum = block_sum(sum, sh);
    if (threadIdx.x == 0) *norm = static_cast<float>(sqrt(sum));
    const float factor = factor_of(sum, max_norm);
    if (in_place && factor == 1.0f) return;
    for (int32_t p = wave; p < b.first_of_group[0]; p += waves) scale_piece<DT, OT, N, LD_WAVE>(b, p, ld_lane(), factor);
}

// A call's lists.
struct Lists {
    const void* const* src;
    void* const* dst;  // NULL: none
    const int64_t* n_elems;
    int32_t n_tensors, src_type, dst_type;
};

// Tensors [t, ...) of the lists as a launch takes them, in pieces of `piece` elements; t moves behind them. With `join` tensors that
// lie one behind the other, and go so, are one to it: the 420 parts of a flat gradient of 5 M elements are clipped in one launch, not three.
template <typename B>
void next_batch(B& b, const Lists& l, int32_t piece, bool join, int32_t& t) {
    int32_t count = 0;
    int64_t pieces = 0, elems = 0;  // of all tensors taken, and of the last
    const unsigned char *src_end = nullptr, *dst_end = nullptr;
    const int64_t src_bytes = ld_type_bytes(l.src_type), dst_bytes = ld_type_bytes(l.dst_type);
    for (; t < l.n_tensors; ++t) {
        if (l.n_elems[t] == 0) continue;
        if (B::kDst && join && count > 0 && l.src[t] == src_end && l.dst[t] == dst_end) {
            elems += l.n_elems[t];
        } else {
            if (count == B::kMost) break;
            b.src[count] = l.src[t];
            if (B::kDst) b.dst[count] = l.dst[t];
            b.first_piece[count] = static_cast<int32_t>(pieces);
            elems = l.n_elems[t];
            ++count;
        }
        const int64_t of_it = (elems + piece - 1) / piece;
        pieces = b.first_piece[count - 1] + of_it;
        b.last[count - 1] = static_cast<int16_t>(elems - (of_it - 1) * piece);
        src_end = static_cast<const unsigned char*>(l.src[t]) + l.n_elems[t] * src_bytes;
        if (B::kDst) dst_end = static_cast<const unsigned char*>(l.dst[t]) + l.n_elems[t] * dst_bytes;
    }
    for (int32_t i = count; i <= B::kMost; ++i) b.first_piece[i] = static_cast<int32_t>(pieces);
    b.first_of_group[0] = static_cast<int32_t>(pieces);
    for (int32_t g = 1; g < kTensorGroup; ++g)
        b.first_of_group[g] = g * kTensorGroup < B::kMost ? b.first_piece[g * kTensorGroup] : static_cast<int32_t>(pieces);
}

constexpr int64_t kMostElems = static_cast<int64_t>(1) << 41;  // of all tensors: 2^29 pieces of 4096, and one more a tensor

ld_status check_lists(const Lists& l, bool with_dst) {
    if (l.n_tensors < 0 || l.n_tensors > LD_MAX_TENSORS || !ld_known_type(l.src_type) || !ld_known_type(l.dst_type)) return LD_ERR_RANGE;
    if (l.n_tensors > 0 && (!l.src || !l.n_elems || (with_dst && !l.dst))) return LD_ERR_NULL;
    int64_t total = 0;
    for (int32_t t = 0; t < l.n_tensors; ++t) {
        if (l.n_elems[t] < 0 || l.n_elems[t] > kMostElems - total) return LD_ERR_RANGE;
        total += l.n_elems[t];
        if (l.n_elems[t] > 0 && (!l.src[t] || (with_dst && !l.dst[t]))) return LD_ERR_NULL;
        if (!ld_aligned(l.src[t], ld_type_bytes(l.src_type)) || (with_dst && !ld_aligned(l.dst[t], ld_type_bytes(l.dst_type)))) return LD_ERR_ALIGN;
    }
    return LD_OK;
}

// Partial sums of all launches, and behind them the sum of squares.
size_t partials_of(int32_t n_tensors) {
    return static_cast<size_t>((n_tensors + SummedTensors::kMost - 1) / SummedTensors::kMost) * kNormGrid;
}

// Enqueues the partial sums; `count` of them are left in `part`. Every tensor by itself, so that the sum's order is that of the sizes.
template <typename B>
ld_status sum_squares(const Lists& l, double* part, int32_t& count, hipStream_t s) {
    count = 0;
    for (int32_t t = 0; t < l.n_tensors;) {
        B b;
        next_batch(b, l, l.src_type == LD_F32 ? piece_elems<4>() : piece_elems<8>(), false, t);
        if (b.first_of_group[0] == 0) continue;
        const int32_t grid = b.first_of_group[0] < kNormGrid ? b.first_of_group[0] : kNormGrid;
        ld_with_type(l.src_type, [&](auto type) { k_sum_squares<type, B><<<dim3(grid), dim3(kThreads), 0, s>>>(b, part + count); });
        if (ld_launch_status() != LD_OK) return LD_ERR_HIP;
        count += grid;
    }
    return LD_OK;
}

ld_status sum_squares(const Lists& l, double* part, int32_t& count, hipStream_t s) {
    return l.n_tensors <= FewSummed::kMost ? sum_squares<FewSummed>(l, part, count, s) : sum_squares<SummedTensors>(l, part, count, s);
}

ld_status finish(const double* part, int32_t count, int32_t accumulate, double* sumsq, float* norm, hipStream_t s) {
    k_norm_finish<<<dim3(1), dim3(kAloneThreads), 0, s>>>(part, count, accumulate, sumsq, norm);
    return ld_launch_status();
}

// Enqueues the scaling by `count` partial sums; with `alone` the sums as well, the call being small.
template <typename B>
ld_status clip(const Lists& l, const double* part, int32_t count, float max_norm, float* norm, bool alone, hipStream_t s) {
    const int32_t piece = l.src_type == LD_F32 || l.dst_type == LD_F32 ? piece_elems<4>() : piece_elems<8>();
    for (int32_t t = 0; t < l.n_tensors;) {
        const int32_t from = t;
        B b;
        next_batch(b, l, piece, !alone, t);
        const int32_t pieces = b.first_of_group[0];
        if (pieces == 0 && !alone) continue;
        int32_t in_place = l.src_type == l.dst_type;
        for (int32_t i = from; i < t; ++i) in_place &= l.n_elems[i] == 0 || l.src[i] == l.dst[i];
        const dim3 grid(ld_clip_grid(pieces, in_place != 0));
        ld_with_type(l.src_type, [&](auto type) {
            ld_with_type(l.dst_type, [&](auto out_type) {
                if (alone) k_clip_alone<type, out_type, B><<<dim3(1), dim3(kAloneThreads), 0, s>>>(b, max_norm, in_place, norm);
                else k_clip<type, out_type, B><<<grid, dim3(kThreads), 0, s>>>(b, part, count, max_norm, in_place, norm);
            });
        });
        if (ld_launch_status() != LD_OK) return LD_ERR_HIP;
    }
    return LD_OK;
}

ld_status clip(const Lists& l, const double* part, int32_t count, float max_norm, float* norm, bool alone, hipStream_t s) {
    return l.n_tensors <= FewClipped::kMost ? clip<FewClipped>(l, part, count, max_norm, norm, alone, s)
                                            : clip<ClippedTensors>(l, part, count, max_norm, norm, alone, s);
}

// Whether one workgroup does a call.
bool done_alone(int32_t n_tensors, const int64_t* n_elems) {
    if (n_tensors <= 0 || n_tensors > ClippedTensors::kMost) return false;
    int64_t total = 0;
    for (int32_t t = 0; t < n_tensors; ++t) {
        if (n_elems[t] < 0 || n_elems[t] > kAloneElems - total) return false;
        total += n_elems[t];
    }
    return true;
}

}  // namespace

extern "C" size_t ld_grad_norm_workspace(int32_t n_tensors) {
    if (n_tensors < 0 || n_tensors > LD_MAX_TENSORS) return 0;
    return ld_round_up((partials_of(n_tensors) + 1) * sizeof(double), 256);
}

extern "C" size_t ld_clip_grad_norm_workspace(int32_t n_tensors, const int64_t* n_elems) {
    return n_elems && done_alone(n_tensors, n_elems) ? 0 : ld_grad_norm_workspace(n_tensors);
}

extern "C" ld_status ld_grad_norm(const void* const* grad, const int64_t* n_elems, int32_t n_tensors, int32_t dtype, int32_t accumulate,
                                  double* sumsq, float* norm, void* workspace, size_t workspace_bytes, ld_stream stream) {
    const Lists l = {grad, nullptr, n_elems, n_tensors, dtype, dtype};
    ld_status st = check_lists(l, false);
    if (st != LD_OK) return st;
    if (!sumsq) return LD_ERR_NULL;
    if (!ld_aligned(sumsq, 8) || !ld_aligned(norm, 4)) return LD_ERR_ALIGN;
    if (!workspace || !ld_aligned(workspace, 256) || workspace_bytes < ld_grad_norm_workspace(n_tensors)) return LD_ERR_WORKSPACE;
    ld_begin_call();
    hipStream_t s = static_cast<hipStream_t>(stream);
    double* part = static_cast<double*>(workspace);
    int32_t count;
    st = sum_squares(l, part, count, s);
    return st != LD_OK ? st : finish(part, count, accumulate, sumsq, norm, s);
}

extern "C" ld_status ld_clip_grads(const void* const* grad, void* const* out, const int64_t* n_elems, int32_t n_tensors, int32_t dtype,
                                   int32_t out_dtype, const double* sumsq, float max_norm, ld_stream stream) {
    const Lists l = {grad, out, n_elems, n_tensors, dtype, out_dtype};
    const ld_status st = check_lists(l, true);
    if (st != LD_OK) return st;
    if (!(max_norm >= 0.0f)) return LD_ERR_RANGE;
    if (!sumsq) return LD_ERR_NULL;
    if (!ld_aligned(sumsq, 8)) return LD_ERR_ALIGN;
    ld_begin_call();
    return clip(l, sumsq, 1, max_norm, nullptr, false, static_cast<hipStream_t>(stream));
}

extern "C" ld_status ld_clip_grad_norm(const void* const* grad, void* const* out, const int64_t* n_elems, int32_t n_tensors, int32_t dtype,
                                       int32_t out_dtype, float max_norm, float* norm, void* workspace, size_t workspace_bytes,
                                       ld_stream stream) {
    const Lists l = {grad, out, n_elems, n_tensors, dtype, out_dtype};
    ld_status st = check_lists(l, true);
    if (st != LD_OK) return st;
    if (!(max_norm >= 0.0f)) return LD_ERR_RANGE;
    if (!norm) return LD_ERR_NULL;
    if (!ld_aligned(norm, 4)) return LD_ERR_ALIGN;
    const bool alone = done_alone(n_tensors, n_elems);
    if (!alone && (!workspace || !ld_aligned(workspace, 256) || workspace_bytes < ld_grad_norm_workspace(n_tensors))) return LD_ERR_WORKSPACE;
    ld_begin_call();
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (alone) return clip(l, nullptr, 0, max_norm, norm, true, s);
    double* part = static_cast<double*>(workspace);
    int32_t count;
    st = sum_squares(l, part, count, s);
    if (st != LD_OK) return st;
    // up to a piece a workgroup, the partial sums are so few that whoever clips adds them up: a launch less (1 M elements 10.4 -> 9.0 us)
    if (count > 0 && count < kNormGrid) return clip(l, part, count, max_norm, norm, false, s);
    double* sumsq = part + partials_of(n_tensors);
    st = finish(part, count, 0, sumsq, norm, s);
    return st != LD_OK ? st : clip(l, sumsq, 1, max_norm, nullptr, false, s);
}
