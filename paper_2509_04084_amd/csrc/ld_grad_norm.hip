// The norm of a step's whole gradient, over many tensors, and clipping by it: what a training loop does between the
// backward pass and ld_compress_topk / ld_snapshot_layers.
//
//   S = sum over all elements of x^2;  norm = sqrt(S);  factor = norm > max_norm ? max_norm / norm : 1
//   out = round(x * factor)
//
// Squares and sums are 64 bits wide: the square of a 32-bit value is exact there and can neither overflow nor vanish.
// Bound by memory: n elements read for S, read again and written for the clipped values; a gradient in place under the limit
// is not touched a second time.
#include <math.h>

#include <type_traits>

#include "ld_elem.h"

namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 4;                 // vectors per thread and piece
constexpr int kTensorGroup = 16;
constexpr int kTensorGroups = 10;
constexpr int kTensorsPerLaunch = kTensorGroup * kTensorGroups;
constexpr int kNormGrid = 2048;            // workgroups of a launch, each with a partial sum

// The tensors of a launch, in its arguments. A tensor is cut into pieces of PIECE elements, the last one ragged.
struct TensorBatch {
    int32_t first_of_group[kTensorGroup];         // [0]: all pieces; then every 16th of first_piece
    int32_t first_piece[kTensorsPerLaunch + 1];   // entries past the last tensor: all pieces
    struct Tensor {
        const void* src;
        void* dst;
    } tensor[kTensorsPerLaunch];
    int16_t last[kTensorsPerLaunch];              // elements of a tensor's last piece
};
static_assert(sizeof(TensorBatch) <= 4000, "the arguments of a kernel must fit 4 KB");

// The tensor that a piece belongs to: two reads of 16 consecutive entries each.
__device__ __forceinline__ int tensor_of(const TensorBatch& b, int32_t piece) {
    int group = 0, t = 0;
#pragma unroll
    for (int i = 1; i < kTensorGroup; ++i) group += b.first_of_group[i] <= piece;
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

template <int DT>
__global__ __launch_bounds__(kThreads) void k_sum_squares(TensorBatch b, double* __restrict__ part) {
    constexpr int N = DT == LD_F32 ? 4 : 8;
    typedef LdVec<DT, N> V;
    __shared__ double sh[kThreads / LD_WAVE];
    double sum = 0.0;
    for (int32_t p = blockIdx.x; p < b.first_of_group[0]; p += gridDim.x) {
        const int t = tensor_of(b, p);
        const typename V::elem* src = static_cast<const typename V::elem*>(b.tensor[t].src) +
                                      static_cast<int64_t>(p - b.first_piece[t]) * piece_elems<N>();
        const int32_t have = p + 1 == b.first_piece[t + 1] ? b.last[t] : piece_elems<N>();
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int32_t at = (u * kThreads + threadIdx.x) * N;
            if (at + N <= have) {
                const typename V::wide x = V::widen(*reinterpret_cast<const typename V::type*>(src + at));
#pragma unroll
                for (int e = 0; e < N; ++e) sum = fma(static_cast<double>(x[e]), static_cast<double>(x[e]), sum);
            } else {
                for (int32_t e = at; e < have && e < at + N; ++e) {
                    const double x = static_cast<double>(static_cast<float>(src[e]));
                    sum = fma(x, x, sum);
                }
            }
        }
    }
    sum = block_sum(sum, sh);
    if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

__global__ __launch_bounds__(1024) void k_norm_finish(const double* __restrict__ part, int32_t count, int32_t accumulate,
                                                      double* __restrict__ sumsq, float* __restrict__ norm) {
    __shared__ double sh[1024 / LD_WAVE];
    double sum = 0.0;
    for (int32_t i = threadIdx.x; i < count; i += blockDim.x) sum += part[i];
    sum = block_sum(sum, sh);
    if (threadIdx.x == 0) {
        if (accumulate) sum += *sumsq;
        *sumsq = sum;
        if (norm) *norm = static_cast<float>(sqrt(sum));
    }
}

template <int DT, int OT>
__global__ __launch_bounds__(kThreads) void k_clip(TensorBatch b, const double* __restrict__ sumsq, float max_norm, int32_t in_place) {
    constexpr int N = DT == LD_F32 || OT == LD_F32 ? 4 : 8;
    typedef LdVec<DT, N> V;
    typedef LdVec<OT, N> O;
    const double norm = sqrt(*sumsq);
    // a norm that is not finite clips nothing: the caller sees it in the norm
    const float factor = norm > max_norm && norm < __builtin_huge_val() ? static_cast<float>(max_norm / norm) : 1.0f;
    if (in_place && factor == 1.0f) return;
    for (int32_t p = blockIdx.x; p < b.first_of_group[0]; p += gridDim.x) {
        const int t = tensor_of(b, p);
        const int64_t first = static_cast<int64_t>(p - b.first_piece[t]) * piece_elems<N>();
        const typename V::elem* src = static_cast<const typename V::elem*>(b.tensor[t].src) + first;
        typename O::elem* dst = static_cast<typename O::elem*>(b.tensor[t].dst) + first;
        const int32_t have = p + 1 == b.first_piece[t + 1] ? b.last[t] : piece_elems<N>();
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int32_t at = (u * kThreads + threadIdx.x) * N;
            if (at + N <= have) {
                const typename V::wide x = V::widen(*reinterpret_cast<const typename V::type*>(src + at));
                *reinterpret_cast<typename O::type*>(dst + at) = O::narrow(x * factor);
            } else {
                for (int32_t e = at; e < have && e < at + N; ++e)
                    dst[e] = static_cast<typename O::elem>(static_cast<float>(src[e]) * factor);
            }
        }
    }
}

// Tensors [t, ...) of the lists as a launch takes them, in pieces of `piece` elements; t moves behind them.
void next_batch(TensorBatch& b, const void* const* src, void* const* dst, const int64_t* n_elems, int32_t n_tensors, int32_t piece,
                int32_t& t) {
    int32_t count = 0;
    int64_t pieces = 0;
    for (; t < n_tensors && count < kTensorsPerLaunch; ++t) {
        const int64_t np = (n_elems[t] + piece - 1) / piece;
        if (np == 0) continue;
        b.tensor[count] = {src[t], dst ? dst[t] : nullptr};
        b.first_piece[count] = static_cast<int32_t>(pieces);
        b.last[count] = static_cast<int16_t>(n_elems[t] - (np - 1) * piece);
        pieces += np;
        ++count;
    }
    for (int32_t i = count; i <= kTensorsPerLaunch; ++i) b.first_piece[i] = static_cast<int32_t>(pieces);
    for (int32_t i = count; i < kTensorsPerLaunch; ++i) {
        b.tensor[i] = {nullptr, nullptr};
        b.last[i] = 0;
    }
    b.first_of_group[0] = static_cast<int32_t>(pieces);
    for (int32_t g = 1; g < kTensorGroup; ++g)
        b.first_of_group[g] = g < kTensorGroups ? b.first_piece[g * kTensorGroup] : static_cast<int32_t>(pieces);
}

constexpr int64_t kMostElems = static_cast<int64_t>(1) << 41;  // of all tensors: 2^29 pieces of 4096, and one more a tensor

ld_status check_lists(const void* const* grad, void* const* out, bool with_out, const int64_t* n_elems, int32_t n_tensors,
                      int32_t dtype, int32_t out_dtype) {
    if (n_tensors < 0 || n_tensors > LD_MAX_TENSORS || !ld_known_type(dtype) || !ld_known_type(out_dtype)) return LD_ERR_RANGE;
    if (n_tensors > 0 && (!grad || !n_elems || (with_out && !out))) return LD_ERR_NULL;
    int64_t total = 0;
    for (int32_t t = 0; t < n_tensors; ++t) {
        if (n_elems[t] < 0 || n_elems[t] > kMostElems - total) return LD_ERR_RANGE;
        total += n_elems[t];
        if (n_elems[t] > 0 && (!grad[t] || (with_out && !out[t]))) return LD_ERR_NULL;
        if (!ld_aligned(grad[t], ld_type_bytes(dtype)) || (with_out && !ld_aligned(out[t], ld_type_bytes(out_dtype)))) return LD_ERR_ALIGN;
    }
    return LD_OK;
}

// Partial sums of all launches, and behind them the sum of squares.
size_t partials_of(int32_t n_tensors) {
    return static_cast<size_t>((n_tensors + kTensorsPerLaunch - 1) / kTensorsPerLaunch) * kNormGrid;
}

ld_status sum_squares(const void* const* grad, const int64_t* n_elems, int32_t n_tensors, int32_t dtype, int32_t accumulate,
                      double* sumsq, float* norm, double* part, hipStream_t s) {
    int32_t count = 0;
    for (int32_t t = 0; t < n_tensors;) {
        TensorBatch b;
        next_batch(b, grad, nullptr, n_elems, n_tensors, dtype == LD_F32 ? piece_elems<4>() : piece_elems<8>(), t);
        if (b.first_of_group[0] == 0) continue;
        const int32_t grid = b.first_of_group[0] < kNormGrid ? b.first_of_group[0] : kNormGrid;
        ld_with_type(dtype, [&](auto type) { k_sum_squares<type><<<dim3(grid), dim3(kThreads), 0, s>>>(b, part + count); });
        if (ld_launch_status() != LD_OK) return LD_ERR_HIP;
        count += grid;
    }
    k_norm_finish<<<dim3(1), dim3(1024), 0, s>>>(part, count, accumulate, sumsq, norm);
    return ld_launch_status();
}

ld_status clip(const void* const* grad, void* const* out, const int64_t* n_elems, int32_t n_tensors, int32_t dtype, int32_t out_dtype,
               const double* sumsq, float max_norm, hipStream_t s) {
    for (int32_t t = 0; t < n_tensors;) {
        const int32_t from = t;
        TensorBatch b;
        next_batch(b, grad, out, n_elems, n_tensors, dtype == LD_F32 || out_dtype == LD_F32 ? piece_elems<4>() : piece_elems<8>(), t);
        if (b.first_of_group[0] == 0) continue;
        int32_t in_place = dtype == out_dtype;
        for (int32_t i = from; i < t; ++i) in_place &= n_elems[i] == 0 || grad[i] == out[i];
        const int32_t grid = b.first_of_group[0] < kNormGrid ? b.first_of_group[0] : kNormGrid;
        ld_with_type(dtype, [&](auto type) {
            ld_with_type(out_dtype, [&](auto out_type) {
                k_clip<type, out_type><<<dim3(grid), dim3(kThreads), 0, s>>>(b, sumsq, max_norm, in_place);
            });
        });
        if (ld_launch_status() != LD_OK) return LD_ERR_HIP;
    }
    return LD_OK;
}

}  // namespace

extern "C" size_t ld_grad_norm_workspace(int32_t n_tensors) {
    if (n_tensors < 0 || n_tensors > LD_MAX_TENSORS) return 0;
    return ld_round_up((partials_of(n_tensors) + 1) * sizeof(double), 256);
}

extern "C" ld_status ld_grad_norm(const void* const* grad, const int64_t* n_elems, int32_t n_tensors, int32_t dtype, int32_t accumulate,
                                  double* sumsq, float* norm, void* workspace, size_t workspace_bytes, ld_stream stream) {
    const ld_status st = check_lists(grad, nullptr, false, n_elems, n_tensors, dtype, dtype);
    if (st != LD_OK) return st;
    if (!sumsq) return LD_ERR_NULL;
    if (!ld_aligned(sumsq, 8) || !ld_aligned(norm, 4)) return LD_ERR_ALIGN;
    if (!workspace || !ld_aligned(workspace, 256) || workspace_bytes < ld_grad_norm_workspace(n_tensors)) return LD_ERR_WORKSPACE;
    ld_begin_call();
    return sum_squares(grad, n_elems, n_tensors, dtype, accumulate, sumsq, norm, static_cast<double*>(workspace),
                       static_cast<hipStream_t>(stream));
}

extern "C" ld_status ld_clip_grads(const void* const* grad, void* const* out, const int64_t* n_elems, int32_t n_tensors, int32_t dtype,
                                   int32_t out_dtype, const double* sumsq, float max_norm, ld_stream stream) {
    const ld_status st = check_lists(grad, out, true, n_elems, n_tensors, dtype, out_dtype);
    if (st != LD_OK) return st;
    if (!(max_norm >= 0.0f)) return LD_ERR_RANGE;
    if (!sumsq) return LD_ERR_NULL;
    if (!ld_aligned(sumsq, 8)) return LD_ERR_ALIGN;
    ld_begin_call();
    return clip(grad, out, n_elems, n_tensors, dtype, out_dtype, sumsq, max_norm, static_cast<hipStream_t>(stream));
}

extern "C" ld_status ld_clip_grad_norm(const void* const* grad, void* const* out, const int64_t* n_elems, int32_t n_tensors, int32_t dtype,
                                       int32_t out_dtype, float max_norm, float* norm, void* workspace, size_t workspace_bytes,
                                       ld_stream stream) {
    const ld_status st = check_lists(grad, out, true, n_elems, n_tensors, dtype, out_dtype);
    if (st != LD_OK) return st;
    if (!(max_norm >= 0.0f)) return LD_ERR_RANGE;
    if (!norm) return LD_ERR_NULL;
    if (!ld_aligned(norm, 4)) return LD_ERR_ALIGN;
    if (!workspace || !ld_aligned(workspace, 256) || workspace_bytes < ld_grad_norm_workspace(n_tensors)) return LD_ERR_WORKSPACE;
    ld_begin_call();
    double* part = static_cast<double*>(workspace);
    double* sumsq = part + partials_of(n_tensors);
    hipStream_t s = static_cast<hipStream_t>(stream);
    const ld_status summed = sum_squares(grad, n_elems, n_tensors, dtype, 0, sumsq, norm, part, s);
    return summed != LD_OK ? summed : clip(grad, out, n_elems, n_tensors, dtype, out_dtype, sumsq, max_norm, s);
}
