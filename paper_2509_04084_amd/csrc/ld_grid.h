// Sizes of launches, apart from their kernels so that host code can be built from it as well: the tests try them at sizes
// that no test allocates.
#pragma once

#include <stdint.h>

// Workgroups of `threads` threads that a launch takes beside `others` of the same size, at most `wanted`: a launch has fewer
// than 2^32 threads in a dimension.
inline int32_t ld_workgroups(int64_t wanted, int32_t threads, int64_t others = 0) {
    const int64_t most = ((static_cast<int64_t>(1) << 32) - 1) / threads - others;
    return static_cast<int32_t>(wanted < most ? wanted : most);
}

// A few tokens' embedding gradient: the workgroups that clear rows beside the `adding` ones.
constexpr int32_t kFewThreads = 1024;
constexpr int32_t kFewClear = 64;  // rows of a clearing workgroup at a time
inline int32_t ld_few_clearing(int64_t V, int32_t adding) { return ld_workgroups((V + kFewClear - 1) / kFewClear, kFewThreads, adding); }

// Clipping: the workgroups that share `pieces` pieces out, a multiple of 8 (XCDs).
constexpr int32_t kClipThreads = 256;
// Workgroups of a launch that clips in place, where all may find that nothing is to be done: GPT-2 XL's norm and clipping under the limit
// 468 us, over it 1594; with one for every piece, as out of place, 507 and 1456, with 2048 465 and 1645. Most steps are under it.
constexpr int32_t kInPlaceGrid = 16384;
inline int32_t ld_clip_grid(int32_t pieces, bool in_place) {
    if (in_place && pieces > kInPlaceGrid) return kInPlaceGrid;
    return ld_workgroups((static_cast<int64_t>(pieces) + 7) / 8 * 8, kClipThreads) / 8 * 8;
}
