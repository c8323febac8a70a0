// Argument checks shared by the C entry points.
#pragma once

#include "hcms.h"

#include <hip/hip_runtime.h>

#include <cstdint>

#include "hcms_internal.h"

namespace hcms {

inline int hip_fail(hipError_t e, const char *what) {
    return fail(HCMS_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

inline int elem_bytes(int dtype) { return dtype == HCMS_BF16 ? 2 : 4; }

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Byte ranges [a, a + na) and [b, b + nb) overlap.
inline bool overlaps(const void *a, int64_t na, const void *b, int64_t nb) {
    if (na <= 0 || nb <= 0) return false;
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + static_cast<uintptr_t>(nb) && y < x + static_cast<uintptr_t>(na);
}

inline int check_dtype(int dtype) {
    if (dtype != HCMS_BF16 && dtype != HCMS_FP32)
        return fail(HCMS_ERR_DTYPE, "dtype %d is neither HCMS_BF16 (0) nor HCMS_FP32 (1)", dtype);
    return HCMS_OK;
}

// Rotation axes from the caller's grid and pair counts: 1..kRopeMaxAxes axes,
// every size >= 1; *tokens = product of the grid, *pairs = sum of the counts,
// *entries = table entries.
inline int rope_axes(const int *grid, const int *axis_pairs, int n_axes, RopeAxes *ax,
              int64_t *tokens, int64_t *pairs, int64_t *entries) {
    if (!grid || !axis_pairs) return fail(HCMS_ERR_NULL, "grid or axis_pairs is NULL");
    if (n_axes < 1 || n_axes > kRopeMaxAxes)
        return fail(HCMS_ERR_ARG, "n_axes=%d must be in [1, %d]", n_axes, kRopeMaxAxes);
    *ax = RopeAxes{};
    ax->n_axes = n_axes;
    int64_t prod = 1, np = 0, off = 0;
    for (int a = 0; a < n_axes; ++a) {
        if (grid[a] < 1 || axis_pairs[a] < 1)
            return fail(HCMS_ERR_SHAPE, "axis %d: grid size %d and pair count %d must be >= 1", a,
                        grid[a], axis_pairs[a]);
        ax->grid[a] = grid[a];
        ax->pairs[a] = axis_pairs[a];
        ax->pair_start[a] = static_cast<int>(np);
        ax->tab_off[a] = static_cast<int>(off);
        prod *= grid[a];
        np += axis_pairs[a];
        off += static_cast<int64_t>(grid[a]) * axis_pairs[a];
        if (prod > 0x7fffffffLL || off > (1LL << 28))
            return fail(HCMS_ERR_SHAPE, "grid too large (%lld tokens, %lld table entries)",
                        static_cast<long long>(prod), static_cast<long long>(off));
    }
    *tokens = prod;
    *pairs = np;
    *entries = off;
    return HCMS_OK;
}

}  // namespace hcms
