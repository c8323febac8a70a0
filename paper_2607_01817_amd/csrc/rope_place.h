// Where a token's rotations lie in the rotation table: shared by the kernels
// that turn head vectors.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "hcms_internal.h"

namespace hcms {

static_assert(kRopeMaxAxes == 4, "RopePlace names the axes one by one");

// Entry of pair p of axis a for one token: r<a> + p; first pairs of the axes behind
// the first one: s<a>.  A token outside the grid has `inside` false and the entries
// of coordinate 0.  (An array, chosen from by pair, would lie in memory.)
struct RopePlace {
    int r0 = 0, r1 = 0, r2 = 0, r3 = 0;
    int s1, s2, s3;
    bool inside = true;
};
// Where the axes' pairs begin.  Read anew for each token: comparisons of pairs with them
// that a loop over tokens kept would take more scalar registers than there are.
__device__ inline void rope_starts(const RopeAxes &ax, RopePlace *at) {
    const auto start = [&](int a) {
        int s = a < ax.n_axes ? ax.pair_start[a] : kRopeMaxPairs;
        asm volatile("" : "+s"(s));
        return s;
    };
    at->s1 = start(1);
    at->s2 = start(2);
    at->s3 = start(3);
}

// The place of the token whose coordinates are positions[index], or, without
// positions, of place `place` of the row-major grid.
__device__ inline RopePlace rope_place(const RopeAxes &ax, const void *positions, bool pos64, int64_t index, int place) {
    RopePlace at;
    rope_starts(ax, &at);
    const auto row = [&](int a, int c) { return ax.tab_off[a] + c * ax.pairs[a] - ax.pair_start[a]; };
    if (positions) {
        const auto axis = [&](int a) {
            if (a >= ax.n_axes) return 0;
            const int64_t i = index * ax.n_axes + a;
            const int64_t c = pos64 ? static_cast<const int64_t *>(positions)[i]
                                    : static_cast<int64_t>(static_cast<const int *>(positions)[i]);
            const bool ok = c >= 0 && c < ax.grid[a];
            at.inside = at.inside && ok;
            return row(a, ok ? static_cast<int>(c) : 0);
        };
        at.r0 = axis(0);
        at.r1 = axis(1);
        at.r2 = axis(2);
        at.r3 = axis(3);
    } else {
        int rest = place;
        const auto axis = [&](int a) {
            if (a >= ax.n_axes) return 0;
            const int c = rest % ax.grid[a];
            rest /= ax.grid[a];
            return row(a, c);
        };
        at.r3 = axis(3);
        at.r2 = axis(2);
        at.r1 = axis(1);
        at.r0 = axis(0);
        at.inside = rest == 0;
    }
    return at;
}

// (cos, sin) of pair p; NaN for a token outside the grid, never another
// position's angle.
__device__ inline float2 rope_entry(const float *table, const RopePlace &at, int p) {
    const int r0 = at.r0, r1 = at.r1, r2 = at.r2, r3 = at.r3;   // values: a choice of members would be one of addresses
    const int row = p < at.s1 ? +r0 : p < at.s2 ? +r1 : p < at.s3 ? +r2 : +r3;
    const float2 cs = reinterpret_cast<const float2 *>(table)[row + p];
    const float nan = __builtin_nanf("");
    return at.inside ? cs : make_float2(nan, nan);
}

}  // namespace hcms
