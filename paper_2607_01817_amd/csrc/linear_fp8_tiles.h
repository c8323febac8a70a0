// The tile of the 8-bit product for an output size: plain C++, no HIP, for the
// launcher and for host tests.
#pragma once

#include <cstdint>

namespace hcms {

// The tiles, and what a round of workgroups and a stage of 128 k take on
// them, in us: a stage with every CU busy, and with few of them busy, where
// the latency of the loads shows; and the start and the epilogue of a round.
struct Fp8TileCost {
    int bm, bn, per_cu;
    double full, alone, fixed;
};
inline constexpr Fp8TileCost kFp8Tiles[] = {
    {256, 256, 1, 1.50, 0.99, 5.0}, {128, 128, 1, 0.49, 0.35, 2.0}, {64, 128, 1, 0.34, 0.26, 1.2},
    {64, 64, 2, 0.37, 0.19, 1.2}};

// The tile with the shortest estimated time: whole rounds of workgroups, then
// a partial one whose stages lie between the two times.  wide: fp32 output,
// whose widened operands do not fit beside the first tile's accumulators.
inline int fp8_tile(int64_t M, int64_t N, int64_t stages, int64_t n_cu, bool wide) {
    const int first = wide ? 1 : 0;
    int best = first;
    double t_best = 0;
    for (int i = first; i < static_cast<int>(sizeof(kFp8Tiles) / sizeof(kFp8Tiles[0])); ++i) {
        const Fp8TileCost &c = kFp8Tiles[i];
        const int64_t tiles = ((M + c.bm - 1) / c.bm) * ((N + c.bn - 1) / c.bn);
        const int64_t slots = n_cu * c.per_cu, rem = tiles % slots;
        const double f = static_cast<double>(rem) / slots;
        double t = (tiles / slots) * (c.fixed + stages * c.full);
        if (rem > 0) t += c.fixed + stages * (c.alone + (c.full - c.alone) * f);
        if (i == first || t < t_best) {
            best = i;
            t_best = t;
        }
    }
    return best;
}

}  // namespace hcms
