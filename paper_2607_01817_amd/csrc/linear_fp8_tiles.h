// The tile of the 8-bit product for an output size: plain C++, no HIP, for the
// launcher and for host tests.
#pragma once

#include <cstdint>

namespace hcms {

// The tiles, and what a round of workgroups and a stage of 128 k take on
// them, in us, measured: a stage with every CU busy, at the clock the power
// limit leaves, and with few of them busy; and the start and the epilogue of a
// round.  `groups`: of waves, which share the stages of a tile between them and
// add up their sums (halves the time of a long k where few tiles are at work).
// On 56160 x 1920 x 5120 the first four take 508, 584, 546 and 595 us; on 1560
// x 5120 x 5120 55, 49, 61 and 58 (the fifth 64); on 1560 x 1920 x 5120 52, 47,
// 32 and 23 (34); on 512 x 512 x 4096 37, 29, 22, 17, 14, 13 and 10.4; on 256 x
// 1920 x 5120 the 64 x 64 ones 15.9 and 12.1, on 100 x 640 x 640 4.5 and 5.1; the
// last 497, 45, 33 on the first three.
struct Fp8TileCost {
    int bm, bn, per_cu, groups;
    double full, alone, fixed;
};
inline constexpr Fp8TileCost kFp8Tiles[] = {
    {256, 256, 1, 1, 1.70, 0.99, 5.0}, {192, 256, 1, 1, 1.30, 0.79, 4.0}, {128, 256, 1, 1, 0.89, 0.70, 2.7},
    {128, 128, 1, 1, 0.54, 0.37, 2.0}, {64, 128, 1, 1, 0.40, 0.26, 1.0},  {64, 64, 2, 1, 0.46, 0.26, 1.0},
    {64, 64, 1, 2, 0.25, 0.18, 2.1},   {192, 192, 1, 1, 1.00, 0.65, 3.4}};
// For fp32 output, whose widened operands run at the bf16 rate and do not fit
// beside the accumulators of a larger tile.  56160 x 1920 x 5120: the first 911
// us, the last 981; 1560 x 5120 x 5120: 117, 114, 127, 140, 83; 256 x 1920 x 5120:
// the 64 x 64 ones 26.7 and 19.3.
inline constexpr Fp8TileCost kFp8WideTiles[] = {
    {256, 128, 1, 1, 1.53, 1.23, 4.5}, {128, 128, 1, 1, 0.98, 0.83, 2.2}, {64, 64, 2, 1, 0.70, 0.57, 1.2},
    {64, 64, 1, 2, 0.40, 0.37, 2.2},   {192, 192, 1, 1, 1.95, 1.79, 3.5}};

// Up to so many rows the kernel for few rows runs (64 rows by N = K = 5120 take
// 17.6 us on it and 15.3 on tiles; by N = 640, 16.1 and 15.3).
inline constexpr int64_t kFp8Rows = 32;
// Its workgroups take 32 columns instead of 16 where those of 16 do not fit
// the CUs at once (1 x 5120 x 5120: 7.6 us against 8.9; 1 x 640 x 5120: 7.4
// against 5.2).
inline bool fp8_rows_wide(int64_t N, int64_t n_cu) { return N > 16 * n_cu; }

// The tile with the shortest estimated time: whole rounds of workgroups, then
// a partial one whose stages lie between the two times.
template <int COUNT>
inline int fp8_tile(const Fp8TileCost (&tiles)[COUNT], int64_t M, int64_t N, int64_t K, int64_t n_cu) {
    const int64_t stages = (K + 127) / 128;
    int best = 0;
    double t_best = 0;
    for (int i = 0; i < COUNT; ++i) {
        const Fp8TileCost &c = tiles[i];
        const int64_t count = ((M + c.bm - 1) / c.bm) * ((N + c.bn - 1) / c.bn);
        const int64_t slots = n_cu * c.per_cu, rem = count % slots;
        const double f = static_cast<double>(rem) / slots;
        double t = (count / slots) * (c.fixed + stages * c.full);
        if (rem > 0) t += c.fixed + stages * (c.alone + (c.full - c.alone) * f);
        if (i == 0 || t < t_best) {
            best = i;
            t_best = t;
        }
    }
    return best;
}

}  // namespace hcms
