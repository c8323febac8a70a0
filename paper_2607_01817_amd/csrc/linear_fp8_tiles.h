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
// In us, in the order of the table, on one card (from card to card the first line
// moves by 5 %: 476 to 500 on 192 x 192):
//   56160 x 1920 x 5120   515  592  556  624  850 1046 1128  494  832
//   1560 x 5120 x 5120     54   48   62   61   67   79   88   41   65
//   1560 x 1920 x 5120     52   45   30   23   33   41   34   32   31
//   1000 x 1920 x 5120     53   43   30   22   19   23   23   32   16.7
//   512 x 512 x 4096       37   29   23   18   15   13.4 10.4 26   12.9
//   1000 x 1536 x 640      10.3  8.4  8.2  6.6  5.9  6.7  9.2  8.4  6.3
struct Fp8TileCost {
    int bm, bn, per_cu, groups;
    double full, alone, fixed;
};
inline constexpr Fp8TileCost kFp8Tiles[] = {
    {256, 256, 1, 1, 1.70, 0.99, 5.0}, {192, 256, 1, 1, 1.30, 0.79, 4.0}, {128, 256, 1, 1, 0.89, 0.70, 2.7},
    {128, 128, 1, 1, 0.54, 0.37, 2.0}, {64, 128, 1, 1, 0.40, 0.26, 1.0},  {64, 64, 2, 1, 0.46, 0.26, 1.0},
    {64, 64, 1, 2, 0.25, 0.18, 2.1},   {192, 192, 1, 1, 0.96, 0.65, 3.4},
    {64, 128, 1, 2, 0.335, 0.27, 2.1}};
// For fp32 output, whose widened operands run at the bf16 rate and do not fit
// beside the accumulators of a larger tile:
//   56160 x 1920 x 5120   950 1054 1647 1762  979
//   1560 x 5120 x 5120    120  107  126  138   82
//   3001 x 1000 x 1936     27.0 18.9 29.7 27.9 34.3
//   256 x 1920 x 5120      54   32   27.5 19.3 73
// (128 x 128 without groups, on eight waves: 1126, 117, 21.9 and 40).
inline constexpr Fp8TileCost kFp8WideTiles[] = {
    {256, 128, 1, 1, 1.53, 1.23, 4.5}, {128, 128, 1, 2, 0.87, 0.66, 2.2}, {64, 64, 2, 1, 0.70, 0.57, 1.2},
    {64, 64, 1, 2, 0.40, 0.37, 2.2},   {192, 192, 1, 1, 1.95, 1.79, 3.5}};

// Up to so many rows the kernel for few rows runs (64 rows by N = K = 5120 take
// 9.8 us on it and 12.2 on tiles; by 1920 x 5120 7.5 and 12.0; by 640 x 640 3.3
// and 5.3).
inline constexpr int64_t kFp8Rows = 64;
// Its workgroups take 32 columns instead of 16 where those of 16 do not fit
// the CUs at once (1 x 5120 x 5120: 4.8 us against 6.5; 64 rows: 9.8 against 14.8;
// 1 x 1920 x 5120: 4.7 against 3.9).
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
