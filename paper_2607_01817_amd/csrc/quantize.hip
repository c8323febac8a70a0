// Quantisation to 8-bit floating point with block scales (fp8.h), as the
// operands of the 8-bit product.
//
// Of x [M][K] any of: q, the values of x by rows, its scales one per row and
// 128 columns or one per 128 x 128; and t, the values of x transposed, its
// scales one per column and 128 rows or one per 128 x 128: the product's
// contraction then runs over M, and a row of t is M values padded with zeros
// to a multiple of 16.  Scales lie in groups of four blocks: [groups][rows of
// the operand, or of its 128 x 128 blocks][4].  Blocks past a row's end, which
// fill its last group, hold the scale of a block of zeros.
//
// What bounds it: bytes, each element read once, whatever is made of it.  bf16,
// read and written bytes: 56160 x 5120 by rows 146 us (5.9 TB/s), with the
// transpose 230 (5.0); 7800 x 5120 19.4 (6.2 TB/s) and 28 (5.7); 1560 x 5120 5.4
// and 9.4; fp32 7800 x 5120 by rows 29.5 (6.8).  The rows alone have a kernel of
// their own, without the tile's detour; by rows, that kernel and the tile: bf16
// 56160 x 5120 146 and 159 us, 7800 x 5120 19.5 and 20.5, 7800 x 1920 8.4 and 10.3,
// 1560 x 5120 5.4 and 6.7 (56160 x 640 20.4 and 19.8; fp32 7800 x 5120 29.6 and 30.4,
// 56160 x 5120 262 and 254).
#include "fp8.h"
#include "hcms_internal.h"

namespace hcms {
namespace {

using fp8::f32x8;
constexpr int kTile = fp8::kBlock;

__device__ inline uint2 pack8(f32x8 v, float by) {
    return {fp8::pack4(v[0] * by, v[1] * by, v[2] * by, v[3] * by),
            fp8::pack4(v[4] * by, v[5] * by, v[6] * by, v[7] * by)};
}
__device__ inline unsigned magnitude8(f32x8 v) {
    unsigned a = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) a = max(a, fp8::magnitude(v[i]));
    return a;
}

// Workgroups (column, row) of the kernels below: a grid has 65535 of them along
// its second axis at most, so rows take the third one too, past whose last row
// nothing is done.
dim3 grid_of(int columns, int64_t rows) {
    const int64_t most = 32768;
    return rows <= most ? dim3(columns, static_cast<unsigned>(rows))
                        : dim3(columns, static_cast<unsigned>(most), static_cast<unsigned>((rows + most - 1) / most));
}
__device__ inline int64_t row_index() { return static_cast<int64_t>(blockIdx.z) * gridDim.y + blockIdx.y; }

// q by rows with a scale per row and 128 columns.  A wave takes a group of
// four blocks of kRows rows.
constexpr int kRows = 4;
template <typename T>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const T *__restrict__ x, int64_t ldx,
                                                            unsigned char *__restrict__ q,
                                                            unsigned *__restrict__ scale, int64_t M, int K) {
    const int lane = threadIdx.x & 63;
    const int g = blockIdx.x;
    const int64_t m0 = (row_index() * 4 + (threadIdx.x >> 6)) * kRows;
    if (m0 >= M) return;
    const int e = g * fp8::kGroup + lane * 8;
    const bool in = e < K;   // K is a multiple of 16
    // Lanes and rows past the ends read the last ones: a load behind a branch
    // would be waited for there.
    decltype(load_raw(x)) raw[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) raw[i] = load_raw(x + min(m0 + i, M - 1) * ldx + min(e, K - 8));
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        if (m0 + i >= M) break;
        const f32x8 v = in ? widen(raw[i]) : f32x8{};
        const unsigned b = fp8::scale_byte(fp8::max16(magnitude8(v)));
        if (in) *reinterpret_cast<uint2 *>(q + (m0 + i) * K + e) = pack8(v, fp8::inverse_scale(b));
        const unsigned four = __builtin_amdgcn_readlane(b, 0) | __builtin_amdgcn_readlane(b, 16) << 8 |
                              __builtin_amdgcn_readlane(b, 32) << 16 | __builtin_amdgcn_readlane(b, 48) << 24;
        if (lane == 0) scale[g * M + m0 + i] = four;
    }
}

// Scale byte `b` of block `blk` of `blocks`, in entry `row` of `rows` of its
// group; the last block fills its group's rest.
__device__ inline void put_scale(unsigned char *scale, int64_t rows, int64_t row, int blk, int blocks, unsigned b) {
    unsigned char *p = scale + ((blk >> 2) * rows + row) * 4;
    p[blk & 3] = static_cast<unsigned char>(b);
    if (blk == blocks - 1)
        for (int i = (blk & 3) + 1; i < 4; ++i) p[i] = 1;
}

// Any of q and t, a 128 x 128 tile per workgroup.  Thread (r, c) holds the 8 x
// 8 elements of rows 8 r .., columns 8 c .., so that 8 rows of a column pack
// into 8 bytes of t; t's tile passes through LDS to leave as 16-byte pieces of
// whole rows.  Unit u (8 bytes) of t's row k sits at place u ^ (k / 8), so that
// the lanes of a write, whose rows are 8 apart, spread over the banks.
template <typename T>
__global__ __launch_bounds__(256) void quantize_tile_kernel(const T *__restrict__ x, int64_t ldx, QuantizeOut o,
                                                            int64_t M, int K, int tiles_k) {
    __shared__ unsigned col_max[16][kTile];
    __shared__ unsigned wave_max[4];
    __shared__ __attribute__((aligned(16))) unsigned char tile[kTile][kTile];
    const int tid = threadIdx.x, c = tid & 15, r = tid >> 4;
    const int kb = blockIdx.x, mb = static_cast<int>(row_index());
    const int tiles_m = static_cast<int>((M + kTile - 1) / kTile);
    if (mb >= tiles_m) return;
    const int64_t m0 = static_cast<int64_t>(mb) * kTile + r * 8;
    const int e = kb * kTile + c * 8;
    // Kept as stored and widened where they are used: 32 registers, not 64.
    using Raw = decltype(load_raw(x));
    // Loads past the ends read the last row or columns (a load behind a branch
    // would be waited for there) and count as zeros.
    Raw v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = load_raw(x + min(m0 + i, M - 1) * ldx + min(e, K - 8));
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (m0 + i >= M || e >= K) v[i] = Raw{};
    unsigned row_max[8], all = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        row_max[i] = magnitude8(widen(v[i]));
        all = max(all, row_max[i]);
        if (o.q && !o.q_square) row_max[i] = fp8::max16(row_max[i]);
    }
    all = fp8::max16(all);
    // Whole-tile maximum, and the maximum of each column.
    unsigned w = max(max(static_cast<unsigned>(__builtin_amdgcn_readlane(all, 0)),
                         static_cast<unsigned>(__builtin_amdgcn_readlane(all, 16))),
                     max(static_cast<unsigned>(__builtin_amdgcn_readlane(all, 32)),
                         static_cast<unsigned>(__builtin_amdgcn_readlane(all, 48))));
    if ((tid & 63) == 0) wave_max[tid >> 6] = w;
    if (o.t && !o.t_square) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            unsigned a = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) a = max(a, fp8::magnitude(widen(v[i])[j]));
            col_max[r][c * 8 + j] = a;
        }
    }
    __syncthreads();
    const unsigned square = fp8::scale_byte(max(max(wave_max[0], wave_max[1]), max(wave_max[2], wave_max[3])));
    if (o.q) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const unsigned b = o.q_square ? square : fp8::scale_byte(row_max[i]);
            if (m0 + i >= M) continue;
            if (e < K) *reinterpret_cast<uint2 *>(o.q + (m0 + i) * K + e) = pack8(widen(v[i]), fp8::inverse_scale(b));
            if (!o.q_square && c == 0) put_scale(o.q_scale, M, m0 + i, kb, tiles_k, b);
        }
        if (o.q_square && tid == 0) put_scale(o.q_scale, tiles_m, mb, kb, tiles_k, square);
    }
    if (!o.t) return;
    if (!o.t_square) {
        // Columns' maxima: thread k < 128 reduces column k and leaves its scale.
        if (tid < kTile) {
            unsigned a = 0;
            for (int i = 0; i < 16; ++i) a = max(a, col_max[i][tid]);
            const unsigned b = fp8::scale_byte(a);
            col_max[0][tid] = b;
            if (kb * kTile + tid < K) put_scale(o.t_scale, K, kb * kTile + tid, mb, tiles_m, b);
        }
        __syncthreads();
    } else if (tid == 0) {
        put_scale(o.t_scale, tiles_k, kb, mb, tiles_m, square);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float by = fp8::inverse_scale(o.t_square ? square : col_max[0][c * 8 + j]);
        const f32x8 col = {widen(v[0])[j], widen(v[1])[j], widen(v[2])[j], widen(v[3])[j],
                           widen(v[4])[j], widen(v[5])[j], widen(v[6])[j], widen(v[7])[j]};
        *reinterpret_cast<uint2 *>(&tile[c * 8 + j][(r ^ c) * 8]) = pack8(col, by);
    }
    __syncthreads();
    const int64_t ldt = (M + 15) / 16 * 16;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int k = i * 32 + (tid >> 3), p = tid & 7, f = k >> 3;
        const int64_t mm = static_cast<int64_t>(mb) * kTile + p * 16;
        const uint4 u = *reinterpret_cast<const uint4 *>(&tile[k][(p ^ (f >> 1)) * 16]);
        if (kb * kTile + k < K && mm < ldt)
            *reinterpret_cast<uint4 *>(o.t + static_cast<int64_t>(kb * kTile + k) * ldt + mm) =
                f & 1 ? uint4{u.z, u.w, u.x, u.y} : u;
    }
}

template <typename T>
hipError_t quantize_typed(const void *x, int64_t ldx, const QuantizeOut &o, int64_t M, int K, hipStream_t stream) {
    if (!o.t && !o.q_square) {
        const int groups = (K + fp8::kGroup - 1) / fp8::kGroup;
        quantize_rows_kernel<T><<<grid_of(groups, (M + 4 * kRows - 1) / (4 * kRows)), 256, 0, stream>>>(
            static_cast<const T *>(x), ldx, o.q, reinterpret_cast<unsigned *>(o.q_scale), M, K);
        return hipGetLastError();
    }
    const int tiles_k = (K + kTile - 1) / kTile;
    quantize_tile_kernel<T><<<grid_of(tiles_k, (M + kTile - 1) / kTile), 256, 0, stream>>>(
        static_cast<const T *>(x), ldx, o, M, K, tiles_k);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize_fp8(const void *x, int64_t ldx, const QuantizeOut &out, int64_t M, int K, int dtype,
                               hipStream_t stream) {
    if (M == 0) return hipSuccess;
    return dtype == 0 ? quantize_typed<__bf16>(x, ldx, out, M, K, stream)
                      : quantize_typed<float>(x, ldx, out, M, K, stream);
}

}  // namespace hcms
