// Root-mean-square norm with the residual's addition, forward and backward:
//   h = x + r,  y = h / sqrt(mean(h^2) + eps) * w        rows of D elements
// h is the residual stream's next value; it is stored rounded to the storage
// type, while y is computed from the unrounded sum.  The statistics are fp32.
//
// What bounds it: bytes.  A row is read once into registers by L lanes (a
// multiple of 64), NC chunks of 8 elements each, summed and written once.  With a
// residual: bf16 56160 x 5120 380 us (6.0 TB/s), 9000 x 16384 197 (6.0); fp32 56160 x
// 5120 940 and 7800 x 5120 130 (4.9; 10 % more is written than there is, a lane's 32
// bytes of a chunk leaving in two stores past the caches).
#include "fp8.h"
#include "hcms_internal.h"

namespace hcms {
namespace {

using fp8::f32x8;

// Lane t of a row's L lanes holds the chunks of 8 elements t, t + L, ...  The
// chunk that the row's end cuts is read from D - 8 on: its first `dup` elements
// are another lane's too, which stores the same values; sums take them from
// that lane alone.  Chunks past the end lie there too, with all 8 doubled.
struct Chunk {
    int e0, dup;
};
__device__ inline Chunk chunk_at(int c, int D) {
    const int e = c * 8, e0 = min(e, D - 8);
    return {e0, e - e0};
}

// The lane's place in a workgroup that takes one row (L = 0), or of 256 threads
// that take one for each L of them.
template <int L>
struct Lane {
    static __device__ int t() { return L ? threadIdx.x & (L - 1) : threadIdx.x; }
    static __device__ int lanes() { return L ? L : blockDim.x; }
    static __device__ int row() { return L ? threadIdx.x / (L ? L : 1) : 0; }
    static constexpr int rows() { return L ? 256 / (L ? L : 1) : 1; }
};

// Sums of N values over the lanes of a row, in a fixed order; `red` holds N
// floats per wave.
template <int L, int N>
__device__ inline void row_sums(float (&v)[N], float (*red)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if constexpr (L == 16 || L == 32) v[i] = lanes_sum<L>(v[i]);
        else v[i] = wave_sum(v[i]);
    }
    if constexpr (L == 0) {
        const int waves = blockDim.x >> 6;
        if (waves == 1) return;
        __syncthreads();   // the sums before have been read
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) red[threadIdx.x >> 6][i] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = red[0][i];
        for (int k = 1; k < waves; ++k)
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] += red[k][i];
    }
}

__device__ inline f32x8 weights(const void *w, bool w_f32, int e0) {
    return w_f32 ? widen(load_raw(static_cast<const float *>(w) + e0))
                 : widen(load_raw(static_cast<const __bf16 *>(w) + e0));
}

// F8: y as e4m3 values q [M][D] and scales [D / 512][M][4] (fp8.h).  RES: with
// the residual.  ONCE: past the caches.  All loads of a row are issued at once:
// lanes past its end read its last chunk, for a load behind a branch is waited
// for there.
template <typename T, typename W, bool F8, int NC, bool RES, bool ONCE>
__global__ __launch_bounds__(1024) void rms_norm_kernel(
    const T *__restrict__ x, const T *__restrict__ r, const W *__restrict__ w, T *__restrict__ y,
    unsigned char *__restrict__ q, unsigned *__restrict__ scale, T *__restrict__ h_out, int64_t M, int D,
    int64_t ldx, int64_t ldr, float eps) {
    __shared__ float red[16][1];
    const int t = threadIdx.x, L = blockDim.x;
    const int64_t m = block_index();
    if (m >= M) return;
    const T *xr = x + m * ldx, *rr = RES ? r + m * ldr : nullptr;
    using Raw = decltype(load_raw(x));
    Raw xv[NC], rv[RES ? NC : 1];
#pragma unroll
    for (int j = 0; j < NC; ++j) {
        const int e0 = chunk_at(j * L + t, D).e0;
        xv[j] = load_raw_if<ONCE>(xr + e0);
        if constexpr (RES) rv[j] = load_raw_if<ONCE>(rr + e0);
    }
    decltype(load_raw(w)) wv[NC];
#pragma unroll
    for (int j = 0; j < NC; ++j) wv[j] = load_raw(w + chunk_at(j * L + t, D).e0);
    f32x8 h[NC];
    float sum[1] = {0};
#pragma unroll
    for (int j = 0; j < NC; ++j) {
        h[j] = widen(xv[j]);
        if constexpr (RES) h[j] += widen(rv[j]);
        const int dup = chunk_at(j * L + t, D).dup;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[0] += i >= dup ? h[j][i] * h[j][i] : 0.0f;
    }
    row_sums<0>(sum, red);
    const float rstd = 1.0f / __builtin_sqrtf(sum[0] / static_cast<float>(D) + eps);
#pragma unroll
    for (int j = 0; j < NC; ++j) {
        const int c = j * L + t;
        const bool in = c * 8 < D;
        const int e0 = chunk_at(c, D).e0;
        f32x8 v{};
        if (in) {
            if constexpr (RES) store_8_if<ONCE>(h_out + m * D + e0, h[j]);
            v = h[j] * rstd * widen(wv[j]);
        }
        if constexpr (!F8) {
            if (in) store_8_if<ONCE>(y + m * D + e0, v);
        } else {
            // 16 lanes hold a block of 128, a wave a group of 4 blocks (none
            // of it past the row's last group).
            if ((c & ~63) * 8 >= D) continue;
            unsigned a = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) a = max(a, fp8::magnitude(v[i]));
            const unsigned b = fp8::scale_byte(fp8::max16(a));
            const float by = fp8::inverse_scale(b);
            if (in) {
                const uint2 o = {fp8::pack4(v[0] * by, v[1] * by, v[2] * by, v[3] * by),
                                 fp8::pack4(v[4] * by, v[5] * by, v[6] * by, v[7] * by)};
                *reinterpret_cast<uint2 *>(q + m * D + e0) = o;
            }
            const unsigned four = __builtin_amdgcn_readlane(b, 0) | __builtin_amdgcn_readlane(b, 16) << 8 |
                                  __builtin_amdgcn_readlane(b, 32) << 16 | __builtin_amdgcn_readlane(b, 48) << 24;
            if ((threadIdx.x & 63) == 0) scale[(c >> 6) * M + m] = four;
        }
    }
}

// Narrow rows (a norm of head vectors), one chunk per lane: L lanes (16 or 32) take a
// row, a workgroup 256 / L of them; with a wave per row 280800 x 128 in bf16 takes 61.6
// us, so 22.3 (6.4 TB/s), 56160 x 256 15.1 and 10.6 (x 512 17.6 and, on 64 lanes,
// 18.1).  The sums are those of the kernel above, in its order, whose lanes past the
// row add zeros.
template <typename T, typename W, int L, bool RES>
__global__ __launch_bounds__(256) void rms_norm_narrow_kernel(
    const T *__restrict__ x, const T *__restrict__ r, const W *__restrict__ w, T *__restrict__ y,
    T *__restrict__ h_out, int64_t M, int D, int64_t ldx, int64_t ldr, float eps) {
    const int t = threadIdx.x & (L - 1);
    const int64_t row = block_index() * (256 / L) + threadIdx.x / L, m = min(row, M - 1);
    const Chunk c = chunk_at(t, D);
    const auto xv = load_raw(x + m * ldx + c.e0);
    decltype(load_raw(x)) rv;
    if constexpr (RES) rv = load_raw(r + m * ldr + c.e0);
    const f32x8 wv = widen(load_raw(w + c.e0));
    f32x8 h = widen(xv);
    if constexpr (RES) h += widen(rv);
    float sum = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += i >= c.dup ? h[i] * h[i] : 0.0f;
    sum = lanes_sum<L>(sum);
    const float rstd = 1.0f / __builtin_sqrtf(sum / static_cast<float>(D) + eps);
    if (row >= M || t * 8 >= D) return;
    if constexpr (RES) store_8(h_out + m * D + c.e0, h);
    store_8(y + m * D + c.e0, h * rstd * wv);
}

// Backward: h = x + r again, unrounded as in the forward (from the stored h,
// rounded, dw would be 1.4 times as far from the exact sum in bf16; reading x
// and r costs one tensor more), n = h rstd, g = dy w,
//   dx = rstd (g - n mean(g n)) + dh,   dw = sum over rows of dy n.
// A workgroup takes every gridDim.x-th set of rows, its next row's loads issued
// ahead of this row's sums (AHEAD; 7800 rows of 5120 with dh 103 us where
// branches around the loads waited for them, 74 without), and keeps its share of
// dw in registers.  Rows that 512 lanes do not hold, whose values and next row
// would not fit the registers, are read twice instead (9000 x 16384 in bf16 with
// residual and dh 325 us, 4.5 TB/s of what is needed once; 2000 rows 81).  fp32 with
// both, 7800 x 5120: 153 us, 5.2 TB/s.  The shares go to partial
// [gridDim.x][D] and are summed by sum_rows_kernel, so no atomics: the order is
// fixed.  RES, DH: with the residual, with dh.  ONCE: past the caches.
template <typename T, int LANES, int NC, int MAX, bool AHEAD, bool RES, bool DH, bool ONCE>
__global__ __launch_bounds__(MAX) void rms_norm_backward_kernel(
    const T *__restrict__ dy, const T *__restrict__ x, const T *__restrict__ r, const T *__restrict__ dh,
    const void *__restrict__ w, bool w_f32, T *__restrict__ dx, float *__restrict__ partial, int64_t M, int D,
    int64_t ldx, int64_t ldr, float eps) {
    __shared__ float red[16][2];
    __shared__ float share[LANES ? LANES * NC * 8 : 1];
    using P = Lane<LANES>;
    const int t = P::t(), L = P::lanes();
    f32x8 acc[NC];
    int e0[NC], dup[NC];
    bool in[NC];
#pragma unroll
    for (int j = 0; j < NC; ++j) {
        const Chunk k = chunk_at(j * L + t, D);
        in[j] = (j * L + t) * 8 < D;
        e0[j] = k.e0;
        dup[j] = k.dup;
        acc[j] = f32x8{};
    }
    const int64_t step = static_cast<int64_t>(gridDim.x) * P::rows();
    int64_t m = static_cast<int64_t>(blockIdx.x) * P::rows() + P::row();
    const auto add = [&](float (&sums)[2], int j, const f32x8 &n, const f32x8 &g, const f32x8 &wv) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            sums[0] += i >= dup[j] ? n[i] * n[i] : 0.0f;
            sums[1] += i >= dup[j] ? g[i] * wv[i] * n[i] : 0.0f;
        }
    };
    float rstd, mean;
    const auto finish_sums = [&](float (&sums)[2]) {
        row_sums<LANES>(sums, red);
        rstd = 1.0f / __builtin_sqrtf(sums[0] / static_cast<float>(D) + eps);
        mean = sums[1] * rstd / static_cast<float>(D);
    };
    // dx without dh, and the chunk's part of dw.
    const auto gradient = [&](int j, const f32x8 &n, const f32x8 &g, const f32x8 &wv) {
        const f32x8 nn = n * rstd;
        acc[j] += g * nn;
        return (g * wv - nn * mean) * rstd;
    };
    using Raw = decltype(load_raw(x));
    if constexpr (AHEAD) {
        f32x8 wv[NC];
        Raw xn[NC], rn[RES ? NC : 1], gn[NC];
        // No branch around loads and stores, which would wait for all that is in
        // flight: lanes past the row's end read its last chunk and store the
        // same values there, and the load past the last row reads that row.
        const auto fetch = [&](int64_t at) {
            at = at < M ? at : M - 1;
#pragma unroll
            for (int j = 0; j < NC; ++j) {
                xn[j] = load_raw_if<ONCE>(x + at * ldx + e0[j]);
                gn[j] = load_raw_if<ONCE>(dy + at * D + e0[j]);
                if constexpr (RES) rn[j] = load_raw_if<ONCE>(r + at * ldr + e0[j]);
            }
        };
#pragma unroll
        for (int j = 0; j < NC; ++j) wv[j] = weights(w, w_f32, e0[j]);
        fetch(m);
        for (; m < M; m += step) {
            f32x8 n[NC], g[NC];
            Raw dhr[DH ? NC : 1];
#pragma unroll
            for (int j = 0; j < NC; ++j) {
                if constexpr (DH) dhr[j] = load_raw_if<ONCE>(dh + m * D + e0[j]);
            }
#pragma unroll
            for (int j = 0; j < NC; ++j) {
                n[j] = widen(xn[j]);
                if constexpr (RES) n[j] += widen(rn[j]);
                g[j] = widen(gn[j]);
            }
            fetch(m + step);
            float sums[2] = {0, 0};
#pragma unroll
            for (int j = 0; j < NC; ++j) add(sums, j, n[j], g[j], wv[j]);
            finish_sums(sums);
#pragma unroll
            for (int j = 0; j < NC; ++j) {
                f32x8 o = gradient(j, n[j], g[j], wv[j]);
                if constexpr (DH) o += widen(dhr[j]);
                store_8_if<ONCE>(dx + m * D + e0[j], o);
            }
        }
    } else {
        for (; m < M; m += step) {
            f32x8 n, g, wv;
            const auto fetch = [&](int j) {
                asm volatile("" : "+v"(e0[j]));   // the second reading is one: nothing is kept
                n = widen(load_raw(x + m * ldx + e0[j]));
                if constexpr (RES) n += widen(load_raw(r + m * ldr + e0[j]));
                g = widen(load_raw(dy + m * D + e0[j]));
                wv = weights(w, w_f32, e0[j]);
            };
            float sums[2] = {0, 0};
#pragma unroll
            for (int j = 0; j < NC; ++j)
                if (in[j]) {
                    fetch(j);
                    add(sums, j, n, g, wv);
                }
            finish_sums(sums);
#pragma unroll
            for (int j = 0; j < NC; ++j)
                if (in[j]) {
                    fetch(j);
                    f32x8 o = gradient(j, n, g, wv);
                    if constexpr (DH) o += widen(load_raw(dh + m * D + e0[j]));
                    store_8(dx + m * D + e0[j], o);
                }
        }
    }
    if constexpr (LANES > 0) {
        // The rows' shares, added in their order.
        constexpr int last = P::rows() - 1;
        for (int k = 0; k <= last; ++k) {
            if (P::row() == k)
#pragma unroll
                for (int j = 0; j < NC; ++j)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        float &s = share[(j * 8 + i) * LANES + t];
                        s = k == 0 ? acc[j][i] : s + acc[j][i];
                        if (k == last) acc[j][i] = s;
                    }
            __syncthreads();
        }
        if (P::row() != last) return;
    }
#pragma unroll
    for (int j = 0; j < NC; ++j)
        if (in[j]) store_8(partial + static_cast<int64_t>(blockIdx.x) * D + e0[j], acc[j]);
}

// out[d] = sum over P rows of partial[P][D]: 16 columns per workgroup, 64 lanes
// each, whose sums are added in a fixed order (16 lanes each: 256 rows of 5120
// 4.3 us in the trace).
template <typename T>
__global__ __launch_bounds__(1024) void sum_rows_kernel(const float *__restrict__ partial, T *__restrict__ out,
                                                        int P, int D) {
    __shared__ float part[64][17];
    const int col = threadIdx.x & 15, k = threadIdx.x >> 4, d = blockIdx.x * 16 + col;
    float s = 0;
    if (d < D)
#pragma unroll 4
        for (int p = k; p < P; p += 64) s += partial[static_cast<int64_t>(p) * D + d];
    part[k][col] = s;
    __syncthreads();
    if (k < 8) {
#pragma unroll
        for (int i = 1; i < 8; ++i) s += part[k + 8 * i][col];
        part[k][col] = s;
    }
    __syncthreads();
    if (k == 0 && d < D) {
#pragma unroll
        for (int i = 1; i < 8; ++i) s += part[i][col];
        out[d] = static_cast<T>(s);
    }
}

struct NormArgs {
    const void *x, *r, *w;
    bool w_f32;
    void *y, *q, *scale, *h;
    int64_t M;
    int D;
    int64_t ldx, ldr;
    float eps;
};

// Lanes of a row of D elements in NC chunks each, in whole waves.
int lanes_for(int D, int NC) { return ((D + 7) / 8 + 64 * NC - 1) / (64 * NC) * 64; }

template <typename T, typename W, bool F8, int NC, bool ONCE>
hipError_t run_norm_of(const NormArgs &a, hipStream_t s) {
    const int threads = lanes_for(a.D, NC);
    if (a.M < 1 || threads > 1024) return hipErrorInvalidValue;
    const auto kernel = a.r ? rms_norm_kernel<T, W, F8, NC, true, ONCE> : rms_norm_kernel<T, W, F8, NC, false, ONCE>;
    kernel<<<grid_of(a.M), threads, 0, s>>>(
        static_cast<const T *>(a.x), static_cast<const T *>(a.r), static_cast<const W *>(a.w),
        static_cast<T *>(a.y), static_cast<unsigned char *>(a.q), static_cast<unsigned *>(a.scale),
        static_cast<T *>(a.h), a.M, a.D, a.ldx, a.ldr, a.eps);
    return hipGetLastError();
}
template <typename T, typename W, int L>
hipError_t run_narrow(const NormArgs &a, hipStream_t s) {
    if (a.M < 1 || a.D > 8 * L) return hipErrorInvalidValue;
    const auto kernel = a.r ? rms_norm_narrow_kernel<T, W, L, true> : rms_norm_narrow_kernel<T, W, L, false>;
    kernel<<<grid_of((a.M + 256 / L - 1) / (256 / L)), 256, 0, s>>>(
        static_cast<const T *>(a.x), static_cast<const T *>(a.r), static_cast<const W *>(a.w), static_cast<T *>(a.y),
        static_cast<T *>(a.h), a.M, a.D, a.ldx, a.ldr, a.eps);
    return hipGetLastError();
}
template <typename T, typename W>
hipError_t narrow_typed(const NormArgs &a, hipStream_t s) {
    if (a.D <= 128) return run_narrow<T, W, 16>(a, s);
    return run_narrow<T, W, 32>(a, s);
}

// Tensors that together are twice what the caches hold (256 MiB) are read and
// written past them (bf16 with a residual: 56160 x 5120 396 us without, 385 with,
// in 8 bits 340 and 329; 15000 x 16384 349 and 318; below, a reader finds them there).
constexpr int64_t kCaches = int64_t{512} << 20;
template <typename T, bool F8, int NC>
hipError_t run_norm(const NormArgs &a, hipStream_t s) {
    if constexpr (NC == 2) {
        if (a.M * a.D * static_cast<int64_t>(sizeof(T)) * (a.r ? 4 : 2) > kCaches)
            return a.w_f32 ? run_norm_of<T, float, F8, 2, true>(a, s) : run_norm_of<T, __bf16, F8, 2, true>(a, s);
    }
    return a.w_f32 ? run_norm_of<T, float, F8, NC, false>(a, s) : run_norm_of<T, __bf16, F8, NC, false>(a, s);
}

// One chunk per lane, two for many long rows and for rows that 1024 lanes do
// not hold.  With one and with two, bf16 with a residual, 56160 rows: D = 5120
// 399 and 396 us (5.8 TB/s), in 8 bits 391 and 340; D = 2560 200 and 198, in 8
// bits 179 and 173; D = 1280 102 and 102.
template <typename T, bool F8>
hipError_t norm_typed(const NormArgs &a, hipStream_t s) {
    if (!F8 && a.D <= 256) return a.w_f32 ? narrow_typed<T, float>(a, s) : narrow_typed<T, __bf16>(a, s);
    if ((a.M >= 1024 && a.D > 2048) || a.D > 8192) return run_norm<T, F8, 2>(a, s);
    return run_norm<T, F8, 1>(a, s);
}

struct BackwardArgs {
    const void *dy, *x, *r, *dh, *w;
    bool w_f32;
    void *dx;
    float *partial;
    int64_t M;
    int D;
    int64_t ldx, ldr;
    float eps;
    int P;
};

template <typename T, int LANES, int NC, int MAX, bool AHEAD, bool ONCE>
hipError_t run_backward_of(const BackwardArgs &a, hipStream_t s) {
    const int threads = LANES ? 256 : lanes_for(a.D, NC);
    if (threads > MAX || (LANES && a.D > LANES * NC * 8)) return hipErrorInvalidValue;
    const auto kernel = a.r ? (a.dh ? rms_norm_backward_kernel<T, LANES, NC, MAX, AHEAD, true, true, ONCE>
                                    : rms_norm_backward_kernel<T, LANES, NC, MAX, AHEAD, true, false, ONCE>)
                            : (a.dh ? rms_norm_backward_kernel<T, LANES, NC, MAX, AHEAD, false, true, ONCE>
                                    : rms_norm_backward_kernel<T, LANES, NC, MAX, AHEAD, false, false, ONCE>);
    kernel<<<a.P, threads, 0, s>>>(
        static_cast<const T *>(a.dy), static_cast<const T *>(a.x), static_cast<const T *>(a.r),
        static_cast<const T *>(a.dh), a.w, a.w_f32, static_cast<T *>(a.dx), a.partial, a.M, a.D, a.ldx, a.ldr,
        a.eps);
    return hipGetLastError();
}
// Tensors that the last-level cache does not hold together are read and written
// past the caches (bf16 with residual and dh: 7800 x 5120, 400 MB, 73 us without and
// 65 with; 56160 x 5120 520 and 476; 30000 x 1280 72 and 63; 3000 x 5120, 154 MB, 27.0
// and 27.5).  Rows that are read twice have to be kept.
template <typename T, int LANES, int NC, int MAX, bool AHEAD>
hipError_t run_backward(const BackwardArgs &a, hipStream_t s) {
    const int64_t bytes = a.M * a.D * static_cast<int64_t>(sizeof(T)) * (3 + (a.r != nullptr) + (a.dh != nullptr));
    if (AHEAD && bytes > int64_t{256} << 20) return run_backward_of<T, LANES, NC, MAX, AHEAD, AHEAD>(a, s);
    return run_backward_of<T, LANES, NC, MAX, AHEAD, false>(a, s);
}

template <typename T>
hipError_t backward_typed(const BackwardArgs &a, hipStream_t s) {
    if (a.D <= 128) return run_backward<T, 16, 1, 256, true>(a, s);
    if (a.D <= 256) return run_backward<T, 32, 1, 256, true>(a, s);
    if (a.D <= 512) return run_backward<T, 64, 1, 256, true>(a, s);
    if (a.D <= 1024) return run_backward<T, 64, 2, 256, true>(a, s);
    if (a.D <= 8192) return run_backward<T, 0, 2, 512, true>(a, s);
    return run_backward<T, 0, 2, 1024, false>(a, s);
}

}  // namespace

int rms_norm_max_width() { return 16384; }

// Workgroups of the backward: up to D = 128 sixteen rows at once, to 256 eight, to
// 1024 four, then one (56160 x 128 with a wave per row 24.6 us, on 16 lanes 13.5;
// 280800 x 128 98 and 38; 56160 x 256 26.0 and, on 32, 19.7); on 256 CUs so many per
// CU as measured best (bf16 with residual and dh; 56160 rows: D = 640 110 with one, 77
// with two, 71 with four, 72 with eight; 30000 rows: D = 1280 130, 94, 70 with three,
// 63 with four; D = 2560 142, 124, 134, 137; D = 3840 178, 202; 56160 x 5120 476 (6.0
// TB/s), 524).
int rms_norm_partials(int64_t M, int D) {
    const int64_t rows = D <= 128 ? 16 : D <= 256 ? 8 : D <= 1024 ? 4 : 1;
    const int waves = lanes_for(D, 2) / 64;   // of a row past D = 1024
    const int64_t most = 256 * (D <= 1024 || waves <= 2 ? 4 : waves == 3 ? 2 : 1);
    const int64_t sets = (M + rows - 1) / rows;
    return static_cast<int>(sets < most ? sets : most);
}

hipError_t launch_rms_norm(const void *x, const void *r, const void *w, bool w_f32, void *y, void *q,
                           void *scale, void *h, int64_t M, int D, int64_t ldx, int64_t ldr, float eps,
                           int dtype, hipStream_t stream) {
    if (M == 0) return hipSuccess;
    const NormArgs a{x, r, w, w_f32, y, q, scale, h, M, D, ldx, ldr, eps};
    if (dtype == 0) return q ? norm_typed<__bf16, true>(a, stream) : norm_typed<__bf16, false>(a, stream);
    return q ? norm_typed<float, true>(a, stream) : norm_typed<float, false>(a, stream);
}

hipError_t launch_rms_norm_backward(const void *dy, const void *x, const void *r, const void *dh, const void *w,
                                    bool w_f32, void *dx, void *dw, float *partial, int64_t M, int D, int64_t ldx,
                                    int64_t ldr, float eps, int dtype, hipStream_t stream) {
    const int P = rms_norm_partials(M, D);
    if (P > 0) {
        const BackwardArgs a{dy, x, r, dh, w, w_f32, dx, partial, M, D, ldx, ldr, eps, P};
        const hipError_t e = dtype == 0 ? backward_typed<__bf16>(a, stream) : backward_typed<float>(a, stream);
        if (e != hipSuccess) return e;
    }
    const int blocks = (D + 15) / 16;
    if (w_f32) sum_rows_kernel<<<blocks, 1024, 0, stream>>>(partial, static_cast<float *>(dw), P, D);
    else sum_rows_kernel<<<blocks, 1024, 0, stream>>>(partial, static_cast<__bf16 *>(dw), P, D);
    return hipGetLastError();
}

}  // namespace hcms
