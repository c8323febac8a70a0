// Root-mean-square norm with the residual's addition, forward and backward:
//   h = x + r,  y = h / sqrt(mean(h^2) + eps) * w        rows of D elements
// h is the residual stream's next value; it is stored rounded to the storage
// type, while y is computed from the unrounded sum.  The statistics are fp32.
//
// What bounds it: bytes.  A row is read once into registers, summed and
// written once, by a wave (64 lanes) where that leaves enough rows to fill
// the CUs, else by 256 or 1024 lanes.
#include "fp8.h"
#include "hcms_internal.h"

namespace hcms {
namespace {

using fp8::f32x8;

// Lane t of a row's TPR lanes holds the chunks of 8 elements t, t + TPR, ...
// The chunk that the row's end cuts is read from D - 8 on: its first `dup`
// elements are another lane's too, which stores the same values; sums take
// them from that lane alone.
struct Chunk {
    int e0, dup;
};
__device__ inline Chunk chunk_at(int c, int D) {
    const int e = c * 8, e0 = min(e, D - 8);
    return {e0, e - e0};
}

// Sum of v over the TPR lanes of a row; `red` holds a float per wave.
template <int TPR>
__device__ inline float row_sum(float v, float *red) {
    v = wave_sum(v);
    if constexpr (TPR > 64) {
        __syncthreads();   // the floats of the sum before have been read
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0;
#pragma unroll
        for (int i = 0; i < TPR / 64; ++i) v += red[i];
    }
    return v;
}

__device__ inline f32x8 weights(const void *w, bool w_f32, int e0) {
    return w_f32 ? widen(load_raw(static_cast<const float *>(w) + e0))
                 : widen(load_raw(static_cast<const __bf16 *>(w) + e0));
}

// F8: y as e4m3 values q [M][D] and scales [D / 512][M][4] (fp8.h).
template <typename T, bool F8, int TPR, int NC>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void rms_norm_kernel(
    const T *__restrict__ x, const T *__restrict__ r, const void *__restrict__ w, bool w_f32,
    T *__restrict__ y, unsigned char *__restrict__ q, unsigned *__restrict__ scale, T *__restrict__ h_out,
    int64_t M, int D, int64_t ldx, int64_t ldr, float eps) {
    __shared__ float red[TPR / 64];
    const int t = threadIdx.x % TPR;
    const int64_t m = TPR >= 256 ? blockIdx.x : static_cast<int64_t>(blockIdx.x) * (256 / TPR) + threadIdx.x / TPR;
    if (TPR < 256 && m >= M) return;   // whole waves, and no barrier follows for them
    const T *xr = x + m * ldx;
    f32x8 h[NC];
#pragma unroll
    for (int j = 0; j < NC; ++j) {
        const int c = j * TPR + t;
        h[j] = c * 8 < D ? widen(load_raw(xr + chunk_at(c, D).e0)) : f32x8{};
    }
    if (r) {
        const T *rr = r + m * ldr;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const int c = j * TPR + t;
            if (c * 8 < D) h[j] += widen(load_raw(rr + chunk_at(c, D).e0));
        }
    }
    float sum = 0;
#pragma unroll
    for (int j = 0; j < NC; ++j) {
        const int dup = chunk_at(j * TPR + t, D).dup;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += i >= dup ? h[j][i] * h[j][i] : 0.0f;
    }
    sum = row_sum<TPR>(sum, red);
    const float rstd = 1.0f / __builtin_sqrtf(sum / static_cast<float>(D) + eps);
#pragma unroll
    for (int j = 0; j < NC; ++j) {
        const int c = j * TPR + t;
        const bool in = c * 8 < D;
        const int e0 = chunk_at(c, D).e0;
        f32x8 v{};
        if (in) {
            if (r) store_8(h_out + m * D + e0, h[j]);
            v = h[j] * rstd * weights(w, w_f32, e0);
        }
        if constexpr (!F8) {
            if (in) store_8(y + m * D + e0, v);
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

// Backward: h = x + r again, unrounded as in the forward (from the stored h,
// rounded, dw would be 1.4 times as far from the exact sum in bf16; reading x
// and r costs one tensor more), n = h rstd, g = dy w,
//   dx = rstd (g - n mean(g n)) + dh,   dw = sum over rows of dy n.
// A workgroup takes every gridDim.x-th set of rows and keeps its share of dw
// in registers; the shares go to partial [gridDim.x][D] and are summed by
// sum_rows_kernel, so no atomics: the order is fixed.
template <typename T, int TPR, int NC>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void rms_norm_backward_kernel(
    const T *__restrict__ dy, const T *__restrict__ x, const T *__restrict__ r, const T *__restrict__ dh,
    const void *__restrict__ w, bool w_f32, T *__restrict__ dx, float *__restrict__ partial, int64_t M, int D,
    int64_t ldx, int64_t ldr, float eps) {
    constexpr int RB = TPR < 256 ? 256 / TPR : 1;   // rows at once
    __shared__ float red[TPR / 64];
    __shared__ float share[RB > 1 ? TPR * NC * 8 : 1];
    const int t = threadIdx.x % TPR;
    f32x8 acc[NC];
#pragma unroll
    for (int j = 0; j < NC; ++j) acc[j] = f32x8{};
    for (int64_t m = static_cast<int64_t>(blockIdx.x) * RB + threadIdx.x / TPR; m < M;
         m += static_cast<int64_t>(gridDim.x) * RB) {
        f32x8 n[NC], g[NC];
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const int c = j * TPR + t;
            n[j] = c * 8 < D ? widen(load_raw(x + m * ldx + chunk_at(c, D).e0)) : f32x8{};
        }
        if (r) {
#pragma unroll
            for (int j = 0; j < NC; ++j) {
                const int c = j * TPR + t;
                if (c * 8 < D) n[j] += widen(load_raw(r + m * ldr + chunk_at(c, D).e0));
            }
        }
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const int c = j * TPR + t;
            g[j] = c * 8 < D ? widen(load_raw(dy + m * D + chunk_at(c, D).e0)) : f32x8{};
        }
        float ss = 0, sg = 0;
        f32x8 wv[NC];
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const int c = j * TPR + t;
            const Chunk k = chunk_at(c, D);
            wv[j] = c * 8 < D ? weights(w, w_f32, k.e0) : f32x8{};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                ss += i >= k.dup ? n[j][i] * n[j][i] : 0.0f;
                sg += i >= k.dup ? g[j][i] * wv[j][i] * n[j][i] : 0.0f;
            }
        }
        ss = row_sum<TPR>(ss, red);
        sg = row_sum<TPR>(sg, red);
        const float rstd = 1.0f / __builtin_sqrtf(ss / static_cast<float>(D) + eps);
        const float mean = sg * rstd / static_cast<float>(D);
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const int c = j * TPR + t;
            if (c * 8 >= D) continue;
            const int e0 = chunk_at(c, D).e0;
            const f32x8 nn = n[j] * rstd;
            acc[j] += g[j] * nn;
            f32x8 o = (g[j] * wv[j] - nn * mean) * rstd;
            if (dh) o += widen(load_raw(dh + m * D + e0));
            store_8(dx + m * D + e0, o);
        }
    }
    if constexpr (RB > 1) {
        // The waves' shares, added in the order of the waves.
        for (int k = 0; k < RB; ++k) {
            if (static_cast<int>(threadIdx.x) / TPR == k)
#pragma unroll
                for (int j = 0; j < NC; ++j)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        float &s = share[(j * 8 + i) * TPR + t];
                        s = k == 0 ? acc[j][i] : s + acc[j][i];
                        if (k == RB - 1) acc[j][i] = s;
                    }
            __syncthreads();
        }
        if (static_cast<int>(threadIdx.x) / TPR != RB - 1) return;
    }
#pragma unroll
    for (int j = 0; j < NC; ++j) {
        const int c = j * TPR + t;
        if (c * 8 < D) store_8(partial + static_cast<int64_t>(blockIdx.x) * D + chunk_at(c, D).e0, acc[j]);
    }
}

// out[d] = sum over P rows of partial[P][D]: 16 columns per workgroup, 16 lanes
// each, whose sums are added in order.
template <typename T>
__global__ __launch_bounds__(256) void sum_rows_kernel(const float *__restrict__ partial, T *__restrict__ out,
                                                       int P, int D) {
    __shared__ float part[16][17];
    const int col = threadIdx.x & 15, k = threadIdx.x >> 4, d = blockIdx.x * 16 + col;
    float s = 0;
    if (d < D)
        for (int p = k; p < P; p += 16) s += partial[static_cast<int64_t>(p) * D + d];
    part[k][col] = s;
    __syncthreads();
    if (k == 0 && d < D) {
        for (int i = 1; i < 16; ++i) s += part[i][col];
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

template <typename T, bool F8, int TPR, int NC>
hipError_t run_norm(const NormArgs &a, hipStream_t s) {
    constexpr int RB = TPR < 256 ? 256 / TPR : 1;
    const int64_t blocks = (a.M + RB - 1) / RB;
    if (blocks < 1 || blocks > 0x7fffffff) return hipErrorInvalidValue;
    rms_norm_kernel<T, F8, TPR, NC><<<static_cast<unsigned>(blocks), TPR < 256 ? 256 : TPR, 0, s>>>(
        static_cast<const T *>(a.x), static_cast<const T *>(a.r), a.w, a.w_f32, static_cast<T *>(a.y),
        static_cast<unsigned char *>(a.q), static_cast<unsigned *>(a.scale), static_cast<T *>(a.h), a.M, a.D,
        a.ldx, a.ldr, a.eps);
    return hipGetLastError();
}

// A wave per row from 1024 rows on, 256 lanes for fewer or longer rows.
template <typename T, bool F8>
hipError_t norm_typed(const NormArgs &a, hipStream_t s) {
    const int D = a.D;
    if (D <= 512) return run_norm<T, F8, 64, 1>(a, s);
    if (a.M >= 1024) {
        if (D <= 1536) return run_norm<T, F8, 64, 3>(a, s);
        if (D <= 2560) return run_norm<T, F8, 64, 5>(a, s);
        if (D <= 5120) return run_norm<T, F8, 64, 10>(a, s);
    }
    if (D <= 2048) return run_norm<T, F8, 256, 1>(a, s);
    if (D <= 6144) return run_norm<T, F8, 256, 3>(a, s);
    return run_norm<T, F8, 256, 8>(a, s);
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

template <typename T, int TPR, int NC>
hipError_t run_backward(const BackwardArgs &a, hipStream_t s) {
    rms_norm_backward_kernel<T, TPR, NC><<<a.P, TPR < 256 ? 256 : TPR, 0, s>>>(
        static_cast<const T *>(a.dy), static_cast<const T *>(a.x), static_cast<const T *>(a.r),
        static_cast<const T *>(a.dh), a.w, a.w_f32, static_cast<T *>(a.dx), a.partial, a.M, a.D, a.ldx, a.ldr,
        a.eps);
    return hipGetLastError();
}

template <typename T>
hipError_t backward_typed(const BackwardArgs &a, hipStream_t s) {
    if (a.D <= 512) return run_backward<T, 64, 1>(a, s);
    if (a.D <= 2048) return run_backward<T, 256, 1>(a, s);
    if (a.D <= 6144) return run_backward<T, 256, 3>(a, s);
    if (a.D <= 8192) return run_backward<T, 1024, 1>(a, s);
    return run_backward<T, 1024, 2>(a, s);
}

}  // namespace

int rms_norm_max_width() { return 16384; }

int rms_norm_partials(int64_t M, int D) {
    const int64_t rows = D <= 512 ? 4 : 1;
    const int64_t sets = (M + rows - 1) / rows;
    return static_cast<int>(sets < 1024 ? sets : 1024);
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
    if (w_f32) sum_rows_kernel<<<blocks, 256, 0, stream>>>(partial, static_cast<float *>(dw), P, D);
    else sum_rows_kernel<<<blocks, 256, 0, stream>>>(partial, static_cast<__bf16 *>(dw), P, D);
    return hipGetLastError();
}

}  // namespace hcms
