// 8-bit floating point with block scales (gfx950): e4m3 values, and per block
// of 128 one power of two, held as its exponent byte (e8m0), which is the form
// the scaled MFMAs take.  The scale s of a block is the smallest power of two
// from 2^-126 on that brings its largest magnitude a to at most 448, the
// largest e4m3 value: x / s is exact in every precision, so a value's rounding
// depends on nothing but the value and its block's exponent, and nothing
// saturates.  e4m3 keeps 3 bits behind the leading one over 15 binades below
// 448, so a scale up to twice as large as a / 448 costs no precision but in
// values below 2^-14 of the largest.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace hcms {
namespace fp8 {

inline constexpr int kBlock = 128;            // elements that share a scale, along a row
inline constexpr int kGroup = 4 * kBlock;     // elements of a group of 4 scales (one dword)

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x8 __attribute__((ext_vector_type(8)));

// Exponent byte of the scale of a block whose largest magnitude has the bits
// `amax`; 448 = 1.75 * 2^8, so the sum carries into the exponent past 1.75.
// 255 (NaN) for a block that holds an infinity or a NaN.
__device__ inline unsigned scale_byte(unsigned amax) {
    if (amax >= 0x7F800000u) return 255u;
    const int e = static_cast<int>((amax + 0x1FFFFFu) >> 23) - 8;
    return e < 1 ? 1u : static_cast<unsigned>(e);
}
// 1 / scale (NaN for 255; otherwise 7 <= 254 - b <= 253 is a normal exponent).
__device__ inline float inverse_scale(unsigned b) {
    return __builtin_bit_cast(float, b == 255u ? 0x7FC00000u : (254u - b) << 23);
}

// Bits of |x|, whose order is that of the magnitudes with NaN above infinity.
__device__ inline unsigned magnitude(float x) { return __builtin_bit_cast(unsigned, x) & 0x7FFFFFFFu; }

// Four values to e4m3, nearest even, the first in the lowest byte.
__device__ inline unsigned pack4(float a, float b, float c, float d) {
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
    return static_cast<unsigned>(r);
}

// Maximum over the 16 lanes of a row (every lane gets it).
__device__ inline unsigned max16(unsigned v) {
#define HCMS_ROR(n) \
    v = max(v, static_cast<unsigned>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x120 + n, 0xF, 0xF, true)))
    HCMS_ROR(8);
    HCMS_ROR(4);
    HCMS_ROR(2);
    HCMS_ROR(1);
#undef HCMS_ROR
    return v;
}

}  // namespace fp8

// Sum over the 64 lanes of a wave (every lane gets it), in a fixed order.
__device__ inline float wave_sum(float v) {
#define HCMS_ROR(n) \
    v += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x120 + n, 0xF, 0xF, true))
    HCMS_ROR(8);
    HCMS_ROR(4);
    HCMS_ROR(2);
    HCMS_ROR(1);
#undef HCMS_ROR
    const int i = __builtin_bit_cast(int, v);
    return (__builtin_bit_cast(float, __builtin_amdgcn_readlane(i, 0)) +
            __builtin_bit_cast(float, __builtin_amdgcn_readlane(i, 16))) +
           (__builtin_bit_cast(float, __builtin_amdgcn_readlane(i, 32)) +
            __builtin_bit_cast(float, __builtin_amdgcn_readlane(i, 48)));
}

// Sum over groups of L lanes (16 or 32), in the order of wave_sum.
template <int L>
__device__ inline float lanes_sum(float v) {
#define HCMS_ROR(n) \
    v += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x120 + n, 0xF, 0xF, true))
    HCMS_ROR(8);
    HCMS_ROR(4);
    HCMS_ROR(2);
    HCMS_ROR(1);
#undef HCMS_ROR
    if constexpr (L == 32) v += __shfl_xor(v, 16);
    return v;
}

// 8 consecutive elements from any element's address (the hardware takes
// 16-byte accesses at every alignment of global memory) as fp32, and back,
// rounded to nearest even.
typedef __bf16 bf16x8_any __attribute__((ext_vector_type(8), aligned(2)));
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
struct raw_f32x8 {
    f32x4_any a, b;
};
__device__ inline bf16x8_any load_raw(const __bf16 *p) { return *reinterpret_cast<const bf16x8_any *>(p); }
__device__ inline raw_f32x8 load_raw(const float *p) {
    return {*reinterpret_cast<const f32x4_any *>(p), *reinterpret_cast<const f32x4_any *>(p + 4)};
}
// The same for data that is not read again (a hint to the caches).
__device__ inline bf16x8_any load_raw_once(const __bf16 *p) {
    return __builtin_nontemporal_load(reinterpret_cast<const bf16x8_any *>(p));
}
__device__ inline raw_f32x8 load_raw_once(const float *p) {
    return {__builtin_nontemporal_load(reinterpret_cast<const f32x4_any *>(p)),
            __builtin_nontemporal_load(reinterpret_cast<const f32x4_any *>(p + 4))};
}
// A launch's threads along one axis of its grid stay below 2^32, so `blocks`
// workgroups of up to 1024 threads may take a second axis, which `block_index`
// joins again; the last ones may have nothing to do.
inline dim3 grid_of(int64_t blocks) {
    const int64_t row = int64_t{1} << 21;
    if (blocks <= row) return dim3(static_cast<unsigned>(blocks));
    return dim3(static_cast<unsigned>(row), 1, static_cast<unsigned>((blocks + row - 1) / row));
}
__device__ inline int64_t block_index() {
    return static_cast<int64_t>(blockIdx.z) * gridDim.x + blockIdx.x;
}

template <bool ONCE, typename T>
__device__ inline auto load_raw_if(const T *p) {
    if constexpr (ONCE) return load_raw_once(p);
    else return load_raw(p);
}
__device__ inline fp8::f32x8 widen(bf16x8_any v) { return __builtin_convertvector(v, fp8::f32x8); }
__device__ inline fp8::f32x8 widen(raw_f32x8 v) {
    return fp8::f32x8{v.a[0], v.a[1], v.a[2], v.a[3], v.b[0], v.b[1], v.b[2], v.b[3]};
}
__device__ inline void store_8(__bf16 *p, fp8::f32x8 v) {
    *reinterpret_cast<bf16x8_any *>(p) = __builtin_convertvector(v, fp8::bf16x8);
}
__device__ inline void store_8(float *p, fp8::f32x8 v) {
    *reinterpret_cast<f32x4_any *>(p) = f32x4_any{v[0], v[1], v[2], v[3]};
    *reinterpret_cast<f32x4_any *>(p + 4) = f32x4_any{v[4], v[5], v[6], v[7]};
}
// The same with the hint.
__device__ inline void store_8_once(__bf16 *p, fp8::f32x8 v) {
    __builtin_nontemporal_store(static_cast<bf16x8_any>(__builtin_convertvector(v, fp8::bf16x8)),
                                reinterpret_cast<bf16x8_any *>(p));
}
__device__ inline void store_8_once(float *p, fp8::f32x8 v) {
    __builtin_nontemporal_store(f32x4_any{v[0], v[1], v[2], v[3]}, reinterpret_cast<f32x4_any *>(p));
    __builtin_nontemporal_store(f32x4_any{v[4], v[5], v[6], v[7]}, reinterpret_cast<f32x4_any *>(p + 4));
}
template <bool ONCE, typename T>
__device__ inline void store_8_if(T *p, fp8::f32x8 v) {
    if constexpr (ONCE) store_8_once(p, v);
    else store_8(p, v);
}

}  // namespace hcms
