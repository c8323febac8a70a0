// The paged cache of keys and values in 4 bits (gfx950), as its kernels read and
// write it.
//
// Values are e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives), with one power
// of two for each 32 consecutive elements of a head vector, held as its exponent
// byte (e8m0): the form that v_cvt_scalef32_pk_bf16_fp4 widens, two values to two
// bf16 per instruction, exactly.  The scale of a block is the smallest power of two
// from 2^-126 on that brings its largest magnitude to at most 6; 255 (NaN) for a
// block that holds an infinity or a NaN.
//
// A page holds a multiple of 64 tokens of every head.  Keys lie token by token.
// Values lie in chunks of 64 tokens with the tokens side by side, in the order in
// which a lane of the score product holds them: the 16 x 16 tile i of a chunk's
// scores gives lane group g the tokens 16 i + 4 g + e, e < 4, and 16 g + 4 i + e is
// their place, so a lane takes its 16 tokens' values of an element pair in one
// 16-byte load and multiplies them with its probabilities without moving either.
// Two elements of one token share a byte, never two tokens, so that tokens are
// written apart from each other.
//   k        [pages][heads][page][d / 2]            element 2 c in the low half of byte c
//   k_scale  [pages][heads][page / 64][d / 32][64]  token t of a chunk at 4 (t % 16) + t / 16
//   v        [pages][heads][page / 64][d / 2][64]   token t at value_place(t)
//   v_scale  [pages][heads][page / 64][d / 32][64]  token t at value_place(t)
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "hcms_internal.h"

namespace hcms {
namespace kv {

inline constexpr int kBlock = 32;   // elements that share a scale
inline constexpr int kChunk = 64;   // tokens of a chunk

__host__ __device__ inline int key_scale_place(int t) { return 4 * (t % 16) + t / 16; }
__host__ __device__ inline int value_place(int t) { return 16 * (t / 4 % 4) + 4 * (t / 16) + t % 4; }

// Exponent byte of the scale of a block whose largest magnitude has the bits `amax`;
// 6 = 1.5 * 2^2, so the sum carries into the exponent past 1.5.
__device__ inline unsigned scale_byte(unsigned amax) {
    if (amax >= 0x7F800000u) return 255u;
    const int e = static_cast<int>((amax + 0x3FFFFFu) >> 23) - 2;
    return e < 1 ? 1u : static_cast<unsigned>(e);
}

// A sequence of a batch: rows [first, first + n) of the packed tensors, which are
// its last tokens, and `length` tokens in all.  Values that a caller must not give
// (a start outside the rows or before the last one, a length below 0 or past the
// page table) never lead outside the buffers.
struct Sequence {
    int first, n, length;
};
__device__ inline Sequence sequence(const KvBatch &batch, int b, int rows) {
    const int s0 = min(max(batch.starts[b], 0), rows);
    const int s1 = min(max(batch.starts[b + 1], s0), rows);
    return {s0, s1 - s0, max(batch.lengths[b], 0)};
}

// A value that is alike in all lanes, as a scalar.
__device__ inline int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ inline int64_t uniform(int64_t x) {
    const unsigned lo = __builtin_amdgcn_readfirstlane(static_cast<int>(x));
    return static_cast<int64_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(x >> 32))) << 32 | lo;
}

// Sums over a batch's sequences of what units(sequence, &a, &b) adds to a and b.
// Called by whole waves.
template <typename F>
__device__ inline void add_up(const KvBatch &batch, int rows, F &&units, int64_t *a, int64_t *b) {
    *a = *b = 0;
    if (batch.B == 1) return units(sequence(batch, 0, rows), a, b);
    for (int i = threadIdx.x % 64; i < batch.B; i += 64) units(sequence(batch, i, rows), a, b);
#pragma unroll
    for (int step = 1; step < 64; step *= 2) {
        *a += __shfl_xor(*a, step);
        *b += __shfl_xor(*b, step);
    }
}

// The sequence that unit `at` of a batch belongs to, and the units before it, where
// units(sequence) says how many a sequence has; false past the last.  Called by whole
// waves, all lanes with the same `at`: 64 sequences at a time.
template <typename F>
__device__ inline bool find_unit(const KvBatch &batch, int rows, int64_t at, F &&units, int *b, int64_t *before,
                                 Sequence *seq) {
    if (batch.B == 1) {
        *b = 0;
        *before = 0;
        *seq = sequence(batch, 0, rows);
        return at < units(*seq);
    }
    const int lane = threadIdx.x % 64;
    int64_t past = 0;   // units of the sequences that have been passed
    for (int base = 0; base < batch.B; base += 64) {
        const int i = base + lane;
        Sequence s{0, 0, 0};
        int64_t count = 0;
        if (i < batch.B) {
            s = sequence(batch, i, rows);
            count = units(s);
        }
        int64_t upto = past + count;
#pragma unroll
        for (int step = 1; step < 64; step *= 2) {
            const int64_t below = __shfl_up(upto - past, step);
            if (lane >= step) upto += below;
        }
        const uint64_t hits = __ballot(upto > at);
        if (hits) {
            const int hit = __ffsll(static_cast<unsigned long long>(hits)) - 1;
            *b = base + hit;
            *before = __shfl(upto - count, hit);
            *seq = {__shfl(s.first, hit), __shfl(s.n, hit), __shfl(s.length, hit)};
            return true;
        }
        past = __shfl(upto, 63);
    }
    return false;
}

}  // namespace kv
}  // namespace hcms
