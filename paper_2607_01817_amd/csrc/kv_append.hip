// Appends keys and values to the paged 4-bit cache, the keys turned by their
// positions on the way:
//   k' = T k,  s = the smallest power of two with max |block of 32| <= 6 s,
//   codes = k' / s rounded to the nearest e2m1 value, ties to the even code.
// The rotation is in fp64 and rounded to fp32 with the lost bits kept in the last
// one, so that a value next to the border of two codes falls on its own side of it.
//
// What bounds it: bytes, k and v once in, 17 / 32 of a byte for each element out,
// and what the cache holds of them where it is asked for.  A workgroup takes the new
// tokens of a sequence in one chunk of 64 of the cache, for one head: keys are
// written as they come, values and scales are put in order in LDS.  A row's loads are
// ahead of the turn before, and of the page's place for the first.  1560 tokens of 40
// heads of 128, bf16, with the held values: 19.7 us, 3.7 TB/s (as they come
// 13.6: the rotation takes the rest); one token of 8 heads 5 us, a launch and the
// dependent loads to its place.
#include <algorithm>

#include "fp8.h"
#include "hcms_internal.h"
#include "kv_cache.h"
#include "rope_place.h"

namespace hcms {
namespace {

using fp8::f32x8;
using kv::kChunk;

// x in fp32 rounded toward zero with the last bit set if that lost something: on
// the same side as x of every value of fewer bits.  Past fp32's range: infinity.
__device__ inline float to_odd(double x) {
    const float f = static_cast<float>(x);
    if (static_cast<double>(f) == x || __builtin_isinf(f)) return f;
    unsigned b = __builtin_bit_cast(unsigned, f);
    if (__builtin_fabs(static_cast<double>(f)) > __builtin_fabs(x)) --b;
    return __builtin_bit_cast(float, b | 1u);
}

// to_odd, where that matters: borders of codes and of scales have at most three bits of
// mantissa, and x rounded to the nearest is on x's side of each but the one that it is.
// The first n elements.
__device__ inline void to_sides(const double (&w)[8], int n, float (&y)[8]) {
    unsigned least = ~0u;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) {
            y[i] = static_cast<float>(w[i]);
            least = min(least, __builtin_bit_cast(unsigned, y[i]) << 12);
        }
    if (least) return;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) y[i] = to_odd(w[i]);
}

__device__ inline unsigned max4(unsigned v) {   // over four lanes that share a scale
    v = max(v, static_cast<unsigned>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x4E, 0xF, 0xF, true)));
    return max(v, static_cast<unsigned>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0xB1, 0xF, 0xF, true)));
}

// 8 elements in 4 bits and their block's scale; called by all four lanes of a block.
struct Coded {
    unsigned bytes, scale;
};
__device__ inline Coded encode(const float (&x)[8]) {
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, fp8::magnitude(x[i]));
    Coded c;
    c.scale = kv::scale_byte(max4(top));
    const float by = fp8::inverse_scale(c.scale);
    c.bytes = 0;
    if (c.scale == 255u) return c;
#define HCMS_PAIR(i) \
    c.bytes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c.bytes, x[2 * i] * by, x[2 * i + 1] * by, 1.0f, i)
    HCMS_PAIR(0);
    HCMS_PAIR(1);
    HCMS_PAIR(2);
    HCMS_PAIR(3);
#undef HCMS_PAIR
    return c;
}
// The values that they stand for.
__device__ inline f32x8 decode(const Coded &c) {
    const float s = c.scale == 255u ? __builtin_nanf("") : __builtin_bit_cast(float, c.scale << 23);
    f32x8 v;
#define HCMS_PAIR(i) \
    { \
        const auto p = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c.bytes, 1.0f, i); \
        v[2 * i] = p[0] * s; \
        v[2 * i + 1] = p[1] * s; \
    }
    HCMS_PAIR(0)
    HCMS_PAIR(1)
    HCMS_PAIR(2)
    HCMS_PAIR(3)
#undef HCMS_PAIR
    return v;
}

// Layout of the pairs: neighbours; halves that units of 8 elements do not straddle; any
// halves.
enum Pairs { kNeighbours, kHalves, kAnyHalves };

// D: elements of a head vector; T: type of the rows.
template <typename T, int D, Pairs PAIRS>
__global__ __launch_bounds__(256) void append_kv_kernel(KvCache cache, KvBatch batch, KvRows rows, const float *table,
                                                        RopeAxes ax, const void *positions, bool pos64, int R) {
    constexpr int UNITS = D / 8, PER = 256 / UNITS;   // lanes of a token, tokens at once
    __shared__ unsigned char values[D / 2][kChunk];
    __shared__ unsigned char scales[2][D / kv::kBlock][kChunk];
    __shared__ __attribute__((aligned(16))) int places[kChunk][4];
    __shared__ bool inside[kChunk];
    __shared__ float turned[PAIRS == kAnyHalves ? 256 : 1][9];
    int b;
    int64_t before;
    kv::Sequence seq;
    const int64_t room = static_cast<int64_t>(batch.W) * cache.page;
    // Chunks that hold new tokens with a place.
    const auto chunks = [&](const kv::Sequence &s) {
        const int64_t lo = max(s.length - s.n, 0), hi = min(static_cast<int64_t>(s.length), room);
        return lo >= hi ? 0 : (hi + kChunk - 1) / kChunk - lo / kChunk;
    };
    if (!kv::find_unit(batch, rows.T, blockIdx.x, chunks, &b, &before, &seq)) return;
    b = kv::uniform(b);
    seq = {kv::uniform(seq.first), kv::uniform(seq.n), kv::uniform(seq.length)};
    const int head = blockIdx.y;
    const int lo = max(seq.length - seq.n, 0);
    const int chunk = lo / kChunk + kv::uniform(static_cast<int>(blockIdx.x - before));
    const int64_t at = static_cast<int64_t>(chunk) * kChunk;   // the chunk's first token
    const int t0 = static_cast<int>(max<int64_t>(lo - at, 0));
    const int t1 = static_cast<int>(min<int64_t>(min(static_cast<int64_t>(seq.length), room) - at, kChunk));
    const int per_page = cache.page / kChunk;
    const int page = batch.page_table[static_cast<int64_t>(b) * batch.W + chunk / per_page];
    const int u = threadIdx.x % UNITS, e = u * 8;
    // A token's rows, loaded a turn ahead, the first ones ahead of the page too.
    int t = t0 + static_cast<int>(threadIdx.x) / UNITS;
    decltype(load_raw(static_cast<const T *>(nullptr))) raw_k, raw_v;
    const auto row_of = [&](int t) { return seq.first + static_cast<int64_t>(at + t - (seq.length - seq.n)); };
    const auto fetch = [&](int t) {
        if (t >= t1) return;
        raw_k = load_raw(static_cast<const T *>(rows.k) + row_of(t) * rows.k_token + head * rows.k_head + e);
        raw_v = load_raw(static_cast<const T *>(rows.v) + row_of(t) * rows.v_token + head * rows.v_head + e);
    };
    fetch(t);
    // The places of the chunk's tokens on the grid, whose divisions each of a token's lanes
    // would do again (1560 tokens of 40 heads 21.3 us so, 19.8 from LDS).
    if (R > 0) {
        const int i = threadIdx.x;
        if (i >= t0 && i < t1) {
            const RopePlace rp = rope_place(ax, positions, pos64, row_of(i), static_cast<int>(at + i));
            places[i][0] = rp.r0;
            places[i][1] = rp.r1;
            places[i][2] = rp.r2;
            places[i][3] = rp.r3;
            inside[i] = rp.inside;
        }
        __syncthreads();
    }
    if (page < 0 || page >= cache.pages) return;   // the whole workgroup
    const int64_t block = (static_cast<int64_t>(page) * cache.heads + head) * per_page + chunk % per_page;
    unsigned char *const ck = cache.k + block * kChunk * (D / 2);
    unsigned char *const cv = cache.v + block * kChunk * (D / 2);
    unsigned char *const sk = cache.k_scale + block * kChunk * (D / kv::kBlock);
    unsigned char *const sv = cache.v_scale + block * kChunk * (D / kv::kBlock);
    // Every lane of a group of UNITS takes the same way, so those of a block stay together.
    for (; t < t1; t += PER) {
        const int64_t row = row_of(t);
        const T *k = static_cast<const T *>(rows.k) + row * rows.k_token + head * rows.k_head;
        const f32x8 xk = widen(raw_k), xv = widen(raw_v);
        if constexpr (PAIRS != kAnyHalves) fetch(t + PER);
        float y[8], z[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            y[i] = xk[i];
            z[i] = xv[i];
        }
        // Comparisons with R anew for each token, as those of rope_place.
        int turning = R;
        asm volatile("" : "+s"(turning));
        if (e < turning) {
            RopePlace rp{places[t][0], places[t][1], places[t][2], places[t][3]};
            rope_starts(ax, &rp);
            rp.inside = inside[t];
            double w[8];
            if constexpr (PAIRS == kHalves) {   // all eight are first elements of their pairs, or all second
                const bool first = e < turning / 2;
                const int p = first ? e : e - turning / 2;
                const f32x8 other = widen(load_raw(k + (first ? p + turning / 2 : p)));
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float2 cs = rope_entry(table, rp, p + i);
                    const double by = first ? -cs.y : cs.y;
                    w[i] = static_cast<double>(xk[i]) * cs.x + static_cast<double>(other[i]) * by;
                }
                to_sides(w, 8, y);
            } else if constexpr (PAIRS == kAnyHalves) {
                // One element behind the other, in LDS: unrolled, their comparisons take more
                // scalar registers than there are.
#pragma unroll
                for (int i = 0; i < 8; ++i) turned[threadIdx.x][i] = y[i];
#pragma unroll 1
                for (int i = 0; i < min(8, turning - e); ++i) {
                    const bool first = e + i < turning / 2;
                    const int p = first ? e + i : e + i - turning / 2;
                    const float2 cs = rope_entry(table, rp, p);
                    const double mine = turned[threadIdx.x][i], other = static_cast<float>(k[first ? p + turning / 2 : p]);
                    turned[threadIdx.x][i] = to_odd(mine * cs.x + other * (first ? -cs.y : cs.y));
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = turned[threadIdx.x][i];
            } else {
#pragma unroll
                for (int i = 0; i < 8; i += 2) {
                    if (e + i >= turning) continue;
                    const float2 cs = rope_entry(table, rp, (e + i) / 2);
                    const double a = xk[i], o = xk[i + 1];
                    w[i] = a * cs.x - o * cs.y;
                    w[i + 1] = a * cs.y + o * cs.x;
                }
                to_sides(w, turning - e, y);
            }
        }
        const Coded ek = encode(y), ev = encode(z);
        *reinterpret_cast<unsigned *>(ck + t * (D / 2) + e / 2) = ek.bytes;
        const int pv = kv::value_place(t);
#pragma unroll
        for (int i = 0; i < 4; ++i) values[e / 2 + i][pv] = static_cast<unsigned char>(ev.bytes >> (8 * i));
        if (u % 4 == 0) {
            scales[0][u / 4][kv::key_scale_place(t)] = static_cast<unsigned char>(ek.scale);
            scales[1][u / 4][pv] = static_cast<unsigned char>(ev.scale);
        }
        if (rows.k_held) {
            const int64_t o = (row * cache.heads + head) * D + e;
            store_8(static_cast<T *>(rows.k_held) + o, decode(ek));
            store_8(static_cast<T *>(rows.v_held) + o, decode(ev));
        }
        if constexpr (PAIRS == kAnyHalves) fetch(t + PER);
    }
    __syncthreads();
    // What the chunk's other tokens hold stays: whole chunks in 16 bytes, else byte by byte.
    if (t1 - t0 == kChunk) {
        typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
        constexpr int V16 = D / 2 * kChunk / 16, S16 = D / kv::kBlock * kChunk / 16;
        for (int i = threadIdx.x; i < V16; i += 256)
            reinterpret_cast<u32x4 *>(cv)[i] = reinterpret_cast<const u32x4 *>(&values[0][0])[i];
        for (int i = threadIdx.x; i < 2 * S16; i += 256) {
            const int side = i / S16, j = i % S16;
            reinterpret_cast<u32x4 *>(side ? sv : sk)[j] = reinterpret_cast<const u32x4 *>(&scales[side][0][0])[j];
        }
        return;
    }
    const int n = t1 - t0;
    for (int i = threadIdx.x; i < n * (D / 2); i += 256) {
        const int t = t0 + i % n, c = i / n, p = kv::value_place(t);
        cv[c * kChunk + p] = values[c][p];
    }
    for (int i = threadIdx.x; i < n * 2 * (D / kv::kBlock); i += 256) {
        const int t = t0 + i % n, j = i / n, side = j % 2, c = j / 2;
        const int p = side ? kv::value_place(t) : kv::key_scale_place(t);
        (side ? sv : sk)[c * kChunk + p] = scales[side][c][p];
    }
}

}  // namespace

hipError_t launch_append_kv(const KvCache &cache, const KvBatch &batch, const KvRows &rows, const float *table,
                            const RopeAxes &ax, const void *positions, bool pos64, int R, bool half, int dtype,
                            hipStream_t stream) {
    if (rows.T == 0 || batch.B == 0 || cache.heads == 0) return hipSuccess;
    // Chunks that n new tokens of a sequence can lie in: at most n, and n / 64 + 2.
    const int64_t tiles = std::min<int64_t>(rows.T, rows.T / kChunk + 2LL * batch.B);
    const dim3 grid(static_cast<unsigned>(tiles), cache.heads);
#define HCMS_RUN(T, D, PAIRS) \
    append_kv_kernel<T, D, PAIRS><<<grid, 256, 0, stream>>>(cache, batch, rows, table, ax, positions, pos64, R)
#define HCMS_PAIRS(T, D) \
    if (!half) HCMS_RUN(T, D, kNeighbours); \
    else if (R % 16 == 0) HCMS_RUN(T, D, kHalves); \
    else HCMS_RUN(T, D, kAnyHalves)
    if (dtype == 0 && cache.d == 128) {
        HCMS_PAIRS(__bf16, 128);
    } else if (dtype == 0) {
        HCMS_PAIRS(__bf16, 64);
    } else if (cache.d == 128) {
        HCMS_PAIRS(float, 128);
    } else {
        HCMS_PAIRS(float, 64);
    }
#undef HCMS_PAIRS
#undef HCMS_RUN
    return hipGetLastError();
}

}  // namespace hcms
