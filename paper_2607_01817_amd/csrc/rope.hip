// Rotary positions: the first R elements of every query and key head vector
// turn, pair by pair, by the (cos, sin) that the rotation table holds for the
// token's coordinates:
//   (a, b) -> (a cos - b sin, a sin + b cos)
// Pair p is the elements (2p, 2p + 1), or (p, p + R/2) in the layout of
// halves.  The inverse flag turns by the negative angle with the table's
// magnitude kept, which is the transpose and so the backward.  Elements past R
// are copied.
//
// What bounds it: bytes, once in and once out (56160 tokens of 10 heads of 128
// in bf16, row-major positions: 50 us, 5.8 TB/s; 7801 tokens of 18 heads of 64
// in fp32 15.8 us, 4.5 TB/s; a few tokens 3.5 us, which is latency).  A thread
// takes one unit (8 elements, in the layout of halves 8 and their partners) of
// one token and goes through the heads with it, so the table entries and the
// coordinates are read once for all of them.
#include "fp8.h"
#include "hcms_internal.h"

namespace hcms {
namespace {

constexpr int kAhead = 4;   // heads whose loads are in flight together

template <typename T, int V>
struct Unit;   // V elements of T in one access, as stored until they are used
template <typename T>
struct Unit<T, 1> {
    T raw;
    template <bool ONCE>
    __device__ void load(const T *p) {
        raw = *p;
    }
    __device__ void get(float (&v)[1]) const { v[0] = static_cast<float>(raw); }
    __device__ void copy(T *p) const { *p = raw; }
    static __device__ void store(T *p, const float (&v)[1]) { *p = static_cast<T>(v[0]); }
};
template <typename T>
struct Unit<T, 8> {
    decltype(load_raw(static_cast<const T *>(nullptr))) raw;
    template <bool ONCE>
    __device__ void load(const T *p) {
        raw = load_raw_if<ONCE>(p);
    }
    __device__ void get(float (&v)[8]) const {
        const fp8::f32x8 x = widen(raw);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = x[i];
    }
    __device__ void copy(T *p) const { store_8(p, widen(raw)); }
    static __device__ void store(T *p, const float (&v)[8]) {
        store_8(p, fp8::f32x8{v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]});
    }
};

// V: elements per access, 8 or 1.  Units of a head vector: the rotated ones,
// then those that are copied (V or, with V = 1, 2 elements).  ONCE: inputs past
// the caches' keeping.
template <typename T, int V, bool HALF, bool ONCE>
__global__ __launch_bounds__(256) void rope_kernel(RopeSide qs, RopeSide ks, const float *__restrict__ table,
                                                   RopeAxes ax, const void *__restrict__ positions, bool pos64,
                                                   int S, int d, int R, bool inverse, int heads_per_block) {
    constexpr int NP = HALF ? V : (V == 1 ? 1 : V / 2);   // pairs per rotated unit
    constexpr bool TWO = HALF || V == 1;                  // a unit is two accesses
    constexpr int CP = V == 1 ? 2 : V;                    // elements per copied unit
    const int turn = R / 2 / NP, units = turn + (d - R + CP - 1) / CP;
    const int per = 256 / units;                          // tokens per workgroup
    const int lt = threadIdx.x / units, u = threadIdx.x - lt * units;
    const int64_t token = block_index() * per + lt;
    if (lt >= per || token >= S) return;

    const bool rotates = u < turn;
    // First elements of the unit's two accesses.
    const int p0 = u * NP;
    const int e0 = rotates ? (HALF ? p0 : 2 * p0) : R + (u - turn) * CP;
    const int e1 = rotates ? (HALF ? p0 + R / 2 : 2 * p0 + 1) : e0 + 1;
    const bool second = TWO && (rotates || (V == 1 && e1 < d));
    const int heads = qs.H + ks.H;
    const int hb = blockIdx.y * heads_per_block, he = min(hb + heads_per_block, heads);
    // The loads of kAhead heads from h0 on, none behind a branch, which would wait
    // for those in flight: heads past the last and second accesses that there are
    // not read what is read anyway.
    Unit<T, V> a[kAhead], b[kAhead];
    const auto fetch = [&](int h0) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int h = min(h0 + k, he - 1);
            const RopeSide &side = h < qs.H ? qs : ks;
            const T *x = static_cast<const T *>(side.x) + token * side.x_token + (h < qs.H ? h : h - qs.H) * side.x_head;
            a[k].template load<ONCE>(x + e0);
            if constexpr (TWO) b[k].template load<ONCE>(x + (second ? e1 : e0));
        }
    };
    fetch(hb);   // ahead of the coordinates and the table: 8 tokens of 48 heads 3.5 us, behind them 3.8
    float c[NP], s[NP];
    if (rotates) {
        int row[kRopeMaxAxes] = {};
        bool inside = true;
        if (positions) {
            for (int a = 0; a < ax.n_axes; ++a) {
                const int64_t i = token * ax.n_axes + a;
                const int64_t at = pos64 ? static_cast<const int64_t *>(positions)[i]
                                         : static_cast<int64_t>(static_cast<const int *>(positions)[i]);
                const bool ok = at >= 0 && at < ax.grid[a];
                inside = inside && ok;
                row[a] = ax.tab_off[a] + (ok ? static_cast<int>(at) : 0) * ax.pairs[a] - ax.pair_start[a];
            }
        } else {
            int rest = static_cast<int>(token);
            for (int a = ax.n_axes - 1; a >= 0; --a) {
                const int cc = rest % ax.grid[a];
                rest /= ax.grid[a];
                row[a] = ax.tab_off[a] + cc * ax.pairs[a] - ax.pair_start[a];
            }
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int p = p0 + i;
            int at = row[0];
#pragma unroll
            for (int a = 1; a < kRopeMaxAxes; ++a)
                if (a < ax.n_axes && p >= ax.pair_start[a]) at = row[a];
            const float2 cs = reinterpret_cast<const float2 *>(table)[at + p];
            // A position outside the grid: NaN, never another position's angle.
            c[i] = inside ? cs.x : __builtin_nanf("");
            s[i] = inside ? (inverse ? -cs.y : cs.y) : __builtin_nanf("");
        }
    }
    for (int h0 = hb; h0 < he; h0 += kAhead) {
        if (h0 > hb) fetch(h0);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int h = h0 + k;
            if (h >= he) break;
            const RopeSide &side = h < qs.H ? qs : ks;
            T *y = static_cast<T *>(side.y) + token * side.y_token + (h < qs.H ? h : h - qs.H) * side.y_head;
            if (!rotates) {
                a[k].copy(y + e0);
                if (second) b[k].copy(y + e1);
                continue;
            }
            float u[V], v[V];
            a[k].get(u);
            if constexpr (TWO) b[k].get(v);
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                float &x0 = u[TWO ? i : 2 * i];
                float &x1 = TWO ? v[i] : u[2 * i + 1];
                const float u0 = x0, u1 = x1;
                x0 = __builtin_fmaf(u0, c[i], -(u1 * s[i]));
                x1 = __builtin_fmaf(u0, s[i], u1 * c[i]);
            }
            Unit<T, V>::store(y + e0, u);
            if constexpr (TWO) Unit<T, V>::store(y + e1, v);
        }
    }
}

// Rotation table from given frequencies: entry of axis a, coordinate c, pair i
// of the axis is magnitude * (cos, sin)(c * freq), computed in fp64.
__global__ __launch_bounds__(256) void rope_table_freqs_kernel(float *table, RopeAxes ax, RopeFreqs f,
                                                               double magnitude, int total) {
    const int e = blockIdx.x * 256 + threadIdx.x;
    if (e >= total) return;
    int a = 0;
    while (a + 1 < ax.n_axes && e >= ax.tab_off[a + 1]) ++a;
    const int rel = e - ax.tab_off[a];
    const double ang = static_cast<double>(rel / ax.pairs[a]) * f.f[ax.pair_start[a] + rel % ax.pairs[a]];
    table[2 * e] = static_cast<float>(magnitude * cos(ang));
    table[2 * e + 1] = static_cast<float>(magnitude * sin(ang));
}

template <typename T, int V, bool HALF>
hipError_t run_rope(const RopeSide &q, const RopeSide &k, const float *table, const RopeAxes &ax,
                    const void *positions, bool pos64, int S, int d, int R, bool inverse, hipStream_t stream) {
    constexpr int NP = HALF ? V : (V == 1 ? 1 : V / 2), CP = V == 1 ? 2 : V;
    const int units = R / 2 / NP + (d - R + CP - 1) / CP;
    if (units < 1 || units > 256) return hipErrorInvalidValue;
    const int per = 256 / units, heads = q.H + k.H;
    const int64_t blocks = (S + static_cast<int64_t>(per) - 1) / per;
    // All heads in one workgroup once the tokens alone make 1024 of them, down
    // to kAhead heads each for a few tokens.
    int split = 1;
    while (split * blocks < 1024 && (heads + split - 1) / split > kAhead) split *= 2;
    const int each = (heads + split - 1) / split;
    dim3 grid = grid_of(blocks);
    grid.y = static_cast<unsigned>((heads + each - 1) / each);
    // Inputs and outputs that the 256 MiB of last-level cache do not hold: the
    // inputs are read past it (56160 tokens of 10 heads of 128 in bf16 take 51 us
    // against 58; 7800 of them would take 11.0 against 9.8; the outputs written
    // past it too, 56).
    const bool once = V > 1 && 2 * static_cast<int64_t>(sizeof(T)) * S * heads * d > (256LL << 20);
    if (V > 1 && once)
        rope_kernel<T, V, HALF, (V > 1)><<<grid, 256, 0, stream>>>(q, k, table, ax, positions, pos64, S, d, R,
                                                                   inverse, each);
    else
        rope_kernel<T, V, HALF, false><<<grid, 256, 0, stream>>>(q, k, table, ax, positions, pos64, S, d, R,
                                                                 inverse, each);
    return hipGetLastError();
}

bool by_eight(const RopeSide &s) {
    return s.H == 0 || (s.x_token % 8 == 0 && s.x_head % 8 == 0 && s.y_token % 8 == 0 && s.y_head % 8 == 0);
}

}  // namespace

hipError_t launch_rope(const RopeSide &q, const RopeSide &k, const float *table, const RopeAxes &ax,
                       const void *positions, bool pos64, int S, int d, int R, bool half, bool inverse,
                       int dtype, hipStream_t stream) {
    if (S == 0 || q.H + k.H == 0) return hipSuccess;
    // 8 elements per access where no access crosses a boundary of the head's
    // parts; else one element.
    const bool wide = d % 8 == 0 && R % (half ? 16 : 8) == 0 && by_eight(q) && by_eight(k);
#define HCMS_RUN(T, V, HALF) return run_rope<T, V, HALF>(q, k, table, ax, positions, pos64, S, d, R, inverse, stream)
    if (dtype == 0) {
        if (wide && half) HCMS_RUN(__bf16, 8, true);
        if (wide) HCMS_RUN(__bf16, 8, false);
        if (half) HCMS_RUN(__bf16, 1, true);
        HCMS_RUN(__bf16, 1, false);
    }
    if (wide && half) HCMS_RUN(float, 8, true);
    if (wide) HCMS_RUN(float, 8, false);
    if (half) HCMS_RUN(float, 1, true);
    HCMS_RUN(float, 1, false);
#undef HCMS_RUN
}

hipError_t launch_rope_table_freqs(float *table, const RopeAxes &ax, const RopeFreqs &freqs, double magnitude,
                                   hipStream_t stream) {
    const int last = ax.n_axes - 1;
    const int total = ax.tab_off[last] + ax.grid[last] * ax.pairs[last];
    if (total == 0) return hipSuccess;
    rope_table_freqs_kernel<<<(total + 255) / 256, 256, 0, stream>>>(table, ax, freqs, magnitude, total);
    return hipGetLastError();
}

}  // namespace hcms
