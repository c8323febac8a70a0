// Norm and rotation of query and key head vectors in one pass, and its
// backward.  Per head vector x of d elements, with the side's weight w [d] and
// the rotation T of the token's position on the first R elements:
//   r = 1 / sqrt(mean(x^2) + eps),  n = x r,  y = T (n w)
// Backward, from x and the gradient dy of y:
//   g = T^t dy,  dw = sum over tokens and heads of g n,
//   u = g w,  dx = r (u - n mean(u n))
// Everything between the loads and the stores is in fp32.
//
// What bounds it: bytes; x once in and y once out, in the backward x and dy in
// and dx out.  LP lanes hold a head vector (8 elements each, in the layout of
// halves 8 and their partners), so the sums are a few steps between lanes of a
// row, and they go through a token's heads with its table entries and the
// weights in registers.  dw is kept in registers over all the tokens of a lane
// (in fp32, chains of a few terms and tokens x heads / 2048 at most), then added
// over a workgroup's lanes through LDS and over the workgroups by a second
// kernel in fp64, all in a fixed order.
//
// bf16, heads of 128: 56160 tokens of 10 heads 61 us, 4.7 TB/s of x and y; 7800 of 80
// heads 55 us, its backward 97, 4.9 TB/s, and the sum of dw 5.
#include <algorithm>

#include "fp8.h"
#include "hcms_internal.h"
#include "rope_place.h"

namespace hcms {
namespace {

constexpr int kAhead = 4;           // heads whose loads are in flight together, at least
constexpr int kMostPartials = 1024;  // workgroups of the backward

using fp8::f32x8;

// Sum over groups of LP lanes, in a fixed order; every lane gets it.
template <int LP>
__device__ inline float group_sum(float v) {
    if constexpr (LP == 64) {
        return wave_sum(v);
    } else if constexpr (LP >= 16) {
        return lanes_sum<LP>(v);
    } else {
        static_assert(LP == 8, "lanes of a head vector");
        const auto add = [](float x, int y) { return x + __builtin_bit_cast(float, y); };
        // lane 7 - i of 8, then i ^ 2 and i ^ 1 of four
        v = add(v, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x141, 0xF, 0xF, true));
        v = add(v, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x4E, 0xF, 0xF, true));
        return add(v, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0xB1, 0xF, 0xF, true));
    }
}

__device__ inline float weight_at(const void *w, bool f32, int i) {
    return f32 ? static_cast<const float *>(w)[i] : static_cast<float>(static_cast<const __bf16 *>(w)[i]);
}
__device__ inline void load_weight(float (&v)[8], const void *w, bool f32, int e) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = weight_at(w, f32, e + i);
}

// One side's heads: x in; y out, or in the backward dx, with the gradient dy of y.
struct Side {
    RopeSide heads;
    const void *dy;
    int64_t dy_token, dy_head;
    const void *w;
};
// 1 / sqrt(x) to an ulp: the hardware's with one step of Newton's, in fewer instructions
// than an exact root and division.  The hardware's takes what is below 2^-126 as 0, so that
// goes in as 2^24 x.  0 gives infinity, and infinity 0.
__device__ inline float inverse_root(float x) {
    const bool small = x < 0x1p-126f;
    const float y = small ? x * 0x1p24f : x;
    const float r = __builtin_amdgcn_rsqf(y);
    const float better = __builtin_fmaf(0.5f * r, __builtin_fmaf(-y * r, r, 1.0f), r);
    return (r > 0.0f && r < __builtin_inff() ? better : r) * (small ? 0x1p12f : 1.0f);
}

// What a launch works on.  A workgroup takes up to `each` heads of one side: the
// queries' groups of heads are counted first, then the keys'.
struct Args {
    Side q, k;
    const float *table;
    RopeAxes ax;
    const void *positions;
    bool pos64, w_f32;
    int S, d, R, each, groups;
    float eps;
};
struct Group {
    bool key;
    int hb, he;   // its heads
    __device__ Group(const Args &a, int y) {
        const int of_q = (a.q.heads.H + a.each - 1) / a.each;
        key = y >= of_q;
        hb = (key ? y - of_q : y) * a.each;
        he = min(hb + a.each, key ? a.k.heads.H : a.q.heads.H);
    }
};

// A lane's share of a head vector: 8 elements from e0 on and, where it turns
// halves, their partners from e1 on; lanes past the vector hold zeros.
template <bool HALF, int LP>
struct Share {
    bool some, turns, two;
    int e0, e1, p0;
    __device__ Share(int lane, int d, int R) {
        const int turn = R / (HALF ? 16 : 8), units = turn + (d - R) / 8;
        some = lane < units;
        turns = lane < turn;
        two = HALF && turns;
        p0 = lane * (HALF ? 8 : 4);
        e0 = !some ? 0 : turns ? lane * 8 : R + (lane - turn) * 8;
        e1 = two ? e0 + R / 2 : e0;
    }
};

// y = T x for the share (INVERSE: the transpose), in place.
template <bool HALF, bool INVERSE>
__device__ inline void turn(float (&a)[8], float (&b)[8], const float (&c)[8], const float (&s)[8]) {
#pragma unroll
    for (int i = 0; i < (HALF ? 8 : 4); ++i) {
        float &x0 = HALF ? a[i] : a[2 * i];
        float &x1 = HALF ? b[i] : a[2 * i + 1];
        const float u0 = x0, u1 = x1, si = INVERSE ? -s[i] : s[i];
        x0 = __builtin_fmaf(u0, c[i], -(u1 * si));
        x1 = __builtin_fmaf(u0, si, u1 * c[i]);
    }
}

template <bool HALF, int LP>
__device__ inline void angles(float (&c)[8], float (&s)[8], const Args &a, const Share<HALF, LP> &sh, int64_t token) {
    if (!sh.turns) return;
    const RopePlace at = rope_place(a.ax, a.positions, a.pos64, token, static_cast<int>(token));
#pragma unroll
    for (int i = 0; i < (HALF ? 8 : 4); ++i) {
        const float2 cs = rope_entry(a.table, at, sh.p0 + i);
        c[i] = cs.x;
        s[i] = cs.y;
    }
}

__device__ inline void get(float (&v)[8], f32x8 x, bool keep) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = keep ? x[i] : 0.0f;
}
template <bool ONCE, typename T>
__device__ inline void put(T *p, const float (&v)[8]) {
    store_8_if<ONCE>(p, f32x8{v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]});
}
template <bool HALF>
__device__ inline float dot(const float (&a)[8], const float (&b)[8], const float (&x)[8], const float (&y)[8]) {
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum = __builtin_fmaf(a[i], x[i], sum);
    if constexpr (HALF) {
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = __builtin_fmaf(b[i], y[i], sum);
    }
    return sum;
}

// ONCE: head vectors past the caches' keeping.  AHEAD: heads whose loads are in flight
// together.
template <typename T, bool HALF, int LP, bool ONCE, int AHEAD>
__global__ __launch_bounds__(256) void head_norm_kernel(Args a) {
    const int lane = threadIdx.x % LP;
    // The groups of a token side by side, as its heads often lie in memory.
    const int64_t id = block_index();
    const int64_t token = id / a.groups * (256 / LP) + threadIdx.x / LP;
    if (token >= a.S) return;
    const Share<HALF, LP> sh(lane, a.d, a.R);
    const Group group(a, static_cast<int>(id % a.groups));
    const Side side = group.key ? a.k : a.q;
    const T *const x = static_cast<const T *>(side.heads.x) + token * side.heads.x_token;
    T *const y = static_cast<T *>(side.heads.y) + token * side.heads.y_token;
    using Raw = decltype(load_raw(static_cast<const T *>(nullptr)));
    Raw ra[AHEAD], rb[AHEAD];
    // Loads of AHEAD heads, none behind a branch; heads past the last read it again.
    const auto fetch = [&](int h0) {
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const T *p = x + min(h0 + j, group.he - 1) * side.heads.x_head;
            ra[j] = load_raw_if<ONCE>(p + sh.e0);
            if constexpr (HALF) rb[j] = load_raw_if<ONCE>(p + sh.e1);
        }
    };
    fetch(group.hb);
    float w0[8], w1[8], c[8], s[8];
    load_weight(w0, side.w, a.w_f32, sh.e0);
    if constexpr (HALF) load_weight(w1, side.w, a.w_f32, sh.e1);
    angles<HALF, LP>(c, s, a, sh, token);
    const float of_d = 1.0f / static_cast<float>(a.d);
    for (int h0 = group.hb; h0 < group.he; h0 += AHEAD) {
        if (h0 > group.hb) fetch(h0);
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            if (h0 + j >= group.he) break;
            float u[8], v[8];
            get(u, widen(ra[j]), sh.some);
            if constexpr (HALF) get(v, widen(rb[j]), sh.two);
            const float r = inverse_root(group_sum<LP>(dot<HALF>(u, v, u, v)) * of_d + a.eps);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                u[i] = u[i] * r * w0[i];
                if constexpr (HALF) v[i] = v[i] * r * w1[i];
            }
            if (sh.turns) turn<HALF, false>(u, v, c, s);
            T *p = y + (h0 + j) * side.heads.y_head;
            if (sh.some) put<false>(p + sh.e0, u);
            if (sh.two) put<false>(p + sh.e1, v);
        }
    }
}

template <typename T, bool HALF, int LP, bool ONCE>
__global__ __launch_bounds__(256) void head_norm_backward_kernel(Args a, float *partial) {
    constexpr int PER = 256 / LP;
    __shared__ float lds[256 * 16];
    const int lane = threadIdx.x % LP, slot = threadIdx.x / LP;
    const Share<HALF, LP> sh(lane, a.d, a.R);
    const Group group(a, blockIdx.y);
    const Side side = group.key ? a.k : a.q;
    const float of_d = 1.0f / static_cast<float>(a.d);
    float w0[8], w1[8], acc0[8] = {}, acc1[8] = {};
    load_weight(w0, side.w, a.w_f32, sh.e0);
    if constexpr (HALF) load_weight(w1, side.w, a.w_f32, sh.e1);
    using Raw = decltype(load_raw(static_cast<const T *>(nullptr)));
    for (int64_t t0 = static_cast<int64_t>(blockIdx.x) * PER; t0 < a.S; t0 += static_cast<int64_t>(gridDim.x) * PER) {
        const int64_t token = t0 + slot;
        if (token >= a.S) break;
        float c[8], s[8];
        angles<HALF, LP>(c, s, a, sh, token);
        const T *x = static_cast<const T *>(side.heads.x) + token * side.heads.x_token + group.hb * side.heads.x_head;
        const T *dy = static_cast<const T *>(side.dy) + token * side.dy_token + group.hb * side.dy_head;
        T *dx = static_cast<T *>(side.heads.y) + token * side.heads.y_token + group.hb * side.heads.y_head;
        // The next head's loads ahead of this one's sums, none behind a branch: the last head
        // is read again.  (fp32 halves take two registers for each of bf16's.)
        constexpr bool AHEAD = !HALF || sizeof(T) == 2;
        Raw x0, x1, g0, g1;
        const auto fetch = [&] {
            x0 = load_raw_if<ONCE>(x + sh.e0);
            g0 = load_raw_if<ONCE>(dy + sh.e0);
            if constexpr (HALF) {
                x1 = load_raw_if<ONCE>(x + sh.e1);
                g1 = load_raw_if<ONCE>(dy + sh.e1);
            }
        };
        if (AHEAD) fetch();
        for (int h = group.hb; h < group.he; ++h, dx += side.heads.y_head) {
            if (!AHEAD) fetch();
            float u[8], v[8], du[8], dv[8];
            get(u, widen(x0), sh.some);
            get(du, widen(g0), sh.some);
            if constexpr (HALF) {
                get(v, widen(x1), sh.two);
                get(dv, widen(g1), sh.two);
            }
            if (h + 1 < group.he) {
                x += side.heads.x_head;
                dy += side.dy_head;
            }
            if (AHEAD) fetch();
            if (sh.turns) turn<HALF, true>(du, dv, c, s);
            const float r = inverse_root(group_sum<LP>(dot<HALF>(u, v, u, v)) * of_d + a.eps);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                u[i] *= r;
                acc0[i] = __builtin_fmaf(du[i], u[i], acc0[i]);
                du[i] *= w0[i];
                if constexpr (HALF) {
                    v[i] *= r;
                    acc1[i] = __builtin_fmaf(dv[i], v[i], acc1[i]);
                    dv[i] *= w1[i];
                }
            }
            const float m = group_sum<LP>(dot<HALF>(u, v, du, dv)) * of_d;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                du[i] = r * (du[i] - u[i] * m);
                if constexpr (HALF) dv[i] = r * (dv[i] - v[i] * m);
            }
            if (sh.some) put<ONCE>(dx + sh.e0, du);
            if (sh.two) put<ONCE>(dx + sh.e1, dv);
        }
    }
    // The workgroup's sums: a row of d.
    float *row = partial + (static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x) * a.d;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (sh.some) lds[slot * a.d + sh.e0 + i] = acc0[i];
        if (sh.two) lds[slot * a.d + sh.e1 + i] = acc1[i];
    }
    __syncthreads();
    for (int e = threadIdx.x; e < a.d; e += 256) {
        double sum = 0.0;   // and in sum_partials_kernel: fp32 are the lanes' own chains alone
        for (int i = 0; i < PER; ++i) sum += lds[i * a.d + e];
        row[e] = static_cast<float>(sum);
    }
}

// Head vectors of any length and stride, element by element: a wave holds one, up
// to kPairs pairs and kOthers elements that do not turn in each lane.
constexpr int kPairs = 4, kOthers = 8;
template <typename T, bool BACKWARD>
__global__ __launch_bounds__(256) void head_norm_any_kernel(Args a, bool half, float *partial) {
    __shared__ float lds[4 * 2 * kRopeMaxPairs];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int pairs = a.R / 2;
    const Group group(a, blockIdx.y);
    const Side side = group.key ? a.k : a.q;
    const float of_d = 1.0f / static_cast<float>(a.d);
    constexpr int N = 2 * kPairs + kOthers;
    // The lane's elements: pairs' first and second ones, then the others; -1: none.
    int at[N];
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
        const int p = lane + 64 * i;
        at[2 * i] = p < pairs ? (half ? p : 2 * p) : -1;
        at[2 * i + 1] = p < pairs ? (half ? p + pairs : 2 * p + 1) : -1;
    }
#pragma unroll
    for (int i = 0; i < kOthers; ++i) at[2 * kPairs + i] = a.R + lane + 64 * i < a.d ? a.R + lane + 64 * i : -1;
    float w[N], acc[N] = {};
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = at[i] < 0 ? 0.0f : weight_at(side.w, a.w_f32, at[i]);
    // Tokens and heads of the wave: the heads of a token in a row.
    const int heads = group.he - group.hb;
    const int64_t first = static_cast<int64_t>(blockIdx.x) * 4 + wave, step = static_cast<int64_t>(gridDim.x) * 4;
    const int step_h = static_cast<int>(step % heads);
    int64_t token = first / heads;
    int h = group.hb + static_cast<int>(first % heads);
    for (; token < a.S; token += step / heads + (h + step_h >= group.he), h += step_h - (h + step_h >= group.he ? heads : 0)) {
        const T *x = static_cast<const T *>(side.heads.x) + token * side.heads.x_token + h * side.heads.x_head;
        T *y = static_cast<T *>(side.heads.y) + token * side.heads.y_token + h * side.heads.y_head;
        const T *dy = static_cast<const T *>(side.dy) + token * side.dy_token + h * side.dy_head;
        const RopePlace place = rope_place(a.ax, a.positions, a.pos64, token, static_cast<int>(token));
        float u[N], du[N], sum = 0.0f;
        // Compared with 0 anew for each vector, as rope_place's pairs.
#pragma unroll
        for (int i = 0; i < N; ++i) asm volatile("" : "+v"(at[i]));
#pragma unroll
        for (int i = 0; i < N; ++i) {
            u[i] = at[i] < 0 ? 0.0f : static_cast<float>(x[at[i]]);
            if (BACKWARD) du[i] = at[i] < 0 ? 0.0f : static_cast<float>(dy[at[i]]);
            sum = __builtin_fmaf(u[i], u[i], sum);
        }
        const float r = inverse_root(wave_sum(sum) * of_d + a.eps);
#pragma unroll
        for (int i = 0; i < N; ++i) u[i] *= BACKWARD ? r : r * w[i];
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
            if (at[2 * i] < 0) continue;
            const float2 cs = rope_entry(a.table, place, lane + 64 * i);
            float &t0 = BACKWARD ? du[2 * i] : u[2 * i], &t1 = BACKWARD ? du[2 * i + 1] : u[2 * i + 1];
            const float x0 = t0, x1 = t1, s = BACKWARD ? -cs.y : cs.y;
            t0 = __builtin_fmaf(x0, cs.x, -(x1 * s));
            t1 = __builtin_fmaf(x0, s, x1 * cs.x);
        }
        if (BACKWARD) {
            float m = 0.0f;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                acc[i] = __builtin_fmaf(du[i], u[i], acc[i]);
                du[i] *= w[i];
                m = __builtin_fmaf(du[i], u[i], m);
            }
            m = wave_sum(m) * of_d;
#pragma unroll
            for (int i = 0; i < N; ++i) u[i] = r * (du[i] - u[i] * m);
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (at[i] >= 0) y[at[i]] = static_cast<T>(u[i]);
    }
    if (!BACKWARD) return;
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (at[i] >= 0) lds[wave * a.d + at[i]] = acc[i];
    __syncthreads();
    float *row = partial + (static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x) * a.d;
    for (int e = threadIdx.x; e < a.d; e += 256)
        row[e] = static_cast<float>((static_cast<double>(lds[e]) + lds[a.d + e]) +
                                    (static_cast<double>(lds[2 * a.d + e]) + lds[3 * a.d + e]));
}

// dw of both sides from the workgroups' rows of d, the queries' q_rows first: 16
// elements of a side per workgroup, 64 lanes along the rows.
__global__ __launch_bounds__(1024) void sum_partials_kernel(const float *__restrict__ partial, int q_rows, int k_rows, int d,
                                                            void *qw, void *kw, bool w_f32) {
    __shared__ double lds[64][17];
    const int col = threadIdx.x % 16, lane = threadIdx.x / 16;
    const int e = blockIdx.x * 16 + col;
    const bool key = blockIdx.y != 0;
    const int first = key ? q_rows : 0, last = first + (key ? k_rows : q_rows);
    double sum = 0.0;
    if (e < d)
        for (int r = first + lane; r < last; r += 64) sum += partial[static_cast<int64_t>(r) * d + e];
    lds[lane][col] = sum;
    __syncthreads();
    void *out = key ? kw : qw;
    if (threadIdx.x >= 16 || e >= d || !out) return;
    sum = 0.0;
    for (int i = 0; i < 64; ++i) sum += lds[i][col];
    if (w_f32) static_cast<float *>(out)[e] = static_cast<float>(sum);
    else static_cast<__bf16 *>(out)[e] = static_cast<__bf16>(static_cast<float>(sum));
}

bool by_eight(const Side &s) {
    const RopeSide &h = s.heads;
    return h.H == 0 || (h.x_token % 8 == 0 && h.x_head % 8 == 0 && h.y_token % 8 == 0 && h.y_head % 8 == 0 &&
                        s.dy_token % 8 == 0 && s.dy_head % 8 == 0);
}
// 8 elements per access where no access crosses a boundary of the head's parts.
bool by_eight(const Args &a, bool half) {
    return a.d % 8 == 0 && a.R % (half ? 16 : 8) == 0 && by_eight(a.q) && by_eight(a.k);
}

// Lanes of a head vector: a power of two from 8 on.
int lanes_of(int d, int R, bool half) {
    const int units = R / (half ? 16 : 8) + (d - R) / 8;
    return units <= 8 ? 8 : units <= 16 ? 16 : units <= 32 ? 32 : 64;
}

int groups_of(const Args &a, int each) {
    return (a.q.heads.H + each - 1) / each + (a.k.heads.H + each - 1) / each;
}
// Heads of a workgroup: all of a side once the tokens alone make 1024 workgroups,
// down to kAhead for a few tokens: a turn's loads are in flight together anyway, and
// more heads reuse the table's entries and the weights.
int heads_each(const Args &a, int64_t blocks) {
    int each = std::max(a.q.heads.H, a.k.heads.H);
    while (each > kAhead && groups_of(a, each) * blocks < 1024) each = (each + 1) / 2;
    return each;
}
// The grid of the backward, at most kMostPartials workgroups and one a head vector.
dim3 backward_grid(Args &a, int64_t blocks) {
    const int64_t x = std::min<int64_t>(blocks, kMostPartials / 2);
    a.each = heads_each(a, x);
    while (groups_of(a, a.each) > kMostPartials / x) a.each *= 2;
    return dim3(static_cast<unsigned>(x), groups_of(a, a.each));
}

template <typename T, bool HALF, int LP, bool ONCE>
hipError_t run_wide(Args &a, float *partial, dim3 *grid, hipStream_t stream) {
    const int per = 256 / LP;
    const int64_t blocks = (a.S + static_cast<int64_t>(per) - 1) / per;
    if (partial) {
        *grid = backward_grid(a, blocks);
        head_norm_backward_kernel<T, HALF, LP, ONCE><<<*grid, 256, 0, stream>>>(a, partial);
    } else {
        a.each = heads_each(a, blocks);
        a.groups = groups_of(a, a.each);
        *grid = grid_of(blocks * a.groups);
        // Four heads at a time or five, as leaves fewer of the last turn's loads for nothing (five
        // key and five query heads: 61 us for 64).
        const int n = std::min(a.each, std::max(a.q.heads.H, a.k.heads.H));
        if ((n + 3) / 4 * 4 > (n + 4) / 5 * 5) head_norm_kernel<T, HALF, LP, ONCE, 5><<<*grid, 256, 0, stream>>>(a);
        else head_norm_kernel<T, HALF, LP, ONCE, kAhead><<<*grid, 256, 0, stream>>>(a);
    }
    return hipGetLastError();
}
// Vectors that the 256 MiB of last-level cache do not hold are read past it, and what the
// backward reads for the last time, x and dy, too (56160 tokens of 10 heads of 128 64 us
// for 67; 7800 of 80, both directions, 164 for 172).
template <typename T, bool HALF, int LP>
hipError_t run_lanes(Args &a, float *partial, dim3 *grid, hipStream_t stream) {
    const int64_t bytes = static_cast<int64_t>(sizeof(T)) * a.S * (a.q.heads.H + a.k.heads.H) * a.d * (partial ? 3 : 2);
    if (bytes > int64_t{256} << 20) return run_wide<T, HALF, LP, true>(a, partial, grid, stream);
    return run_wide<T, HALF, LP, false>(a, partial, grid, stream);
}

// The forward, or the backward where `partial` is given, which writes a row for
// each workgroup of the grid.
template <typename T>
hipError_t run(Args &a, bool half, float *partial, dim3 *grid, hipStream_t stream) {
    if (by_eight(a, half)) {
        const int lanes = lanes_of(a.d, a.R, half);
#define HCMS_RUN(LP) half ? run_lanes<T, true, LP>(a, partial, grid, stream) : run_lanes<T, false, LP>(a, partial, grid, stream)
        return lanes == 8 ? HCMS_RUN(8) : lanes == 16 ? HCMS_RUN(16) : lanes == 32 ? HCMS_RUN(32) : HCMS_RUN(64);
#undef HCMS_RUN
    }
    a.each = std::max(a.q.heads.H, a.k.heads.H);
    const int64_t blocks = (static_cast<int64_t>(a.S) * a.each + 3) / 4;   // the waves go on past the grid
    *grid = dim3(static_cast<unsigned>(std::min<int64_t>(blocks, partial ? kMostPartials / 2 : 1 << 20)),
                 groups_of(a, a.each));
    if (partial) head_norm_any_kernel<T, true><<<*grid, 256, 0, stream>>>(a, half, partial);
    else head_norm_any_kernel<T, false><<<*grid, 256, 0, stream>>>(a, half, nullptr);
    return hipGetLastError();
}

}  // namespace

int head_norm_partials(int64_t S, int64_t heads) {
    return static_cast<int>(std::min<int64_t>(S * heads, kMostPartials));
}

hipError_t launch_head_norm(const RopeSide &q, const RopeSide &k, const void *qw, const void *kw, bool w_f32,
                            const float *table, const RopeAxes &ax, const void *positions, bool pos64, int S, int d,
                            int R, bool half, float eps, int dtype, hipStream_t stream) {
    if (S == 0 || q.H + k.H == 0) return hipSuccess;
    Args a{{q, nullptr, 0, 0, qw}, {k, nullptr, 0, 0, kw}, table, ax, positions, pos64, w_f32, S, d, R, 0, 0, eps};
    dim3 grid;
    return dtype == 0 ? run<__bf16>(a, half, nullptr, &grid, stream) : run<float>(a, half, nullptr, &grid, stream);
}

hipError_t launch_head_norm_backward(const RopeSide &q, const RopeSide &k, const RopeSide &dq, const RopeSide &dk,
                                     const void *qw, const void *kw, bool w_f32, void *dqw, void *dkw, float *partial,
                                     const float *table, const RopeAxes &ax, const void *positions, bool pos64, int S,
                                     int d, int R, bool half, float eps, int dtype, hipStream_t stream) {
    int q_rows = 0, k_rows = 0;
    if (S > 0 && q.H + k.H > 0) {
        const auto side = [](const RopeSide &x, const RopeSide &g, const void *w) {
            return Side{{x.x, g.y, x.x_token, x.x_head, g.y_token, g.y_head, x.H}, g.x, g.x_token, g.x_head, w};
        };
        Args a{side(q, dq, qw), side(k, dk, kw), table, ax, positions, pos64, w_f32, S, d, R, 0, 0, eps};
        dim3 grid;
        const hipError_t e = dtype == 0 ? run<__bf16>(a, half, partial, &grid, stream)
                                        : run<float>(a, half, partial, &grid, stream);
        if (e != hipSuccess) return e;
        q_rows = static_cast<int>(grid.x) * ((q.H + a.each - 1) / a.each);
        k_rows = static_cast<int>(grid.x) * ((k.H + a.each - 1) / a.each);
    }
    sum_partials_kernel<<<dim3((d + 15) / 16, 2), 1024, 0, stream>>>(partial, q_rows, k_rows, d, dqw, dkw, w_f32);
    return hipGetLastError();
}

}  // namespace hcms
