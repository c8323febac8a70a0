// Attention over the paged 4-bit cache (kv_cache.h): for each query row, the
// cached tokens j in [begin, end) that it sees,
//   o = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale <q, k_j> - max)
// in one pass over the cache with a running maximum and sum.  A row that sees
// nothing gives zeros.
//
// The rows of a key head are its sequence's new tokens times the query heads that
// share it.  Scores are computed transposed, S^T = K Q^T, so each lane of the
// accumulator holds one row and some tokens, which is what O^T += V^T P^T takes as its
// operand: probabilities never leave the lane.  Two kernels:
//   * few rows (the next tokens): tiles of 16 rows.  The cache's layout gives both
//     products' operands in 16-byte loads from global memory (the contraction of K Q^T
//     runs through the elements in an order of its own), so each wave streams chunks of
//     its own through registers, and the states of a workgroup's waves, and of workgroups
//     that share a long sequence, are joined at the end;
//   * many rows (a prompt's piece, a frame): tiles of 32 rows a wave.  A workgroup
//     widens each chunk once into LDS, in the order of the operands, and all its waves
//     read it there; a wave computes the next chunk's scores while it takes the
//     exponentials of this one's.
// Widening is one instruction for two elements, exact in bf16.
//
// fp32 rows: Q and P are taken apart into three bf16 each, whose sum is exact, and
// K and V are exact anyway, so the products are those of fp32.  bf16 rows: P is
// rounded to bf16, 2^-9 relative at most, where its sum is not.
#include <algorithm>
#include <cmath>

#include "fp8.h"
#include "hcms_internal.h"
#include "kv_cache.h"

namespace hcms {
namespace {

using kv::kChunk;

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

constexpr int kRows = 16;    // rows of a tile, and
constexpr int kWaves = 4;    // waves of a workgroup, each with chunks of its own, for few rows
constexpr int kWaveRows = 32;                                    // rows of a wave, and
// waves of a workgroup for many: two a SIMD, or one where its registers take the room
// of two (fp32 rows of 128)
template <typename T, int D>
constexpr int kPieceWaves = D == 128 && sizeof(T) == 2 ? 8 : 4;
template <typename T, int D>
constexpr int kPiecePerSimd = D == 128 && sizeof(T) == 4 ? 1 : 2;
template <typename T, int D>
constexpr int kPieceRows = kWaveRows * kPieceWaves<T, D>;
constexpr float kNone = -__builtin_inff();

// How far a row's scores may pass its running maximum before O and the sum are
// rescaled: probabilities stay below 2^8.
constexpr float kHeadroom = 8.0f;

struct Args {
    KvCache cache;
    KvBatch batch;
    KvQueries rows;
    float c;          // |scale| log2(e), above 0; the queries take its sign
    int group;        // query heads of a key head
    int from, to;     // the launch takes the sequences of [from, to] rows
    int tiles;        // at most so many tiles of them
    int splits;       // workgroups of a tile along the tokens
    int least;        // chunks of a split, at least
    float *partial;   // of splits: [split][tile][key head][rows of a tile][d + 4]
};

// A tile: rows [row0, row0 + n) of its sequence's n_new * group, and the chunks
// [c0, c1) that they see.
struct Tile {
    int b, row0, n, c0, c1;
    kv::Sequence seq;
    bool lost;   // the sequence is longer than its pages: NaN
};

__device__ inline int row_end(const Args &a, const kv::Sequence &s, int query) {
    return max(a.rows.causal ? s.length - s.n + query + 1 : s.length, 0);
}
__device__ inline int row_begin(const Args &a, int end) { return a.rows.window ? max(end - a.rows.window, 0) : 0; }

template <int ROWS>
__device__ inline bool tile_at(const Args &a, int64_t at, Tile *t) {
    int tile;
    const auto tiles = [&](const kv::Sequence &s) {
        const int rows = s.n * a.group;
        return rows < a.from || rows > a.to ? 0 : (rows + ROWS - 1) / ROWS;
    };
    if (!kv::find_tile(a.batch, a.rows.T, at, tiles, &t->b, &tile, &t->seq)) return false;
    t->row0 = tile * ROWS;
    t->n = min(ROWS, t->seq.n * a.group - t->row0);
    const int64_t room = static_cast<int64_t>(a.batch.W) * a.cache.page;
    t->lost = t->seq.length > room;
    t->c0 = row_begin(a, row_end(a, t->seq, t->row0 / a.group)) / kChunk;
    t->c1 = static_cast<int>((static_cast<int64_t>(row_end(a, t->seq, (t->row0 + t->n - 1) / a.group)) + kChunk - 1) / kChunk);
    if (t->lost) {   // any one chunk
        t->c0 = 0;
        t->c1 = 1;
    }
    return true;
}
// Chunks of a split, and how many splits have some.
__device__ inline int split_chunks(const Args &a, const Tile &t) {
    return max(a.least, (t.c1 - t.c0 + a.splits - 1) / a.splits);
}
__device__ inline int split_count(const Args &a, const Tile &t) {
    const int per = split_chunks(a, t);
    return max((t.c1 - t.c0 + per - 1) / per, 1);
}

// A chunk of one head as loaded: for 16-token tile i the lane's keys (D / 4 elements
// of token 16 i + lane % 16), and for block b of 32 elements the values of element
// pair 16 b + lane % 16 and 16 tokens.
template <int D>
struct Raw {
    using Key = std::conditional_t<D == 128, u32x4, u32x2>;
    Key k[4];
    unsigned k_scale;   // byte i: tile i
    u32x4 v[D / 32], v_scale[D / 32];
    bool bad;           // a page that there is not

    __device__ void load(const Args &a, int head, int page, int chunk, int lane) {
        const int per_page = a.cache.page / kChunk, r = lane % 16, g = lane / 16;
        bad = page < 0 || page >= a.cache.pages;
        const int64_t block = (static_cast<int64_t>(bad ? 0 : page) * a.cache.heads + head) * per_page + chunk % per_page;
        const unsigned char *kp = a.cache.k + block * kChunk * (D / 2) + r * (D / 2) + g * (D / 8);
        const unsigned char *vp = a.cache.v + block * kChunk * (D / 2) + r * kChunk + 16 * g;
        const unsigned char *sk = a.cache.k_scale + block * kChunk * (D / 32) + g * (D / 32) / 4 * kChunk + 4 * r;
        const unsigned char *sv = a.cache.v_scale + block * kChunk * (D / 32) + 16 * g;
#pragma unroll
        for (int i = 0; i < 4; ++i) k[i] = *reinterpret_cast<const Key *>(kp + i * 16 * (D / 2));
        k_scale = *reinterpret_cast<const unsigned *>(sk);
#pragma unroll
        for (int b = 0; b < D / 32; ++b) {
            v[b] = *reinterpret_cast<const u32x4 *>(vp + b * 16 * kChunk);
            v_scale[b] = *reinterpret_cast<const u32x4 *>(sv + b * kChunk);
        }
    }
};

// Byte i of x as a scale: the power of two in fp32, NaN's exponent for 255.
__device__ inline float scale_of(unsigned x, int i) {
    return __builtin_bit_cast(float, (x >> (8 * i) & 0xFFu) << 23);
}

template <int SEL>
__device__ inline unsigned widen2(unsigned x, float scale) {
    return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, SEL));
}
// 8 elements of one token.
__device__ inline bf16x8 widen8(unsigned x, float scale) {
    return __builtin_bit_cast(bf16x8, u32x4{widen2<0>(x, scale), widen2<1>(x, scale), widen2<2>(x, scale), widen2<3>(x, scale)});
}
// An element pair of four tokens (the bytes of x), their scales the bytes of s: the
// even and the odd elements.
__device__ inline void widen_tokens(unsigned x, unsigned s, unsigned (&even)[2], unsigned (&odd)[2]) {
    const unsigned p0 = widen2<0>(x, scale_of(s, 0)), p1 = widen2<1>(x, scale_of(s, 1));
    const unsigned p2 = widen2<2>(x, scale_of(s, 2)), p3 = widen2<3>(x, scale_of(s, 3));
    even[0] = __builtin_amdgcn_perm(p1, p0, 0x05040100u);
    odd[0] = __builtin_amdgcn_perm(p1, p0, 0x07060302u);
    even[1] = __builtin_amdgcn_perm(p3, p2, 0x05040100u);
    odd[1] = __builtin_amdgcn_perm(p3, p2, 0x07060302u);
}

__device__ inline f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// x as the sum of NP bf16 vectors, the largest first (exact with three).
template <int NP>
__device__ inline void take_apart(const float (&x)[8], bf16x8 (&part)[NP]) {
    float rest[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) rest[e] = x[e];
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            part[p][e] = static_cast<__bf16>(rest[e]);
            rest[e] -= static_cast<float>(part[p][e]);
        }
}

__device__ inline float over_groups(float x, bool maximum) {   // lanes l, l ^ 16, l ^ 32, l ^ 48
    const float y = __shfl_xor(x, 16);
    x = maximum ? fmaxf(x, y) : x + y;
    const float z = __shfl_xor(x, 32);
    return maximum ? fmaxf(x, z) : x + z;
}

// Bytes of x that are 253 or more: scales whose values bf16 does not hold.
__device__ inline unsigned not_finite(unsigned x) { return ((x & 0x7F7F7F7Fu) + 0x03030303u) & x & 0x80808080u; }

// What a wave knows of its rows: lane l holds row l % 16, of the accumulators the
// elements 32 b + 8 (l / 16) + 2 e + p in o[b][p][e].
template <int D>
struct State {
    float m = kNone, limit = kNone, sum = 0.0f;   // sum: of the lane's own tokens
    f32x4 o[D / 32][2] = {};
};

template <int D, int NP>
__device__ inline void attend(const Args &a, const Raw<D> &raw, const bf16x8 (&q)[D / 32][NP], State<D> &st, int token0,
                              int begin, int end, bool masked, bool lost) {
    const float c = a.c;
    f32x4 s[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float by = scale_of(raw.k_scale, i);
        s[i] = f32x4{};
#pragma unroll
        for (int j = 0; j < D / 32; ++j) {
            const bf16x8 k = widen8(raw.k[i][j], by);
#pragma unroll
            for (int p = NP - 1; p >= 0; --p) s[i] = mfma(k, q[j][p], s[i]);
        }
    }
    if (lost || raw.bad) {
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = f32x4{} + __builtin_nanf("");
    }
    if (masked) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int t = token0 + 16 * i + e;
                s[i][e] = t >= begin && t < end ? s[i][e] : kNone;
            }
    }
    float top = kNone;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) top = fmaxf(top, s[i][e]);
    if (__ballot(top > st.limit)) {
        const float m = over_groups(fmaxf(top, st.m), true);
        const float by = st.m == kNone ? 0.0f : __builtin_amdgcn_exp2f((st.m - m) * c);
        st.sum *= by;
#pragma unroll
        for (int b = 0; b < D / 32; ++b)
#pragma unroll
            for (int p = 0; p < 2; ++p) st.o[b][p] *= by;
        st.m = m;
        st.limit = m == kNone ? kNone : m + kHeadroom / c;
    }
    const float mc = st.m == kNone ? 0.0f : st.m * c;
    bf16x8 pr[2][NP];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[2 * h + e / 4][e % 4], c, -mc));
            st.sum += x[e];
        }
        take_apart<NP>(x, pr[h]);
    }
    // Where rows see different tokens of the chunk, a value that is not finite must not
    // reach those that do not see it (0 times NaN): it counts as 0 in the product and
    // makes those NaN that do.
    unsigned wrong = 0;
    if (masked) {
#pragma unroll
        for (int b = 0; b < D / 32; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) wrong |= not_finite(raw.v_scale[b][i]);
    }
    const bool repair = masked && __ballot(wrong != 0) != 0;
#pragma unroll
    for (int b = 0; b < D / 32; ++b) {
        u32x4 scale = raw.v_scale[b];
        if (repair) {
            f32x4 seen = {};
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                bf16x8 is, sees;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int i = 2 * h + e / 4, t = token0 + 16 * i + e % 4;
                    const bool bad = not_finite(scale[i]) >> (8 * (e % 4) + 7) & 1u;
                    is[e] = static_cast<__bf16>(bad ? 1.0f : 0.0f);
                    sees[e] = static_cast<__bf16>(t >= begin && t < end ? 1.0f : 0.0f);
                }
                seen = mfma(is, sees, seen);
            }
            const float add = seen[0] > 0.0f ? __builtin_nanf("") : 0.0f;   // alike for all elements of the block
            st.o[b][0] += add;
            st.o[b][1] += add;
#pragma unroll
            for (int i = 0; i < 4; ++i) scale[i] &= ~((not_finite(scale[i]) >> 7) * 0xFFu);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            unsigned even[2][2], odd[2][2];
            widen_tokens(raw.v[b][2 * h], scale[2 * h], even[0], odd[0]);
            widen_tokens(raw.v[b][2 * h + 1], scale[2 * h + 1], even[1], odd[1]);
            const bf16x8 v0 = __builtin_bit_cast(bf16x8, u32x4{even[0][0], even[0][1], even[1][0], even[1][1]});
            const bf16x8 v1 = __builtin_bit_cast(bf16x8, u32x4{odd[0][0], odd[0][1], odd[1][0], odd[1][1]});
#pragma unroll
            for (int p = NP - 1; p >= 0; --p) {
                st.o[b][0] = mfma(v0, pr[h][p], st.o[b][0]);
                st.o[b][1] = mfma(v1, pr[h][p], st.o[b][1]);
            }
        }
    }
}

// The weight of a state of maximum m in one of maximum `all`.
__device__ inline float weight_of(float m, float all, float c) {
    return m == kNone ? 0.0f : __builtin_amdgcn_exp2f((m - all) * c);
}

template <int ROWS, int D>
__device__ inline float *partial_at(const Args &a, int split, int tile, int head, int row) {
    return a.partial + (((static_cast<int64_t>(split) * a.tiles + tile) * a.cache.heads + head) * ROWS + row) * (D + 4);
}
template <typename T>
__device__ inline T *out_at(const Args &a, const Tile &t, int head, int row) {
    return static_cast<T *>(a.rows.out) +
           (static_cast<int64_t>(t.seq.first + row / a.group) * a.rows.H + head * a.group + row % a.group) * a.cache.d;
}
template <typename T>
__device__ inline const T *query_at(const Args &a, const Tile &t, int head, int row) {
    return static_cast<const T *>(a.rows.q) + static_cast<int64_t>(t.seq.first + row / a.group) * a.rows.q_token +
           static_cast<int64_t>(head * a.group + row % a.group) * a.rows.q_head;
}

template <typename T, int D>
__global__ __launch_bounds__(64 * kWaves, 2) void cache_attention_kernel(Args a) {
    constexpr int NP = sizeof(T) == 2 ? 1 : 3, LD = D + 4;
    __shared__ float o_lds[kWaves][kRows][LD], m_lds[kWaves][kRows], l_lds[kWaves][kRows];
    Tile t;
    if (!tile_at<kRows>(a, blockIdx.x, &t)) return;
    const int head = blockIdx.y, lane = threadIdx.x % 64, wave = threadIdx.x / 64, r = lane % 16, g = lane / 16;
    const int per = split_chunks(a, t), count = split_count(a, t);
    if (static_cast<int>(blockIdx.z) >= count) return;
    const int first = t.c0 + static_cast<int>(blockIdx.z) * per, last = min(first + per, t.c1);

    const int row = t.row0 + min(r, t.n - 1), query = row / a.group;
    const int end = row_end(a, t.seq, query), begin = row_begin(a, end);
    // The tokens that every row of the tile sees.
    const int all_end = row_end(a, t.seq, t.row0 / a.group);
    const int all_begin = row_begin(a, row_end(a, t.seq, (t.row0 + t.n - 1) / a.group));

    State<D> st;
    const int *const pages = a.batch.page_table + static_cast<int64_t>(t.b) * a.batch.W;
    const int per_page = a.cache.page / kChunk;
    int chunk = first + wave;
    if (chunk < last) {
        Raw<D> raw;
        raw.load(a, head, pages[chunk / per_page], chunk, lane);
        bf16x8 q[D / 32][NP];
        const T *qp = query_at<T>(a, t, head, row) + g * (D / 4);
        const float sign = a.rows.scale < 0.0f ? -1.0f : 1.0f;
#pragma unroll
        for (int j = 0; j < D / 32; ++j) {
            const fp8::f32x8 x = widen(load_raw(qp + 8 * j));
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = x[e] * sign;
            take_apart<NP>(y, q[j]);
        }
        // The next chunk's loads ahead of this one's products, where the registers hold both.
        constexpr bool AHEAD = NP == 1 || D == 64;
        while (true) {
            const int next = chunk + kWaves;
            Raw<D> ahead;
            if (AHEAD && next < last) ahead.load(a, head, pages[next / per_page], next, lane);
            const int token0 = chunk * kChunk;
            const bool masked = !t.lost && (token0 < all_begin || token0 + kChunk > all_end);
            attend<D, NP>(a, raw, q, st, token0 + 4 * g, begin, end, masked, t.lost);
            if (next >= last) break;
            if constexpr (AHEAD) raw = ahead;
            else raw.load(a, head, pages[next / per_page], next, lane);
            chunk = next;
        }
    }

    // The waves' states in one, in the order of the waves.
    const float sum = over_groups(st.sum, false);
    if (g == 0) {
        m_lds[wave][r] = st.m;
        l_lds[wave][r] = sum;
    }
#pragma unroll
    for (int b = 0; b < D / 32; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            o_lds[wave][r][32 * b + 8 * g + 2 * e] = st.o[b][0][e];
            o_lds[wave][r][32 * b + 8 * g + 2 * e + 1] = st.o[b][1][e];
        }
    __syncthreads();
    constexpr int LANES = 64 * kWaves / kRows, EACH = D / LANES;   // threads of a row, elements of each
    const int out_row = threadIdx.x / LANES, e0 = threadIdx.x % LANES * EACH;
    if (out_row >= t.n) return;
    float m = kNone, l = 0.0f, o[EACH] = {};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) m = fmaxf(m, m_lds[w][out_row]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const float by = weight_of(m_lds[w][out_row], m, a.c);
        l = __builtin_fmaf(l_lds[w][out_row], by, l);
#pragma unroll
        for (int e = 0; e < EACH; ++e) o[e] = __builtin_fmaf(o_lds[w][out_row][e0 + e], by, o[e]);
    }
    if (count > 1) {
        float *p = partial_at<kRows, D>(a, blockIdx.z, blockIdx.x, head, out_row);
#pragma unroll
        for (int e = 0; e < EACH; ++e) p[e0 + e] = o[e];
        if (e0 == 0) {
            p[D] = m;
            p[D + 1] = l;
        }
        return;
    }
    T *out = out_at<T>(a, t, head, t.row0 + out_row) + e0;
    const float by = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int e = 0; e < EACH; ++e) out[e] = static_cast<T>(o[e] * by);
}

// ---------------------------------------------------------------------------
// Many rows
// ---------------------------------------------------------------------------
typedef float f32x16 __attribute__((ext_vector_type(16)));

__device__ inline f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// A chunk in LDS: keys token by token, and values element by element with each 16
// tokens in the order in which a lane holds its probabilities (those of the lower half
// of a wave, 4 h + e and 8 + 4 h + e, then those of the upper).  Rows are padded by 16
// bytes, so that 16 rows' operands lie in different banks.
template <int D>
struct Widened {
    static constexpr int KS = D + 8, VS = kChunk + 8;
    __bf16 k[kChunk * KS];
    __bf16 v[D * VS];
    unsigned char wrong[D / 32][kChunk];   // of masked chunks: values that are not finite, taken as 0
};

// A thread's share of a chunk as loaded: half of the workgroup's waves take the keys,
// 32 elements of a token each, half the values, an element pair of 16 tokens.
template <int D>
struct Share {
    u32x4 x, scale;

    __device__ void load_keys(const Args &a, int head, int page, int chunk, int t) {
        const int per_page = a.cache.page / kChunk;
        const bool bad = page < 0 || page >= a.cache.pages;
        const int64_t block = (static_cast<int64_t>(bad ? 0 : page) * a.cache.heads + head) * per_page + chunk % per_page;
        x = *reinterpret_cast<const u32x4 *>(a.cache.k + block * kChunk * (D / 2) + 16 * t);
        const int token = t / (D / 32), b = t % (D / 32);
        scale[0] = bad ? 255u : a.cache.k_scale[(block * (D / 32) + b) * kChunk + kv::key_scale_place(token)];
    }
    __device__ void load_values(const Args &a, int head, int page, int chunk, int t) {
        const int per_page = a.cache.page / kChunk;
        const bool bad = page < 0 || page >= a.cache.pages;
        const int64_t block = (static_cast<int64_t>(bad ? 0 : page) * a.cache.heads + head) * per_page + chunk % per_page;
        const int c = t / 4, at = 16 * (t & 1) + 8 * (t >> 1 & 1);
        const unsigned char *p = a.cache.v + block * kChunk * (D / 2) + c * kChunk + at;
        const unsigned char *s = a.cache.v_scale + (block * (D / 32) + c / 16) * kChunk + at;
        const u32x2 x0 = *reinterpret_cast<const u32x2 *>(p), x1 = *reinterpret_cast<const u32x2 *>(p + 32);
        const u32x2 s0 = *reinterpret_cast<const u32x2 *>(s), s1 = *reinterpret_cast<const u32x2 *>(s + 32);
        x = u32x4{x0[0], x0[1], x1[0], x1[1]};
        scale = u32x4{s0[0], s0[1], s1[0], s1[1]};
    }
    __device__ void store_keys(Widened<D> &lds, int t) const {
        __bf16 *p = lds.k + t / (D / 32) * Widened<D>::KS + t % (D / 32) * 32;
        const float by = scale_of(scale[0], 0);
#pragma unroll
        for (int j = 0; j < 4; ++j) *reinterpret_cast<bf16x8 *>(p + 8 * j) = widen8(x[j], by);
    }
    __device__ void store_values(Widened<D> &lds, int t, bool is_masked) const {
        const int c = t / 4, h = t & 1, i0 = 2 * (t >> 1 & 1);
        u32x4 s = scale;
        if (is_masked) {
            u32x4 wrong;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                wrong[i] = not_finite(s[i]) >> 7;
                s[i] &= ~(wrong[i] * 0xFFu);
            }
            if (c % 16 == 0)
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    *reinterpret_cast<u32x2 *>(&lds.wrong[c / 16][(i0 + i) * 16 + 8 * h]) = u32x2{wrong[i], wrong[2 + i]};
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            unsigned e0[2], o0[2], e1[2], o1[2];
            widen_tokens(x[i], s[i], e0, o0);
            widen_tokens(x[2 + i], s[2 + i], e1, o1);
            __bf16 *p = lds.v + 2 * c * Widened<D>::VS + (i0 + i) * 16 + 8 * h;
            *reinterpret_cast<u32x4 *>(p) = u32x4{e0[0], e0[1], e1[0], e1[1]};
            *reinterpret_cast<u32x4 *>(p + Widened<D>::VS) = u32x4{o0[0], o0[1], o1[0], o1[1]};
        }
    }
};

// Both halves of a wave hold the same rows: x of the lower and of the upper half, in
// every lane.
__device__ inline float of_halves(float x, bool maximum) {
    const unsigned b = __builtin_bit_cast(unsigned, x);
    const auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    const float lo = __builtin_bit_cast(float, static_cast<unsigned>(r[0]));
    const float hi = __builtin_bit_cast(float, static_cast<unsigned>(r[1]));
    return maximum ? fmaxf(lo, hi) : lo + hi;
}

// Lane (li, g) of a wave: of a chunk's scores the row li and the tokens 32 mt + 8 (r / 4)
// + 4 g + r % 4 in s[mt][r], of the output the elements 32 dt + 8 (r / 4) + 4 g + r % 4
// in o[dt][r].
template <typename T, int D>
__global__ __launch_bounds__((64 * kPieceWaves<T, D>), (kPiecePerSimd<T, D>)) void cache_attention_piece_kernel(Args a) {
    constexpr int NP = sizeof(T) == 2 ? 1 : 3, WAVES = kPieceWaves<T, D>, ROWS = kPieceRows<T, D>, KK = D / 16, DT = D / 32;
    constexpr int KS = Widened<D>::KS, VS = Widened<D>::VS;
    __shared__ Widened<D> lds[2];

    // Workgroup b runs on XCD b % 8; each XCD gets a range of the launch, whose
    // neighbours are the tiles that read the same chunks.
    const int nb = gridDim.x, id = blockIdx.x, xcd = id & 7;
    int at = xcd * (nb >> 3) + min(xcd, nb & 7) + (id >> 3);
    const int tile = at % a.tiles;
    at /= a.tiles;
    const int head = at % a.cache.heads, split = at / a.cache.heads;
    Tile t;
    if (!tile_at<ROWS>(a, tile, &t)) return;
    const int per = split_chunks(a, t), count = split_count(a, t);
    if (split >= count) return;
    const int first = t.c0 + split * per, chunks = min(per, t.c1 - first);

    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, li = lane % 32, g = lane / 32;
    const bool active = wave * kWaveRows < t.n;
    // Half of the threads take keys and half values, or each takes both.
    constexpr bool BOTH = 64 * WAVES == 2 * D;
    static_assert(BOTH || 64 * WAVES == 4 * D, "2 D shares of keys and of values");
    const bool keys = wave < WAVES / 2;
    const int share = threadIdx.x % (2 * D);
    const int row = t.row0 + min(wave * kWaveRows + li, t.n - 1);
    const int end = row_end(a, t.seq, row / a.group), begin = row_begin(a, end);
    const int all_end = row_end(a, t.seq, t.row0 / a.group);
    const int all_begin = row_begin(a, row_end(a, t.seq, (t.row0 + t.n - 1) / a.group));
    const auto masked = [&](int j) {
        const int token0 = (first + j) * kChunk;
        return !t.lost && (token0 < all_begin || token0 + kChunk > all_end);
    };

    bf16x8 q[KK][NP];
    {
        const T *qp = query_at<T>(a, t, head, row) + 8 * g;
        const float sign = a.rows.scale < 0.0f ? -1.0f : 1.0f;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
            const fp8::f32x8 x = widen(load_raw(qp + 16 * kk));
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = x[e] * sign;
            take_apart<NP>(y, q[kk]);
        }
    }

    const int *const pages = a.batch.page_table + static_cast<int64_t>(t.b) * a.batch.W;
    const int per_page = a.cache.page / kChunk;
    Share<D> of_keys, of_values;
    const auto page_of = [&](int j) { return t.lost ? -1 : pages[(first + min(j, chunks - 1)) / per_page]; };
    int page = page_of(0);
    const auto load = [&](int j) {   // chunk j's share (past the last one, that again) and the next one's page
        const int chunk = first + min(j, chunks - 1), at = page;
        page = page_of(j + 1);
        if (BOTH || keys) of_keys.load_keys(a, head, at, chunk, share);
        if (BOTH || !keys) (BOTH ? of_values : of_keys).load_values(a, head, at, chunk, share);
    };
    const auto store = [&](int j) {
        if (BOTH || keys) of_keys.store_keys(lds[j & 1], share);
        if (BOTH || !keys) (BOTH ? of_values : of_keys).store_values(lds[j & 1], share, masked(j));
    };

    const float c = a.c;
    float m = kNone, mc = 0.0f, sum = 0.0f;
    f32x16 o[DT] = {};
    load(0);
    store(0);
    load(1);
    __syncthreads();
    for (int j = 0; j < chunks; ++j) {
        const Widened<D> &buf = lds[j & 1];
        if (j + 1 < chunks) {
            store(j + 1);
            load(j + 2);
        }
        if (active) {
            f32x16 s[2] = {};
#pragma unroll
            for (int kk = 0; kk < KK; ++kk)
#pragma unroll
                for (int mt = 0; mt < 2; ++mt) {
                    const bf16x8 k = *reinterpret_cast<const bf16x8 *>(buf.k + (32 * mt + li) * KS + 16 * kk + 8 * g);
#pragma unroll
                    for (int p = NP - 1; p >= 0; --p) s[mt] = mfma32(k, q[kk][p], s[mt]);
                }
            const bool mask = masked(j);
            const int token0 = (first + j) * kChunk + 4 * g;
            if (mask) {
#pragma unroll
                for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int token = token0 + 32 * mt + 8 * (r / 4) + r % 4;
                        s[mt][r] = token >= begin && token < end ? s[mt][r] : kNone;
                    }
            }
            float top = kNone;
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, fmaxf(s[0][r], s[1][r]));
            if (__ballot(m == kNone ? top > kNone : (top - m) * c > kHeadroom)) {
                const float up = of_halves(fmaxf(top, m), true);
                const float by = m == kNone ? 0.0f : __builtin_amdgcn_exp2f((m - up) * c);
                sum *= by;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) o[dt] *= by;
                m = up;
                mc = m == kNone ? 0.0f : m * c;
            }
            bf16x8 pr[4][NP];
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) {
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    x[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[ks / 2][8 * (ks % 2) + e], c, -mc));
                    sum += x[e];
                }
                take_apart<NP>(x, pr[ks]);
            }
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    const bf16x8 v = *reinterpret_cast<const bf16x8 *>(buf.v + (32 * dt + li) * VS + 16 * ks + 8 * g);
#pragma unroll
                    for (int p = NP - 1; p >= 0; --p) o[dt] = mfma32(v, pr[ks][p], o[dt]);
                }
            if (mask) {
                // As in attend: values that are not finite make the rows NaN that see them.
                unsigned any = 0;
                if (lane < D / 32 * kChunk / 4) any = reinterpret_cast<const unsigned *>(&buf.wrong[0][0])[lane];
                if (__ballot(any != 0)) {
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) {
                        f32x16 seen = {};
#pragma unroll
                        for (int ks = 0; ks < 4; ++ks) {
                            bf16x8 is, sees;
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                const int token = token0 + 16 * ks + 8 * (e / 4) + e % 4;
                                is[e] = static_cast<__bf16>(buf.wrong[dt][16 * ks + 8 * g + e] ? 1.0f : 0.0f);
                                sees[e] = static_cast<__bf16>(token >= begin && token < end ? 1.0f : 0.0f);
                            }
                            seen = mfma32(is, sees, seen);
                        }
                        o[dt] += seen[0] > 0.0f ? __builtin_nanf("") : 0.0f;
                    }
                }
            }
        }
        __syncthreads();
    }

    if (wave * kWaveRows + li >= t.n) return;
    sum = of_halves(sum, false);
    if (count > 1) {
        float *p = partial_at<ROWS, D>(a, split, tile, head, wave * kWaveRows + li);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int r = 0; r < 16; ++r) p[32 * dt + 8 * (r / 4) + 4 * g + r % 4] = o[dt][r];
        if (g == 0) {
            p[D] = m;
            p[D + 1] = sum;
        }
        return;
    }
    T *out = out_at<T>(a, t, head, row);
    const float by = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) out[32 * dt + 8 * (r / 4) + 4 * g + r % 4] = static_cast<T>(o[dt][r] * by);
}

// ---------------------------------------------------------------------------
// The splits of a tile in one, in a fixed order
// ---------------------------------------------------------------------------
// A row's state over the splits z, z + by, ..., EACH elements of it from p on; `ahead`
// splits' loads are in flight together.
template <int EACH>
struct Joined {
    float m = kNone, l = 0.0f, o[EACH] = {};

    // p: the element of split 0, ml: its maximum and sum, `step` floats from split to split.
    __device__ void add(const float *p, const float *ml, int64_t step, int z, int by, int count, float c) {
        constexpr int AHEAD = 8;
        for (; z < count; z += AHEAD * by) {
            float pm[AHEAD], pl[AHEAD], po[AHEAD][EACH], up = m;
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const int64_t at = min(z + i * by, count - 1) * step;
                pm[i] = z + i * by < count ? ml[at] : kNone;
                pl[i] = ml[at + 1];
#pragma unroll
                for (int e = 0; e < EACH; ++e) po[i][e] = p[at + e];
            }
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) up = fmaxf(up, pm[i]);
            scale(weight_of(m, up, c));
            m = up;
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                if (z + i * by >= count) break;
                const float w = weight_of(pm[i], up, c);
                l = __builtin_fmaf(pl[i], w, l);
#pragma unroll
                for (int e = 0; e < EACH; ++e) o[e] = __builtin_fmaf(po[i][e], w, o[e]);
            }
        }
    }
    __device__ void scale(float by) {
        l *= by;
#pragma unroll
        for (int e = 0; e < EACH; ++e) o[e] *= by;
    }
};

// Few splits: 16 lanes a row, 16 rows a workgroup.  Many (WIDE): a workgroup a row, its
// waves every fourth split each.
template <typename T, int D, int ROWS, bool WIDE>
__global__ __launch_bounds__(256) void join_splits_kernel(Args a) {
    constexpr int PER = WIDE ? 1 : 16, LANES = WIDE ? 64 : 16, EACH = D / LANES;   // rows, lanes of one, their elements
    const int tile = blockIdx.x / (ROWS / PER), head = blockIdx.y;
    Tile t;
    if (!tile_at<ROWS>(a, tile, &t)) return;
    const int count = split_count(a, t);
    const int r = blockIdx.x % (ROWS / PER) * PER + (WIDE ? 0 : threadIdx.x / LANES);
    if (count == 1 || r >= t.n) return;
    const int e0 = threadIdx.x % LANES * EACH;
    const float *const row = partial_at<ROWS, D>(a, 0, tile, head, r);
    const int64_t step = partial_at<ROWS, D>(a, 1, tile, head, r) - row;
    Joined<EACH> j;
    if constexpr (!WIDE) {
        j.add(row + e0, row + D, step, 0, 1, count, a.c);
        T *out = out_at<T>(a, t, head, t.row0 + r) + e0;
        const float by = j.l == 0.0f ? 0.0f : 1.0f / j.l;
#pragma unroll
        for (int e = 0; e < EACH; ++e) out[e] = static_cast<T>(j.o[e] * by);
    } else {
        __shared__ float o_lds[4][D], ml_lds[4][2];
        const int wave = threadIdx.x / 64;
        j.add(row + e0, row + D, step, wave, 4, count, a.c);
#pragma unroll
        for (int e = 0; e < EACH; ++e) o_lds[wave][e0 + e] = j.o[e];
        if (e0 == 0) {
            ml_lds[wave][0] = j.m;
            ml_lds[wave][1] = j.l;
        }
        __syncthreads();
        if (threadIdx.x >= D) return;
        float all = kNone, sum = 0.0f, x = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) all = fmaxf(all, ml_lds[w][0]);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float by = weight_of(ml_lds[w][0], all, a.c);
            sum = __builtin_fmaf(ml_lds[w][1], by, sum);
            x = __builtin_fmaf(o_lds[w][threadIdx.x], by, x);
        }
        out_at<T>(a, t, head, t.row0 + r)[threadIdx.x] = static_cast<T>(sum == 0.0f ? 0.0f : x / sum);
    }
}

// ---------------------------------------------------------------------------
// What is launched
// ---------------------------------------------------------------------------
// Sequences of more rows than this are taken by the kernel for many, where there are
// both kinds.
constexpr int kFewRows = 32;

// What writing a tile's partial state and reading it again costs, in chunks.
constexpr int kStateChunks = 7;
#ifndef FEW_TARGET
#define FEW_TARGET 1024
#endif

// A launch over the sequences of [from, to] rows.
struct Launch {
    int from = 1, to = 0, tiles = 0, splits = 1, least = 1;
    bool some() const { return from <= to; }
    int64_t partial(const KvCache &cache, int rows) const {
        return some() && splits > 1
                   ? static_cast<int64_t>(splits) * tiles * cache.heads * rows * (cache.d + 4) : 0;
    }
};
struct Plan {
    Launch few, many;
};

int piece_rows(int d, int dtype) { return d == 128 && dtype == 0 ? kPieceRows<__bf16, 128> : kPieceRows<float, 64>; }
static_assert(kPieceRows<float, 128> == kPieceRows<float, 64> && kPieceRows<__bf16, 64> == kPieceRows<float, 64>, "piece_rows");

Plan plan_of(const KvCache &cache, const KvBatch &batch, int T, int H, int window, int dtype) {
    Plan p;
    const int group = H / cache.heads, most = std::min(batch.B, T);
    const int64_t rows = static_cast<int64_t>(T) * group;
    const bool pieces = rows > static_cast<int64_t>(kFewRows) * batch.B;
    const int64_t cached = static_cast<int64_t>(batch.W) * (cache.page / kChunk);
    const auto chunks = [&](int tile_rows) {   // that a tile sees, at most
        return window ? std::min<int64_t>(cached, (static_cast<int64_t>(window) + tile_rows / group) / kChunk + 2) : cached;
    };
    if (!pieces || batch.B > 1) {
        Launch &f = p.few;
        f.to = pieces ? kFewRows : INT32_MAX;
        f.tiles = static_cast<int>(pieces ? std::min<int64_t>(rows, most * static_cast<int64_t>(kFewRows / kRows))
                                          : (rows + static_cast<int64_t>(most) * (kRows - 1)) / kRows);
        f.least = 2 * kWaves;
        const int64_t work = static_cast<int64_t>(f.tiles) * cache.heads;
        f.splits = static_cast<int>(std::min<int64_t>(
            {(FEW_TARGET + work - 1) / work, std::max<int64_t>((chunks(kRows) + f.least - 1) / f.least, 1), 256}));
    }
    if (pieces) {
        Launch &m = p.many;
        const int each = piece_rows(cache.d, dtype);
        m.from = batch.B > 1 ? kFewRows + 1 : 1;
        m.to = INT32_MAX;
        const int64_t seqs = std::min<int64_t>(most, rows / m.from);
        m.tiles = static_cast<int>((rows + seqs * (each - 1)) / each);
        m.least = 8;
        // Splits by the time they take in chunks: the rounds of workgroups on 256 CUs (of
        // sequences of equal rows), each as long as its chunks and, with splits, the
        // states that it writes and that are read again.
        const int64_t tiles = batch.B * ((rows / batch.B + each - 1) / each) * cache.heads, n = chunks(each);
        const int64_t at_once = 256 * (cache.d == 128 ? 1 : 2);
        int64_t best = 0;
        for (int64_t z = 1; z <= 32 && (z == 1 || z * m.least <= n); ++z) {
            const int64_t cost = (tiles * z + at_once - 1) / at_once * ((n + z - 1) / z + (z > 1 ? kStateChunks : 0));
            if (z == 1 || cost < best) {
                best = cost;
                m.splits = static_cast<int>(z);
            }
        }
    }
    return p;
}

Args with(Args a, const Launch &l, float *partial) {
    a.from = l.from;
    a.to = l.to;
    a.tiles = l.tiles;
    a.splits = l.splits;
    a.least = l.least;
    a.partial = partial;
    return a;
}

template <typename T, int D, int ROWS>
void join(const Args &a, hipStream_t stream) {
    if (a.splits == 1) return;
    const dim3 rows(static_cast<unsigned>(a.tiles) * ROWS, a.cache.heads);
    if (a.splits > 8) join_splits_kernel<T, D, ROWS, true><<<rows, 256, 0, stream>>>(a);
    else join_splits_kernel<T, D, ROWS, false><<<dim3(rows.x / 16, rows.y), 256, 0, stream>>>(a);
}

template <typename T, int D>
hipError_t run(const Args &args, const Plan &p, float *workspace, hipStream_t stream) {
    const unsigned heads = args.cache.heads;
    if (p.few.some()) {
        const Args a = with(args, p.few, workspace);
        cache_attention_kernel<T, D><<<dim3(a.tiles, heads, a.splits), 64 * kWaves, 0, stream>>>(a);
        join<T, D, kRows>(a, stream);
    }
    if (p.many.some()) {
        const Args a = with(args, p.many, workspace + p.few.partial(args.cache, kRows));
        cache_attention_piece_kernel<T, D><<<static_cast<unsigned>(a.tiles) * heads * a.splits, (64 * kPieceWaves<T, D>), 0,
                                             stream>>>(a);
        join<T, D, kPieceRows<T, D>>(a, stream);
    }
    return hipGetLastError();
}

}  // namespace

int64_t cache_attention_workspace(const KvCache &cache, const KvBatch &batch, int T, int H, int window, int dtype) {
    if (T == 0 || batch.B == 0 || H == 0) return 0;
    const Plan p = plan_of(cache, batch, T, H, window, dtype);
    return 4 * (p.few.partial(cache, kRows) + p.many.partial(cache, piece_rows(cache.d, dtype)));
}

hipError_t launch_cache_attention(const KvCache &cache, const KvBatch &batch, const KvQueries &rows, void *workspace,
                                  int dtype, hipStream_t stream) {
    if (rows.T == 0 || batch.B == 0 || rows.H == 0) return hipSuccess;
    // At least 2^-126, which makes exp2 of any finite score 1 as a scale of 0 does, and
    // leaves masked scores at minus infinity.
    const float c = std::max(std::fabs(rows.scale) * 1.44269504088896340736f, 1.17549435e-38f);
    const Args a{cache, batch, rows, c, rows.H / cache.heads, 0, 0, 0, 0, 0, nullptr};
    const Plan p = plan_of(cache, batch, rows.T, rows.H, rows.window, dtype);
    float *w = static_cast<float *>(workspace);
    if (dtype == 0) return cache.d == 128 ? run<__bf16, 128>(a, p, w, stream) : run<__bf16, 64>(a, p, w, stream);
    return cache.d == 128 ? run<float, 128>(a, p, w, stream) : run<float, 64>(a, p, w, stream);
}

}  // namespace hcms
