// Attention over the paged 4-bit cache (kv_cache.h): for each query row, the
// cached tokens j in [begin, end) that it sees,
//   o = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale <q, k_j> - max)
// in one pass over the cache with a running maximum and sum.  A row that sees
// nothing gives zeros.
//
// The rows of a key head are its sequence's new tokens times the query heads that
// share it, in tiles of 16.  Scores are computed transposed, S^T = K Q^T, so each
// lane of the accumulator holds one row and four tokens of a 16 x 16 tile, which is
// what O^T += V^T P^T takes as its operand: probabilities never leave the lane.  The
// cache's layout gives both products' operands in 16-byte loads from global memory
// (the contraction of K Q^T runs through the elements in an order of its own), and
// widening them is one instruction for two elements, exact in bf16.
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

constexpr int kRows = 16;    // rows of a tile
constexpr int kWaves = 8;    // waves of a workgroup, each with chunks of its own
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
    int splits;       // workgroups of a tile along the tokens
    int least;        // chunks of a split, at least
    float *partial;   // of splits: [split][tile][key head][kRows][d + 2]
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

__device__ inline bool tile_at(const Args &a, int64_t at, Tile *t) {
    int tile;
    const auto tiles = [&](const kv::Sequence &s) { return (s.n * a.group + kRows - 1) / kRows; };
    if (!kv::find_tile(a.batch, a.rows.T, at, tiles, &t->b, &tile, &t->seq)) return false;
    t->row0 = tile * kRows;
    t->n = min(kRows, t->seq.n * a.group - t->row0);
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

template <typename T, int D>
__global__ __launch_bounds__(64 * kWaves) void cache_attention_kernel(Args a) {
    constexpr int NP = sizeof(T) == 2 ? 1 : 3, LD = D + 4;
    __shared__ float o_lds[kWaves][kRows][LD], m_lds[kWaves][kRows], l_lds[kWaves][kRows];
    Tile t;
    if (!tile_at(a, blockIdx.x, &t)) return;
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
        const T *qp = static_cast<const T *>(a.rows.q) + static_cast<int64_t>(t.seq.first + query) * a.rows.q_token +
                      static_cast<int64_t>(head * a.group + row % a.group) * a.rows.q_head + g * (D / 4);
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
        const int64_t slot = (static_cast<int64_t>(blockIdx.z) * gridDim.x + blockIdx.x) * gridDim.y + head;
        float *p = a.partial + (slot * kRows + out_row) * (D + 2);
#pragma unroll
        for (int e = 0; e < EACH; ++e) p[e0 + e] = o[e];
        if (e0 == 0) {
            p[D] = m;
            p[D + 1] = l;
        }
        return;
    }
    const int orow = t.row0 + out_row;
    T *out = static_cast<T *>(a.rows.out) +
             (static_cast<int64_t>(t.seq.first + orow / a.group) * a.rows.H + head * a.group + orow % a.group) * D + e0;
    const float by = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int e = 0; e < EACH; ++e) out[e] = static_cast<T>(o[e] * by);
}

// The splits of a tile in one, in their order.
template <typename T, int D>
__global__ __launch_bounds__(256) void join_splits_kernel(Args a) {
    Tile t;
    if (!tile_at(a, blockIdx.x, &t)) return;
    const int count = split_count(a, t), head = blockIdx.y;
    if (count == 1) return;
    constexpr int LANES = 256 / kRows, EACH = D / LANES;
    const int r = threadIdx.x / LANES, e0 = threadIdx.x % LANES * EACH;
    if (r >= t.n) return;
    const int64_t step = static_cast<int64_t>(gridDim.x) * gridDim.y * kRows * (D + 2);
    const float *p = a.partial + ((static_cast<int64_t>(blockIdx.x) * gridDim.y + head) * kRows + r) * (D + 2);
    float m = kNone, l = 0.0f, o[EACH] = {};
    for (int z = 0; z < count; ++z) m = fmaxf(m, p[z * step + D]);
    for (int z = 0; z < count; ++z) {
        const float by = weight_of(p[z * step + D], m, a.c);
        l = __builtin_fmaf(p[z * step + D + 1], by, l);
#pragma unroll
        for (int e = 0; e < EACH; ++e) o[e] = __builtin_fmaf(p[z * step + e0 + e], by, o[e]);
    }
    const int row = t.row0 + r;
    T *out = static_cast<T *>(a.rows.out) +
             (static_cast<int64_t>(t.seq.first + row / a.group) * a.rows.H + head * a.group + row % a.group) * D + e0;
    const float by = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int e = 0; e < EACH; ++e) out[e] = static_cast<T>(o[e] * by);
}

// Tiles of T rows of tokens in B sequences, at most.
int64_t tiles_of(const KvBatch &batch, int T, int group) {
    return static_cast<int64_t>(T) * group / kRows + std::min(batch.B, T);
}

constexpr int kLeastChunks = kWaves;   // of a split: one for each wave

int splits_of(const KvCache &cache, const KvBatch &batch, int T, int H, int window) {
    const int64_t work = tiles_of(batch, T, H / cache.heads) * cache.heads;
    int64_t chunks = static_cast<int64_t>(batch.W) * (cache.page / kChunk);
    if (window) chunks = std::min<int64_t>(chunks, (static_cast<int64_t>(window) + kRows) / kChunk + 2);
    const int64_t most = std::max<int64_t>((chunks + kLeastChunks - 1) / kLeastChunks, 1);
    return static_cast<int>(std::min<int64_t>(std::min<int64_t>((1024 + work - 1) / work, most), 256));
}

template <typename T, int D>
hipError_t run(const Args &a, int64_t tiles, hipStream_t stream) {
    const dim3 grid(static_cast<unsigned>(tiles), a.cache.heads, a.splits);
    cache_attention_kernel<T, D><<<grid, 64 * kWaves, 0, stream>>>(a);
    if (a.splits > 1) join_splits_kernel<T, D><<<dim3(grid.x, grid.y), 256, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace

int64_t cache_attention_workspace(const KvCache &cache, const KvBatch &batch, int T, int H, int window, int dtype) {
    (void)dtype;
    if (T == 0 || batch.B == 0 || H == 0) return 0;
    const int splits = splits_of(cache, batch, T, H, window);
    if (splits == 1) return 0;
    return splits * tiles_of(batch, T, H / cache.heads) * cache.heads * kRows * (cache.d + 2) * 4;
}

hipError_t launch_cache_attention(const KvCache &cache, const KvBatch &batch, const KvQueries &rows, void *workspace,
                                  int dtype, hipStream_t stream) {
    if (rows.T == 0 || batch.B == 0 || rows.H == 0) return hipSuccess;
    const int group = rows.H / cache.heads;
    // At least 2^-126, which makes exp2 of any finite score 1 as a scale of 0 does, and
    // leaves masked scores at minus infinity.
    const float c = std::max(std::fabs(rows.scale) * 1.44269504088896340736f, 1.17549435e-38f);
    const Args a{cache, batch, rows, c, group,
                 splits_of(cache, batch, rows.T, rows.H, rows.window), kLeastChunks, static_cast<float *>(workspace)};
    const int64_t tiles = tiles_of(batch, rows.T, group);
    if (dtype == 0) return cache.d == 128 ? run<__bf16, 128>(a, tiles, stream) : run<__bf16, 64>(a, tiles, stream);
    return cache.d == 128 ? run<float, 128>(a, tiles, stream) : run<float, 64>(a, tiles, stream);
}

}  // namespace hcms
