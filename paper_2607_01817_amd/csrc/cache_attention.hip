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
//   * few rows (the next tokens; bounded by the cache's bytes): tiles of 16 rows.  The cache's layout gives both
//     products' operands in 16-byte loads from global memory (the contraction of K Q^T
//     runs through the elements in an order of its own), so each wave streams chunks of
//     its own through registers, and the states of a workgroup's waves, and of workgroups
//     that share a long sequence, are joined at the end.  bf16, 8 key heads of 128 shared
//     by five: 64 next tokens, sequences of up to 8192 tokens 64 us (286 MB, 4.5 TB/s), two
//     of 131072 58 us (4.9 TB/s), one of 1001 11 us, a launch, the search for its place
//     and loads that depend on each other;
//   * many rows (a prompt's piece, a frame; bounded by the matrix units, whose LDS reads
//     and exponentials take as long and overlap in part): tiles of 32 rows a wave.  A
//     workgroup widens each chunk once into LDS, in the order of the operands, and all its
//     waves read it there.  bf16, 128: 2 x 2048 rows of 40 heads over 16384 tokens 1212 to
//     1294 us in all, by card (1.06 to 1.00 PFLOP/s), 1560 of 5 heads over 56160 254 to 265
//     (0.89 to 0.85: the last of 7 tiles has 24 of 256 rows); fp32, 1024 of 64 heads on 8
//     key heads over 9216 872 us (1.0 PFLOP/s of the three products).
// Widening is one instruction for two elements, exact in bf16.
//
// fp32 rows: Q and P are taken apart into three bf16 each, whose sum is exact, and
// K and V are exact anyway, so the products are those of fp32.  bf16 rows: P is
// rounded to bf16, 2^-8 relative at most, where its sum is not.  That takes the output's
// error in norm from the 1.66e-3 of its own rounding to 2.1e-3 to 2.35e-3; P in two parts,
// which would save that, takes a third longer with many rows (1225 -> 1685 us, 254 -> 335)
// and 2 to 12 % with few (one next token of 64 sequences 81.6 -> 83.3, 8 next tokens of 16
// sequences of 8192 101 -> 110, a prompt of 64 behind 8192 52 -> 59).  fp16 would hold
// three bits more, but not those of probabilities below 2^-21 of the largest, which are all
// that an element has whose other tokens' values are 0.
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
constexpr int kWaves = 4;    // waves of a workgroup, for few rows
constexpr int kTeamWaves = 8;   // where they work at the same part
constexpr int kTeamChunks = 4 * kTeamWaves;     // up to which they take a whole tile
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
constexpr float kMostSum = 256.0f;   // 2^kHeadroom, of a chunk's probabilities together
// A probability's power of two is one multiply-add of its score, c score - c maximum, where
// the maximum's product, rounded first, is up to this: off by 2^-13 at most.  Rows whose
// maximum lies farther out take c (score - maximum), as that rounding would soon be all
// there is.
constexpr float kFar = 4096.0f;

struct Args {
    KvCache cache;
    KvBatch batch;
    KvQueries rows;
    float c;          // |scale| log2(e), above 0; the queries take its sign
    int group;        // query heads of a key head
    int from, to;     // the launch takes the sequences of [from, to] rows
    int groups;       // workgroups
    int least;        // chunks of a workgroup, at least, but where there are more tiles
    bool whole;       // a group a tile
    struct Begun *begun;   // [groups]
    float *partial;        // [2 groups][rows of a tile][d + 4]: states of parts of tiles
};

// The tile that a workgroup begins and others end: how many workgroups work at it (0:
// none is begun), its key head, its first row and their number in the sequence, and the
// sequence's first row.
struct Begun {
    int parts, head, row0, n, first;
};

// The division of a launch's work.  A tile is some rows of a sequence and key head and
// weighs as many chunks as they see.  All tiles lie one behind the other,
// the tiles of a sequence and head in a row, sequence by sequence, head by head, and each
// workgroup takes an equal piece of that line: the end of one tile, whole ones, and the
// beginning of another.  Lengths are read here, so the pieces are equal whatever the
// sequences are.  Parts of tiles leave their states in `partial`, two for a workgroup.
//
// The weights of a sequence's tiles are taken to rise evenly from the first one's chunks
// to the last one's, so that those before tile k are known at once; a part of a tile is
// that part of the chunks that it has.
__device__ inline int row_end(const Args &a, const kv::Sequence &s, int query) {
    return max(a.rows.causal ? s.length - s.n + query + 1 : s.length, 0);
}
__device__ inline int row_begin(const Args &a, int end) { return a.rows.window ? max(end - a.rows.window, 0) : 0; }

// A tile: rows [row0, row0 + n) of its sequence's, and the chunks [c0, c1) that they see.
struct Tile {
    int row0, n, c0, c1;
    bool lost;   // the sequence is longer than its pages: NaN
};
template <int ROWS>
__device__ inline Tile tile_of(const Args &a, const kv::Sequence &s, int k) {
    Tile t;
    t.row0 = k * ROWS;
    t.n = min(ROWS, s.n * a.group - t.row0);
    t.lost = s.length > static_cast<int64_t>(a.batch.W) * a.cache.page;
    t.c0 = t.lost ? 0 : row_begin(a, row_end(a, s, t.row0 / a.group)) / kChunk;
    const int64_t end = row_end(a, s, (t.row0 + t.n - 1) / a.group);
    t.c1 = t.lost ? 1 : max(static_cast<int>((end + kChunk - 1) / kChunk), t.c0);   // lost: any one chunk
    return t;
}

// The tiles of a sequence: how many, and the weights of the first and last.  Divisions
// are in fp64, a tenth of the instructions of those of 64-bit integers: their operands
// are whole numbers below 2^53, and what they give grows with k as it has to.
template <int ROWS>
struct Tiles {
    int count = 0, first = 0;
    double rise = 0.0;   // of a weight, half of it from tile to tile
    __device__ Tiles(const Args &a, const kv::Sequence &s) {
        const int rows = s.n * a.group;
        if (rows < a.from || rows > a.to) return;
        count = (rows + ROWS - 1) / ROWS;
        const Tile x = tile_of<ROWS>(a, s, 0), y = tile_of<ROWS>(a, s, count - 1);
        first = max(x.c1 - x.c0, 1);
        rise = count < 2 ? 0.0 : static_cast<double>(max(y.c1 - y.c0 - first, 0)) / (2.0 * (count - 1));
    }
    // Weights of the tiles before tile k.
    __device__ int64_t before(int k) const {
        return static_cast<int64_t>(k) * first + static_cast<int64_t>(rise * (static_cast<double>(k) * (k - 1)));
    }
    __device__ int64_t all() const { return before(count); }
    // The tile of unit `at` of them.
    __device__ int find(int64_t at) const {
        int lo = 0, hi = count - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) / 2;
            if (before(mid) <= at) lo = mid;
            else hi = mid - 1;
        }
        return lo;
    }
};

// All of a launch's work: units of a head, and what the workgroups share them by.
template <int ROWS>
struct Work {
    int64_t head, all;
    int groups;    // that have some
    double each;   // units of a group
    Work() = default;
    __device__ explicit Work(const Args &a) {
        int64_t tiles;
        kv::add_up(a.batch, a.rows.T, [&](const kv::Sequence &s, int64_t *units, int64_t *tiles) {
            const Tiles<ROWS> t(a, s);
            *units += t.all();
            *tiles += t.count;
        }, &head, &tiles);
        all = head * a.cache.heads;
        tiles *= a.cache.heads;
        // Groups of at least so many units, or a whole number of groups to a tile, where a
        // group then has at most as many units more as it has at least, or, of many rows, not
        // half as many: parts of tiles alike begin and end with groups, and a group's second
        // part costs about those units (12 sequences of 8 key heads of 128: 3840 tokens 25.7 us
        // in equal pieces and 22.8 in two groups a tile, 32768 92 and 102; of 5 heads 1560 rows
        // over 32768 203 and 189, 1536 184 and 204).  Many rows, bf16 and fp32, of 64 and 128,
        // in 11 forms: at most 4 % slower than in equal pieces always, and than with 1.0, which
        // takes up to 17 % longer (1536 rows of 5 heads over 32768 217 us for 185).
        constexpr double MORE = ROWS > kRows ? 0.45 : 1.0;
        const double room = a.groups, some = static_cast<double>(tiles), units = static_cast<double>(all);
        const double fit = min(units / a.least, room), even = some * floor(fit / some);
        const bool whole_number = even > 0.0 && units / even - units / fit <= a.least * MORE;
        groups = static_cast<int>(whole_number ? even : min(max(some, fit), room));
        each = static_cast<double>(all) / max(groups, 1);
    }
    // Rounded up a little, so that a whole number of groups to a tile ends with the tile.
    __device__ int64_t begin(int group) const {
        return group < groups ? static_cast<int64_t>(__builtin_fma(static_cast<double>(group), each, 0x1p-20)) : all;
    }
    // The workgroup of a unit.
    __device__ int group_of(int64_t unit) const {
        int g = min(static_cast<int>(static_cast<double>(unit) / each), groups - 1);
        while (begin(g + 1) <= unit) ++g;
        while (begin(g) > unit) --g;
        return g;
    }
};

// A part of a tile: its place, and its part [u0, u1) of the tile's weight.
template <int ROWS>
struct Piece;
template <int ROWS>
struct Part {
    int b, k, head;
    kv::Sequence seq;
    int u0, u1, weight;
    // Where a group takes a tile: the heads of a tile in a row; false past the last tile.
    __device__ bool whole_tile(const Args &a, int group) {
        const int unit = group / a.cache.heads;
        int64_t before = 0;
        if (!kv::find_unit(a.batch, a.rows.T, unit, [&](const kv::Sequence &s) {
                const int rows = s.n * a.group;
                return static_cast<int64_t>(rows < a.from || rows > a.to ? 0 : (rows + ROWS - 1) / ROWS);
            }, &b, &before, &seq))
            return false;
        head = group % a.cache.heads;
        k = unit - static_cast<int>(before);
        u0 = 0;
        u1 = weight = 1;
        return true;
    }
    Part() = default;
    // The part that begins at unit `at` of a line of `of_head` units a head, and ends
    // with its tile or at `end`.
    __device__ Part(const Args &a, int64_t of_head, int64_t at, int64_t end) {
        head = static_cast<int>(static_cast<double>(at) / static_cast<double>(of_head));   // exact below 2^53
        int64_t before = 0;
        kv::find_unit(a.batch, a.rows.T, at - head * of_head, [&](const kv::Sequence &s) { return Tiles<ROWS>(a, s).all(); },
                      &b, &before, &seq);
        const Tiles<ROWS> t(a, seq);
        const int64_t in = at - head * of_head - before;
        k = t.find(in);
        const int64_t first = t.before(k);
        weight = static_cast<int>(t.before(k + 1) - first);
        u0 = static_cast<int>(in - first);
        u1 = static_cast<int>(min(static_cast<int64_t>(weight), u0 + (end - at)));
    }
    // What is alike in all lanes, but reckoned in vector registers, as scalar ones are few.
    __device__ void settle() {
        head = kv::uniform(head);
        b = kv::uniform(b);
        k = kv::uniform(k);
        seq = {kv::uniform(seq.first), kv::uniform(seq.n), kv::uniform(seq.length)};
        weight = kv::uniform(weight);
        u0 = kv::uniform(u0);
        u1 = kv::uniform(u1);
    }
    __device__ bool whole() const { return u0 == 0 && u1 == weight; }
    // Its chunks.
    __device__ int chunk(const Tile &t, int u) const {
        return t.c0 + static_cast<int>(static_cast<double>(t.c1 - t.c0) * u / weight);   // all of them for all of it
    }
    // Where its state goes: a workgroup's first part that begins inside a tile, or its last.
    __device__ int slot(const Piece<ROWS> &piece) const;
};

// A workgroup's piece of the line, in LDS between its parts, where it takes no registers.
template <int ROWS>
struct Piece {
    Work<ROWS> work;
    int64_t at, end;
    int group;
};
// The kernel's arguments (its only parameter, so they lie first in its argument
// segment), read anew for each part: they, and what is made of them (a division's
// factors, strides in bytes), kept over all parts would take more scalar registers than
// there are.
__device__ inline Args arguments() {
    typedef const __attribute__((address_space(4))) unsigned Word;
    struct Words {
        unsigned w[sizeof(Args) / 4];
    } words;
    static_assert(sizeof(Args) % 4 == 0, "whole words");
    Word *p = (Word *)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
#pragma unroll
    for (unsigned i = 0; i < sizeof(Args) / 4; ++i) words.w[i] = p[i];
    return __builtin_bit_cast(Args, words);
}
template <int ROWS>
__device__ inline int Part<ROWS>::slot(const Piece<ROWS> &piece) const { return 2 * piece.group + (u0 == 0 ? 1 : 0); }

// Calls each(arguments, part) for the parts of a group's piece.  WAVES: all waves of a
// workgroup call it for one group; else each wave for its own, with an `lds` of its own,
// which all its lanes write alike.
template <int ROWS, bool WAVES, typename F>
__device__ inline void for_parts(int group, Piece<ROWS> &lds, F &&each) {
    const auto sync = [] {
        if constexpr (WAVES) __syncthreads();
    };
    const auto writes = [] { return !WAVES || threadIdx.x == 0; };
    {
        const Args a = arguments();
        if (group >= a.groups) return;
        if (!a.whole) {
            const Work<ROWS> work(a);
            if (writes()) {
                a.begun[group].parts = 0;
                lds.work = work;
                lds.at = work.begin(min(group, work.groups));
                lds.end = work.begin(min(group + 1, work.groups));
                lds.group = group;
            }
        }
    }
    for (bool again = false;; again = true) {
        const Args a = arguments();
        Part<ROWS> part;
        if (a.whole) {
            if (again || !part.whole_tile(a, group)) return;
        } else {
            sync();
            const int64_t at = lds.at, end = lds.end;
            if (kv::uniform(static_cast<int>(at >= end))) return;
            part = Part<ROWS>(a, lds.work.head, at, end);
            sync();
            if (writes()) {
                lds.at = at + (part.u1 - part.u0);
                if (part.u0 == 0 && part.u1 < part.weight) {   // the last one
                    const Tile t = tile_of<ROWS>(a, part.seq, part.k);
                    a.begun[group] = {lds.work.group_of(at + part.weight - 1) - group + 1, part.head, t.row0, t.n,
                                      part.seq.first};
                }
            }
        }
        part.settle();
        each(a, part);
    }
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
    unsigned some;      // four bytes of v_scale: all lanes' together are all that the wave has
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
        some = *reinterpret_cast<const unsigned *>(sv + r / 4 % (D / 32) * kChunk + r % 4 * 4);
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

// The larger one, up to fp32's largest: the median with that, one instruction, where
// fmaxf makes each operand a quiet NaN first.  A NaN does not count.
__device__ inline float larger(float a, float b) { return __builtin_amdgcn_fmed3f(a, b, 3.4028235e38f); }

// Bytes of x that are 253 or more: scales whose values bf16 does not hold.
__device__ inline unsigned not_finite(unsigned x) { return ((x & 0x7F7F7F7Fu) + 0x03030303u) & x & 0x80808080u; }
// All ones in these bytes.
__device__ inline unsigned not_finite_bytes(unsigned x) {
    const unsigned y = not_finite(x);
    return (y << 1) - (y >> 7);
}

// What a wave knows of its rows: lane l holds row l % 16, of the accumulators the
// elements 32 b + 8 (l / 16) + 2 e + p in o[b][p][e].
template <int D>
struct State {
    float m = kNone, limit = kNone, mc = 0.0f, sum = 0.0f;   // sum: of the lane's own tokens
    f32x4 o[D / 32][2] = {};
};

template <int D, int NP>
__device__ inline void attend(const Args &a, const Raw<D> &raw, const bf16x8 (&q)[D / 32][NP], State<D> &st, int token0,
                              int begin, int end, bool masked, bool lost) {
    const float c = a.c;
    f32x4 s[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float by = scale_of(raw.k_scale | not_finite_bytes(raw.k_scale), i);
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
    float tops[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) tops[i] = larger(larger(s[i][0], s[i][1]), larger(s[i][2], s[i][3]));
    const float top = larger(larger(tops[0], tops[1]), larger(tops[2], tops[3]));
    if (__ballot(top > st.limit)) {
        // Far rows' limit is none: they come here with each chunk of which they see something.
        const float all = over_groups(fmaxf(top, st.m), true), m = all > st.limit ? all : st.m;
        const float by = st.m == kNone ? 0.0f : __builtin_amdgcn_exp2f((st.m - m) * c);
        st.sum *= by;
#pragma unroll
        for (int b = 0; b < D / 32; ++b)
#pragma unroll
            for (int p = 0; p < 2; ++p) st.o[b][p] *= by;
        const bool near = __builtin_fabsf(m * c) <= kFar;
        st.m = m;
        st.limit = near ? m + kHeadroom / c : kNone;
        st.mc = near ? m * c : 0.0f;
        const float from = near || m == kNone ? 0.0f : m;
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] -= from;
    }
    const float mc = st.mc;
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
    // A value that is not finite must not reach rows that do not see it (0 times NaN): it
    // counts as 0 in the product and makes those NaN that see it.
    const bool repair = __ballot(not_finite(raw.some) != 0) != 0;
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
            for (int i = 0; i < 4; ++i) scale[i] &= ~not_finite_bytes(scale[i]);
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
__device__ inline float *partial_at(const Args &a, int slot, int row) {
    return a.partial + (static_cast<int64_t>(slot) * ROWS + row) * (D + 4);
}
template <typename T>
__device__ inline T *out_at(const Args &a, int first, int head, int row) {
    return static_cast<T *>(a.rows.out) +
           (static_cast<int64_t>(first + row / a.group) * a.rows.H + head * a.group + row % a.group) * a.cache.d;
}
template <typename T>
__device__ inline const T *query_at(const Args &a, const kv::Sequence &s, int head, int row) {
    return static_cast<const T *>(a.rows.q) + static_cast<int64_t>(s.first + row / a.group) * a.rows.q_token +
           static_cast<int64_t>(head * a.group + row % a.group) * a.rows.q_head;
}

// A wave's state of a part of a tile of 16 rows: every `step`-th of its chunks.
template <typename T, int D>
__device__ inline void few_rows(const Args &a, const Part<kRows> &part, const Tile &t, int chunk, int step, State<D> &st) {
    constexpr int NP = sizeof(T) == 2 ? 1 : 3;
    const int lane = threadIdx.x % 64, r = lane % 16, g = lane / 16;
    const int last = part.chunk(t, part.u1), head = part.head;
    if (chunk >= last) return;
    const int row = t.row0 + min(r, t.n - 1), query = row / a.group;
    const int end = row_end(a, part.seq, query), begin = row_begin(a, end);
    // The tokens that every row of the tile sees.
    const int all_end = row_end(a, part.seq, t.row0 / a.group);
    const int all_begin = row_begin(a, row_end(a, part.seq, (t.row0 + t.n - 1) / a.group));
    const int *const pages = a.batch.page_table + static_cast<int64_t>(part.b) * a.batch.W;
    const int per_page = a.cache.page / kChunk;
    Raw<D> raw;
    raw.load(a, head, pages[chunk / per_page], chunk, lane);
    bf16x8 q[D / 32][NP];
    const T *qp = query_at<T>(a, part.seq, head, row) + g * (D / 4);
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
        const int next = chunk + step;
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

// Waves with pieces of their own: none waits for another, so that one's beginnings and
// ends of tiles are covered by the others' loads.
template <typename T, int D>
__global__ __launch_bounds__(64 * kWaves, 2) void cache_attention_kernel(Args) {
    __shared__ Piece<kRows> pieces[kWaves];
    const int wave = kv::uniform(static_cast<int>(threadIdx.x / 64));
    Piece<kRows> &piece = pieces[wave];
    for_parts<kRows, false>(blockIdx.x * kWaves + wave, piece, [&](const Args &a, const Part<kRows> &part) {
        const Tile t = tile_of<kRows>(a, part.seq, part.k);
        State<D> st;
        few_rows<T, D>(a, part, t, part.chunk(t, part.u0), 1, st);
        const int lane = threadIdx.x % 64, r = lane % 16, g = lane / 16;
        const float sum = over_groups(st.sum, false);
        if (r >= t.n) return;
        const bool whole = part.whole();
        float *const p = partial_at<kRows, D>(a, part.slot(piece), r);
        T *const out = out_at<T>(a, part.seq.first, part.head, t.row0 + r);
        const float by = whole ? (sum == 0.0f ? 0.0f : 1.0f / sum) : 1.0f;
#pragma unroll
        for (int b = 0; b < D / 32; ++b) {
            fp8::f32x8 x;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[2 * e] = st.o[b][0][e] * by;
                x[2 * e + 1] = st.o[b][1][e] * by;
            }
            if (whole) store_8(out + 32 * b + 8 * g, x);
            else store_8(p + 32 * b + 8 * g, x);
        }
        if (!whole && g == 0) {
            p[D] = st.m;
            p[D + 1] = sum;
        }
    });
}

// Workgroups with pieces of their own, for few tiles: the chunks of a part go by turns to
// the waves, whose states are joined in their order.
template <typename T, int D>
__global__ __launch_bounds__(64 * kTeamWaves, 2) void cache_attention_team_kernel(Args) {
    __shared__ float o_lds[kTeamWaves][kRows][D + 4], m_lds[kTeamWaves][kRows], l_lds[kTeamWaves][kRows];
    __shared__ Piece<kRows> piece;
    for_parts<kRows, true>(static_cast<int>(block_index()), piece, [&](const Args &a, const Part<kRows> &part) {
        const Tile t = tile_of<kRows>(a, part.seq, part.k);
        const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, r = lane % 16, g = lane / 16;
        State<D> st;
        few_rows<T, D>(a, part, t, part.chunk(t, part.u0) + wave, kTeamWaves, st);
        const float mine = over_groups(st.sum, false);
        if (g == 0) {
            m_lds[wave][r] = st.m;
            l_lds[wave][r] = mine;
        }
#pragma unroll
        for (int b = 0; b < D / 32; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                o_lds[wave][r][32 * b + 8 * g + 2 * e] = st.o[b][0][e];
                o_lds[wave][r][32 * b + 8 * g + 2 * e + 1] = st.o[b][1][e];
            }
        __syncthreads();
        const bool whole = part.whole();
        for (int i = threadIdx.x; i < t.n * D; i += 64 * kTeamWaves) {
            const int row = i / D, e = i % D;
            float m = kNone, sum = 0.0f, x = 0.0f;
#pragma unroll
            for (int w = 0; w < kTeamWaves; ++w) m = fmaxf(m, m_lds[w][row]);
#pragma unroll
            for (int w = 0; w < kTeamWaves; ++w) {
                const float by = weight_of(m_lds[w][row], m, a.c);
                sum = __builtin_fmaf(l_lds[w][row], by, sum);
                x = __builtin_fmaf(o_lds[w][row][e], by, x);
            }
            if (whole) {
                out_at<T>(a, part.seq.first, part.head, t.row0 + row)[e] = static_cast<T>(sum == 0.0f ? 0.0f : x / sum);
                continue;
            }
            float *const p = partial_at<kRows, D>(a, part.slot(piece), row);
            p[e] = x;
            if (e == 0) {
                p[D] = m;
                p[D + 1] = sum;
            }
        }
    });
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
    const unsigned char *data, *scales;   // the cache's, and
    unsigned at, scale_at;                // its place in a chunk of it
    u32x4 x, scale;

    __device__ void at_keys(const Args &a, int t) {
        data = a.cache.k;
        scales = a.cache.k_scale;
        at = 16 * t;
        scale_at = t % (D / 32) * kChunk + kv::key_scale_place(t / (D / 32));
    }
    __device__ void at_values(const Args &a, int t) {
        const int c = t / 4, in = 16 * (t & 1) + 8 * (t >> 1 & 1);
        data = a.cache.v;
        scales = a.cache.v_scale;
        at = c * kChunk + in;
        scale_at = c / 16 * kChunk + in;
    }
    // Chunk `block` of the cache; bad: of a page that there is not.
    __device__ void load_keys(int64_t block, bool bad) {
        x = *reinterpret_cast<const u32x4 *>(data + block * (kChunk * (D / 2)) + at);
        scale[0] = bad ? 255u : (scales + block * (kChunk * (D / 32)))[scale_at];
    }
    __device__ void load_values(int64_t block) {
        const unsigned char *p = data + block * (kChunk * (D / 2)) + at, *s = scales + block * (kChunk * (D / 32)) + scale_at;
        const u32x2 x0 = *reinterpret_cast<const u32x2 *>(p), x1 = *reinterpret_cast<const u32x2 *>(p + 32);
        const u32x2 s0 = *reinterpret_cast<const u32x2 *>(s), s1 = *reinterpret_cast<const u32x2 *>(s + 32);
        x = u32x4{x0[0], x0[1], x1[0], x1[1]};
        scale = u32x4{s0[0], s0[1], s1[0], s1[1]};
    }
    __device__ void store_keys(Widened<D> &lds, int t) const {
        __bf16 *p = lds.k + t / (D / 32) * Widened<D>::KS + t % (D / 32) * 32;
        const float by = scale_of(scale[0] < 253u ? scale[0] : 255u, 0);   // not finite: NaN
#pragma unroll
        for (int j = 0; j < 4; ++j) *reinterpret_cast<bf16x8 *>(p + 8 * j) = widen8(x[j], by);
    }
    __device__ void store_values(Widened<D> &lds, int t, bool is_masked) const {
        const int c = t / 4, h = t & 1, i0 = 2 * (t >> 1 & 1);
        u32x4 s = scale;
        if (!is_masked) {
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i] |= not_finite_bytes(s[i]);
        } else {
            u32x4 wrong;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                wrong[i] = not_finite(s[i]) >> 7;
                s[i] &= ~not_finite_bytes(s[i]);
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

// A hint to the scheduler: N operands are read from LDS, each for NP products, AHEAD of
// them before the first product and each of the others behind another one's.
template <int N, int NP, int AHEAD>
__device__ inline void in_order() {
    __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);   // LDS reads
#pragma unroll
    for (int i = 0; i < N; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, NP, 0);   // products
        if (i + AHEAD < N) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
}

// Lane (li, g) of a wave: of a chunk's scores the row li and the tokens 32 mt + 8 (r / 4)
// + 4 g + r % 4 in s[mt][r], of the output the elements 32 dt + 8 (r / 4) + 4 g + r % 4
// in o[dt][r].
template <typename T, int D>
__device__ inline void many_rows(const Args &a, const Part<kPieceRows<T, D>> &part, const Piece<kPieceRows<T, D>> &piece, Widened<D> (&lds)[2]) {
    constexpr int NP = sizeof(T) == 2 ? 1 : 3, WAVES = kPieceWaves<T, D>, ROWS = kPieceRows<T, D>, KK = D / 16, DT = D / 32;
    constexpr int KS = Widened<D>::KS, VS = Widened<D>::VS;
    const Tile t = tile_of<ROWS>(a, part.seq, part.k);
    const int head = part.head, first = part.chunk(t, part.u0), chunks = part.chunk(t, part.u1) - first;
    const int lane = threadIdx.x % 64, wave = kv::uniform(static_cast<int>(threadIdx.x / 64)), li = lane % 32, g = lane / 32;
    const bool active = wave * kWaveRows < t.n;
    // Half of the threads take keys and half values, or each takes both.
    constexpr bool BOTH = 64 * WAVES == 2 * D;
    static_assert(BOTH || 64 * WAVES == 4 * D, "2 D shares of keys and of values");
    const bool keys = wave < WAVES / 2;
    const int share = threadIdx.x % (2 * D);
    const int row = t.row0 + min(wave * kWaveRows + li, t.n - 1);
    const int end = row_end(a, part.seq, row / a.group), begin = row_begin(a, end);
    const int all_end = row_end(a, part.seq, t.row0 / a.group);
    const int all_begin = row_begin(a, row_end(a, part.seq, (t.row0 + t.n - 1) / a.group));
    const auto masked = [&](int j) {
        const int token0 = (first + j) * kChunk;
        return !t.lost && (token0 < all_begin || token0 + kChunk > all_end);
    };

    bf16x8 q[KK][NP];
    {
        const T *qp = query_at<T>(a, part.seq, head, row) + 8 * g;
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

    // Chunk by chunk: the page's place in the table and the chunk's in the page.
    const int per_page = a.cache.page / kChunk;
    const int *pages = a.batch.page_table + static_cast<int64_t>(part.b) * a.batch.W + first / per_page;
    int in_page = first % per_page, page = t.lost || chunks == 0 ? -1 : *pages;
    Share<D> of_keys, of_values;
    if (BOTH || keys) of_keys.at_keys(a, share);
    if (BOTH || !keys) (BOTH ? of_values : of_keys).at_values(a, share);
    const auto load = [&](int j) {   // chunk j's share, if there is one, and the next one's page
        if (j >= chunks) return;
        const bool bad = page < 0 || page >= a.cache.pages;
        const int64_t block = (static_cast<int64_t>(bad ? 0 : page) * a.cache.heads + head) * per_page + in_page;
        if (++in_page == per_page) {
            in_page = 0;
            ++pages;
            if (j + 1 < chunks) page = *pages;
        }
        if (BOTH || keys) of_keys.load_keys(block, bad);
        if (BOTH || !keys) (BOTH ? of_values : of_keys).load_values(block);
    };
    const auto store = [&](int j) {
        if (BOTH || keys) of_keys.store_keys(lds[j & 1], share);
        if (BOTH || !keys) (BOTH ? of_values : of_keys).store_values(lds[j & 1], share, masked(j));
    };

    const float c = a.c;
    float m = kNone, sum = 0.0f;
    float mc = __builtin_nanf("");   // m times c; NaN where there is none, or it is far
    f32x16 o[DT] = {};
    // Scores of chunk j.
    const auto scores = [&](int j, f32x16 (&s)[2]) {
        const __bf16 *const k = lds[j & 1].k + li * KS + 8 * g;
        s[0] = s[1] = f32x16{};
#pragma unroll
        for (int kk = 0; kk < KK; ++kk)
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) {
                const bf16x8 x = *reinterpret_cast<const bf16x8 *>(k + 32 * mt * KS + 16 * kk);
#pragma unroll
                for (int p = NP - 1; p >= 0; --p) s[mt] = mfma32(x, q[kk][p], s[mt]);
            }
    };
    // What lane g's token r of tile mt of chunk j is, and whether its row sees it.
    const auto sees = [&](int j, int at) {
        return static_cast<unsigned>((first + j) * kChunk + 4 * g + at - begin) < static_cast<unsigned>(end - begin);
    };
    const auto hide = [&](int j, f32x16 (&s)[2]) {
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[mt][r] = sees(j, 32 * mt + 8 * (r / 4) + r % 4) ? s[mt][r] : kNone;
                if (r % 4 == 3) __builtin_amdgcn_sched_barrier(0);   // else all comparisons' masks at once
            }
    };
    // Probabilities of powers c (s - from) - off, and the lane's sum of them.
    const auto weights = [&](const f32x16 (&s)[2], float from, float off, bf16x8 (&pr)[4][NP]) {
        float all = 0.0f;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[ks / 2][8 * (ks % 2) + e] - from, c, -off));
                all += x[e];
            }
            take_apart<NP>(x, pr[ks]);
        }
        return all;
    };
    const auto product = [&](int j, const bf16x8 (&pr)[4][NP]) {
        const __bf16 *const v = lds[j & 1].v + li * VS + 8 * g;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks)
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                const bf16x8 x = *reinterpret_cast<const bf16x8 *>(v + 32 * dt * VS + 16 * ks);
#pragma unroll
                for (int p = NP - 1; p >= 0; --p) o[dt] = mfma32(x, pr[ks][p], o[dt]);
            }
    };
    const auto maximum = [&](const f32x16 (&s)[2]) {   // of the chunk's scores of the row
        float top[2] = {kNone, kNone};
#pragma unroll
        for (int r = 0; r < 16; ++r)
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) top[mt] = larger(top[mt], s[mt][r]);
        return of_halves(larger(top[0], top[1]), true);
    };
    const auto raise = [&](float to) {
        const float by = m == kNone ? 0.0f : __builtin_amdgcn_exp2f((m - to) * c);
        sum *= by;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[dt] *= by;
        m = to;
        mc = __builtin_fabsf(m * c) <= kFar ? m * c : __builtin_nanf("");
    };
    // What the powers of a row's probabilities are taken from (of far rows: all of m).
    const auto far = [&] { return mc != mc; };
    const auto from = [&] { return far() && m != kNone ? m : 0.0f; };
    const auto off = [&] { return far() ? 0.0f : mc; };
    // As in attend: values that are not finite make the rows NaN that see them, at the end
    // (bit dt: the elements of o[dt]).
    unsigned lost = 0;
    const auto note_wrong = [&](int j) {
        const Widened<D> &buf = lds[j & 1];
        unsigned any = 0;
        if (lane < D / 32 * kChunk / 4) any = reinterpret_cast<const unsigned *>(&buf.wrong[0][0])[lane];
        if (!__ballot(any != 0)) return;
#pragma unroll 1
        for (int i = 0; i < D / 32 * kChunk; ++i) {   // in the order of the operands
            const int at = i % kChunk;
            const int token = (first + j) * kChunk + at / 16 * 16 + at / 8 % 2 * 4 + at % 8 / 4 * 8 + at % 4;
            if ((&buf.wrong[0][0])[i] && token >= begin && token < end) lost |= 1u << (i / kChunk);
        }
    };

    load(0);
    if (chunks > 0) store(0);
    load(1);
    __syncthreads();
    for (int j = 0; j < chunks; ++j) {
        if (j + 1 < chunks) {
            store(j + 1);
            load(j + 2);
        }
        if (active) {
            f32x16 s[2];
            scores(j, s);
            in_order<2 * KK, NP, 6>();
            const bool mask = masked(j);
            if (mask) hide(j, s);
            if constexpr (NP == 1) {
                // The maximum is raised, and the chunk's probabilities taken again, where their
                // sum passes kMostSum, so that none is needed otherwise, and where it is NaN:
                // until a chunk of which the row sees something, and of far rows always.
                bf16x8 pr[4][NP];
                float all = weights(s, 0.0f, mc, pr);
                const bool high = !(of_halves(all, false) <= kMostSum);
                if (__ballot(high)) {
                    const float top = maximum(s);
                    raise(high ? fmaxf(m, top) : m);
                    all = weights(s, from(), off(), pr);
                }
                sum += all;
                product(j, pr);
            } else {
                const float top = maximum(s);
                if (__ballot(m == kNone ? top > kNone : far() || (top - m) * c > kHeadroom)) {
                    raise(fmaxf(m, top));
                    if (__ballot(far())) {   // the scores are not needed again
#pragma unroll
                        for (int mt = 0; mt < 2; ++mt) s[mt] -= from();
                    }
                }
                bf16x8 pr[4][NP];
                sum += weights(s, 0.0f, off(), pr);
                product(j, pr);
            }
            in_order<4 * DT, NP, 6>();
            if (mask) note_wrong(j);
        }
        __syncthreads();
    }

    if (wave * kWaveRows + li >= t.n) return;
    sum = of_halves(sum, false);
    if (lost) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[dt] += lost >> dt & 1u ? __builtin_nanf("") : 0.0f;
    }
    if (!part.whole()) {
        float *p = partial_at<ROWS, D>(a, part.slot(piece), wave * kWaveRows + li);
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
    T *out = out_at<T>(a, part.seq.first, head, row);
    const float by = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) out[32 * dt + 8 * (r / 4) + 4 * g + r % 4] = static_cast<T>(o[dt][r] * by);
}

template <typename T, int D>
__global__ __launch_bounds__((64 * kPieceWaves<T, D>), (kPiecePerSimd<T, D>)) void cache_attention_piece_kernel(Args) {
    constexpr int ROWS = kPieceRows<T, D>;
    __shared__ Widened<D> lds[2];
    __shared__ Piece<ROWS> piece;
    // Workgroup b runs on XCD b % 8; each XCD takes a range of the line, whose neighbours
    // are tiles that read the same chunks.
    const int nb = gridDim.x, id = blockIdx.x, xcd = id & 7;
    const int group = xcd * (nb >> 3) + min(xcd, nb & 7) + (id >> 3);
    for_parts<ROWS, true>(group, piece, [&](const Args &a, const Part<ROWS> &part) { many_rows<T, D>(a, part, piece, lds); });
}

// ---------------------------------------------------------------------------
// The parts of a tile in one, in their order
// ---------------------------------------------------------------------------
// A row's state over the parts z, z + by, ... of its tile, EACH elements of it; the loads
// of some parts are in flight together.
template <int EACH>
struct Joined {
    float m = kNone, l = 0.0f, o[EACH] = {};

    // state(z): a part's row.
    template <typename F>
    __device__ void add(F &&state, int e0, int d, int z, int by, int count, float c) {
        constexpr int AHEAD = 8;
        for (; z < count; z += AHEAD * by) {
            float pm[AHEAD], pl[AHEAD], po[AHEAD][EACH], up = m;
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const float *p = state(min(z + i * by, count - 1));
                pm[i] = z + i * by < count ? p[d] : kNone;
                pl[i] = p[d + 1];
#pragma unroll
                for (int e = 0; e < EACH; ++e) po[i][e] = p[e0 + e];
            }
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) up = fmaxf(up, pm[i]);
            const float keep = weight_of(m, up, c);
            l *= keep;
#pragma unroll
            for (int e = 0; e < EACH; ++e) o[e] *= keep;
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
};

// A workgroup joins rows of the tile that its group of the launch before has begun, 16
// lanes a row: 16 rows, or, of tiles of many parts (WIDE), four, whose parts its waves
// share.
template <typename T, int D, int ROWS, bool WIDE>
__global__ __launch_bounds__(256) void join_parts_kernel(Args a) {
    constexpr int LANES = 16, EACH = D / LANES, WAVES = 4;
    const int group = blockIdx.x, wave = threadIdx.x / 64, lane = threadIdx.x % 64, e0 = lane % LANES * EACH;
    const int r0 = WIDE ? blockIdx.y * 4 : blockIdx.y * 16 + 4 * wave;
    const Begun tile = a.begun[group];
    if (tile.parts == 0 || r0 >= tile.n) return;
    const int r = min(r0 + lane / LANES, tile.n - 1);
    Joined<EACH> j;
    j.add([&](int z) { return partial_at<ROWS, D>(a, 2 * (group + z) + (z == 0 ? 1 : 0), r); }, e0, D, WIDE ? wave : 0,
          WIDE ? WAVES : 1, tile.parts, a.c);
    if constexpr (!WIDE) {
        if (r0 + lane / LANES >= tile.n) return;
        T *out = out_at<T>(a, tile.first, tile.head, tile.row0 + r) + e0;
        const float by = j.l == 0.0f ? 0.0f : 1.0f / j.l;
#pragma unroll
        for (int e = 0; e < EACH; ++e) out[e] = static_cast<T>(j.o[e] * by);
    } else {
        __shared__ float o_lds[WAVES][4][D], ml_lds[WAVES][4][2];
#pragma unroll
        for (int e = 0; e < EACH; ++e) o_lds[wave][lane / LANES][e0 + e] = j.o[e];
        if (e0 == 0) {
            ml_lds[wave][lane / LANES][0] = j.m;
            ml_lds[wave][lane / LANES][1] = j.l;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < 4 * D; i += 256) {
            const int row = i / D, e = i % D;
            if (r0 + row >= tile.n) break;
            float all = kNone, sum = 0.0f, x = 0.0f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) all = fmaxf(all, ml_lds[w][row][0]);
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const float by = weight_of(ml_lds[w][row][0], all, a.c);
                sum = __builtin_fmaf(ml_lds[w][row][1], by, sum);
                x = __builtin_fmaf(o_lds[w][row][e], by, x);
            }
            out_at<T>(a, tile.first, tile.head, tile.row0 + r0 + row)[e] = static_cast<T>(sum == 0.0f ? 0.0f : x / sum);
        }
    }
}

// ---------------------------------------------------------------------------
// What is launched
// ---------------------------------------------------------------------------
// Beside sequences of many rows, those of up to this many are next tokens: the kernel
// for few takes them (16 sequences of 8192 tokens, 8 key heads of 128, in both kernels:
// 64 rows 102 and 124 us, 96 rows 143 and 131).
constexpr int kFewRows = 64;

// A launch over the sequences of [from, to] rows.
struct Launch {
    int from = 1, to = 0, groups = 0, least = 1;
    bool whole = false;   // a group a tile
    bool wide = false;    // tiles have many parts
    bool some() const { return from <= to; }
    // Words of workspace: the states, then what has been begun (a multiple of 16 bytes).
    int64_t partial(int d, int rows) const { return some() && !whole ? 2LL * groups * rows * (d + 4) : 0; }
    int64_t words(int d, int rows) const {
        return some() && !whole ? partial(d, rows) + (groups * (sizeof(Begun) / 4) + 3) / 4 * 4 : 0;
    }
    // At most `tiles`, `alike` if the sequences are, of up to n chunks: on `room` groups
    // at once, each of at least `each` chunks but where there are more tiles.  A group a
    // tile, which joins nothing, where n is at most `small`, or `more` and the tiles fill
    // a quarter of the room, or `most` and they fill it (teams, 64 tiles of 24 chunks: 13 us
    // against 21, 256 of 64 29 against 33, but 64 of them 26 against 18; many rows of 64, 256
    // tiles of 20 chunks 31 against 40, 128 of 32 50 against 39).
    void divide(int64_t tiles, int64_t alike, int64_t n, int each, int small, int more, int most, int room) {
        least = each;
        whole = n <= small || (n <= more && 4 * alike >= room) || (n <= most && alike >= room);
        const int64_t fit = std::max<int64_t>(tiles, tiles * n / each);
        groups = static_cast<int>(whole ? tiles : std::min<int64_t>(fit, room));
        wide = groups > 8 * alike;
    }
};
struct Plan {
    Launch few, many;
    bool team = false;   // the few rows' kernel
};

int piece_rows(int d, int dtype) { return d == 128 && dtype == 0 ? kPieceRows<__bf16, 128> : kPieceRows<float, 64>; }

Plan plan_of(const KvCache &cache, const KvBatch &batch, int T, int H, int window, int dtype) {
    Plan p;
    const int group = H / cache.heads, most = std::min(batch.B, T);
    const int64_t rows = static_cast<int64_t>(T) * group;
    const auto chunks = [&](int tile_rows) {   // that a tile sees, at most
        const int64_t cached = static_cast<int64_t>(batch.W) * (cache.page / kChunk);
        return window ? std::min<int64_t>(cached, (static_cast<int64_t>(window) + tile_rows / group) / kChunk + 3) : cached;
    };
    // Tiles of a key head: at most, of rows in sequences of which each has a multiple of
    // the group, and of sequences alike.
    const auto tiles_of = [&](int64_t seqs, int each) {
        int step = 1;
        while (2 * step <= each && group % (2 * step) == 0) step *= 2;
        return (rows + seqs * (each - step)) / each;
    };
    const auto alike_of = [&](int64_t seqs, int each) { return seqs * std::max<int64_t>((rows / seqs + each - 1) / each, 1); };
    // Rows for the kernel for many: of sequences alike, or where one may well have them
    // beside others' next tokens, and enough of them for its start and its tiles of 128
    // or 256 rows, which the long sequences pay back first (8 key heads of 128, in both
    // kernels: 8192 tokens of 512 rows 50 and 81 us, of 1024 99 and 85; 32768 tokens of 256
    // 88 and 111, of 512 159 and 137; 1024 tokens of 1024 24 and 46, of 4096 84 and 48).  Heads
    // of 64 and fp32 turn at the same place: of 13 prompts each behind 1024, 8192 and 32768
    // tokens, 64 rows a token, the rule takes the faster kernel or one 3 % behind, but for fp32,
    // 128, 1024 tokens behind 1024 (216 us, 196 in the other).
    const int64_t n = chunks(kRows);
    const double beyond = static_cast<double>((static_cast<int64_t>(T) - batch.B) * H / kRows);   // tiles
    const bool pieces = (rows > static_cast<int64_t>(kFewRows) * batch.B || T > 8LL * batch.B) && T > batch.B &&
                        beyond * beyond * static_cast<double>(n) >= 3 << 23;
    if (!pieces || batch.B > 1) {
        p.few.to = pieces ? kFewRows : INT32_MAX;
        const int64_t tiles = cache.heads * (pieces ? std::min<int64_t>(rows, most * static_cast<int64_t>(kFewRows / kRows))
                                                    : tiles_of(most, kRows));
        const int64_t alike = cache.heads * (pieces ? most : alike_of(most, kRows));
        // Eight waves a CU, alone or together.  Together they share what starting and
        // joining a part costs, up to a tile a CU, and of short tiles; of more tiles, waves
        // alone have whole ones and wait for nothing (8192 tokens of 16 sequences, 8 key heads,
        // 128: 128 tiles 35 us together and 45 alone, 256 55 and 70, 440 84 and 83, 1024 165
        // both; 1000 tiles of 18 chunks, fp32, 64: 50 and 41).
        p.team = n <= kTeamChunks / 2 || alike <= 256;
        if (p.team) p.few.divide(tiles, alike, n, 2 * kTeamWaves, kTeamChunks, kTeamChunks, 2 * kTeamChunks, 256);
        else p.few.divide(tiles, alike, n, 4, 0, 0, 0, 8 * 256);
    }
    if (pieces) {
        const int each = piece_rows(cache.d, dtype);
        p.many.from = batch.B > 1 ? kFewRows + 1 : 1;
        p.many.to = INT32_MAX;
        const int64_t seqs = std::min<int64_t>(most, std::max<int64_t>(rows / p.many.from, 1));
        p.many.divide(cache.heads * tiles_of(seqs, each), cache.heads * alike_of(seqs, each), chunks(each), 8, 8, 24, 32,
                      cache.d == 128 ? 256 : 512);
    }
    return p;
}

Args with(Args a, const Launch &l, float *workspace, int rows) {
    a.from = l.from;
    a.to = l.to;
    a.groups = l.groups;
    a.least = l.least;
    a.whole = l.whole;
    a.partial = workspace;
    a.begun = reinterpret_cast<Begun *>(workspace + l.partial(a.cache.d, rows));
    return a;
}

template <typename T, int D, int ROWS>
void join(const Args &a, const Launch &l, hipStream_t stream) {
    if (l.whole) return;
    if (l.wide) join_parts_kernel<T, D, ROWS, true><<<dim3(a.groups, ROWS / 4), 256, 0, stream>>>(a);
    else join_parts_kernel<T, D, ROWS, false><<<dim3(a.groups, ROWS / 16), 256, 0, stream>>>(a);
}

template <typename T, int D>
hipError_t run(const Args &args, const Plan &p, float *workspace, hipStream_t stream) {
    if (p.few.some()) {
        const Args a = with(args, p.few, workspace, kRows);
        // Whole tiles of 16 rows are up to 2^25 + 2^21, whose threads pass 32 bits; those of many
        // rows, at most 2^22 of 512 threads or 2^23 of 256, do not.
        if (p.team) cache_attention_team_kernel<T, D><<<grid_of(a.groups), 64 * kTeamWaves, 0, stream>>>(a);
        else cache_attention_kernel<T, D><<<(a.groups + kWaves - 1) / kWaves, 64 * kWaves, 0, stream>>>(a);
        join<T, D, kRows>(a, p.few, stream);
    }
    if (p.many.some()) {
        constexpr int ROWS = kPieceRows<T, D>;
        const Args a = with(args, p.many, workspace + p.few.words(D, kRows), ROWS);
        cache_attention_piece_kernel<T, D><<<a.groups, (64 * kPieceWaves<T, D>), 0, stream>>>(a);
        join<T, D, ROWS>(a, p.many, stream);
    }
    return hipGetLastError();
}

}  // namespace

int64_t cache_attention_workspace(const KvCache &cache, const KvBatch &batch, int T, int H, int window, int dtype) {
    if (T == 0 || batch.B == 0 || H == 0) return 0;
    const Plan p = plan_of(cache, batch, T, H, window, dtype);
    return 4 * (p.few.words(cache.d, kRows) + p.many.words(cache.d, piece_rows(cache.d, dtype)));
}

hipError_t launch_cache_attention(const KvCache &cache, const KvBatch &batch, const KvQueries &rows, void *workspace,
                                  int dtype, hipStream_t stream) {
    if (rows.T == 0 || batch.B == 0 || rows.H == 0) return hipSuccess;
    // At least 2^-149, which makes exp2 of any finite score 1 as a scale of 0 does, and
    // leaves masked scores at minus infinity; at most the largest number, so that scores of
    // 0 stay 0.
    const float c = std::min(std::max(std::fabs(rows.scale) * 1.44269504088896340736f, 0x1p-149f), 0x1.fffffep127f);
    const Args a{cache, batch, rows, c, rows.H / cache.heads, 0, 0, 0, 0, false, nullptr, nullptr};
    const Plan p = plan_of(cache, batch, rows.T, rows.H, rows.window, dtype);
    float *w = static_cast<float *>(workspace);
    if (dtype == 0) return cache.d == 128 ? run<__bf16, 128>(a, p, w, stream) : run<__bf16, 64>(a, p, w, stream);
    return cache.d == 128 ? run<float, 128>(a, p, w, stream) : run<float, 64>(a, p, w, stream);
}

}  // namespace hcms
