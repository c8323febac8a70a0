// 8-bit product for gfx950 (MI355X), scaled MFMA with fp32 accumulation:
//   Y[m][n] = sum_b 2^(sx[m][b] + sw[n / 128][b]) sum_{k in b} X[m][k] W[n][k]
// X [M][K] and W [N][K] e4m3, b the blocks of 128 k, sx and sw the exponents
// of fp8.h.  v_mfma_scale_f32_32x32x64_f8f6f4 takes the exponents as operands,
// so the scales cost no arithmetic and the sum over blocks stays in the MFMA's
// accumulators.
//
// Work decomposition
//   * one workgroup computes a BM x BN tile of Y, its waves WM x WN rectangles
//     of 32 x 32 MFMA tiles of Y^T: D[n][m], W rows as the A operand, X rows
//     as the B operand, each lane holding one row m.  Every element sums its
//     products in the order of k, whatever the tile, but for tiles with groups
//     of waves, each of which takes every KG-th stage: their sums are added in
//     the order of the groups;
//   * k advances in stages of 128 bytes per row, one block of the scales,
//     which go from global memory straight into one of ST LDS buffers, as the
//     stage's scales do (one dword, a group of four blocks, per row of X and
//     per 32 rows of W);
//   * one barrier per stage, placed where the operands of the stage's last
//     k-step are already in registers: past it the stage's buffer is free and
//     the next stage is in LDS;
//   * workgroups are persistent (without groups), their tiles form one stream
//     of stages, and the tile order gives each XCD a contiguous range of each
//     round (8 row tiles at a time), so that its L2 serves shared panels.
//
// What bounds it.  Large products: the power limit (the matrix cores alone take
// 8-bit operands at 3200-3500 TFLOP/s for a short while) and what is not MFMAs:
// 56160 x 1920 x 5120 runs at 2210-2320 TFLOP/s (476-500 us, by the card) with the MFMAs busy
// 58 % of the SIMDs' cycles at 1.86 GHz, 2.5 us of each tile's 41 its start and epilogue; 8192^3
// at 2700.  Each stage also moves its operands through LDS, WN times for X and WM
// times for W, at 128 bytes per clock: 0.95 us per stage of a 256 x 256 tile against
// 0.85 of MFMAs, which is why the waves' rectangles are large.  Few tiles: the
// stages' latencies (0.37 us on 128 x 128).
//
// Tails: rows past M or N and k past K are read as zeros through buffer
// resources; rows past M and columns past N are not stored.  K is a multiple
// of 16 and N / parts of 8 (checked by the caller).
#include <type_traits>

#include "attention_tiles.h"
#include "fp8.h"
#include "hcms_internal.h"
#include "linear_fp8_tiles.h"

namespace hcms {
namespace {

using namespace tiles;

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kGroupM = 8;   // row tiles per group of the tile order

template <int BM_, int BN_, int WM_, int WN_, int ST_, int PER_CU_, int KG_ = 1>
struct Tile {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, ST = ST_, PER_CU = PER_CU_, KG = KG_;
    static constexpr int W = WM * WN, THREADS = 64 * W * KG;     // W: waves of a group of k
    static constexpr int WAVES = PER_CU * W * KG / 4;            // per SIMD
    static constexpr int MT = BM / WM / 32, NT = BN / WN / 32;   // 32 x 32 tiles per wave
    static constexpr int XL = BM / 8 / W, WL = BN / 8 / W;       // operand loads per wave and stage
    static constexpr int SL = (BM / 64 + W) / W;                 // scale loads per wave and stage
    static constexpr int SW = 128 % (NT * 32) ? NT : 1;          // scale blocks of a wave's W rows
    static constexpr int SCALE_B = (BM + 64) * 4;                // scales of a stage: X rows, 32 W rows each
    static constexpr int STAGE_B = (BM + BN) * 128 + SCALE_B;
    static constexpr int OUT_B = 2048;                           // output staging per wave
    static constexpr int RING_B = KG * ST * STAGE_B;
    // With groups of k the sums and the output pass through the ring.
    static constexpr int LDS_B = RING_B + (KG == 1 ? W * OUT_B : 0);
    static_assert(XL * 8 * W == BM && WL * 8 * W == BN && (W % 2 == 0 || KG > 1), "whole loads per wave");
    static_assert(KG == 1 || KG == 2, "a sum of two does not depend on their order");
    static_assert(KG == 1 || (NT * MT % KG == 0 && KG * BM * BN * 4 <= RING_B), "sums of the groups");
    static_assert(BM % 64 == 0, "whole scale loads");
    static_assert(LDS_B * PER_CU <= 160 * 1024 && ST >= 2, "LDS of a CU");
};

// Resource over `bytes` bytes (at most 2^28) from base on.
__device__ inline __amdgpu_buffer_rsrc_t span(const void *base, int bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(base), 0, bytes, 0x00020000);
}

// 8 of an operand's 32 values, quarter t, widened to bf16 and scaled by the
// fp32 number whose exponent s holds: exact.
__device__ inline bf16x8 widened(const i32x8 &v, int t, int s) {
    const float by = __builtin_bit_cast(float, s);
    const bf16x2 p0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[2 * t], by, false);
    const bf16x2 p1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[2 * t], by, true);
    const bf16x2 p2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[2 * t + 1], by, false);
    const bf16x2 p3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[2 * t + 1], by, true);
    return bf16x8{p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
}

// A wave's MT x NT tiles at rows mb .., columns nb .. of Y.  Lane (li, g)
// holds row mb + 32 mt + li and, per 32 x 32 tile, runs of 4 consecutive
// columns 8 rb + 4 g; they pass through a private 2 KiB of LDS, 32 rows by 64
// bytes at a time, to leave as 16 bytes per lane and 64 per row.  Chunk c of
// staged row r sits at position c ^ (r / 4 % 4).  Column n of Y lies in part
// n / np (np is a multiple of 8, so no chunk crosses parts).  Of KG groups
// of waves group `grp` stores every KG-th tile.
// FULL: the wave's rows and columns all lie inside of Y, and no store is skipped.
template <typename T, typename C, bool FULL>
__device__ inline void store_tile(f32x16 (&acc)[C::NT][C::MT], char *stage, T *y, int np, int mb, int nb, int M,
                                  int N, int lane, int grp) {
    constexpr int SEG = sizeof(T) == 2 ? 1 : 2;          // segments per 32 columns
    constexpr int E = 16 / static_cast<int>(sizeof(T));  // elements per chunk
    const int li = lane & 31, g = lane >> 5;
    // A segment's stores wait for its reads from LDS, so they stand behind the
    // next segment's writes and reads.
    u32x4 o[2];
    T *to = nullptr;
    int row = 0, n = 0;
    const auto store = [&]() {
#pragma unroll
        for (int q = 0; q < 2; ++q)
            if (FULL || (row + q * 16 < M && n < N)) *reinterpret_cast<u32x4 *>(to + static_cast<int64_t>(q * 16) * np) = o[q];
    };
#pragma unroll
    for (int mt = 0; mt < C::MT; ++mt) {
#pragma unroll
        for (int sg = 0; sg < C::NT * SEG; ++sg) {
            if (C::KG > 1 && (sg / SEG * C::MT + mt) % C::KG != grp) continue;
            const f32x16 &t = acc[sg / SEG][mt];
#pragma unroll
            for (int i = 0; i < 4 / SEG; ++i) {
                const int rb = (sg % SEG) * 2 + i;
                const f32x4 v = {t[rb * 4 + 0], t[rb * 4 + 1], t[rb * 4 + 2], t[rb * 4 + 3]};
                if constexpr (sizeof(T) == 2)
                    *reinterpret_cast<bf16x4 *>(stage + li * 64 + ((i ^ ((li >> 2) & 3)) << 4) + g * 8) =
                        __builtin_convertvector(v, bf16x4);
                else
                    *reinterpret_cast<f32x4 *>(stage + li * 64 + (((i * 2 + g) ^ ((li >> 2) & 3)) << 4)) = v;
            }
            const int ch = lane & 3;
            u32x4 next[2];
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int r = q * 16 + (lane >> 2);
                next[q] = *reinterpret_cast<const u32x4 *>(stage + r * 64 + ((ch ^ ((r >> 2) & 3)) << 4));
            }
            if (to) store();
            n = nb + sg * (32 / SEG) + ch * E;
            row = mb + mt * 32 + (lane >> 2);
            const int part = n / np;
            to = y + static_cast<int64_t>(part) * M * np + (n - part * np) + static_cast<int64_t>(row) * np;
            o[0] = next[0];
            o[1] = next[1];
        }
    }
    store();
}

template <typename T, typename C>
__global__ __launch_bounds__(C::THREADS, C::WAVES) void linear_fp8_kernel(
    const unsigned char *__restrict__ x, const unsigned *__restrict__ xs, const unsigned char *__restrict__ w,
    const unsigned *__restrict__ ws, T *__restrict__ y, int M, int N, int K, int np, int tiles_m, int tiles_n) {
    constexpr int MT = C::MT, NT = C::NT, ST = C::ST, W = C::W, KG = C::KG;
    constexpr int LPW = C::XL + C::WL + C::SL;   // loads per wave and stage, the last ones of scales
    constexpr int kHalf = (LPW + 1) / 2;         // of them right behind the barrier
    __shared__ __attribute__((aligned(1024))) char lds[C::LDS_B];

    const int G = gridDim.x, b = blockIdx.x;
    const int xcd = b & 7, per = G >> 3, rem = G & 7;
    const int slot = xcd * per + min(xcd, rem) + (b >> 3);
    const int n_tiles = tiles_m * tiles_n;
    if (slot >= n_tiles) return;
    const int n_mine = KG > 1 ? 1 : (n_tiles - 1 - slot) / G + 1;
    auto origin = [&](int r, int &m0, int &n0) {
        const int L = r * G + slot;
        const int group = L / (kGroupM * tiles_n);
        const int first_m = group * kGroupM;
        const int gm = min(tiles_m - first_m, kGroupM);
        const int in_group = L - group * kGroupM * tiles_n;
        m0 = (first_m + in_group % gm) * C::BM;
        n0 = (in_group / gm) * C::BN;
    };

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave_all = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int grp = KG == 1 ? 0 : wave_all / W, wave = wave_all - grp * W;
    const int li = lane & 31, g = lane >> 5;
    const int wm = wave / C::WN, wn = wave % C::WN;
    const int nkb = (K + 127) / 128, n_blocks = (N + 127) / 128;
    const int steps = (nkb + KG - 1) / KG;   // step s of group `grp` is block s KG + grp

    // Load i of a wave brings rows 8 (i W + wave) + lane / 8 of the stage's X
    // rows (then of its W rows), 16 bytes per lane; the lane at position
    // lane % 8 of its row fetches chunk (lane % 8) ^ (row / 2 % 8), so that 16
    // rows of one chunk lie in 16 different groups of 4 banks.  A chunk past K
    // is fetched from past the resource: zeros.
    const unsigned chunk = ((lane & 7) ^ ((4 * wave + (lane >> 4)) & 7)) << 4;
    const unsigned voff_in = (8 * wave + (lane >> 3)) * static_cast<unsigned>(K) + chunk;
    const unsigned voff_end = (nkb - 1) * 128u + chunk < static_cast<unsigned>(K) ? voff_in : 0x80000000u;
    const unsigned pass_bytes = 8u * W * K;
    char *const ring = lds + grp * ST * C::STAGE_B;
    const unsigned lds0 = static_cast<unsigned>(reinterpret_cast<uintptr_t>(ring));
    unsigned w_scale;   // W's scales: lane l fetches that of rows 32 l .. of the panel
    // Offsets of block kb: those of a block past K (a group's last step may be
    // one) are past the resource.
    const auto offsets = [&](int kb) { return kb < nkb - 1 ? voff_in : kb == nkb - 1 ? voff_end : 0x80000000u; };

    // The stages of the workgroup's tiles form one stream.  A stage past its
    // end is loaded through empty resources: zeros into a buffer that nobody
    // reads, so that every step issues the same number of loads.
    int ld_r = 0, ld_kb = grp;
    int lm0, ln0;
    unsigned voff;
    __amdgpu_buffer_rsrc_t lxs, lws, lss[C::SL];
    // Scales of stage ld_kb: load i of wave w brings piece i W + w, 64 rows of X
    // each while they last, then (all alike) W's.
    auto scales = [&]() {
        const int64_t four = ld_kb >> 2;
#pragma unroll
        for (int i = 0; i < C::SL; ++i)
            lss[i] = i * W + wave < C::BM / 64
                         ? span(xs + four * M + lm0, min(M - lm0, C::BM) * 4)
                         : span(ws + four * n_blocks + ln0 / 128, min(n_blocks - ln0 / 128, 64) * 4);
    };
    auto panels = [&]() {
        origin(ld_r, lm0, ln0);
        lxs = span(x + static_cast<int64_t>(lm0) * K, min(M - lm0, C::BM) * K);
        lws = span(w + static_cast<int64_t>(ln0) * K, min(N - ln0, C::BN) * K);
        w_scale = ((ln0 >> 5 & 3) + lane) >> 2 << 2;
        scales();
    };
    panels();
    voff = offsets(ld_kb);
    auto load_one = [&](int i, int buf) {
        if (i >= C::XL + C::WL) {
            const int piece = min((i - C::XL - C::WL) * W + wave, C::BM / 64);
            load_lds_b32(lds0 + buf * C::STAGE_B + (C::BM + C::BN) * 128 + piece * 256, lss[i - C::XL - C::WL],
                         piece < C::BM / 64 ? lane * 4 : w_scale,
                         piece < C::BM / 64 ? piece * 256 : 0);
            return;
        }
        // Opaque, so that no sums and multiples of them are kept: scalar
        // registers are short.
        unsigned dst = lds0 + wave * 1024, pass = pass_bytes;
        asm volatile("" : "+s"(dst), "+s"(pass));
        dst += buf * C::STAGE_B + i * W * 1024;
        const unsigned soff = ld_kb * 128;
        if (i < C::XL) load_lds(dst, lxs, voff, soff + i * pass);
        else load_lds(dst, lws, voff, soff + (i - C::XL) * pass);
    };
    auto advance = [&]() {
        ld_kb += KG;
        if (ld_kb < steps * KG) {
            if ((ld_kb & 3) < KG && ld_r < n_mine) scales();
            voff = offsets(ld_kb);
            return;
        }
        ld_kb = grp;
        voff = offsets(ld_kb);
        if (++ld_r < n_mine) {
            panels();
        } else {
            lxs = lws = span(nullptr, 0);
#pragma unroll
            for (int i = 0; i < C::SL; ++i) lss[i] = span(nullptr, 0);
        }
    };

    const unsigned rd = li * 128 + ((g ^ ((li >> 1) & 7)) << 4);
    const char *const xrd = ring + wm * MT * 32 * 128;
    const char *const wrd = ring + C::BM * 128 + wn * NT * 32 * 128;
    const char *const xsrd = ring + (C::BM + C::BN) * 128 + (wm * MT * 32 + li) * 4;
    const char *const wsrd = ring + (C::BM + C::BN) * 128 + C::BM * 4 + wn * NT * 4;

    // fp32 output: the 8-bit MFMA aligns groups of 8 products to the largest sum
    // of operand exponents among them and cuts each 13 binary places below it
    // (relative error 1.4e-5 on normal operands, a hundredth of the rounding to bf16), so for
    // fp32 output the operands are widened to bf16, exactly, scales included,
    // and multiplied at the bf16 rate, whose MFMA keeps fp32 sums (6e-8).
    constexpr bool kWide = sizeof(T) == 4;
    f32x16 acc[NT][MT];
    i32x8 a[2][NT], bx[2][MT];
    int sx[MT], sw[C::SW], sx_next[MT], sw_next[C::SW];
    // Operand of k-step ks (64 k, 4 chunks of a staged row): lane half g takes
    // chunks g and 2 + g of them, of both operands alike.
    auto operand = [&](const char *p, int ks) {
        const i32x4 lo = *reinterpret_cast<const i32x4 *>(p + (rd ^ (ks << 6)));
        const i32x4 hi = *reinterpret_cast<const i32x4 *>(p + (rd ^ (ks << 6) ^ 32));
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    // Operand i (W's NT, then X's MT) of k-step ks into `set`.
    auto read_op = [&](int i, int set, int ks, int buf) {
        const int base = buf * C::STAGE_B;
        if (i < NT) a[set][i] = operand(wrd + base + i * 32 * 128, ks);
        else bx[set][i - NT] = operand(xrd + base + (i - NT) * 32 * 128, ks);
    };
    auto read_scales = [&](int buf) {
        const int base = buf * C::STAGE_B;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) sx_next[mt] = *reinterpret_cast<const int *>(xsrd + base + mt * 32 * 4);
#pragma unroll
        for (int nt = 0; nt < C::SW; ++nt) sw_next[nt] = *reinterpret_cast<const int *>(wsrd + base + nt * 4);
    };
    // The stage's byte of the group's four into the lowest place (of a block past
    // K, whose products are zeros, one bit of it: never the scale NaN).
    auto take_scales = [&](int kb) {
        const int sh = KG == 1 || kb < nkb ? (kb & 3) * 8 : 31;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) sx[mt] = static_cast<unsigned>(sx_next[mt]) >> sh;
#pragma unroll
        for (int nt = 0; nt < C::SW; ++nt) sw[nt] = static_cast<unsigned>(sw_next[nt]) >> sh;
        if constexpr (kWide) {   // as fp32 exponents
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) sx[mt] = (sx[mt] & 255) << 23;
#pragma unroll
            for (int nt = 0; nt < C::SW; ++nt) sw[nt] = (sw[nt] & 255) << 23;
        }
    };
    auto mfma = [&](int set, int i) {
        const int nt = i / MT, mt = i % MT;
        acc[nt][mt] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a[set][nt], bx[set][mt], acc[nt][mt], 0, 0, 0,
                                                                      sw[C::SW == 1 ? 0 : nt], 0, sx[mt]);
    };

#pragma unroll 1
    for (int st = 0; st < ST - 1; ++st) {
#pragma unroll
        for (int i = 0; i < LPW; ++i) load_one(i, st);
        advance();
    }
#pragma unroll
    for (int i = 0; i < kHalf; ++i) load_one(i, ST - 1);
    wait_vm<(ST - 2) * LPW + kHalf>();
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NT + MT; ++i) read_op(i, 0, 0, 0);
    read_scales(0);

    // MFMAs of operand set `set`, between them the operand reads of k-step ks
    // of buffer `from` into the other set (all at once ahead of the MFMAs, the
    // waves' reads fill the LDS queue and the matrix cores wait behind them),
    // and the loads l0 .. l1 - 1 into `into`.
    auto phase = [&](int set, int ks, int from, int l0, int l1, int into) {
        // In the order in which the next MFMAs take them: W's first, X's, W's others,
        // over 3/4 of the MFMAs ahead of the barrier and over all of them behind it,
        // against W's first and 3/4: 1920 x 5120 x 7808 on 192 x 256 72 us against 75,
        // on 64 x 128 116 against 120, but with three of W's and more in a wave that
        // has its SIMD alone 488 against 483 (56160 x 1920 x 5120 on 192 x 192) and 76
        // against 73 (7800 x 5120 x 1920 on 128 x 256).  Over half of the MFMAs of
        // widened operands, which take longer (3/4: 3001 x 1000 x 1936 19.1 us, half 18.6).
        constexpr int kOps = NT + MT, kMf = NT * MT * (kWide ? 4 : 1);
        constexpr bool kByUse = kWide || C::WAVES > 1 || NT < 3;
        const int kOver = kWide ? (kMf + 1) / 2 : kByUse && ks == 0 ? kMf : (kMf * 3 + 3) / 4;
        bf16x8 aw[NT], bw[MT];
#pragma unroll
        for (int i = 0; i < kMf; ++i) {
            if constexpr (kWide) {
                const int t = i / (NT * MT), nt = i % (NT * MT) / MT, mt = i % MT;
                if (i % (NT * MT) == 0) {
#pragma unroll
                    for (int k = 0; k < NT; ++k) aw[k] = widened(a[set][k], t, sw[C::SW == 1 ? 0 : k]);
#pragma unroll
                    for (int k = 0; k < MT; ++k) bw[k] = widened(bx[set][k], t, sx[k]);
                }
                acc[nt][mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(aw[nt], bw[mt], acc[nt][mt], 0, 0, 0);
            } else {
                mfma(set, i);
            }
#pragma unroll
            for (int o = 0; o < kOps; ++o)
                if (o * kOver / kOps == i)
                    read_op(!kByUse || o == 0 ? o : o <= MT ? NT + o - 1 : o - MT, set ^ 1, ks, from);
            if (i == kMf - 1 && ks == 0) read_scales(from);
#pragma unroll
            for (int l = 0; l < LPW; ++l)
                if (l >= l0 && l < l1 && (l - l0) * kMf / (l1 - l0) == i) load_one(l, into);
            __builtin_amdgcn_sched_barrier(0);
        }
        // Keeps the MFMAs here: with their results not read in this basic block
        // the compiler sinks them into the next one, past the barrier.
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                if constexpr (C::WAVES == 1) asm volatile("" : "+a"(acc[nt][mt]));
                else asm volatile("" : "+v"(acc[nt][mt]));
            }
        __builtin_amdgcn_sched_barrier(0);
    };
    constexpr int kStores = NT * MT * (sizeof(T) == 2 ? 2 : 4);   // of a wave's whole tile
    static_assert((ST - 2) * LPW + kStores < 64, "counted by vmcnt");
    bool behind = false;   // kStores stores were issued behind the tile before
    int buf = 0, prev = ST - 1;
    for (int r = 0; r < n_mine; ++r) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) acc[nt][mt] = f32x16{};
        // End the scalar loads of the code before the loop (simm16: lgkmcnt 0,
        // the others open).
        __builtin_amdgcn_s_waitcnt(0xC07F);
        take_scales(grp);
        for (int s = 0; s < steps; ++s) {
            // The first k-step, beside the operand reads of the second; it
            // also issues the second half of the loads into the buffer that
            // the step before freed.
            phase(0, 1, buf, kHalf, LPW, prev);
            advance();
            // The second k-step's operands are in registers: past this barrier
            // the stage's buffer is free and the next stage is in LDS.
            // With three buffers and more that stage's loads are older than the
            // stores of the tile before, which may then go on (vector memory ends in
            // the order of issue); with two, half of them were issued just now.
            if (ST > 2 && s == 0 && behind) wait_vm<(ST - 2) * LPW + (ST > 2 ? kStores : 0)>();
            else wait_vm<(ST - 2) * LPW>();
            __syncthreads();
            const int next = buf + 1 == ST ? 0 : buf + 1;
            phase(1, 0, next, 0, kHalf, buf);
            if (s + 1 < steps) take_scales((s + 1) * KG + grp);
            prev = buf;
            buf = next;
        }
        if constexpr (KG > 1) {
            // The only tile of the workgroup: each group leaves the other's 32 x
            // 32 tiles and adds up its own.
            wait_vm<0>();
            __syncthreads();
            const auto place = [&](int from, int t, int piece) {
                return reinterpret_cast<f32x4 *>(lds + (((from * NT * MT + t) * W + wave) * 4 + piece) * 1024) + lane;
            };
#pragma unroll
            for (int t = 0; t < NT * MT; ++t)
                if (t % KG != grp)
#pragma unroll
                    for (int p = 0; p < 4; ++p) {
                        const f32x16 &v = acc[t / MT][t % MT];
                        *place(grp, t, p) = f32x4{v[4 * p], v[4 * p + 1], v[4 * p + 2], v[4 * p + 3]};
                    }
            __syncthreads();
#pragma unroll
            for (int t = 0; t < NT * MT; ++t)
                if (t % KG == grp)
#pragma unroll
                    for (int p = 0; p < 4; ++p) {
                        f32x16 &v = acc[t / MT][t % MT];
                        const f32x4 o = *place(grp ^ 1, t, p);
#pragma unroll
                        for (int i = 0; i < 4; ++i) v[4 * p + i] += o[i];
                    }
            __syncthreads();
        }
        // What the addresses need is worked out here, not kept over the loop.
        if constexpr (KG == 1) asm volatile("" : "+s"(M), "+s"(N), "+s"(np));
        int m0, n0;
        origin(r, m0, n0);
        const int mb = m0 + wm * MT * 32, nb = n0 + wn * NT * 32;
        char *const out = lds + (KG == 1 ? ST * C::STAGE_B : 0) + wave_all * C::OUT_B;
        behind = KG == 1 && mb + MT * 32 <= M && nb + NT * 32 <= N;
        if (behind) store_tile<T, C, true>(acc, out, y, np, mb, nb, M, N, lane, grp);
        else store_tile<T, C, false>(acc, out, y, np, mb, nb, M, N, lane, grp);
    }
    wait_vm<0>();   // no load into LDS is pending when the workgroup ends
}

// Few rows: what counts is that all of W is in flight at once and that a load
// covers whole lines: 16 consecutive lanes of a load that read 16 rows cost 16
// look-ups, and straight from memory into the MFMA's operands (lane li holds row
// li) every load is of that kind: 1 x 5120 x 5120 7.5 us, 16 rows 9.2, 32 rows 12.0.
// So 8 lanes load a row's block of 128, and the operands pass through LDS, a place
// of each wave's own: 4.8 us (5.4 TB/s; 7.4 with W from memory), 5.2 and 7.1; 64
// rows 9.8, on 64 x 64 tiles, whose stages wait for each other, 12.2.  From 17 rows on
// the registers that hold X's blocks leave fewer of W's in flight (kDeep), so the
// time grows while W's bytes do not.  A workgroup
// takes 16 NT columns of Y and all rows (16 MT hold them), its waves the blocks of
// k in turn, and the waves' sums are added through LDS in the order of the waves.
// MFMA 16 x 16 x 128 (for fp32 output 16 x 16 x 32 in bf16): lane (li, g) holds 32
// k of one row of W and of X (chunks g and 4 + g of the block's eight), and of Y^T
// row m = li, columns 4 g .. 4 g + 3.
template <typename T, int NT, int MT>
__global__ __launch_bounds__(512) void linear_fp8_rows_kernel(
    const unsigned char *__restrict__ x, const unsigned *__restrict__ xs, const unsigned char *__restrict__ w,
    const unsigned *__restrict__ ws, T *__restrict__ y, int M, int N, int K, int np) {
    constexpr bool kWide = sizeof(T) == 4;
    // Blocks whose loads are in flight together, as many as the registers hold (32
    // rows by 5120 x 5120 from memory: 4 of them 10.9 us, 3 11.1, 5 spill).
    constexpr int kDeep = NT + MT == 2 ? 8 : NT + MT == 3 ? 6 : MT == 2 ? 4 : 2;
    __shared__ __attribute__((aligned(16))) char stage[8][(NT + MT) * 2048];
    __shared__ f32x4 part[8][NT][MT][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const int li = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.x * (16 * NT), nkb = (K + 127) / 128, n_blocks = (N + 127) / 128;
    // Lane l loads chunk l % 8 of rows l / 8 and 8 + l / 8 of each 16.
    const int row = lane >> 3, chunk = (lane & 7) * 16;
    const unsigned char *wr[NT][2], *xr[MT][2];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
#pragma unroll
        for (int i = 0; i < NT; ++i)
            wr[i][c] = w + static_cast<int64_t>(min(n0 + 16 * i + 8 * c + row, N - 1)) * K;
#pragma unroll
        for (int i = 0; i < MT; ++i) xr[i][c] = x + static_cast<int64_t>(min(16 * i + 8 * c + row, M - 1)) * K;
    }
    // Chunk q of staged row r sits at place q ^ (r / 2 % 8): the 16 rows of a read
    // lie in 16 different groups of 4 banks.
    char *const mine = stage[wave];
    char *const put = mine + row * 128 + (chunk ^ ((row >> 1) << 4));          // of row 8 + row: place ^ 4
    const char *const get = mine + li * 128 + ((g ^ (li >> 1)) << 4);          // of chunk 4 + g: place ^ 4
    f32x4 acc[NT][MT]{};
    // Else X's last 8 staged rows are nobody's, and are neither loaded nor staged (1 x
    // 5120 x 5120 5.2 us with them).
    const bool upper = M > 16 * MT - 8;
    // D blocks from kb0 on, without a branch around the loads, which would wait for
    // them there: rows past the ends read the last row (their sums are not stored),
    // chunks past K the row's last one, and are made zeros before they are used.
    const auto blocks = [&](int kb0, auto depth) {
        constexpr int D = depth();
        i32x4 a[D][NT][2], b[D][MT][2];
        unsigned sa[D], sb[D][MT];
#pragma unroll
        for (int d = 0; d < D; ++d) {
            const int kb = kb0 + d * waves, at = min(kb * 128 + chunk, K - 16);
#pragma unroll
            for (int c = 0; c < 2; ++c) {
#pragma unroll
                for (int i = 0; i < NT; ++i) a[d][i][c] = *reinterpret_cast<const i32x4 *>(wr[i][c] + at);
#pragma unroll
                for (int i = 0; i < MT; ++i)
                    if (c == 0 || i < MT - 1 || upper) b[d][i][c] = *reinterpret_cast<const i32x4 *>(xr[i][c] + at);
            }
            const int64_t grp = kb >> 2;
            sa[d] = ws[grp * n_blocks + n0 / 128];
#pragma unroll
            for (int i = 0; i < MT; ++i) sb[d][i] = xs[grp * M + min(16 * i + li, M - 1)];
        }
#pragma unroll
        for (int d = 0; d < D; ++d) {
            const int kb = kb0 + d * waves, sh = (kb & 3) * 8;
            if (d == D - 1 && kb * 128 + chunk >= K) {
#pragma unroll
                for (int c = 0; c < 2; ++c) {
#pragma unroll
                    for (int i = 0; i < NT; ++i) a[d][i][c] = i32x4{};
#pragma unroll
                    for (int i = 0; i < MT; ++i) b[d][i][c] = i32x4{};
                }
            }
            // The wave's own place, whose accesses stay in order: no barrier.
#pragma unroll
            for (int i = 0; i < NT + MT; ++i)
#pragma unroll
                for (int c = 0; c < 2; ++c)
                    if (c == 0 || i < NT + MT - 1 || upper) {
                        char *const to = c == 0 ? put + i * 2048 : mine + i * 2048 + 1024 + ((put - mine) ^ 64);
                        *reinterpret_cast<i32x4 *>(to) = i < NT ? a[d][i][c] : b[d][i - NT][c];
                    }
            const auto operand = [&](int i) {
                const i32x4 lo = *reinterpret_cast<const i32x4 *>(get + i * 2048);
                const i32x4 hi = *reinterpret_cast<const i32x4 *>(mine + i * 2048 + ((get - mine) ^ 64));
                return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            };
            const unsigned wa = sa[d] >> sh & 255;
            i32x8 av[NT];
#pragma unroll
            for (int i = 0; i < NT; ++i) av[i] = operand(i);
#pragma unroll
            for (int j = 0; j < MT; ++j) {
                const i32x8 bv = operand(NT + j);
                const unsigned wb = sb[d][j] >> sh & 255;
#pragma unroll
                for (int i = 0; i < NT; ++i) {
                    if constexpr (kWide) {
#pragma unroll
                        for (int q = 0; q < 4; ++q)
                            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                                widened(av[i], q, wa << 23), widened(bv, q, wb << 23), acc[i][j], 0, 0, 0);
                    } else {
                        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(av[i], bv, acc[i][j], 0, 0, 0, wa,
                                                                                    0, wb);
                    }
                }
            }
        }
    };
    int kb0 = wave;
    for (; kb0 + (kDeep - 1) * waves < nkb; kb0 += kDeep * waves) blocks(kb0, std::integral_constant<int, kDeep>{});
    const int left = kb0 < nkb ? (nkb - 1 - kb0) / waves + 1 : 0;
    const auto rest = [&](auto self, auto n) {
        if constexpr (n() < kDeep) {
            if (left == n()) blocks(kb0, n);
            else self(self, std::integral_constant<int, n() + 1>{});
        }
    };
    rest(rest, std::integral_constant<int, 1>{});
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j) part[wave][i][j][lane] = acc[i][j];
    __syncthreads();
    for (int o = threadIdx.x; o < NT * MT * 64; o += blockDim.x) {
        const int l = o & 63, i = o / (64 * MT), j = o / 64 % MT;
        f32x4 v = part[0][i][j][l];
        for (int k = 1; k < waves; ++k) v += part[k][i][j][l];
        const int mm = 16 * j + (l & 15), n = n0 + 16 * i + 4 * (l >> 4);
        if (mm >= M || n >= N) continue;
        const int z = n / np;
        store4(y + static_cast<int64_t>(z) * M * np + static_cast<int64_t>(mm) * np + (n - z * np), v);
    }
}

template <typename T, int NT, int MT>
hipError_t launch_rows(const void *x, const void *xs, const void *w, const void *ws, void *y, int M, int N, int K,
                       int np, hipStream_t stream) {
    if (M > 16 * MT) return hipErrorInvalidValue;
    const int waves = min(8, (K + 127) / 128);
    linear_fp8_rows_kernel<T, NT, MT><<<(N + 16 * NT - 1) / (16 * NT), 64 * waves, 0, stream>>>(
        static_cast<const unsigned char *>(x), static_cast<const unsigned *>(xs),
        static_cast<const unsigned char *>(w), static_cast<const unsigned *>(ws), static_cast<T *>(y), M, N, K, np);
    return hipGetLastError();
}

template <typename T, typename C>
hipError_t launch_tile(const void *x, const void *xs, const void *w, const void *ws, void *y, int M, int N, int K,
                       int np, int n_cu, hipStream_t stream) {
    const int tiles_m = (M + C::BM - 1) / C::BM, tiles_n = (N + C::BN - 1) / C::BN;
    const int64_t tiles = static_cast<int64_t>(tiles_m) * tiles_n;
    if (tiles < 1 || tiles > 0x3fffffff) return hipErrorInvalidValue;
    const int64_t slots = static_cast<int64_t>(n_cu) * C::PER_CU;
    const int64_t blocks = C::KG == 1 && tiles > slots ? slots : tiles;
    linear_fp8_kernel<T, C><<<static_cast<unsigned>(blocks), C::THREADS, 0, stream>>>(
        static_cast<const unsigned char *>(x), static_cast<const unsigned *>(xs),
        static_cast<const unsigned char *>(w), static_cast<const unsigned *>(ws), static_cast<T *>(y), M, N, K, np,
        tiles_m, tiles_n);
    return hipGetLastError();
}

// The tiles in the order of kFp8Tiles and of kFp8WideTiles.
template <typename... C>
struct Tiles {
    static constexpr bool match(const Fp8TileCost *c) {
        int i = 0;
        return ((c[i].bm == C::BM && c[i].bn == C::BN && c[i].per_cu == C::PER_CU && c[i++].groups == C::KG) && ...);
    }
};
using Narrow = Tiles<Tile<256, 256, 4, 2, 2, 1>, Tile<192, 256, 2, 4, 2, 1>, Tile<128, 256, 2, 2, 3, 1>,
                     Tile<128, 128, 2, 2, 4, 1>, Tile<64, 128, 2, 2, 4, 1>, Tile<64, 64, 2, 2, 4, 2>,
                     Tile<64, 64, 1, 2, 4, 1, 2>, Tile<192, 192, 2, 2, 3, 1>, Tile<64, 128, 2, 2, 3, 1, 2>>;
using Wide = Tiles<Tile<256, 128, 4, 2, 2, 1>, Tile<128, 128, 2, 2, 2, 1, 2>, Tile<64, 64, 2, 2, 4, 2>,
                   Tile<64, 64, 1, 2, 4, 1, 2>, Tile<192, 192, 2, 2, 3, 1>>;
static_assert(Narrow::match(kFp8Tiles) && Wide::match(kFp8WideTiles));

struct ProductArgs {
    const void *x, *xs, *w, *ws;
    void *y;
    int M, N, K, np, n_cu;
    hipStream_t stream;
};
template <typename T, typename... C>
hipError_t launch_nth(Tiles<C...>, int n, const ProductArgs &p) {
    hipError_t e = hipErrorInvalidValue;
    int i = 0;
    ((i++ == n ? (void)(e = launch_tile<T, C>(p.x, p.xs, p.w, p.ws, p.y, p.M, p.N, p.K, p.np, p.n_cu, p.stream))
               : (void)0),
     ...);
    return e;
}

template <typename T>
hipError_t launch_few(const ProductArgs &p, bool wide) {
    const auto run = [&](auto nt, auto mt) {
        return launch_rows<T, nt(), mt()>(p.x, p.xs, p.w, p.ws, p.y, p.M, p.N, p.K, p.np, p.stream);
    };
    using One = std::integral_constant<int, 1>;
    using Two = std::integral_constant<int, 2>;
    using Four = std::integral_constant<int, 4>;
    if (p.M <= 16) return wide ? run(Two{}, One{}) : run(One{}, One{});
    if (p.M <= 32) return wide ? run(Two{}, Two{}) : run(One{}, Two{});
    return wide ? run(Two{}, Four{}) : run(One{}, Four{});
}

}  // namespace

hipError_t launch_linear_fp8(const void *x, const void *x_scale, const void *w, const void *w_scale, void *y, int M,
                             int N, int K, int parts, int dtype, hipStream_t stream) {
    if (M == 0 || N == 0) return hipSuccess;
    int device = 0, n_cu = 0;
    hipError_t e = hipGetDevice(&device);
    if (e == hipSuccess) e = hipDeviceGetAttribute(&n_cu, hipDeviceAttributeMultiprocessorCount, device);
    if (e != hipSuccess) return e;
    if (n_cu < 1) return hipErrorInvalidValue;
    const ProductArgs p{x, x_scale, w, w_scale, y, M, N, K, N / parts, n_cu, stream};
    if (M <= kFp8Rows) {
        const bool wide = fp8_rows_wide(N, n_cu);
        if (dtype == 0) return launch_few<__bf16>(p, wide);
        return launch_few<float>(p, wide);
    }
    if (dtype == 0) return launch_nth<__bf16>(Narrow{}, fp8_tile(kFp8Tiles, M, N, K, n_cu), p);
    return launch_nth<float>(Wide{}, fp8_tile(kFp8WideTiles, M, N, K, n_cu), p);
}

}  // namespace hcms
