// C entry points of the operators beside the chunk loop: the RMS norm, the
// 8-bit product with its quantisation, the rotary positions, and the norm and
// rotation of head vectors in one pass.  Declarations and the contract live in
// hcms.h.
#include "hcms.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "checks.h"
#include "fp8.h"
#include "hcms_internal.h"
#include "rope_heads.h"

namespace {

using hcms::aligned;
using hcms::aligned16;
using hcms::Buffer;
using hcms::check_disjoint;
using hcms::check_dtype;
using hcms::elem_bytes;
using hcms::fail;
using hcms::hip_fail;
using hcms::kMostSpan;
using hcms::ok;
using hcms::rope_axes;

// Bytes from the first to the last element of M rows of n, ld elements apart.
int64_t span_bytes(int64_t M, int64_t n, int64_t ld, int es) { return M < 1 ? 0 : ((M - 1) * ld + n) * es; }

// Bytes of the scales of `rows` rows (or blocks of rows) of K elements.
int64_t scale_bytes(int64_t rows, int64_t K) { return (K + hcms::fp8::kGroup - 1) / hcms::fp8::kGroup * rows * 4; }

int check_eps(float eps) {
    if (!std::isfinite(eps) || eps < 0.0f)
        return fail(HCMS_ERR_ARG, "eps must be finite and >= 0 (got %g)", static_cast<double>(eps));
    return HCMS_OK;
}

int check_norm_shape(int M, int D, int dtype, int weight_dtype, float eps) {
    int st;
    if ((st = check_dtype(dtype)) != HCMS_OK || (st = check_dtype(weight_dtype)) != HCMS_OK) return st;
    if (M < 0) return fail(HCMS_ERR_SHAPE, "need M >= 0 (M=%d)", M);
    if (D < 8 || D > hcms::rms_norm_max_width())
        return fail(HCMS_ERR_SHAPE, "D=%d must be in [8, %d]", D, hcms::rms_norm_max_width());
    return check_eps(eps);
}

// M rows of n elements, ld apart: the span of any type's bytes fits 63 bits.
int check_stride(int64_t ld, int n, int M, const char *name) {
    if (ld < n || ld > (1LL << 40))
        return fail(HCMS_ERR_SHAPE, "%s=%lld is below the row's %d elements or above 2^40", name,
                    static_cast<long long>(ld), n);
    if (M > 1 && ld > kMostSpan / (M - 1))
        return fail(HCMS_ERR_SHAPE, "%d rows %lld elements apart span more than 2^60 elements", M,
                    static_cast<long long>(ld));
    return HCMS_OK;
}

int norm_forward(const void *x, const void *residual, const void *weight, void *y, void *q, void *scale, void *h,
                 int M, int D, int64_t ldx, int64_t ldr, float eps, int dtype, int weight_dtype, void *stream) {
    int st;
    if ((st = check_norm_shape(M, D, dtype, weight_dtype, eps)) != HCMS_OK) return st;
    if ((st = check_stride(ldx, D, M, "ldx")) != HCMS_OK) return st;
    if (residual && (st = check_stride(ldr, D, M, "ldr")) != HCMS_OK) return st;
    const bool f8 = q || scale;
    if (f8 && D % 16 != 0) return fail(HCMS_ERR_SHAPE, "D=%d must be a multiple of 16 for 8-bit output", D);
    if (M == 0) return ok();
    if (!x || !weight || (f8 ? !q || !scale : !y)) return fail(HCMS_ERR_NULL, "x, weight or an output is NULL");
    if ((residual == nullptr) != (h == nullptr))
        return fail(HCMS_ERR_NULL, "residual and h are given together or not at all");
    const int es = elem_bytes(dtype);
    if (!aligned(x, es) || !aligned(residual, es) || !aligned(weight, elem_bytes(weight_dtype)) || !aligned(y, es) ||
        !aligned(h, es) || !aligned16(q) || !aligned16(scale))
        return fail(HCMS_ERR_ALIGN, "buffers must be aligned to their elements, q and scale to 16 bytes");
    const int64_t n = static_cast<int64_t>(M) * D;
    const Buffer in[] = {{"x", x, span_bytes(M, D, ldx, es)},
                         {"residual", residual, span_bytes(M, D, ldr, es)},
                         {"weight", weight, static_cast<int64_t>(D) * elem_bytes(weight_dtype)}};
    const Buffer out[] = {{"y", y, n * es}, {"q", q, n}, {"scale", scale, scale_bytes(M, D)}, {"h", h, n * es}};
    if ((st = check_disjoint(out, 4, in, 3)) != HCMS_OK) return st;
    const hipError_t e = hcms::launch_rms_norm(x, residual, weight, weight_dtype == HCMS_FP32, y, q, scale, h, M, D,
                                               ldx, ldr, eps, dtype, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "rms norm launch");
    return ok();
}

// A rotation's axes, positions and head dimension; *pairs of it and its table's
// *entries.
int check_rotation(const int *grid, const int *axis_pairs, int n_axes, const void *positions, int position_bytes, int S,
                   int d, int layout, hcms::RopeAxes *ax, int64_t *pairs, int64_t *entries) {
    int64_t tokens = 0;
    const int st = rope_axes(grid, axis_pairs, n_axes, ax, &tokens, pairs, entries);
    if (st != HCMS_OK) return st;
    if (S < 0 || d < 2 || d > 2 * hcms::kRopeMaxPairs || 2 * *pairs > d)
        return fail(HCMS_ERR_SHAPE, "need S >= 0, 2 <= d <= %d and at most d / 2 pairs (S=%d d=%d pairs=%lld)",
                    2 * hcms::kRopeMaxPairs, S, d, static_cast<long long>(*pairs));
    if (layout != HCMS_ROPE_INTERLEAVED && layout != HCMS_ROPE_HALF) return fail(HCMS_ERR_ARG, "layout=%d", layout);
    if (positions ? position_bytes != 4 && position_bytes != 8 : position_bytes != 0)
        return fail(HCMS_ERR_ARG, "position_bytes=%d: 4 or 8 with positions, 0 without", position_bytes);
    if (!positions && S > tokens)
        return fail(HCMS_ERR_SHAPE, "S=%d tokens on a grid of %lld", S, static_cast<long long>(tokens));
    return HCMS_OK;
}

// The heads of a side that are read: count, address, strides, alignment.
int check_heads_in(const hcms_rope_heads *h, int S, int es, int i) {
    if (h->heads < 0 || h->heads > (1 << 16)) return fail(HCMS_ERR_SHAPE, "heads=%d", h->heads);
    if (!h->x) return fail(HCMS_ERR_NULL, "the %s heads' input is NULL", i ? "key" : "query");
    for (const int64_t s : {h->x_token, h->x_head})
        if (s < 0 || s > (1LL << 40)) return fail(HCMS_ERR_SHAPE, "strides must be in [0, 2^40]");
    if (S > 1 && h->x_token > kMostSpan / (S - 1))
        return fail(HCMS_ERR_SHAPE, "%d tokens %lld elements apart span more than 2^60 elements", S,
                    static_cast<long long>(h->x_token));
    if (!aligned(h->x, es)) return fail(HCMS_ERR_ALIGN, "buffers must be aligned to their elements");
    return HCMS_OK;
}

// What a norm of head vectors reads beside them: the table, the positions and the
// weights of the sides that have heads.
int check_norm_rope_inputs(const hcms_rope_heads *const (&sides)[2], const void *const (&weights)[2], const float *table,
                           int64_t entries, const void *positions, int position_bytes, int n_axes, int S, int d,
                           int weight_dtype, Buffer *in) {
    if (S > 0 && !table) return fail(HCMS_ERR_NULL, "table is NULL");
    if (!aligned(table, 8) || !aligned(positions, position_bytes ? position_bytes : 1))
        return fail(HCMS_ERR_ALIGN, "table must be 8-byte aligned, positions to their elements");
    in[0] = {"table", table, entries * 8};
    in[1] = {"positions", positions, static_cast<int64_t>(S) * n_axes * position_bytes};
    static const char *const name[2] = {"q_weight", "k_weight"};
    const int ws = elem_bytes(weight_dtype);
    for (int i = 0; i < 2; ++i) {
        const bool used = S > 0 && sides[i] && sides[i]->heads > 0;
        if (used && !weights[i]) return fail(HCMS_ERR_NULL, "%s is NULL", name[i]);
        if (!aligned(weights[i], ws)) return fail(HCMS_ERR_ALIGN, "%s must be aligned to its elements", name[i]);
        in[2 + i] = {name[i], weights[i], static_cast<int64_t>(d) * ws};
    }
    return HCMS_OK;
}

// The sides of a rotation, queries and keys, of S tokens and head vectors of d, whose
// outputs overlap none of the `shared` buffers, nor each other or the other's input.
int check_sides(const hcms_rope_heads *q, const hcms_rope_heads *k, const Buffer *shared, int n_shared, int S, int d,
                int dtype, hcms::RopeSide (&side)[2]) {
    int st;
    const int es = elem_bytes(dtype);
    const hcms_rope_heads *sides[2] = {q, k};
    static const char *const in_name[2] = {"q", "k"}, *const out_name[2] = {"the rotated q", "the rotated k"};
    hcms::HeadBlock in[2], out[2];   // of the sides that have heads
    bool in_place[2] = {};
    for (int i = 0; i < 2; ++i) {
        const hcms_rope_heads *h = sides[i];
        if (!h) continue;
        if (h->heads < 0 || h->heads > (1 << 16)) return fail(HCMS_ERR_SHAPE, "heads=%d", h->heads);
        if (h->heads == 0 || S == 0) continue;
        if (!h->x || !h->y) return fail(HCMS_ERR_NULL, "the %s heads' input or output is NULL", i ? "key" : "query");
        const int64_t strides[4] = {h->x_token, h->x_head, h->y_token, h->y_head};
        for (const int64_t s : strides)
            if (s < 0 || s > (1LL << 40)) return fail(HCMS_ERR_SHAPE, "strides must be in [0, 2^40]");
        for (const int64_t s : {h->x_token, h->y_token})
            if (S > 1 && s > kMostSpan / (S - 1))
                return fail(HCMS_ERR_SHAPE, "%d tokens %lld elements apart span more than 2^60 elements", S,
                            static_cast<long long>(s));
        // Distinct heads and tokens of the output do not overlap.
        const bool by_token = h->y_token >= h->y_head;
        if (h->y_head < d && h->heads > 1) return fail(HCMS_ERR_SHAPE, "output heads overlap");
        if (S > 1 && (h->y_token < d || (by_token ? h->y_token < (h->heads - 1) * h->y_head + d
                                                  : h->y_head < (S - 1) * h->y_token + d && h->heads > 1)))
            return fail(HCMS_ERR_SHAPE, "output tokens overlap");
        if (!aligned(h->x, es) || !aligned(h->y, es))
            return fail(HCMS_ERR_ALIGN, "buffers must be aligned to their elements");
        side[i] = {h->x, h->y, h->x_token, h->x_head, h->y_token, h->y_head, h->heads};
        in[i] = {reinterpret_cast<uintptr_t>(h->x), h->x_token * es, h->x_head * es, S, d * es, h->heads};
        out[i] = {reinterpret_cast<uintptr_t>(h->y), h->y_token * es, h->y_head * es, S, d * es, h->heads};
        // The strides of a single token and of a single head say nothing.
        in_place[i] = h->x == h->y && (S == 1 || h->x_token == h->y_token) && (h->heads == 1 || h->x_head == h->y_head);
        const Buffer y[] = {{out_name[i], h->y, hcms::heads_span(out[i])}};
        if ((st = check_disjoint(y, 1, shared, n_shared)) != HCMS_OK) return st;
    }
    // A head is written by one workgroup and read by it alone.  Heads are compared, not
    // a side's first and last byte: both sides may lie in one packed buffer.
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2; ++j) {
            if (side[i].H == 0 || side[j].H == 0) continue;
            if ((i != j || !in_place[i]) && hcms::heads_meet(out[i], in[j]))
                return fail(HCMS_ERR_ALIAS, "%s overlaps %s", out_name[i], in_name[j]);
            if (i < j && hcms::heads_meet(out[i], out[j]))
                return fail(HCMS_ERR_ALIAS, "%s overlaps %s", out_name[i], out_name[j]);
        }
    return HCMS_OK;
}

}  // namespace

extern "C" {

int hcms_rms_norm(const void *x, const void *residual, const void *weight, void *y, void *h, int M, int D,
                  int64_t ldx, int64_t ldr, float eps, int dtype, int weight_dtype, void *stream) {
    return norm_forward(x, residual, weight, y, nullptr, nullptr, h, M, D, ldx, ldr, eps, dtype, weight_dtype,
                        stream);
}

int hcms_rms_norm_fp8(const void *x, const void *residual, const void *weight, void *q, void *scale, void *h, int M,
                      int D, int64_t ldx, int64_t ldr, float eps, int dtype, int weight_dtype, void *stream) {
    if (M > 0 && (!q || !scale)) return fail(HCMS_ERR_NULL, "q or scale is NULL");
    if (M == 0 && D % 16 != 0) return fail(HCMS_ERR_SHAPE, "D=%d must be a multiple of 16 for 8-bit output", D);
    return norm_forward(x, residual, weight, nullptr, q, scale, h, M, D, ldx, ldr, eps, dtype, weight_dtype, stream);
}

int hcms_rms_norm_partials(int M, int D) {
    const int st = check_norm_shape(M, D, HCMS_BF16, HCMS_BF16, 0.0f);
    if (st != HCMS_OK) return st;
    ok();
    return hcms::rms_norm_partials(M, D);
}

int hcms_rms_norm_backward(const void *dy, const void *x, const void *residual, const void *dh, const void *weight,
                           void *dx, void *dw, float *partial, int M, int D, int64_t ldx, int64_t ldr, float eps,
                           int dtype, int weight_dtype, void *stream) {
    int st;
    if ((st = check_norm_shape(M, D, dtype, weight_dtype, eps)) != HCMS_OK) return st;
    if ((st = check_stride(ldx, D, M, "ldx")) != HCMS_OK) return st;
    if (residual && (st = check_stride(ldr, D, M, "ldr")) != HCMS_OK) return st;
    if (!dw) return fail(HCMS_ERR_NULL, "dw is NULL");
    if (M > 0 && (!dy || !x || !weight || !dx || !partial))
        return fail(HCMS_ERR_NULL, "dy, x, weight, dx or partial is NULL");
    const int es = elem_bytes(dtype), ws = elem_bytes(weight_dtype);
    if (!aligned(dy, es) || !aligned(x, es) || !aligned(residual, es) || !aligned(dh, es) || !aligned(weight, ws) || !aligned(dx, es) ||
        !aligned(dw, ws) || !aligned(partial, 4))
        return fail(HCMS_ERR_ALIGN, "buffers must be aligned to their elements");
    const int64_t n = static_cast<int64_t>(M) * D;
    const Buffer in[] = {{"dy", dy, n * es},
                         {"x", x, span_bytes(M, D, ldx, es)},
                         {"residual", residual, span_bytes(M, D, ldr, es)},
                         {"dh", dh, n * es},
                         {"weight", weight, static_cast<int64_t>(D) * ws}};
    const Buffer out[] = {{"dx", dx, n * es},
                          {"dw", dw, static_cast<int64_t>(D) * ws},
                          {"partial", partial, 4LL * hcms::rms_norm_partials(M, D) * D}};
    if ((st = check_disjoint(out, 3, in, 5)) != HCMS_OK) return st;
    const hipError_t e =
        hcms::launch_rms_norm_backward(dy, x, residual, dh, weight, weight_dtype == HCMS_FP32, dx, dw, partial, M, D,
                                       ldx, ldr, eps, dtype, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "rms norm backward launch");
    return ok();
}

int hcms_quantize_fp8(const void *x, void *q, void *q_scale, int q_block, void *t, void *t_scale, int t_block, int M,
                      int K, int64_t ldx, int dtype, void *stream) {
    int st;
    if ((st = check_dtype(dtype)) != HCMS_OK) return st;
    if (M < 0 || K < 16 || K % 16 != 0 || K > (1 << 20))
        return fail(HCMS_ERR_SHAPE, "need M >= 0 and K a positive multiple of 16, at most 2^20 (M=%d K=%d)", M, K);
    if ((st = check_stride(ldx, K, M, "ldx")) != HCMS_OK) return st;
    if ((q_block != 1 && q_block != hcms::fp8::kBlock) || (t_block != 1 && t_block != hcms::fp8::kBlock))
        return fail(HCMS_ERR_ARG, "scale blocks have 1 or 128 rows (q_block=%d t_block=%d)", q_block, t_block);
    if ((q == nullptr) != (q_scale == nullptr) || (t == nullptr) != (t_scale == nullptr))
        return fail(HCMS_ERR_NULL, "values and scales are given together or not at all");
    if (M == 0 || (!q && !t)) return ok();
    if (!x) return fail(HCMS_ERR_NULL, "x is NULL");
    const int es = elem_bytes(dtype);
    if (!aligned(x, es) || !aligned16(q) || !aligned16(q_scale) || !aligned16(t) || !aligned16(t_scale))
        return fail(HCMS_ERR_ALIGN, "x must be aligned to its elements, the outputs to 16 bytes");
    const int64_t mb = (static_cast<int64_t>(M) + 127) / 128, kb = (K + 127) / 128;
    const Buffer in[] = {{"x", x, span_bytes(M, K, ldx, es)}};
    const Buffer out[] = {{"q", q, static_cast<int64_t>(M) * K},
                          {"q_scale", q_scale, scale_bytes(q_block == 1 ? M : mb, K)},
                          {"t", t, (static_cast<int64_t>(M) + 15) / 16 * 16 * K},
                          {"t_scale", t_scale, scale_bytes(t_block == 1 ? K : kb, M)}};
    if ((st = check_disjoint(out, 4, in, 1)) != HCMS_OK) return st;
    hcms::QuantizeOut o{};
    o.q = static_cast<unsigned char *>(q);
    o.q_scale = static_cast<unsigned char *>(q_scale);
    o.q_square = q_block != 1;
    o.t = static_cast<unsigned char *>(t);
    o.t_scale = static_cast<unsigned char *>(t_scale);
    o.t_square = t_block != 1;
    const hipError_t e = hcms::launch_quantize_fp8(x, ldx, o, M, K, dtype, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "quantisation launch");
    return ok();
}

int hcms_linear_fp8(const void *x, const void *x_scale, const void *w, const void *w_scale, void *y, int M, int N,
                    int K, int parts, int dtype, void *stream) {
    int st;
    if ((st = check_dtype(dtype)) != HCMS_OK) return st;
    // The last tile's rows are counted in 32 bits too.
    if (M < 0 || M > INT32_MAX - 255 || N < 0 || N > (1 << 20))
        return fail(HCMS_ERR_SHAPE, "need 0 <= M <= 2^31 - 256 and 0 <= N <= 2^20 (M=%d N=%d)", M, N);
    if (K < 16 || K % 16 != 0 || K > (1 << 20))
        return fail(HCMS_ERR_SHAPE, "K=%d must be a positive multiple of 16, at most 2^20", K);
    if (parts < 1 || N % (8LL * parts) != 0)
        return fail(HCMS_ERR_SHAPE, "N=%d must be %d parts of a multiple of 8", N, parts);
    if (M == 0 || N == 0) return ok();
    if (!x || !x_scale || !w || !w_scale || !y) return fail(HCMS_ERR_NULL, "an operand, a scale or y is NULL");
    if (!aligned16(x) || !aligned16(x_scale) || !aligned16(w) || !aligned16(w_scale) || !aligned16(y))
        return fail(HCMS_ERR_ALIGN, "buffers must be 16-byte aligned");
    const Buffer in[] = {{"x", x, static_cast<int64_t>(M) * K},
                         {"x_scale", x_scale, scale_bytes(M, K)},
                         {"w", w, static_cast<int64_t>(N) * K},
                         {"w_scale", w_scale, scale_bytes((N + 127) / 128, K)}};
    const Buffer out[] = {{"y", y, static_cast<int64_t>(M) * N * elem_bytes(dtype)}};
    if ((st = check_disjoint(out, 1, in, 4)) != HCMS_OK) return st;
    const hipError_t e = hcms::launch_linear_fp8(x, x_scale, w, w_scale, y, M, N, K, parts, dtype,
                                                 static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "8-bit linear launch");
    return ok();
}

int hcms_rope_frequencies(int pairs, double base, int scaling, double factor, double original_length,
                          double beta_fast, double beta_slow, double *freqs, double *magnitude) {
    if (!freqs || !magnitude) return fail(HCMS_ERR_NULL, "freqs or magnitude is NULL");
    if (pairs < 1 || pairs > hcms::kRopeMaxPairs)
        return fail(HCMS_ERR_SHAPE, "pairs=%d must be in [1, %d]", pairs, hcms::kRopeMaxPairs);
    if (!std::isfinite(base) || !(base > 1.0)) return fail(HCMS_ERR_ARG, "base must be finite and > 1 (got %g)", base);
    if (scaling < HCMS_ROPE_UNSCALED || scaling > HCMS_ROPE_YARN) return fail(HCMS_ERR_ARG, "scaling=%d", scaling);
    if (scaling != HCMS_ROPE_UNSCALED && (!std::isfinite(factor) || !(factor >= 1.0)))
        return fail(HCMS_ERR_ARG, "factor must be finite and >= 1 (got %g)", factor);
    const double two_pi = 6.283185307179586476925;
    double fast = 0, slow = 0, lo = 0, hi = 0;
    if (scaling == HCMS_ROPE_YARN) {
        if (!std::isfinite(original_length) || !(original_length > 0) || !std::isfinite(beta_fast) ||
            !std::isfinite(beta_slow) || !(beta_slow > 0) || !(beta_fast >= beta_slow))
            return fail(HCMS_ERR_ARG, "need original_length > 0 and beta_fast >= beta_slow > 0");
        // The pair, not rounded, that turns `beta` times over the original length.
        const auto at = [&](double beta) {
            return pairs * std::log(original_length / (two_pi * beta)) / std::log(base);
        };
        fast = at(beta_fast);
        slow = at(beta_slow);
        // The mixture's ends.  The upper one may lie past the last pair, which then is
        // not slowed in full: it turns more than beta_slow times.
        lo = std::max(std::floor(fast), 0.0);
        hi = std::min(std::ceil(slow), 2.0 * pairs - 1.0);
    }
    const double b = scaling == HCMS_ROPE_NTK && pairs > 1 ? base * std::pow(factor, pairs / (pairs - 1.0)) : base;
    *magnitude = scaling == HCMS_ROPE_YARN ? 0.1 * std::log(factor) + 1.0 : 1.0;
    for (int i = 0; i < pairs; ++i) {
        double f = std::pow(b, -static_cast<double>(i) / pairs);
        if (scaling == HCMS_ROPE_LINEAR) f /= factor;
        if (scaling == HCMS_ROPE_YARN) {
            const double keep = i <= fast ? 1.0 : i >= slow ? 0.0 : 1.0 - std::min((i - lo) / (hi - lo), 1.0);
            f = f * keep + f / factor * (1.0 - keep);
        }
        freqs[i] = f;
    }
    return ok();
}

int hcms_rope_table_freqs(float *table, const int *grid, const int *axis_pairs, int n_axes, const double *freqs,
                          double magnitude, void *stream) {
    hcms::RopeAxes ax;
    int64_t tokens = 0, pairs = 0, entries = 0;
    int st;
    if ((st = rope_axes(grid, axis_pairs, n_axes, &ax, &tokens, &pairs, &entries)) != HCMS_OK) return st;
    if (!table || !freqs) return fail(HCMS_ERR_NULL, "table or freqs is NULL");
    if (pairs > hcms::kRopeMaxPairs)
        return fail(HCMS_ERR_SHAPE, "%lld pairs; the limit is %d", static_cast<long long>(pairs), hcms::kRopeMaxPairs);
    if (!aligned16(table)) return fail(HCMS_ERR_ALIGN, "table must be 16-byte aligned");
    if (!std::isfinite(magnitude)) return fail(HCMS_ERR_ARG, "magnitude must be finite (got %g)", magnitude);
    hcms::RopeFreqs f{};
    for (int i = 0; i < pairs; ++i) {
        if (!std::isfinite(freqs[i])) return fail(HCMS_ERR_ARG, "frequency %d is not finite", i);
        f.f[i] = freqs[i];
    }
    const hipError_t e = hcms::launch_rope_table_freqs(table, ax, f, magnitude, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "rope table launch");
    return ok();
}

int hcms_rope(const hcms_rope_heads *q, const hcms_rope_heads *k, const float *table, const int *grid,
              const int *axis_pairs, int n_axes, const void *positions, int position_bytes, int S, int d, int layout,
              int inverse, int dtype, void *stream) {
    int st;
    if (!q) return fail(HCMS_ERR_NULL, "q is NULL");
    if ((st = check_dtype(dtype)) != HCMS_OK) return st;
    hcms::RopeAxes ax;
    int64_t pairs = 0, entries = 0;
    if ((st = check_rotation(grid, axis_pairs, n_axes, positions, position_bytes, S, d, layout, &ax, &pairs, &entries)) !=
        HCMS_OK)
        return st;
    if (S > 0 && !table) return fail(HCMS_ERR_NULL, "table is NULL");
    if (!aligned(table, 8) || !aligned(positions, position_bytes ? position_bytes : 1))
        return fail(HCMS_ERR_ALIGN, "table must be 8-byte aligned, positions to their elements");
    const Buffer shared[2] = {{"table", table, entries * 8},
                              {"positions", positions, static_cast<int64_t>(S) * n_axes * position_bytes}};
    hcms::RopeSide side[2] = {};
    if ((st = check_sides(q, k, shared, 2, S, d, dtype, side)) != HCMS_OK) return st;
    if (S == 0 || side[0].H + side[1].H == 0) return ok();
    const hipError_t e = hcms::launch_rope(side[0], side[1], table, ax, positions, position_bytes == 8, S, d,
                                           static_cast<int>(2 * pairs), layout == HCMS_ROPE_HALF, inverse != 0, dtype,
                                           static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "rope launch");
    return ok();
}

int hcms_qk_norm_rope(const hcms_rope_heads *q, const hcms_rope_heads *k, const void *q_weight, const void *k_weight,
                      const float *table, const int *grid, const int *axis_pairs, int n_axes, const void *positions,
                      int position_bytes, int S, int d, int layout, float eps, int dtype, int weight_dtype,
                      void *stream) {
    int st;
    if (!q) return fail(HCMS_ERR_NULL, "q is NULL");
    if ((st = check_dtype(dtype)) != HCMS_OK || (st = check_dtype(weight_dtype)) != HCMS_OK) return st;
    hcms::RopeAxes ax;
    int64_t pairs = 0, entries = 0;
    if ((st = check_rotation(grid, axis_pairs, n_axes, positions, position_bytes, S, d, layout, &ax, &pairs, &entries)) !=
        HCMS_OK)
        return st;
    if ((st = check_eps(eps)) != HCMS_OK) return st;
    Buffer shared[4];
    const hcms_rope_heads *const sides[2] = {q, k};
    const void *const weights[2] = {q_weight, k_weight};
    if ((st = check_norm_rope_inputs(sides, weights, table, entries, positions, position_bytes, n_axes, S, d,
                                     weight_dtype, shared)) != HCMS_OK)
        return st;
    hcms::RopeSide side[2] = {};
    if ((st = check_sides(q, k, shared, 4, S, d, dtype, side)) != HCMS_OK) return st;
    if (S == 0 || side[0].H + side[1].H == 0) return ok();
    const hipError_t e = hcms::launch_head_norm(side[0], side[1], q_weight, k_weight, weight_dtype == HCMS_FP32, table,
                                                ax, positions, position_bytes == 8, S, d, static_cast<int>(2 * pairs),
                                                layout == HCMS_ROPE_HALF, eps, dtype, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "head norm launch");
    return ok();
}

int hcms_qk_norm_rope_partials(int S, int heads) {
    if (S < 0 || heads < 0) return fail(HCMS_ERR_SHAPE, "need S >= 0 and heads >= 0 (S=%d heads=%d)", S, heads);
    ok();
    return hcms::head_norm_partials(S, heads);
}

int hcms_qk_norm_rope_backward(const hcms_rope_heads *dq, const hcms_rope_heads *dk, const hcms_rope_heads *q,
                               const hcms_rope_heads *k, const void *q_weight, const void *k_weight, void *dq_weight,
                               void *dk_weight, float *partial, const float *table, const int *grid,
                               const int *axis_pairs, int n_axes, const void *positions, int position_bytes, int S,
                               int d, int layout, float eps, int dtype, int weight_dtype, void *stream) {
    int st;
    if (!dq || !q) return fail(HCMS_ERR_NULL, "dq or q is NULL");
    if ((dk == nullptr) != (k == nullptr)) return fail(HCMS_ERR_NULL, "k and dk are given together or not at all");
    if ((st = check_dtype(dtype)) != HCMS_OK || (st = check_dtype(weight_dtype)) != HCMS_OK) return st;
    hcms::RopeAxes ax;
    int64_t pairs = 0, entries = 0;
    if ((st = check_rotation(grid, axis_pairs, n_axes, positions, position_bytes, S, d, layout, &ax, &pairs, &entries)) !=
        HCMS_OK)
        return st;
    if ((st = check_eps(eps)) != HCMS_OK) return st;
    if (dq->heads != q->heads || (k && dk->heads != k->heads))
        return fail(HCMS_ERR_SHAPE, "the gradients have other heads than their inputs");
    Buffer in[6];
    const hcms_rope_heads *const sides[2] = {q, k};
    const void *const weights[2] = {q_weight, k_weight};
    if ((st = check_norm_rope_inputs(sides, weights, table, entries, positions, position_bytes, n_axes, S, d,
                                     weight_dtype, in)) != HCMS_OK)
        return st;
    // The inputs' heads: read only, within the strides that outputs have.
    hcms::RopeSide of[2] = {}, side[2] = {};
    static const char *const name[2] = {"q", "k"};
    const int es = elem_bytes(dtype);
    for (int i = 0; i < 2; ++i) {
        in[4 + i] = {name[i], nullptr, 0};
        const hcms_rope_heads *h = sides[i];
        if (!h || h->heads == 0 || S == 0) continue;
        if ((st = check_heads_in(h, S, es, i)) != HCMS_OK) return st;
        of[i] = {h->x, nullptr, h->x_token, h->x_head, 0, 0, h->heads};
        const hcms::HeadBlock b{reinterpret_cast<uintptr_t>(h->x), h->x_token * es, h->x_head * es, S, d * es, h->heads};
        in[4 + i].p = h->x;
        in[4 + i].bytes = hcms::heads_span(b);
    }
    if ((st = check_sides(dq, dk, in, 6, S, d, dtype, side)) != HCMS_OK) return st;
    const int heads = side[0].H + side[1].H, ws = elem_bytes(weight_dtype);
    if (heads > 0 && !partial) return fail(HCMS_ERR_NULL, "partial is NULL");
    if (!aligned(dq_weight, ws) || !aligned(dk_weight, ws) || !aligned(partial, 4))
        return fail(HCMS_ERR_ALIGN, "buffers must be aligned to their elements");
    const int64_t wb = static_cast<int64_t>(d) * ws;
    const Buffer out[] = {{"dq_weight", dq_weight, wb},
                          {"dk_weight", dk_weight, wb},
                          {"partial", partial, 4LL * hcms::head_norm_partials(S, heads) * d}};
    if ((st = check_disjoint(out, 3, in, 6)) != HCMS_OK) return st;
    // The gradients' heads, from first to last byte.
    Buffer heads_of[4];
    for (int i = 0; i < 2; ++i) {
        const hcms::HeadBlock g{0, side[i].x_token * es, side[i].x_head * es, S, d * es, side[i].H};
        const hcms::HeadBlock o{0, side[i].y_token * es, side[i].y_head * es, S, d * es, side[i].H};
        const bool some = side[i].H > 0;
        heads_of[2 * i] = {i ? "dk" : "dq", side[i].x, some ? hcms::heads_span(g) : 0};
        heads_of[2 * i + 1] = {i ? "the gradient of k" : "the gradient of q", side[i].y, some ? hcms::heads_span(o) : 0};
    }
    if ((st = check_disjoint(out, 3, heads_of, 4)) != HCMS_OK) return st;
    if (!dq_weight && !dk_weight && heads == 0) return ok();
    const hipError_t e = hcms::launch_head_norm_backward(
        of[0], of[1], side[0], side[1], q_weight, k_weight, weight_dtype == HCMS_FP32, dq_weight, dk_weight, partial,
        table, ax, positions, position_bytes == 8, S, d, static_cast<int>(2 * pairs), layout == HCMS_ROPE_HALF, eps,
        dtype, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "head norm backward launch");
    return ok();
}

}  // extern "C"
