// C entry points of the paged 4-bit cache: the append and the attention over it.
// Declarations and the contract live in hcms.h.
#include "hcms.h"

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "checks.h"
#include "hcms_internal.h"
#include "kv_cache.h"

namespace {

using hcms::aligned;
using hcms::aligned16;
using hcms::Buffer;
using hcms::check_disjoint;
using hcms::check_dtype;
using hcms::elem_bytes;
using hcms::fail;
using hcms::hip_fail;
using hcms::ok;

constexpr int kMostHeads = 1 << 15;   // the second axis of a grid
constexpr int64_t kMostCache = 1LL << 48;   // tokens of all heads: their bytes fit 63 bits

// Sizes of a cache and a batch over it.
int check_sizes(const hcms_kv_cache *c, const hcms_kv_batch *b, int T) {
    if (!c || !b) return fail(HCMS_ERR_NULL, "cache or batch is NULL");
    if (c->d != 64 && c->d != 128) return fail(HCMS_ERR_SHAPE, "d=%d must be 64 or 128", c->d);
    if (c->page < hcms::kv::kChunk || c->page % hcms::kv::kChunk != 0 || c->page > (1 << 20))
        return fail(HCMS_ERR_SHAPE, "page=%d must be a multiple of %d, at most 2^20", c->page, hcms::kv::kChunk);
    if (c->pages < 1 || c->heads < 1 || c->heads > kMostHeads)
        return fail(HCMS_ERR_SHAPE, "need pages >= 1 and heads in [1, 2^15] (pages=%d heads=%d)", c->pages, c->heads);
    if (T < 0 || b->B < 0 || b->W < 1)
        return fail(HCMS_ERR_SHAPE, "need T >= 0, B >= 0 and W >= 1 (T=%d B=%d W=%d)", T, b->B, b->W);
    // Tokens' places are counted in 32 bits, a chunk past the last one's too.
    if (static_cast<int64_t>(b->W) * c->page > INT32_MAX - 1023)
        return fail(HCMS_ERR_SHAPE, "W=%d pages of %d tokens: at most 2^31 - 1024 tokens", b->W, c->page);
    if (static_cast<int64_t>(c->pages) * c->heads > kMostCache / c->page)
        return fail(HCMS_ERR_SHAPE, "%d pages of %d heads and %d tokens: at most 2^48 together", c->pages, c->heads, c->page);
    // The grids' first axis, in threads.
    if (static_cast<int64_t>(T) + 2LL * b->B > (1 << 22))
        return fail(HCMS_ERR_SHAPE, "T=%d rows and B=%d sequences: at most 2^22 rows and half as many sequences", T, b->B);
    return HCMS_OK;
}

int64_t cache_tokens(const hcms_kv_cache *c) { return static_cast<int64_t>(c->pages) * c->heads * c->page; }

// The buffers of a cache and a batch, which are there and aligned.
int check_buffers(const hcms_kv_cache *c, const hcms_kv_batch *b, Buffer (&cache)[4], Buffer (&batch)[3]) {
    if (!c->k || !c->v || !c->k_scale || !c->v_scale) return fail(HCMS_ERR_NULL, "a buffer of the cache is NULL");
    if (!b->page_table || !b->lengths || !b->starts)
        return fail(HCMS_ERR_NULL, "page_table, lengths or starts is NULL");
    if (!aligned16(c->k) || !aligned16(c->v) || !aligned16(c->k_scale) || !aligned16(c->v_scale))
        return fail(HCMS_ERR_ALIGN, "the cache's buffers must be 16-byte aligned");
    if (!aligned(b->page_table, 4) || !aligned(b->lengths, 4) || !aligned(b->starts, 4))
        return fail(HCMS_ERR_ALIGN, "page_table, lengths and starts must be aligned to their elements");
    const int64_t n = cache_tokens(c);
    cache[0] = {"the cache's k", c->k, n * (c->d / 2)};
    cache[1] = {"the cache's v", c->v, n * (c->d / 2)};
    cache[2] = {"k_scale", c->k_scale, n * (c->d / hcms::kv::kBlock)};
    cache[3] = {"v_scale", c->v_scale, n * (c->d / hcms::kv::kBlock)};
    batch[0] = {"page_table", b->page_table, 4LL * b->B * b->W};
    batch[1] = {"lengths", b->lengths, 4LL * b->B};
    batch[2] = {"starts", b->starts, 4LL * (b->B + 1)};
    return HCMS_OK;
}

// T rows of `heads` heads that are read.
int check_rows(const hcms_kv_rows *r, const char *name, int T, int heads, int d, int es, Buffer *out) {
    if (!r->x) return fail(HCMS_ERR_NULL, "%s is NULL", name);
    for (const int64_t s : {r->token, r->head})
        if (s < 0 || s > (1LL << 40)) return fail(HCMS_ERR_SHAPE, "strides of %s must be in [0, 2^40]", name);
    if (T > 1 && r->token > hcms::kMostSpan / (T - 1))
        return fail(HCMS_ERR_SHAPE, "%d rows %lld elements apart span more than 2^60 elements", T,
                    static_cast<long long>(r->token));
    const int64_t rest = hcms::kMostSpan - (T - 1) * r->token;
    if (heads > 1 && r->head > rest / (heads - 1))
        return fail(HCMS_ERR_SHAPE, "%d heads %lld elements apart in %d rows %lld apart span more than 2^60 elements",
                    heads, static_cast<long long>(r->head), T, static_cast<long long>(r->token));
    if (!aligned(r->x, es)) return fail(HCMS_ERR_ALIGN, "%s must be aligned to its elements", name);
    *out = {name, r->x, ((T - 1) * r->token + (heads - 1) * r->head + d) * es};
    return HCMS_OK;
}

hcms::KvCache cache_of(const hcms_kv_cache *c) {
    return {static_cast<unsigned char *>(c->k), static_cast<unsigned char *>(c->v),
            static_cast<unsigned char *>(c->k_scale), static_cast<unsigned char *>(c->v_scale), c->pages, c->heads,
            c->d, c->page};
}
hcms::KvBatch batch_of(const hcms_kv_batch *b) { return {b->page_table, b->lengths, b->starts, b->B, b->W}; }

int check_queries(const hcms_kv_cache *c, int B, int T, int H, int window, int dtype) {
    int st;
    if ((st = check_dtype(dtype)) != HCMS_OK) return st;
    if (H < 0 || H % c->heads != 0) return fail(HCMS_ERR_SHAPE, "H=%d must be a multiple of the cache's %d heads", H, c->heads);
    // Rows of all heads, their tiles and those that sequences' ends cut are counted in 32 bits.
    if (static_cast<int64_t>(H) * T > (1 << 29) || static_cast<int64_t>(c->heads) * B > (1 << 21))
        return fail(HCMS_ERR_SHAPE, "T=%d rows of H=%d heads: at most 2^29 together; B=%d sequences of %d key heads: 2^21", T,
                    H, B, c->heads);
    if (window < 0) return fail(HCMS_ERR_ARG, "window=%d", window);
    return HCMS_OK;
}

}  // namespace

extern "C" {

int hcms_append_kv(const hcms_kv_cache *cache, const hcms_kv_batch *batch, const hcms_kv_rows *k, const hcms_kv_rows *v,
                   void *k_held, void *v_held, int T, const float *table, const int *grid, const int *axis_pairs,
                   int n_axes, const void *positions, int position_bytes, int layout, int dtype, void *stream) {
    int st;
    if ((st = check_sizes(cache, batch, T)) != HCMS_OK || (st = check_dtype(dtype)) != HCMS_OK) return st;
    if (!k || !v) return fail(HCMS_ERR_NULL, "k or v is NULL");
    if ((k_held == nullptr) != (v_held == nullptr))
        return fail(HCMS_ERR_NULL, "k_held and v_held are given together or not at all");
    hcms::RopeAxes ax{};
    int64_t tokens = 0, pairs = 0, entries = 0;
    if (table) {
        if ((st = hcms::rope_axes(grid, axis_pairs, n_axes, &ax, &tokens, &pairs, &entries)) != HCMS_OK) return st;
        if (2 * pairs > cache->d)
            return fail(HCMS_ERR_SHAPE, "%lld pairs in head vectors of %d", static_cast<long long>(pairs), cache->d);
    } else if (positions) {
        return fail(HCMS_ERR_NULL, "positions without a table");
    }
    if (layout != HCMS_ROPE_INTERLEAVED && layout != HCMS_ROPE_HALF) return fail(HCMS_ERR_ARG, "layout=%d", layout);
    if (positions ? position_bytes != 4 && position_bytes != 8 : position_bytes != 0)
        return fail(HCMS_ERR_ARG, "position_bytes=%d: 4 or 8 with positions, 0 without", position_bytes);
    if (T == 0 || batch->B == 0) return ok();
    Buffer held_by[4], of_batch[3], in[7];
    if ((st = check_buffers(cache, batch, held_by, of_batch)) != HCMS_OK) return st;
    const int es = elem_bytes(dtype);
    if ((st = check_rows(k, "k", T, cache->heads, cache->d, es, &in[0])) != HCMS_OK) return st;
    if ((st = check_rows(v, "v", T, cache->heads, cache->d, es, &in[1])) != HCMS_OK) return st;
    if (!aligned(table, 8) || !aligned(positions, position_bytes ? position_bytes : 1))
        return fail(HCMS_ERR_ALIGN, "table must be 8-byte aligned, positions to their elements");
    if (!aligned(k_held, es) || !aligned(v_held, es))
        return fail(HCMS_ERR_ALIGN, "k_held and v_held must be aligned to their elements");
    in[2] = {"table", table, entries * 8};
    in[3] = {"positions", positions, static_cast<int64_t>(T) * n_axes * position_bytes};
    for (int i = 0; i < 3; ++i) in[4 + i] = of_batch[i];
    const int64_t n = static_cast<int64_t>(T) * cache->heads * cache->d * es;
    const Buffer out[6] = {held_by[0], held_by[1], held_by[2], held_by[3], {"k_held", k_held, n}, {"v_held", v_held, n}};
    if ((st = check_disjoint(out, 6, in, 7)) != HCMS_OK) return st;
    const hcms::KvRows rows{k->x, v->x, k->token, k->head, v->token, v->head, k_held, v_held, T};
    const hipError_t e = hcms::launch_append_kv(cache_of(cache), batch_of(batch), rows, table, ax, positions,
                                                position_bytes == 8, static_cast<int>(2 * pairs),
                                                layout == HCMS_ROPE_HALF, dtype, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "append launch");
    return ok();
}

int hcms_cache_attention_workspace(const hcms_kv_cache *cache, const hcms_kv_batch *batch, int T, int H, int window,
                                   int dtype, int64_t *bytes) {
    int st;
    if ((st = check_sizes(cache, batch, T)) != HCMS_OK) return st;
    if (!bytes) return fail(HCMS_ERR_NULL, "bytes is NULL");
    if ((st = check_queries(cache, batch->B, T, H, window, dtype)) != HCMS_OK) return st;
    *bytes = hcms::cache_attention_workspace(cache_of(cache), batch_of(batch), T, H, window, dtype);
    return ok();
}

int hcms_cache_attention(const hcms_kv_cache *cache, const hcms_kv_batch *batch, const hcms_kv_rows *q, void *out,
                         void *workspace, int T, int H, float scale, int causal, int window, int dtype, void *stream) {
    int st;
    if ((st = check_sizes(cache, batch, T)) != HCMS_OK) return st;
    if (!q) return fail(HCMS_ERR_NULL, "q is NULL");
    if ((st = check_queries(cache, batch->B, T, H, window, dtype)) != HCMS_OK) return st;
    if (!std::isfinite(scale)) return fail(HCMS_ERR_ARG, "scale must be finite (got %g)", static_cast<double>(scale));
    if (T == 0 || batch->B == 0 || H == 0) return ok();
    Buffer in[8], held_by[4], of_batch[3];
    if ((st = check_buffers(cache, batch, held_by, of_batch)) != HCMS_OK) return st;
    const int es = elem_bytes(dtype);
    if ((st = check_rows(q, "q", T, H, cache->d, es, &in[0])) != HCMS_OK) return st;
    for (int i = 0; i < 4; ++i) in[1 + i] = held_by[i];
    for (int i = 0; i < 3; ++i) in[5 + i] = of_batch[i];
    const int64_t bytes = hcms::cache_attention_workspace(cache_of(cache), batch_of(batch), T, H, window, dtype);
    if (!out || (bytes > 0 && !workspace)) return fail(HCMS_ERR_NULL, "out or workspace is NULL");
    if (!aligned(out, es) || !aligned16(workspace))
        return fail(HCMS_ERR_ALIGN, "out must be aligned to its elements, workspace to 16 bytes");
    const Buffer o[2] = {{"out", out, static_cast<int64_t>(T) * H * cache->d * es}, {"workspace", workspace, bytes}};
    if ((st = check_disjoint(o, 2, in, 8)) != HCMS_OK) return st;
    const hcms::KvQueries rows{q->x, q->token, q->head, out, T, H, scale, causal != 0, window};
    const hipError_t e = hcms::launch_cache_attention(cache_of(cache), batch_of(batch), rows, workspace, dtype,
                                                      static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "cache attention launch");
    return ok();
}

}  // extern "C"
