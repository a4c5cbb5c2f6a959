// Entry points of the attention calls: what they accept, and how a call is cut into workgroups.
#include <math.h>

#include "attention.h"

clada_status clada_check_kv(clada_ctx *ctx, const clada_kv_cache *c, const char *what, bool data)
{
    if (data && (!c->k || !c->v)) return clada_fail(ctx, CLADA_ERR_NULL, "%s: a pointer is NULL", what);
    if (c->dtype != CLADA_F32 && c->dtype != CLADA_BF16) return clada_fail(ctx, CLADA_ERR_DTYPE, "%s: unknown dtype %d", what, (int)c->dtype);
    if (c->d < 8 || c->d > CLADA_ATTN_MAX_D || c->d % 8)
        return clada_fail(ctx, CLADA_ERR_SHAPE, "%s: heads of %d values, not a multiple of 8 in [8,%d]", what, c->d, CLADA_ATTN_MAX_D);
    if (c->batch < 1 || c->heads < 1 || c->heads > CLADA_ATTN_MAX_HEADS || c->capacity < 1 || c->capacity > CLADA_ATTN_MAX_CAPACITY)
        return clada_fail(ctx, CLADA_ERR_SHAPE, "%s: %d sequences, %d heads, %d rows", what, c->batch, c->heads, c->capacity);
    if (c->n_sink < 0 || c->ring < 0 || (c->ring && (int64_t)c->n_sink + c->ring > c->capacity))
        return clada_fail(ctx, CLADA_ERR_SHAPE, "%s: n_sink=%d and a ring of %d rows in a capacity of %d", what, c->n_sink, c->ring, c->capacity);
    const int64_t step = 16 / (int64_t)dtype_size(c->dtype);
    if (c->stride_b < 0 || c->stride_h < 0 || c->stride_n < 0)
        return clada_fail(ctx, CLADA_ERR_SHAPE, "%s: a stride is negative", what);
    if (c->stride_b % step || c->stride_h % step || c->stride_n % step || (data && (!aligned16(c->k) || !aligned16(c->v))))
        return clada_fail(ctx, CLADA_ERR_ALIGN, "%s: pointers and strides must be multiples of 16 bytes", what);
    return CLADA_OK;
}

clada_status clada_check_heads(clada_ctx *ctx, const clada_heads *h, int32_t dtype, const char *what)
{
    if (!h) return clada_fail(ctx, CLADA_ERR_NULL, "%s is NULL", what);
    if (!h->data) return clada_fail(ctx, CLADA_ERR_NULL, "%s: the pointer is NULL", what);
    if (h->stride_b < 0 || h->stride_t < 0 || h->stride_h < 0) return clada_fail(ctx, CLADA_ERR_SHAPE, "%s: a stride is negative", what);
    const int64_t step = 16 / (int64_t)dtype_size(dtype);
    if (h->stride_b % step || h->stride_t % step || h->stride_h % step || !aligned16(h->data))
        return clada_fail(ctx, CLADA_ERR_ALIGN, "%s: pointer and strides must be multiples of 16 bytes", what);
    return CLADA_OK;
}

clada_status clada_check_out(clada_ctx *ctx, const clada_heads *h, int32_t dtype, int32_t B, int32_t T, int32_t H, int32_t d, const char *what)
{
    const clada_status st = clada_check_heads(ctx, h, dtype, what);
    if (st != CLADA_OK) return st;
    if ((B > 1 && h->stride_b < d) || (T > 1 && h->stride_t < d) || (H > 1 && h->stride_h < d))
        return clada_fail(ctx, CLADA_ERR_SHAPE, "%s: a stride below %d values puts heads on top of each other", what, d);
    return CLADA_OK;
}

namespace {

constexpr int MAX_SPLITS = 256;                              // of one row's keys
constexpr int MAX_CU = 256;                                  // of the device that the workspace bound is made for

size_t part_bytes(int64_t parts, int d) { return align_up((size_t)parts * 8, 256) + (size_t)parts * d * 4; }

AttnKV kv_of(const clada_kv_cache *c)
{
    const int64_t es = (int64_t)dtype_size(c->dtype);
    return {(const char *)c->k, (const char *)c->v, c->stride_b * es, c->stride_h * es, c->stride_n * es, c->capacity, c->n_sink, c->ring};
}

clada_status check_call(clada_ctx *ctx, const clada_kv_cache *cache, int32_t B, int32_t T, int32_t Hq, float scale, const void *lens, const void *q_lens,
                        const float *lse)
{
    if (B < 1 || T < 1 || B > CLADA_ATTN_MAX_BATCH || (int64_t)B * T > CLADA_ATTN_MAX_ROWS)
        return clada_fail(ctx, CLADA_ERR_SHAPE, "B=%d, T=%d: need B in [1,%d], T >= 1 and B*T <= %d", B, T, CLADA_ATTN_MAX_BATCH, CLADA_ATTN_MAX_ROWS);
    if (Hq < 1 || Hq > CLADA_ATTN_MAX_HEADS || Hq % cache->heads)
        return clada_fail(ctx, CLADA_ERR_SHAPE, "%d query heads: need a multiple of the cache's %d in [1,%d]", Hq, cache->heads, CLADA_ATTN_MAX_HEADS);
    if (cache->batch < B) return clada_fail(ctx, CLADA_ERR_SHAPE, "the cache holds %d sequences, the call has %d", cache->batch, B);
    if (!isfinite((float)(scale * 1.4426950408889634))) return clada_fail(ctx, CLADA_ERR_VALUE, "scale=%g is not finite, or not in base 2", scale);
    if (((uintptr_t)lens | (uintptr_t)q_lens | (uintptr_t)lse) & 3u) return clada_fail(ctx, CLADA_ERR_ALIGN, "lens, q_lens and lse must be 4-byte aligned");
    return CLADA_OK;
}

void fill(AttnArgs &a, const clada_heads *q, const clada_heads *out, const clada_kv_cache *cache, const int32_t *lens, int32_t B, int32_t T, int32_t Hq,
          float scale, float *lse)
{
    const int64_t es = (int64_t)dtype_size(cache->dtype);
    a.q = (const char *)q->data;
    a.q_sb = q->stride_b * es;
    a.q_st = q->stride_t * es;
    a.q_sh = q->stride_h * es;
    a.out = (char *)out->data;
    a.o_sb = out->stride_b * es;
    a.o_st = out->stride_t * es;
    a.o_sh = out->stride_h * es;
    a.lse = lse;
    a.kv = kv_of(cache);
    a.lens = lens;
    a.B = B;
    a.T = T;
    a.Hq = Hq;
    a.Hkv = cache->heads;
    a.G = Hq / cache->heads;
    a.D = cache->d;
    a.scale2 = (float)((double)scale * 1.4426950408889634);
}

}  // namespace

// Splits of `keys` keys for `units` tiles, so that the launch has about `wgs` workgroups; no split under 128 keys (one step of the few-row kernel's
// waves; two tiles).  One workgroup for all keys of a short sequence costs more than the launch that joins splits (513 keys of one
// head of 256 values: 26 us against 15).
int clada_attn_splits(int64_t units, int64_t keys, int64_t wgs)
{
    const int64_t want = (wgs + units - 1) / units, most = (keys + 127) / 128;
    int64_t s = want < most ? want : most;
    if (s > MAX_SPLITS) s = MAX_SPLITS;
    return s < 1 ? 1 : (int)s;
}

// Partial results into the workspace.
clada_status clada_attn_place(clada_ctx *ctx, AttnArgs &a)
{
    const int64_t parts = (int64_t)a.B * a.T * a.Hq * (a.splits + a.pre_splits);
    const size_t need = part_bytes(parts, a.D);
    if (CLADA_WS_HEADER + need > ctx->ws_bytes)
        return clada_fail(ctx, CLADA_ERR_WORKSPACE, "workspace %zu < %zu bytes", ctx->ws_bytes, CLADA_WS_HEADER + need);
    a.part_ml = (float2 *)(ctx->ws + CLADA_WS_HEADER);
    a.part_o = (float *)(ctx->ws + CLADA_WS_HEADER + align_up((size_t)parts * 8, 256));
    return CLADA_OK;
}

extern "C" {

size_t clada_attn_workspace_bytes(int32_t B, int32_t T, int32_t Hq, int32_t d)
{
    if (B < 1 || T < 1 || Hq < 1 || d < 1) return 256;
    // Partial results, one a row and split, of the largest call up to these sizes.  Tiles of 128 rows are split where there are fewer than 2 MAX_CU,
    // into 2 MAX_CU / tiles + 1 at most; tiles of 16, and a prefix's of 128, where there are fewer than MAX_CU, into MAX_CU / tiles + 1.  (A single
    // token may need the last two together.)
    const int64_t one = (int64_t)B * Hq, rows = one * T, wide = 128 * 2 * MAX_CU;
    int64_t parts = (16 + 128) * MAX_CU + 2 * one;
    if (parts > one * 2 * MAX_SPLITS) parts = one * 2 * MAX_SPLITS;
    if (T > 1) {
        int64_t many = wide + (rows < wide ? rows : wide);
        if (many > rows * MAX_SPLITS) many = rows * MAX_SPLITS;
        if (many > parts) parts = many;
    }
    return part_bytes(parts, d) + 256;
}

clada_status clada_window_attn(clada_ctx *ctx, const clada_heads *q, const clada_kv_cache *cache, const int32_t *lens, const int32_t *q_lens,
                               int32_t B, int32_t T, int32_t Hq, int32_t window, int32_t sinks, float scale, const clada_heads *out, float *lse,
                               void *hip_stream)
{
    if (!ctx) return CLADA_ERR_NULL;
    if (!cache || !lens) return clada_fail(ctx, CLADA_ERR_NULL, "cache or lens is NULL");
    clada_status st = clada_check_kv(ctx, cache, "cache", true);
    if (st != CLADA_OK) return st;
    if ((st = check_call(ctx, cache, B, T, Hq, scale, lens, q_lens, lse)) != CLADA_OK) return st;
    if (window < 0 || sinks < 0) return clada_fail(ctx, CLADA_ERR_VALUE, "window=%d, sinks=%d: negative", window, sinks);
    if (cache->ring && (window == 0 || (int64_t)window + T - 1 > cache->ring || sinks > cache->n_sink))
        return clada_fail(ctx, CLADA_ERR_SHAPE, "a ring of %d rows behind %d does not hold a window of %d for %d queries and %d sinks", cache->ring,
                          cache->n_sink, window, T, sinks);
    if ((st = clada_check_heads(ctx, q, cache->dtype, "q")) != CLADA_OK) return st;
    if ((st = clada_check_out(ctx, out, cache->dtype, B, T, Hq, cache->d, "out")) != CLADA_OK) return st;
    if (ctx->ws_bytes == 0) return clada_fail(ctx, CLADA_ERR_WORKSPACE, "context has no device");

    AttnArgs a = {};
    fill(a, q, out, cache, lens, B, T, Hq, scale, lse);
    a.q_lens = q_lens;
    a.window = cache->ring == 0 && window >= cache->capacity ? 0 : window;       // (as wide as the cache: everything)
    a.sinks = a.window ? (sinks < cache->capacity ? sinks : cache->capacity) : 0;
    const int es = (int)dtype_size(cache->dtype);
    const AttnPath path = T == 1 || T * a.G <= 16 ? ATTN_ROWS : ATTN_TILES;
    const int tile = path == ATTN_ROWS ? 16 : 128;
    a.own_tiles = (T * a.G + tile - 1) / tile;
    const int64_t units = (int64_t)B * a.Hkv * a.own_tiles;
    int64_t keys = cache->capacity;                          // what a tile can see at most
    if (a.window) {
        const int64_t seen = (int64_t)a.window + a.sinks + tile / a.G;
        if (seen < keys) keys = seen;
    }
    // Few rows: one workgroup a compute unit streams heads of 128 values and more as fast as two, with half the partial results (8 sequences of 8192
    // rows, 8 key heads of 128 values: 54.8 against 57 us); narrower ones it does not (64 values: 37.8 against 33).  Tiles take two.
    a.splits = clada_attn_splits(units, keys, path == ATTN_ROWS && cache->d >= 128 ? ctx->num_cu : 2 * ctx->num_cu);
    if (a.splits > 1 && (st = clada_attn_place(ctx, a)) != CLADA_OK) return st;
    CLADA_CHECK_HIP(ctx, clada_attn_launch(a, es, path, ctx->num_cu, (hipStream_t)hip_stream));
    return CLADA_OK;
}

clada_status clada_shared_prefix_attn(clada_ctx *ctx, const clada_heads *q, const clada_kv_cache *prefix, int32_t prefix_len,
                                      const clada_kv_cache *cache, const int32_t *lens, int32_t B, int32_t Hq, float scale, const clada_heads *out,
                                      float *lse, void *hip_stream)
{
    if (!ctx) return CLADA_ERR_NULL;
    if (!prefix || !cache || !lens) return clada_fail(ctx, CLADA_ERR_NULL, "prefix, cache or lens is NULL");
    clada_status st = clada_check_kv(ctx, cache, "cache", true);
    if (st != CLADA_OK) return st;
    if ((st = clada_check_kv(ctx, prefix, "prefix", true)) != CLADA_OK) return st;
    if ((st = check_call(ctx, cache, B, 1, Hq, scale, lens, nullptr, lse)) != CLADA_OK) return st;
    if (prefix->dtype != cache->dtype || prefix->d != cache->d || prefix->heads != cache->heads)
        return clada_fail(ctx, CLADA_ERR_SHAPE, "prefix and cache differ in type, heads or values a head");
    if (prefix->ring || cache->ring) return clada_fail(ctx, CLADA_ERR_VALUE, "rings hold a window, not a sequence behind a prefix");
    if (prefix_len < 1 || prefix_len > prefix->capacity)
        return clada_fail(ctx, CLADA_ERR_SHAPE, "prefix_len=%d outside [1,%d]", prefix_len, prefix->capacity);
    if ((st = clada_check_heads(ctx, q, cache->dtype, "q")) != CLADA_OK) return st;
    if ((st = clada_check_out(ctx, out, cache->dtype, B, 1, Hq, cache->d, "out")) != CLADA_OK) return st;
    if (ctx->ws_bytes == 0) return clada_fail(ctx, CLADA_ERR_WORKSPACE, "context has no device");

    AttnArgs a = {};
    fill(a, q, out, cache, lens, B, 1, Hq, scale, lse);
    a.pre = kv_of(prefix);
    a.pre_n = prefix_len;
    const int es = (int)dtype_size(cache->dtype);
    const AttnPath path = B * a.G <= 16 ? ATTN_ROWS : ATTN_PREFIX;
    const int tile = path == ATTN_ROWS ? 16 : 128;
    a.pre_tiles = (B * a.G + tile - 1) / tile;
    a.own_tiles = (a.G + 15) / 16;
    // One workgroup a compute unit for the prefix and one for the sequences' own keys: 16 sequences behind 8192 rows 20.2 us, with two each 27.2
    // (48 behind 4095: 38.2 and 44).
    a.pre_splits = clada_attn_splits((int64_t)a.Hkv * a.pre_tiles, prefix_len, ctx->num_cu);
    a.splits = clada_attn_splits((int64_t)B * a.Hkv * a.own_tiles, cache->capacity, ctx->num_cu);
    if ((st = clada_attn_place(ctx, a)) != CLADA_OK) return st;
    CLADA_CHECK_HIP(ctx, clada_attn_launch(a, es, path, ctx->num_cu, (hipStream_t)hip_stream));
    return CLADA_OK;
}

}  // extern "C"
