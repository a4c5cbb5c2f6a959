// clada_paged_attn: what it accepts, and how a call is cut into workgroups.
#include <float.h>
#include <math.h>

#include "paged.h"

extern "C" clada_status clada_paged_attn(clada_ctx *ctx, const clada_heads *q, const clada_paged_cache *cache, const int32_t *lens, const int32_t *q_lens,
                                         int32_t B, int32_t T, int32_t Hq, int32_t max_len, const clada_attn_scores *scores, const clada_heads *out,
                                         float *lse, void *hip_stream)
{
    if (!ctx) return CLADA_ERR_NULL;
    if (!cache || !lens || !scores) return clada_fail(ctx, CLADA_ERR_NULL, "cache, lens or scores is NULL");
    clada_status st = clada_check_paged(ctx, cache, "cache", true);
    if (st != CLADA_OK) return st;
    if (B < 1 || T < 1 || B > CLADA_ATTN_MAX_BATCH || (int64_t)B * T > CLADA_ATTN_MAX_ROWS)
        return clada_fail(ctx, CLADA_ERR_SHAPE, "B=%d, T=%d: need B in [1,%d], T >= 1 and B*T <= %d", B, T, CLADA_ATTN_MAX_BATCH, CLADA_ATTN_MAX_ROWS);
    if (Hq < 1 || Hq > CLADA_ATTN_MAX_HEADS || Hq % cache->heads)
        return clada_fail(ctx, CLADA_ERR_SHAPE, "%d query heads: need a multiple of the cache's %d in [1,%d]", Hq, cache->heads, CLADA_ATTN_MAX_HEADS);
    if (cache->batch < B) return clada_fail(ctx, CLADA_ERR_SHAPE, "the cache holds %d sequences, the call has %d", cache->batch, B);
    if (!isfinite(scores->scale)) return clada_fail(ctx, CLADA_ERR_VALUE, "scale is not finite");
    if (!(scores->cap >= 0.0f) || !isfinite(scores->cap)) return clada_fail(ctx, CLADA_ERR_VALUE, "cap=%g is negative or not finite", scores->cap);
    // A cap 2^100 scales away is none for products below 2^88 (tanh is its argument there to 2^-24), and its quotient could leave fp32's range; one that
    // is nothing beside the scale cuts all products but zero, as the largest quotient does.  What the scores are formed with has to be a number of
    // fp32 in base 2 too.
    const double log2e = 1.4426950408889634, quotient = scores->cap > 0.0f ? (double)scores->scale / scores->cap : 0.0;
    const bool capped = scores->cap > 0.0f && (scores->scale == 0.0f ? scores->cap * log2e <= FLT_MAX : fabs(quotient) >= 0x1p-100);
    if (fabs((capped ? scores->cap : scores->scale) * log2e) > FLT_MAX)
        return clada_fail(ctx, CLADA_ERR_VALUE, "scale=%g, cap=%g: scores beyond fp32", scores->scale, scores->cap);
    if (scores->window < 0 || max_len < 0) return clada_fail(ctx, CLADA_ERR_VALUE, "window=%d, max_len=%d: negative", scores->window, max_len);
    if (((uintptr_t)lens | (uintptr_t)q_lens | (uintptr_t)lse | (uintptr_t)scores->slopes | (uintptr_t)scores->prefix_lens | (uintptr_t)scores->first) & 3u)
        return clada_fail(ctx, CLADA_ERR_ALIGN, "lens, q_lens, lse, slopes, prefix_lens and first must be 4-byte aligned");
    const int32_t dtype = paged_dtype(cache);
    if ((st = clada_check_heads(ctx, q, dtype, "q")) != CLADA_OK) return st;
    if ((st = clada_check_out(ctx, out, dtype, B, T, Hq, cache->d, "out")) != CLADA_OK) return st;
    if (ctx->ws_bytes == 0) return clada_fail(ctx, CLADA_ERR_WORKSPACE, "context has no device");

    const int64_t es = (int64_t)dtype_size(dtype);
    PagedArgs a = {};
    a.q = (const char *)q->data;
    a.q_sb = q->stride_b * es;
    a.q_st = q->stride_t * es;
    a.q_sh = q->stride_h * es;
    a.out = (char *)out->data;
    a.o_sb = out->stride_b * es;
    a.o_st = out->stride_t * es;
    a.o_sh = out->stride_h * es;
    a.lse = lse;
    a.lens = lens;
    a.q_lens = q_lens;
    a.B = B;
    a.T = T;
    a.Hq = Hq;
    a.Hkv = cache->heads;
    a.G = Hq / cache->heads;
    a.D = cache->d;
    a.pg = clada_paged_of(cache);
    a.kv.capacity = cache->max_pages * cache->page_size;     // what lens is cut to
    if (max_len && max_len < a.kv.capacity) a.kv.capacity = max_len;
    a.window = scores->window >= a.kv.capacity ? 0 : scores->window;       // (as wide as the sequences: everything)
    a.first = scores->first;
    a.prefix_lens = scores->prefix_lens;
    a.slopes = scores->slopes;
    a.scale2 = (float)(scores->scale * log2e);
    if (capped) {
        a.cap2 = (float)(scores->cap * log2e);
        a.inv_cap_scale = (float)fmax(fmin(quotient, 3e38), -3e38);
        // The polynomial's coefficients are cap2 ratio, cap2 ratio^3 .. cap2 ratio^9 times 1 to 0.013: all of them normal numbers of fp32, or none is
        // used (an infinite one times a product of zero is no zero).
        const double ratio = fabs((double)a.inv_cap_scale), c1 = a.cap2 * ratio, c9 = a.cap2 * pow(ratio, 9.0);
        const bool fits = ratio >= 0x1p-12 && ratio <= 0x1p12 && fmin(c1, c9) >= 0x1p-118 && fmax(c1, c9) <= 0x1p120;
        a.cap_limit = fits ? 0.7f / fabsf(a.inv_cap_scale) : -1.0f;
    }
    const AttnPath path = T == 1 || T * a.G <= 16 ? ATTN_ROWS : ATTN_TILES;
    const int tile = a.tile_rows = path == ATTN_TILES ? 128 : cache->type != CLADA_PAGE_F32 && T * a.G <= 8 ? 8 : 16;
    a.own_tiles = (T * a.G + tile - 1) / tile;
    const int64_t units = (int64_t)B * a.Hkv * a.own_tiles;
    int64_t keys = a.kv.capacity;                            // what a tile can see at most
    if (a.window && !a.prefix_lens) {
        const int64_t seen = (int64_t)a.window + tile / a.G;
        if (seen < keys) keys = seen;
    }
    const bool eight_waves = cache->type == CLADA_PAGE_MX4 && cache->d <= 128;
    a.splits = clada_attn_splits(units, keys, path == ATTN_ROWS && (eight_waves || cache->d >= 128) ? ctx->num_cu : 2 * ctx->num_cu);
    a.snake = path == ATTN_TILES && units * a.splits <= 2 * ctx->num_cu;
    if (units > PAGED_MAX_ARRIVED) a.splits = 1;             // (there is a counter for each; 512 units are one split each already)
    a.arrived = (int *)(ctx->ws + PAGED_ARRIVED);
    if (a.splits > 1 && (st = clada_attn_place(ctx, a)) != CLADA_OK) return st;
    const auto launch = cache->type == CLADA_PAGE_MX4 ? clada_paged_launch_mx4 : cache->type == CLADA_PAGE_BF16 ? clada_paged_launch_bf16 : clada_paged_launch_f32;
    CLADA_CHECK_HIP(ctx, launch(a, path, ctx->num_cu, (hipStream_t)hip_stream));
    return CLADA_OK;
}
