// The paged cache: what a call accepts as one, and clada_paged_read.
#include "paged.h"

clada_status clada_check_paged(clada_ctx *ctx, const clada_paged_cache *c, const char *what, bool data)
{
    if (data && (!c->k || !c->v || !c->table)) return clada_fail(ctx, CLADA_ERR_NULL, "%s: a pointer is NULL", what);
    if (c->type != CLADA_PAGE_F32 && c->type != CLADA_PAGE_BF16 && c->type != CLADA_PAGE_MX4)
        return clada_fail(ctx, CLADA_ERR_DTYPE, "%s: unknown page type %d", what, (int)c->type);
    const bool four = c->type == CLADA_PAGE_MX4;
    if (data && four && (!c->k_scales || !c->v_scales)) return clada_fail(ctx, CLADA_ERR_NULL, "%s: pages of 4 bits need scales", what);
    if (c->d < 8 || c->d > CLADA_ATTN_MAX_D || c->d % (four ? 32 : 8))
        return clada_fail(ctx, CLADA_ERR_SHAPE, "%s: heads of %d values, not a multiple of %d in [8,%d]", what, c->d, four ? 32 : 8, CLADA_ATTN_MAX_D);
    if (c->page_size < CLADA_PAGE_MIN || c->page_size > CLADA_PAGE_MAX || (c->page_size & (c->page_size - 1)))
        return clada_fail(ctx, CLADA_ERR_SHAPE, "%s: pages of %d rows, not a power of two in [%d,%d]", what, c->page_size, CLADA_PAGE_MIN, CLADA_PAGE_MAX);
    if (c->pages < 1 || c->heads < 1 || c->heads > CLADA_ATTN_MAX_HEADS || c->batch < 1 || c->max_pages < 1 ||
        (int64_t)c->max_pages * c->page_size > CLADA_ATTN_MAX_CAPACITY)
        return clada_fail(ctx, CLADA_ERR_SHAPE, "%s: %d pages of %d rows, %d heads, a table of %d x %d", what, c->pages, c->page_size, c->heads, c->batch, c->max_pages);
    if (c->stride_p < 0 || c->stride_h < 0 || c->stride_n < 0 || c->table_stride < 0) return clada_fail(ctx, CLADA_ERR_SHAPE, "%s: a stride is negative", what);
    if (c->stride_n > (INT64_C(1) << 26) || c->stride_p > (INT64_C(1) << 33))
        return clada_fail(ctx, CLADA_ERR_SHAPE, "%s: rows %lld and pages %lld values apart", what, (long long)c->stride_n, (long long)c->stride_p);
    const int64_t step = c->type == CLADA_PAGE_F32 ? 4 : four ? 32 : 8;
    if (c->stride_p % step || c->stride_h % step || c->stride_n % step || (data && (!aligned16(c->k) || !aligned16(c->v) || ((uintptr_t)c->table & 3u))))
        return clada_fail(ctx, CLADA_ERR_ALIGN, "%s: pointers and strides must be multiples of 16 bytes, the table 4-byte aligned", what);
    return CLADA_OK;
}

PagedKV clada_paged_of(const clada_paged_cache *c)
{
    PagedKV p = {};
    const bool four = c->type == CLADA_PAGE_MX4;
    auto units = [&](int64_t n) { return c->type == CLADA_PAGE_F32 ? n / 4 : four ? n / 32 : n / 8; };
    p.k = (const char *)c->k;
    p.v = (const char *)c->v;
    p.sh = units(c->stride_h);
    p.sp = (unsigned int)units(c->stride_p);
    p.sn = (unsigned int)units(c->stride_n);
    p.ks = four ? c->k_scales : nullptr;
    p.vs = four ? c->v_scales : nullptr;
    p.table = c->table;
    p.table_stride = c->table_stride;
    p.pages = c->pages;
    p.max_pages = c->max_pages;
    while ((1 << p.shift) < c->page_size) ++p.shift;
    return p;
}

namespace {

struct ReadArgs {
    PagedKV pg;
    char *k, *v;
    int64_t k_s[3], v_s[3];                                  // bytes: sequence, token, head
    const int32_t *positions;
    int T, H, chunks;                                        // 16-byte chunks of a row that is written
    int64_t items;
};

// A thread for every 16 bytes that are written: eight values of 4 bits are one word.  Bound by the bytes of both sides (HBM).
template <PagedType TY>
__global__ void __launch_bounds__(256)
k_paged_read(const ReadArgs a)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= a.items) return;
    const int c = (int)(i % a.chunks), h = (int)(i / a.chunks % a.H);
    const int64_t rest = i / a.chunks / a.H;
    const bool values = a.k ? a.v && (rest & 1) : true;
    const int token = (int)(a.k && a.v ? rest >> 1 : rest), b = token / a.T, t = token - b * a.T;
    const int pos = a.positions[token], page = pos < 0 ? -1 : paged_page(a.pg, b, pos);
    u32x4 x = {0, 0, 0, 0};
    if (page >= 0) {
        const int at = pos & ((1 << a.pg.shift) - 1);
        const int64_t unit = paged_unit_at(a.pg, page, at) + h * a.pg.sh;
        const char *from = (values ? a.pg.v : a.pg.k) + unit * 16;
        if (TY == PAGED_4BIT) {
            const unsigned char scale = (values ? a.pg.vs : a.pg.ks)[unit + c / 4];
            x = paged_bf16x8(reinterpret_cast<const unsigned int *>(from)[c], paged_scale(scale));
        } else
            x = reinterpret_cast<const u32x4 *>(from)[c];
    }
    const int64_t(&s)[3] = values ? a.v_s : a.k_s;
    *reinterpret_cast<u32x4 *>((values ? a.v : a.k) + b * s[0] + t * s[1] + h * s[2] + c * 16) = x;
}

}  // namespace

extern "C" clada_status clada_paged_read(clada_ctx *ctx, const clada_paged_cache *cache, const int32_t *positions, int32_t B, int32_t T,
                                         const clada_heads *k_out, const clada_heads *v_out, void *hip_stream)
{
    if (!ctx) return CLADA_ERR_NULL;
    if (!cache || !positions || (!k_out && !v_out)) return clada_fail(ctx, CLADA_ERR_NULL, "cache, positions or both outputs are NULL");
    clada_status st = clada_check_paged(ctx, cache, "cache", true);
    if (st != CLADA_OK) return st;
    if (B < 1 || T < 1 || B > CLADA_ATTN_MAX_BATCH || (int64_t)B * T > CLADA_ATTN_MAX_ROWS)
        return clada_fail(ctx, CLADA_ERR_SHAPE, "B=%d, T=%d: need B in [1,%d], T >= 1 and B*T <= %d", B, T, CLADA_ATTN_MAX_BATCH, CLADA_ATTN_MAX_ROWS);
    if (cache->batch < B) return clada_fail(ctx, CLADA_ERR_SHAPE, "the cache holds %d sequences, the call has %d", cache->batch, B);
    if ((uintptr_t)positions & 3u) return clada_fail(ctx, CLADA_ERR_ALIGN, "positions must be 4-byte aligned");
    const int32_t dtype = paged_dtype(cache);
    if (k_out && (st = clada_check_out(ctx, k_out, dtype, B, T, cache->heads, cache->d, "k_out")) != CLADA_OK) return st;
    if (v_out && (st = clada_check_out(ctx, v_out, dtype, B, T, cache->heads, cache->d, "v_out")) != CLADA_OK) return st;
    if (ctx->ws_bytes == 0) return clada_fail(ctx, CLADA_ERR_WORKSPACE, "context has no device");

    const int es = (int)dtype_size(dtype);
    ReadArgs a = {};
    auto view = [es](const clada_heads *h, int64_t (&s)[3]) {
        s[0] = h->stride_b * es;
        s[1] = h->stride_t * es;
        s[2] = h->stride_h * es;
        return (char *)h->data;
    };
    if (k_out) a.k = view(k_out, a.k_s);
    if (v_out) a.v = view(v_out, a.v_s);
    a.pg = clada_paged_of(cache);
    a.positions = positions;
    a.T = T;
    a.H = cache->heads;
    a.chunks = cache->d * es / 16;
    a.items = (int64_t)B * T * ((k_out ? 1 : 0) + (v_out ? 1 : 0)) * a.H * a.chunks;
    if (a.items > (INT64_C(1) << 31)) return clada_fail(ctx, CLADA_ERR_SHAPE, "the call has too many heads and tokens");
    const dim3 grid((unsigned int)((a.items + 255) / 256)), block(256);
    hipStream_t s = (hipStream_t)hip_stream;
    if (cache->type == CLADA_PAGE_MX4) hipLaunchKernelGGL(k_paged_read<PAGED_4BIT>, grid, block, 0, s, a);
    else if (cache->type == CLADA_PAGE_BF16) hipLaunchKernelGGL(k_paged_read<PAGED_BF16>, grid, block, 0, s, a);
    else hipLaunchKernelGGL(k_paged_read<PAGED_F32>, grid, block, 0, s, a);
    CLADA_CHECK_HIP(ctx, hipGetLastError());
    return CLADA_OK;
}
