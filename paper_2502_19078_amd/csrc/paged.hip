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
    int T, H, chunks, tokens;                                // chunks: of 16 bytes, of a row that is written
    int items;                                               // chunks of a token, of both outputs
};

// A thread for 16 bytes that are written, of READ_TOKENS tokens one behind the other, whose pages and rows are on their way together; eight values of
// 4 bits are one word.  Bound by the bytes of both sides (HBM): 4 x 4001 rows of 8 heads of 128 values out of 4 bits 15.4 us, 4.2 TB/s (20.7
// with a token a thread and its place by division of 64 bits; 21.8 with loads that pass by the caches).
constexpr int READ_TOKENS = 4;
template <PagedType TY>
__global__ void __launch_bounds__(256)
k_paged_read(const ReadArgs a)
{
    const int item = blockIdx.y * 256 + threadIdx.x;
    if (item >= a.items) return;
    const int c = item % a.chunks, row = item / a.chunks;
    const bool values = !a.k || row >= a.H;
    const int h = values && a.k ? row - a.H : row;
    const int64_t(&s)[3] = values ? a.v_s : a.k_s;
    const char *pool = (values ? a.pg.v : a.pg.k) + h * a.pg.sh * 16;
    const unsigned char *scales = (values ? a.pg.vs : a.pg.ks) + h * a.pg.sh;
    char *to = (values ? a.v : a.k) + h * s[2] + c * 16;
    const int first = blockIdx.x * READ_TOKENS;
    int64_t unit[READ_TOKENS];
#pragma unroll
    for (int j = 0; j < READ_TOKENS; ++j) {
        const int token = min(first + j, a.tokens - 1), pos = a.positions[token];
        const int page = pos < 0 ? -1 : paged_page(a.pg, token / a.T, pos);
        unit[j] = page < 0 ? -1 : paged_unit_at(a.pg, page, pos & ((1 << a.pg.shift) - 1));
    }
    u32x4 x[READ_TOKENS];
    unsigned int codes[READ_TOKENS], scale[READ_TOKENS];
#pragma unroll
    for (int j = 0; j < READ_TOKENS; ++j) {
        const int64_t u = unit[j] < 0 ? 0 : unit[j];         // (a row that is not there: read as the pool's first, not used)
        if (TY == PAGED_4BIT) {
            codes[j] = reinterpret_cast<const unsigned int *>(pool + u * 16)[c];
            scale[j] = scales[u + c / 4];
        } else
            x[j] = reinterpret_cast<const u32x4 *>(pool + u * 16)[c];
    }
#pragma unroll
    for (int j = 0; j < READ_TOKENS; ++j) {
        if (TY == PAGED_4BIT) x[j] = paged_bf16x8(codes[j], paged_scale(scale[j]));
        if (unit[j] < 0) x[j] = u32x4{0, 0, 0, 0};
        const int token = first + j, b = token / a.T;
        if (token < a.tokens) *reinterpret_cast<u32x4 *>(to + b * s[0] + (token - b * a.T) * s[1]) = x[j];
    }
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
    a.tokens = B * T;
    a.items = ((k_out ? 1 : 0) + (v_out ? 1 : 0)) * a.H * a.chunks;
    const dim3 grid((unsigned int)((a.tokens + READ_TOKENS - 1) / READ_TOKENS), (unsigned int)((a.items + 255) / 256)), block(256);
    hipStream_t s = (hipStream_t)hip_stream;
    if (cache->type == CLADA_PAGE_MX4) hipLaunchKernelGGL(k_paged_read<PAGED_4BIT>, grid, block, 0, s, a);
    else if (cache->type == CLADA_PAGE_BF16) hipLaunchKernelGGL(k_paged_read<PAGED_BF16>, grid, block, 0, s, a);
    else hipLaunchKernelGGL(k_paged_read<PAGED_F32>, grid, block, 0, s, a);
    CLADA_CHECK_HIP(ctx, hipGetLastError());
    return CLADA_OK;
}
