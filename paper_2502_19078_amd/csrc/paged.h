// Shared by the sources of the paged cache: where a row lies, what 4 bits stand for, which keys a query sees and what is done to its scores.
#pragma once
#include "attention.h"

enum PagedType { PAGED_F32 = CLADA_PAGE_F32, PAGED_BF16 = CLADA_PAGE_BF16, PAGED_4BIT = CLADA_PAGE_MX4 };

// Strides in units of 16 bytes.  16 bytes of 4 bits have one byte of scales, so a row's unit is also its first scale's byte.
struct PagedKV {
    const char *k, *v;
    const unsigned char *ks, *vs;
    int64_t sh;                                              // head
    unsigned int sp, sn;                                     // page, row
    const int32_t *table;
    int64_t table_stride;
    int pages, shift, max_pages;                             // rows of a page: 2^shift
};

struct PagedArgs : AttnArgs {
    PagedKV pg;
    const int32_t *first, *prefix_lens;
    const float *slopes;
    int *arrived;                                            // splits of a tile that are done, 0 between the calls
    int snake;                                               // order of the row tiles (paged_tiles.h)
    int tile_rows;                                           // rows of a tile: 8, 16 or 128
    float cap2, inv_cap_scale;                               // cap log2(e) (0: none), scale / cap
    float cap_limit;                                         // products up to which a steady tile's polynomial serves (paged_tiles.h)
};

hipError_t clada_paged_launch_f32(const PagedArgs &a, AttnPath path, int num_cu, hipStream_t stream);
hipError_t clada_paged_launch_bf16(const PagedArgs &a, AttnPath path, int num_cu, hipStream_t stream);
hipError_t clada_paged_launch_mx4(const PagedArgs &a, AttnPath path, int num_cu, hipStream_t stream);
clada_status clada_check_paged(clada_ctx *ctx, const clada_paged_cache *c, const char *what, bool data);
PagedKV clada_paged_of(const clada_paged_cache *c);
static inline int32_t paged_dtype(const clada_paged_cache *c) { return c->type == CLADA_PAGE_F32 ? CLADA_F32 : CLADA_BF16; }

#ifdef __HIPCC__
constexpr int paged_es(PagedType ty) { return ty == PAGED_F32 ? 4 : 2; }      // bytes of a query's value
constexpr int paged_row_bytes(PagedType ty, int d) { return ty == PAGED_4BIT ? d / 2 : d * paged_es(ty); }

// The page of a sequence's position, or -1.
__device__ __forceinline__ int paged_page(const PagedKV &pg, int b, int p)
{
    const int at = p >> pg.shift;
    const int page = at < pg.max_pages ? pg.table[b * pg.table_stride + at] : -1;
    return (unsigned int)page < (unsigned int)pg.pages ? page : -1;
}

// Unit of a page's row, heads aside.
__device__ __forceinline__ int64_t paged_unit_at(const PagedKV &pg, int page, int row)
{
    return (int64_t)((unsigned long long)(unsigned int)page * pg.sp + (unsigned long long)(unsigned int)row * pg.sn);
}

// What the conversions below take for 2^(byte - 127): they use its exponent alone, so that 0 is 2^-127 too, and 255 (an infinity) gives NaN.
__device__ __forceinline__ float paged_scale(unsigned int byte) { return __uint_as_float(byte << 23); }

// Eight values of 4 bits (a word) as eight bf16.
__device__ __forceinline__ u32x4 paged_bf16x8(unsigned int codes, float unit)
{
    u32x4 v;
    v[0] = __builtin_bit_cast(unsigned int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 0));
    v[1] = __builtin_bit_cast(unsigned int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 1));
    v[2] = __builtin_bit_cast(unsigned int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 2));
    v[3] = __builtin_bit_cast(unsigned int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 3));
    return v;
}

// Keys [begin, end) that query t of sequence b sees, at position pos; all zero for one that sees nothing.
struct RowSpan { int begin, end, pos; };
__device__ __forceinline__ RowSpan paged_span(const PagedArgs &a, int b, int t, int len, int qlen)
{
    RowSpan s = {0, 0, 0};
    const int pos = len - qlen + t;
    if (t >= qlen || pos < 0) return s;
    s.pos = pos;
    s.end = pos + 1;
    if (a.prefix_lens) s.end = min(len, max(s.end, a.prefix_lens[b]));
    if (a.window) s.begin = max(0, pos - a.window + 1);
    if (a.first) s.begin = max(s.begin, a.first[(int64_t)b * a.T + t]);
    if (s.begin >= s.end) s.begin = s.end = 0;
    return s;
}

// cap log2(e) tanh(u), u = x / cap.  In 16 and 4 bits: up to |u| = 0.7 an odd polynomial of five terms (least largest error, 1.6 2^-24, found by
// weighted least squares; seven instructions of a clock each in place of three and two that take four), beyond it 1 - 2 / (1 + exp(2 u)).  Both are off
// by a few 2^-24 of cap; in fp32 calls, whose scores may be small beside it, tanhf is not.
// In units of 2^-24 cap, |u| <= 0.7: the argument's two roundings 0.9 (u / cosh^2 u <= 0.45), the polynomial 1.6, its steps 1, the products and cap2 1.8: below
// 6.  With the scale in the coefficients (paged_tiles.h), each k-th power's off by 2 k + 3 at most: 4.9, the polynomial 1.6, its steps 1.1: below 8.
constexpr float PAGED_CAP_POLY = 0.7f;
__device__ __forceinline__ float paged_cap_poly(float cap2, float u)
{
    const float s = u * u;
    float p = fmaf(0.013194188f, s, -0.05019526f);
    p = fmaf(p, s, 0.13257454f);
    p = fmaf(p, s, -0.33326973f);
    p = fmaf(p, s, 0.99999850f);
    return u * cap2 * p;
}
__device__ __forceinline__ float paged_cap_far(float cap2, float u)      // (halves, so that twice the cap, which fp32 may not hold, is never formed)
{
    return fmaf(-cap2, __builtin_amdgcn_rcpf(fmaf(0.5f, __builtin_amdgcn_exp2f(u * 2.8853900817779268f), 0.5f)), cap2);
}
template <PagedType TY>
__device__ __forceinline__ float paged_capped(float cap2, float u)
{
    if (TY == PAGED_F32) return cap2 * tanhf(u);
    return fabsf(u) > PAGED_CAP_POLY ? paged_cap_far(cap2, u) : paged_cap_poly(cap2, u);
}

// q . k of a key at `far` positions from its query -> score in log2 units.  slope2: slope log2(e).
template <PagedType TY>
__device__ __forceinline__ float paged_score(const PagedArgs &a, float dot, float slope2, float far)
{
    const float x = a.cap2 == 0.0f ? dot * a.scale2 : paged_capped<TY>(a.cap2, dot * a.inv_cap_scale);
    return a.slopes ? fmaf(-slope2, fabsf(far), x) : x;
}

// The same for a lane's scores s[k][e], e < N, of keys `far` + at(k, e) from their query.
template <PagedType TY, int N, class V, int K, class At>
__device__ __forceinline__ void paged_scores(const PagedArgs &a, V (&s)[K], float slope2, float far, At &&at)
{
    const float factor = a.cap2 == 0.0f ? a.scale2 : a.inv_cap_scale;
    unrolled<K * N>([&](auto x) { s[x / N][x % N] *= factor; });
    if (a.cap2 != 0.0f) {
        float most = 0.0f;
        if constexpr (TY != PAGED_F32) unrolled<K * N>([&](auto x) { most = fmaxf(most, fabsf(s[x / N][x % N])); });
        if (TY != PAGED_F32 && !__any(most > PAGED_CAP_POLY))
            unrolled<K * N>([&](auto x) { s[x / N][x % N] = paged_cap_poly(a.cap2, s[x / N][x % N]); });
        else
            unrolled<K * N>([&](auto x) { s[x / N][x % N] = paged_capped<TY>(a.cap2, s[x / N][x % N]); });
    }
    if (a.slopes) unrolled<K * N>([&](auto x) { s[x / N][x % N] = fmaf(-slope2, fabsf(far + (float)at(x / N, x % N)), s[x / N][x % N]); });
}

__device__ __forceinline__ float paged_slope2(const PagedArgs &a, int hq) { return a.slopes ? a.slopes[hq] * 1.4426950408889634f : 0.0f; }

// Value d of a row: `row` its first byte, `units` its first exponent.
template <PagedType TY>
__device__ __forceinline__ float paged_value(const char *row, const unsigned char *units, int d)
{
    if constexpr (TY == PAGED_4BIT) {
        typedef __attribute__((ext_vector_type(2))) float f32x2;
        const unsigned int both = reinterpret_cast<const unsigned char *>(row)[d >> 1];
        const f32x2 v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(both, paged_scale(units[d >> 5]), 0);
        return d & 1 ? v[1] : v[0];
    } else
        return attn_value<paged_es(TY)>(row, d);
}

// One row by one wave, key by key as it sees them: 64 keys' scores at once, a lane each, then their values one after the other, a lane for every 64th
// dimension.  Keys [k0, k1) of sequence b and key head h, those that the row sees.
template <PagedType TY>
__device__ __forceinline__ RowAgain paged_row(const PagedArgs &a, int b, int h, const char *q, const RowSpan &s, float slope2, int k0, int k1)
{
    const int lane = threadIdx.x & 63;
    const PagedKV &pg = a.pg;
    RowAgain r;
    r.m = NEG_INF;
    r.l = 0.0f;
    for (int j = 0; j < CLADA_ATTN_MAX_D / 64; ++j) r.o[j] = 0.0f;
    for (int base = max(k0, s.begin); base < min(k1, s.end); base += 64) {
        const int key = base + lane;
        const int page = key < min(k1, s.end) ? paged_page(pg, b, key) : -1;
        const bool see = page >= 0;
        const int at = key & ((1 << pg.shift) - 1);
        const int64_t unit = see ? paged_unit_at(pg, page, at) + h * pg.sh : 0;
        float x = NEG_INF;
        if (see) {
            float dot = 0.0f;
            for (int d = 0; d < a.D; ++d) dot = fmaf(paged_value<TY>(pg.k + unit * 16, pg.ks + unit, d), attn_value<paged_es(TY)>(q, d), dot);
            x = paged_score<TY>(a, dot, slope2, (float)(key - s.pos));
        }
        const float mn = fmaxf(r.m, wave_max(x)), f = r.m == NEG_INF ? 0.0f : __builtin_amdgcn_exp2f(r.m - mn);
        const float w = see ? __builtin_amdgcn_exp2f(x - (mn == NEG_INF ? 0.0f : mn)) : 0.0f;
        r.l = r.l * f + wave_sum(w);
        for (int j = 0; j < CLADA_ATTN_MAX_D / 64; ++j)
            if (r.m != NEG_INF) r.o[j] *= f;
        r.m = mn;
        for (unsigned long long left = __ballot(see); left; left &= left - 1) {
            const int t = __builtin_ctzll(left);
            const float wt = __shfl(w, t);
            const int64_t row = __shfl(unit, t);
            for (int j = 0; j < CLADA_ATTN_MAX_D / 64; ++j)
                if (lane + 64 * j < a.D) r.o[j] = fmaf(wt, paged_value<TY>(pg.v + row * 16, pg.vs + row, lane + 64 * j), r.o[j]);
        }
    }
    return r;
}

// Partial results go to memory and come from there, past the L2, which the workgroup that joins them need not share: a fence for the whole L2 (tried in
// every wave) took 100 us of a call.
__device__ __forceinline__ void store_past(void *to, float2 v)
{
    __hip_atomic_store(reinterpret_cast<unsigned long long *>(to), __builtin_bit_cast(unsigned long long, v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 load_past(const void *from)
{
    return __builtin_bit_cast(float2, __hip_atomic_load(reinterpret_cast<const unsigned long long *>(from), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}

// Four values of the partial outputs at once, the same way: `at` counts values from part_o on (fewer than 2^24 of them: splits are made up to two workgroups a compute unit).
constexpr int PAST_CACHES = 16;                              // the instructions' sc1
__device__ __forceinline__ void store_past4(float *part_o, unsigned int at, f32x4 v)
{
    const __amdgpu_buffer_rsrc_t all = __builtin_amdgcn_make_buffer_rsrc(part_o, 0, -1, 0x00027000);
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), all, at * 4, 0, PAST_CACHES);
}
__device__ __forceinline__ f32x4 load_past4(float *part_o, unsigned int at)
{
    const __amdgpu_buffer_rsrc_t all = __builtin_amdgcn_make_buffer_rsrc(part_o, 0, -1, 0x00027000);
    return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(all, at * 4, 0, PAST_CACHES));
}

// What a row of a split, or of a call without splits, leaves behind: by a wave that holds it as above.
template <int ES>
__device__ __forceinline__ void paged_store_row(const PagedArgs &a, const RowAgain &r, const RowAt &at, int part)
{
    const int lane = threadIdx.x & 63;
    if (a.splits > 1) {
        if (lane == 0) store_past(&a.part_ml[at.lse * a.splits + part], make_float2(r.m, r.l));
    } else if (a.lse && lane == 0)
        a.lse[at.lse] = r.l == 0.0f ? NEG_INF : r.m * 0.69314718055994531f + logf(r.l);
    for (int j = 0; j < CLADA_ATTN_MAX_D / 64; ++j) {
        const int d = lane + 64 * j;
        if (d >= a.D) continue;
        const float y = r.l == 0.0f ? 0.0f : r.o[j] / r.l;
        if (a.splits > 1) __hip_atomic_store(&a.part_o[(at.lse * a.splits + part) * a.D + d], r.o[j], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        else if (ES == 2) reinterpret_cast<unsigned short *>(a.out + at.o)[d] = (unsigned short)f32_to_bf16_bits(y);
        else reinterpret_cast<float *>(a.out + at.o)[d] = y;
    }
}
// For attention_join.h: a row whose weights sum up to nothing saw no key, or only scores of -inf.
__device__ __forceinline__ bool joined_none(const PagedArgs &, int, int, float l) { return l == 0.0f; }
#endif
