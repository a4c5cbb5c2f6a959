// clada_qk_rope, clada_paged_rope: norms of queries and keys for each head, rotary positions, keys and values stored into the cache, in one pass.
//
// Every value is read once and written once (HBM): a row (one head of one token) lies on a group of lanes, two 16-byte chunks each; the group
// sums the squares for the norm, and the value that a rotation pairs with lies in the same chunk (neighbouring pairs) or in the same
// lane (halves: a lane holds the two chunks that face each other).  A group takes several heads of its token, so the angles and the
// norm's weights are taken once for them.  4096 tokens of 32 + 8 + 8 heads of 128 bf16 values with norms, one input
// time and again, which the last-level cache holds: 24 us (44 with a chunk a lane, every angle twice and weights value by value); inputs in turn, into pages:
// 33 us, 3.1 TB/s, and 1998 tokens of 96 fp32 heads of 80 33 us, 3.9.  Into pages of 4 bits those 4096 tokens take 31 us: a quarter of the bytes
// stored for k and v, but by stores of 4 bytes.
//
// The angle of pair i at position p is p * f_i.  In fp32 that product is off by 2^-24 p f_i radians: at position 100 000 more than a bf16
// value's rounding.  f_i is therefore held as a 64-bit fraction of a turn, and the integer product wraps whole turns away exactly.
#include <math.h>

#include <type_traits>

#include "paged.h"

namespace {

struct RopeArgs {
    const char *q, *k, *v;
    char *q_out, *kc, *vc;
    int64_t q_s[3], k_s[3], v_s[3], o_s[3], c_s[3];   // bytes: sequence, token (cache: row), head
    const int32_t *positions, *slots;
    const unsigned long long *turns;
    const void *qw, *kw;
    int T, tokens, Hq, Hk, D, R;                      // Hk: key heads stored (0: queries only)
    int slabs, capacity, n_sink, ring;
    float eps, offset, magnitude, inv_d;
    int norm;
    PagedKV pg;                                       // pages: kc, vc and c_s (page, row, head) as for a cache, the rest here
};

// What k and v go into: the rows of a cache, pages of the same type, pages of 4 bits.
enum RopeInto { INTO_ROWS, INTO_PAGES, INTO_4BIT };

template <int ES>
__device__ __forceinline__ u32x4 pack_row16(const float *f)
{
    u32x4 v;
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = ES == 2 ? pack_bf16(f[2 * k], f[2 * k + 1]) : __float_as_uint(f[k]);
    return v;
}

// Sum over groups of LG lanes, in every lane.
template <int LG>
__device__ __forceinline__ float group_sum(float v)
{
    v += dpp_move<0xB1, 0xf>(v);                             // quad_perm [1,0,3,2]
    v += dpp_move<0x4E, 0xf>(v);                             // quad_perm [2,3,0,1]
    if (LG >= 8) v += dpp_move<0x141, 0xf>(v);               // row_half_mirror
    if (LG >= 16) v += dpp_move<0x140, 0xf>(v);              // row_mirror
    if (LG >= 32) v += __shfl_xor(v, 16);
    return v;
}

template <int CTRL>
__device__ __forceinline__ unsigned int quad_move(unsigned int v) { return __float_as_uint(dpp_move<CTRL, 0xf>(__uint_as_float(v))); }

// A rotated value is r (x_i w_i cos + x_j w_j (+-sin)), j its partner and r the norm's factor: two coefficients for every value of a lane,
// the same for all query heads of a token, and for all key heads.
// LG lanes a row, two 16-byte chunks each.  FACE (halves, R/2 whole chunks): the two that turn into each other, so that each angle is
// computed once; otherwise neighbours.  PAIRS: neighbouring values turn together.  Neither: halves that begin inside a chunk, and in 4 bits
// those that are not whole blocks of 32, whose maximum is found over neighbouring lanes; partners are loaded one by one (4096 tokens of 32 + 8 + 8 heads of 128
// bf16 values of which 24 turn: 46 us, 22 where 32 do, one input; in 4 bits 32 of 128, or 96 of 96: 68, inputs in turn, 31 where all 128 do).
template <int ES, int LG, bool PAIRS, bool FACE, RopeInto INTO>
__global__ void __launch_bounds__(256)
k_qk_rope(const RopeArgs a)
{
    constexpr int E = 16 / ES;
    const int item = blockIdx.x * (256 / LG) + (int)threadIdx.x / LG;
    if (item >= a.tokens * a.slabs) return;                  // (whole groups leave)
    const int p = threadIdx.x % LG, half = a.R / 2;
    int ch[2] = {2 * p, 2 * p + 1};                          // this lane's chunks: values ch * E on
    if (FACE) {
        const int hc = half / E;
        ch[0] = p < hc ? p : 2 * p;
        ch[1] = p < hc ? p + hc : 2 * p + 1;
    }
    const int token = item / a.slabs, slab = item - token * a.slabs;
    const int b = token / a.T, t = token - b * a.T;
    const int pos = a.positions[token];
    const bool mine[2] = {ch[0] * E < a.D, ch[1] * E < a.D};
    auto partner = [&](int i) { return PAIRS ? i ^ 1 : i < half ? i + half : i - half; };

    // the turns of a chunk's values, as vectors where the chunk turns as a whole
    constexpr int FT = PAIRS ? E / 2 : E;
    unsigned long long f[2][FT];
#pragma unroll
    for (int k = 0; k < (FACE ? 1 : 2); ++k) {
        const int i0 = ch[k] * E;
        if ((FACE || PAIRS) && i0 + E <= a.R) {
            const ulonglong2 *from = reinterpret_cast<const ulonglong2 *>(a.turns + (PAIRS ? i0 / 2 : i0));
#pragma unroll
            for (int e = 0; e < FT; e += 2) {
                const ulonglong2 two = from[e / 2];
                f[k][e] = two.x;
                f[k][e + 1] = two.y;
            }
        } else {
#pragma unroll
            for (int e = 0; e < FT; ++e) {
                const int i = i0 + (PAIRS ? 2 * e : e);
                f[k][e] = i < a.R ? a.turns[PAIRS ? i / 2 : i < half ? i : i - half] : 0;
            }
        }
    }
    float cs[2][E], sn[2][E];                                // a value outside the rotated part turns by nothing
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if (FACE && k == 1) {                            // the same angles, the other sign
                cs[1][e] = cs[0][e];
                sn[1][e] = -sn[0][e];
                continue;
            }
            if (PAIRS && (e & 1)) {
                cs[k][e] = cs[k][e - 1];
                sn[k][e] = -sn[k][e - 1];
                continue;
            }
            cs[k][e] = 1.0f;
            sn[k][e] = 0.0f;
            const int i = ch[k] * E + e;
            if (i >= a.R || pos < 0) continue;
            const unsigned long long fi = f[k][PAIRS ? e / 2 : e];
            const unsigned int top = __umulhi((unsigned int)pos, (unsigned int)fi) + (unsigned int)pos * (unsigned int)(fi >> 32);
            const float turn = (float)(int)top * 0x1p-32f;   // [-1/2, 1/2]
            float s, co;
            if (ES == 2) {                                   // the hardware's functions take turns; off by 2^-22.9 (measured, 4 Mi turns from -1/2 to 1/2), a bf16 by 2^-9
                s = __builtin_amdgcn_sinf(turn);
                co = __builtin_amdgcn_cosf(turn);
            } else
                sincospif(2.0f * turn, &s, &co);
            cs[k][e] = a.magnitude * co;
            sn[k][e] = a.magnitude * (!PAIRS && i >= half ? s : -s);
        }

    int64_t slot = -1, home = b;                             // row of the cache, and its sequence or page
    if (INTO != INTO_ROWS) {
        home = a.Hk && pos >= 0 ? paged_page(a.pg, b, pos) : -1;
        slot = home < 0 ? -1 : pos & ((1 << a.pg.shift) - 1);
    } else if (a.Hk && pos >= 0) {
        if (a.slots) slot = a.slots[token];
        else slot = a.ring == 0 || pos < a.n_sink ? pos : a.n_sink + (pos - a.n_sink) % a.ring;
        if (slot >= a.capacity) slot = -1;
    }

    // Both chunks' values into a row of 4 bits.  The 32 values of a block lie in the same chunk slot of four neighbouring lanes (where FACE turns), or in
    // both slots of two; the largest magnitude's bits, as a number, are above infinity's where a value is NaN.
    auto store_4bit = [&](const float (&z)[2][E], char *row, unsigned char *unit) {
        if constexpr (ES == 2) {
            unsigned int top[2] = {0, 0};
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (mine[k]) top[k] = max(top[k], __float_as_uint(z[k][e]) & 0x7fffffffu);
            const bool quad = FACE && p < half / E;
            const unsigned int pair = max(top[0], top[1]), both = max(pair, quad_move<0xB1>(pair));
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                unsigned int t = max(top[k], quad_move<0xB1>(top[k]));
                t = max(t, quad_move<0x4E>(t));
                const unsigned int bits = quad ? t : both;
                const int exponent = min(max((int)((bits + 0x200000u) >> 23) - 2, 1), 252);      // (6 * 2^125 is finite, 4 * 2^126 is not)
                const bool finite = bits < 0x7f800000u;
                const float scale = finite ? __uint_as_float((unsigned int)exponent << 23) : 1.0f;
                unsigned int codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, z[k][0], z[k][1], scale, 0);
                codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, z[k][2], z[k][3], scale, 1);
                codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, z[k][4], z[k][5], scale, 2);
                codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, z[k][6], z[k][7], scale, 3);
                if (!mine[k]) continue;
                *reinterpret_cast<unsigned int *>(row + ch[k] * 4) = codes;
                if (ch[k] % 4 == 0) unit[ch[k] / 4] = finite ? (unsigned char)exponent : 255;
            }
        }
    };

    // Heads first, first + slabs, .. below n, two at once (their loads are in flight together), with the coefficients u and v.
    constexpr int N = 2;
    auto turn_heads = [&](auto four, const char *src, int64_t src_h, char *dst, int64_t dst_h, unsigned char *unit, int first, int n, const float (&u)[2][E],
                          const float (&v)[2][E]) {
        for (int h = first; h < n; h += N * a.slabs) {
            u32x4 raw[N][2];
#pragma unroll
            for (int j = 0; j < N; ++j)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    raw[j][k] = u32x4{0, 0, 0, 0};
                    if (mine[k] && h + j * a.slabs < n) raw[j][k] = *reinterpret_cast<const u32x4 *>(src + (h + j * a.slabs) * src_h + ch[k] * 16);
                }
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const int hj = h + j * a.slabs;
                if (hj >= n) break;
                float x[2][E], y[2][E];                      // own values, and those that they pair with
#pragma unroll
                for (int k = 0; k < 2; ++k) unpack_row16(raw[j][k], x[k]);
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const int i = ch[k] * E + e;
                        y[k][e] = PAIRS ? x[k][e ^ 1] : FACE ? x[1 - k][e] : i < a.R ? attn_value<ES>(src + hj * src_h, partner(i)) : 0.0f;
                    }
                float r = 1.0f;
                if (a.norm) {
                    float ss = 0.0f;
#pragma unroll
                    for (int k = 0; k < 2; ++k)
#pragma unroll
                        for (int e = 0; e < E; ++e) ss = fmaf(x[k][e], x[k][e], ss);
                    r = rsqrtf(fmaf(group_sum<LG>(ss), a.inv_d, a.eps));      // (the bare instruction takes a subnormal mean for 0)
                }
                float z[2][E];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        // (what does not turn meets no other value)
                        z[k][e] = ch[k] * E + e < a.R ? fmaf(x[k][e], u[k][e], y[k][e] * v[k][e]) : x[k][e] * u[k][e];
                        if (a.norm) z[k][e] *= r;
                    }
                    if (!four.value && mine[k]) *reinterpret_cast<u32x4 *>(dst + hj * dst_h + ch[k] * 16) = pack_row16<ES>(z[k]);
                }
                if (four.value) store_4bit(z, dst + hj * dst_h, unit + hj * a.pg.sh);
            }
        }
    };
    auto coefficients = [&](const char *w, float (&u)[2][E], float (&v)[2][E]) {
        float own[2][E];
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int e = 0; e < E; ++e) own[k][e] = 1.0f;
        const bool scaled = a.norm && w;
        if (scaled) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                if (!mine[k]) continue;
                unpack_row16(*reinterpret_cast<const u32x4 *>(w + ch[k] * 16), own[k]);
#pragma unroll
                for (int e = 0; e < E; ++e) own[k][e] += a.offset;
            }
        }
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int i = ch[k] * E + e;
                u[k][e] = cs[k][e] * own[k][e];
                v[k][e] = sn[k][e] * (PAIRS ? own[k][e ^ 1] : FACE ? own[1 - k][e] : scaled && i < a.R ? attn_value<ES>(w, partner(i)) + a.offset : 1.0f);
            }
    };

    float u[2][E], v[2][E];
    if (slab < a.Hq) {
        const char *src = a.q + b * a.q_s[0] + t * a.q_s[1];
        char *dst = a.q_out + b * a.o_s[0] + t * a.o_s[1];
        if (pos < 0) {                                       // padding: queries of zeros
            for (int h = slab; h < a.Hq; h += a.slabs)
                for (int k = 0; k < 2; ++k)
                    if (mine[k]) *reinterpret_cast<u32x4 *>(dst + h * a.o_s[2] + ch[k] * 16) = u32x4{0, 0, 0, 0};
            return;
        }
        coefficients((const char *)a.qw, u, v);
        turn_heads(std::false_type{}, src, a.q_s[2], dst, a.o_s[2], nullptr, slab, a.Hq, u, v);
    }
    if (slot < 0) return;
    const int k0 = (slab + a.slabs - a.Hq % a.slabs) % a.slabs, v0 = (slab + a.slabs - (a.Hq + a.Hk) % a.slabs) % a.slabs;
    char *kc = a.kc + home * a.c_s[0] + slot * a.c_s[1], *vc = a.vc + home * a.c_s[0] + slot * a.c_s[1];
    const int64_t units = INTO == INTO_4BIT ? paged_unit_at(a.pg, (int)home, (int)slot) : 0;      // of the scales
    if (k0 < a.Hk) {
        coefficients((const char *)a.kw, u, v);
        turn_heads(std::bool_constant<INTO == INTO_4BIT>{}, a.k + b * a.k_s[0] + t * a.k_s[1], a.k_s[2], kc, a.c_s[2], const_cast<unsigned char *>(a.pg.ks) + units,
                   k0, a.Hk, u, v);
    }
    const char *vs = a.v + b * a.v_s[0] + t * a.v_s[1];
    if (INTO == INTO_4BIT) {
        for (int h = v0; h < a.Hk; h += a.slabs) {
            float z[2][E];
#pragma unroll
            for (int k = 0; k < 2; ++k)
                unpack_row16(mine[k] ? *reinterpret_cast<const u32x4 *>(vs + h * a.v_s[2] + ch[k] * 16) : u32x4{0, 0, 0, 0}, z[k]);
            store_4bit(z, vc + h * a.c_s[2], const_cast<unsigned char *>(a.pg.vs) + units + h * a.pg.sh);
        }
        return;
    }
    for (int h = v0; h < a.Hk; h += a.slabs)                 // values go to the cache as they are
        for (int k = 0; k < 2; ++k)
            if (mine[k]) *reinterpret_cast<u32x4 *>(vc + h * a.c_s[2] + ch[k] * 16) = *reinterpret_cast<const u32x4 *>(vs + h * a.v_s[2] + ch[k] * 16);
}

template <int ES, int LG, RopeInto INTO>
void launch_into(const RopeArgs &a, bool pairs, hipStream_t stream)
{
    const int per = 256 / LG;
    const dim3 grid((unsigned int)(((int64_t)a.tokens * a.slabs + per - 1) / per)), block(256);
    if (pairs)
        hipLaunchKernelGGL((k_qk_rope<ES, LG, true, false, INTO>), grid, block, 0, stream, a);
    else if ((a.R / 2) % (INTO == INTO_4BIT ? 32 : 16 / ES) == 0)
        hipLaunchKernelGGL((k_qk_rope<ES, LG, false, true, INTO>), grid, block, 0, stream, a);
    else
        hipLaunchKernelGGL((k_qk_rope<ES, LG, false, false, INTO>), grid, block, 0, stream, a);
}

template <int ES, int LG>
void launch_rope(const RopeArgs &a, RopeInto into, bool pairs, hipStream_t stream)
{
    if (into == INTO_ROWS) launch_into<ES, LG, INTO_ROWS>(a, pairs, stream);
    else if (into == INTO_PAGES) launch_into<ES, LG, INTO_PAGES>(a, pairs, stream);
    else if constexpr (ES == 2) launch_into<ES, LG, INTO_4BIT>(a, pairs, stream);
}

}  // namespace

extern "C" clada_status clada_rope_turns(clada_ctx *ctx, int32_t rotary_dim, const clada_rope_scaling *s, uint64_t *turns, float *magnitude)
{
    if (!ctx) return CLADA_ERR_NULL;
    if (!s || !turns || !magnitude) return clada_fail(ctx, CLADA_ERR_NULL, "a pointer is NULL");
    if (rotary_dim < 2 || rotary_dim > CLADA_ATTN_MAX_D || rotary_dim % 2)
        return clada_fail(ctx, CLADA_ERR_SHAPE, "rotary_dim=%d is not an even number in [2,%d]", rotary_dim, CLADA_ATTN_MAX_D);
    const double pi2 = 6.283185307179586476925;
    if (!(s->theta >= 1.0) || !isfinite(s->theta)) return clada_fail(ctx, CLADA_ERR_VALUE, "theta=%g is not in [1,inf)", s->theta);
    if (s->kind < CLADA_ROPE_SCALE_NONE || s->kind > CLADA_ROPE_SCALE_RAMP) return clada_fail(ctx, CLADA_ERR_VALUE, "unknown scaling %d", (int)s->kind);
    const bool scaled = s->kind != CLADA_ROPE_SCALE_NONE, banded = s->kind == CLADA_ROPE_SCALE_BANDS || s->kind == CLADA_ROPE_SCALE_RAMP;
    if (scaled && (!(s->factor >= 1.0) || !isfinite(s->factor))) return clada_fail(ctx, CLADA_ERR_VALUE, "factor=%g is not in [1,inf)", s->factor);
    if (banded && (!(s->original_len >= 1.0) || !isfinite(s->original_len) || !(s->low > 0.0) || !(s->high > s->low) || !isfinite(s->high)))
        return clada_fail(ctx, CLADA_ERR_VALUE, "original_len=%g, low=%g, high=%g: need a length of 1 or more and 0 < low < high", s->original_len, s->low, s->high);
    if (s->kind == CLADA_ROPE_SCALE_RAMP && !(s->theta > 1.0)) return clada_fail(ctx, CLADA_ERR_VALUE, "the ramp needs theta > 1");
    double theta = s->theta;
    if (s->kind == CLADA_ROPE_SCALE_BASE && rotary_dim > 2) theta *= pow(s->factor, (double)rotary_dim / (rotary_dim - 2));
    double from = 0.0, to = 0.0;                             // pairs between which the ramp falls
    if (s->kind == CLADA_ROPE_SCALE_RAMP) {
        from = fmax(floor(rotary_dim * log(s->original_len / (s->high * pi2)) / (2.0 * log(theta))), 0.0);
        to = fmin(ceil(rotary_dim * log(s->original_len / (s->low * pi2)) / (2.0 * log(theta))), rotary_dim - 1.0);
    }
    for (int i = 0; i < rotary_dim / 2; ++i) {
        const double f = pow(theta, -2.0 * i / rotary_dim);
        double keep = 1.0;                                   // share of the unscaled frequency
        if (s->kind == CLADA_ROPE_SCALE_LINEAR) keep = 0.0;
        if (s->kind == CLADA_ROPE_SCALE_BANDS) keep = fmin(fmax((s->original_len * f / pi2 - s->low) / (s->high - s->low), 0.0), 1.0);
        if (s->kind == CLADA_ROPE_SCALE_RAMP) keep = 1.0 - fmin(fmax((i - from) / fmax(to - from, 0.001), 0.0), 1.0);
        const double g = scaled && s->kind != CLADA_ROPE_SCALE_BASE ? f / s->factor * (1.0 - keep) + f * keep : f;
        turns[i] = (uint64_t)(g / pi2 * 18446744073709551616.0);      // g <= 1: below 2^62
    }
    *magnitude = s->kind == CLADA_ROPE_SCALE_RAMP ? (float)(0.1 * log(s->factor) + 1.0) : 1.0f;
    return CLADA_OK;
}

namespace {

// What the two calls have in common behind their caches' own checks: k and v go to `rows` or to `paged`.
clada_status rope_call(clada_ctx *ctx, const clada_rope *rope, const clada_head_norm *norm, int32_t B, int32_t T, int32_t Hq, const clada_heads *q,
                       const clada_heads *k, const clada_heads *v, const int32_t *positions, const int32_t *slots, const clada_heads *q_out,
                       const clada_kv_cache *rows, const clada_paged_cache *paged, void *hip_stream)
{
    const int32_t d = rows ? rows->d : paged->d, heads = rows ? rows->heads : paged->heads, batch = rows ? rows->batch : paged->batch;
    const int32_t dtype = rows ? rows->dtype : paged_dtype(paged);
    clada_status st;
    if (B < 1 || T < 1 || B > CLADA_ATTN_MAX_BATCH || (int64_t)B * T > CLADA_ATTN_MAX_ROWS)
        return clada_fail(ctx, CLADA_ERR_SHAPE, "B=%d, T=%d: need B in [1,%d], T >= 1 and B*T <= %d", B, T, CLADA_ATTN_MAX_BATCH, CLADA_ATTN_MAX_ROWS);
    if (q && (Hq < 1 || Hq > CLADA_ATTN_MAX_HEADS)) return clada_fail(ctx, CLADA_ERR_SHAPE, "Hq=%d outside [1,%d]", Hq, CLADA_ATTN_MAX_HEADS);
    if (k && batch < B) return clada_fail(ctx, CLADA_ERR_SHAPE, "the cache holds %d sequences, the call has %d", batch, B);
    if (k && rows && ((heads > 1 && rows->stride_h < d) || (T > 1 && rows->capacity > 1 && rows->stride_n < d)))
        return clada_fail(ctx, CLADA_ERR_SHAPE, "cache: a stride below %d values puts what is stored on top of each other", d);
    if (k && paged && ((heads > 1 && paged->stride_h < d) || paged->stride_n < d || (paged->pages > 1 && paged->stride_p < d)))
        return clada_fail(ctx, CLADA_ERR_SHAPE, "cache: a stride below %d values puts what is stored on top of each other", d);
    if (k && rows && !slots && rows->ring && T > rows->ring)
        return clada_fail(ctx, CLADA_ERR_SHAPE, "%d tokens a sequence do not fit a ring of %d rows", T, rows->ring);
    const int R = rope->rotary_dim;
    if (R < 0 || R > d || R % 2) return clada_fail(ctx, CLADA_ERR_SHAPE, "rotary_dim=%d is not an even number in [0,%d]", R, d);
    if (R && !rope->turns) return clada_fail(ctx, CLADA_ERR_NULL, "rope->turns is NULL");
    if (rope->layout != CLADA_ROPE_HALF && rope->layout != CLADA_ROPE_PAIRS) return clada_fail(ctx, CLADA_ERR_VALUE, "unknown rotary layout %d", (int)rope->layout);
    if (!isfinite(rope->magnitude)) return clada_fail(ctx, CLADA_ERR_VALUE, "magnitude is not finite");
    if (norm && (!(norm->eps >= 0.0f) || !isfinite(norm->eps) || !isfinite(norm->offset))) return clada_fail(ctx, CLADA_ERR_VALUE, "eps or offset out of range");
    if ((((uintptr_t)positions | (uintptr_t)slots) & 3u) || !aligned16(rope->turns) || (norm && (!aligned16(norm->q_weight) || !aligned16(norm->k_weight))))
        return clada_fail(ctx, CLADA_ERR_ALIGN, "turns and weights must be 16-byte, positions and slots 4-byte aligned");
    if (q && (st = clada_check_heads(ctx, q, dtype, "q")) != CLADA_OK) return st;
    if (q && (st = clada_check_out(ctx, q_out, dtype, B, T, Hq, d, "q_out")) != CLADA_OK) return st;
    if (k && (st = clada_check_heads(ctx, k, dtype, "k")) != CLADA_OK) return st;
    if (k && (st = clada_check_heads(ctx, v, dtype, "v")) != CLADA_OK) return st;
    if (ctx->ws_bytes == 0) return clada_fail(ctx, CLADA_ERR_WORKSPACE, "context has no device");

    const int es = (int)dtype_size(dtype);
    RopeArgs a = {};
    auto view = [es](const clada_heads *h, int64_t (&s)[3]) {
        s[0] = h->stride_b * es;
        s[1] = h->stride_t * es;
        s[2] = h->stride_h * es;
        return (char *)h->data;
    };
    if (q) {
        a.q = view(q, a.q_s);
        a.q_out = view(q_out, a.o_s);
        a.Hq = Hq;
    }
    if (k) {
        a.k = view(k, a.k_s);
        a.v = view(v, a.v_s);
        a.Hk = heads;
        if (rows) {
            a.kc = (char *)rows->k;
            a.vc = (char *)rows->v;
            a.c_s[0] = rows->stride_b * es;
            a.c_s[1] = rows->stride_n * es;
            a.c_s[2] = rows->stride_h * es;
        } else {
            a.pg = clada_paged_of(paged);
            a.kc = (char *)paged->k;
            a.vc = (char *)paged->v;
            a.c_s[0] = 16 * (int64_t)a.pg.sp;
            a.c_s[1] = 16 * (int64_t)a.pg.sn;
            a.c_s[2] = 16 * a.pg.sh;
        }
    }
    a.positions = positions;
    a.slots = slots;
    a.turns = (const unsigned long long *)rope->turns;
    a.T = T;
    a.tokens = B * T;
    a.D = d;
    a.R = R;
    if (rows) {
        a.capacity = rows->capacity;
        a.n_sink = rows->n_sink;
        a.ring = rows->ring;
    }
    a.magnitude = rope->magnitude;
    a.inv_d = 1.0f / (float)d;
    if (norm) {
        a.norm = 1;
        a.qw = norm->q_weight;
        a.kw = norm->k_weight;
        a.eps = norm->eps;
        a.offset = norm->offset;
    }
    // A group takes up to eight heads of a token where that leaves sixteen waves for every compute unit; fewer tokens spread over more groups.
    const int all_heads = a.Hq + 2 * a.Hk, pairs_of_chunks = (a.D * es / 16 + 1) / 2;
    int lg = 4;
    while (lg < pairs_of_chunks) lg *= 2;
    int per = 8;
    while (per > 1 && (int64_t)a.tokens * ((all_heads + per - 1) / per) * lg < (int64_t)ctx->num_cu * 1024) per /= 2;
    a.slabs = (all_heads + per - 1) / per;
    if ((int64_t)a.tokens * a.slabs * lg > (INT64_C(1) << 31)) return clada_fail(ctx, CLADA_ERR_SHAPE, "the call has too many heads and tokens");
    const bool pairs = rope->layout == CLADA_ROPE_PAIRS;
    const RopeInto into = rows ? INTO_ROWS : paged->type == CLADA_PAGE_MX4 ? INTO_4BIT : INTO_PAGES;
    hipStream_t s = (hipStream_t)hip_stream;
    if (es == 2) {
        if (lg == 4) launch_rope<2, 4>(a, into, pairs, s);
        else if (lg == 8) launch_rope<2, 8>(a, into, pairs, s);
        else launch_rope<2, 16>(a, into, pairs, s);
    } else {
        if (lg == 4) launch_rope<4, 4>(a, into, pairs, s);
        else if (lg == 8) launch_rope<4, 8>(a, into, pairs, s);
        else if (lg == 16) launch_rope<4, 16>(a, into, pairs, s);
        else launch_rope<4, 32>(a, into, pairs, s);
    }
    CLADA_CHECK_HIP(ctx, hipGetLastError());
    return CLADA_OK;
}

}  // namespace

extern "C" clada_status clada_qk_rope(clada_ctx *ctx, const clada_rope *rope, const clada_head_norm *norm, int32_t B, int32_t T, int32_t Hq,
                                      const clada_heads *q, const clada_heads *k, const clada_heads *v, const int32_t *positions,
                                      const int32_t *slots, const clada_heads *q_out, const clada_kv_cache *cache, void *hip_stream)
{
    if (!ctx) return CLADA_ERR_NULL;
    if (!rope || !positions || !cache) return clada_fail(ctx, CLADA_ERR_NULL, "rope, positions or cache is NULL");
    if (!q && !k) return clada_fail(ctx, CLADA_ERR_NULL, "neither queries nor keys are given");
    if ((q && !q_out) || (!k != !v)) return clada_fail(ctx, CLADA_ERR_NULL, "queries need q_out, keys need values");
    const clada_status st = clada_check_kv(ctx, cache, "cache", k != nullptr);
    if (st != CLADA_OK) return st;
    return rope_call(ctx, rope, norm, B, T, Hq, q, k, v, positions, slots, q_out, cache, nullptr, hip_stream);
}

extern "C" clada_status clada_paged_rope(clada_ctx *ctx, const clada_rope *rope, const clada_head_norm *norm, int32_t B, int32_t T, int32_t Hq,
                                         const clada_heads *q, const clada_heads *k, const clada_heads *v, const int32_t *positions,
                                         const clada_heads *q_out, const clada_paged_cache *cache, void *hip_stream)
{
    if (!ctx) return CLADA_ERR_NULL;
    if (!rope || !positions || !cache) return clada_fail(ctx, CLADA_ERR_NULL, "rope, positions or cache is NULL");
    if (!q && !k) return clada_fail(ctx, CLADA_ERR_NULL, "neither queries nor keys are given");
    if ((q && !q_out) || (!k != !v)) return clada_fail(ctx, CLADA_ERR_NULL, "queries need q_out, keys need values");
    const clada_status st = clada_check_paged(ctx, cache, "cache", k != nullptr);
    if (st != CLADA_OK) return st;
    return rope_call(ctx, rope, norm, B, T, Hq, q, k, v, positions, nullptr, q_out, nullptr, cache, hip_stream);
}
