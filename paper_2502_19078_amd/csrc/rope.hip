// clada_qk_rope: norms of queries and keys for each head, rotary positions, keys and values stored into the cache, in one pass.
//
// Every value is read once and written once (HBM): a row (one head of one token) of D values lies on a group of lanes, 16 bytes each; the
// group sums the squares for the norm, and the value that a rotation pairs with comes from the same chunk (neighbouring pairs) or from a
// second load that the first level cache answers (halves).  A group takes several heads of its token, so the angles are computed once for them.
//
// The angle of pair i at position p is p * f_i.  In fp32 that product is off by 2^-24 p f_i radians: at position 100 000 more than a bf16
// value's rounding.  f_i is therefore held as a 64-bit fraction of a turn, and the integer product wraps whole turns away exactly.
#include <math.h>

#include "clada_internal.h"

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
    float eps, offset, magnitude;
    int norm;
};

template <int ES>
__device__ __forceinline__ u32x4 pack_row16(const float *f)
{
    u32x4 v;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        v[k] = ES == 2 ? (f32_to_bf16_bits(f[2 * k]) | (f32_to_bf16_bits(f[2 * k + 1]) << 16)) : __float_as_uint(f[k]);
    return v;
}

template <int ES>
__device__ __forceinline__ float load_value(const char *p, int i)
{
    return ES == 2 ? __uint_as_float((unsigned int)reinterpret_cast<const unsigned short *>(p)[i] << 16) : reinterpret_cast<const float *>(p)[i];
}

// LG lanes a row.  PAIRS: neighbouring values turn together; otherwise i and i + R/2, whose chunks face each other (FACE) or not.
template <int ES, int LG, bool PAIRS, bool FACE>
__global__ void __launch_bounds__(256)
k_qk_rope(const RopeArgs a)
{
    constexpr int E = 16 / ES;
    const int item = blockIdx.x * (256 / LG) + (int)threadIdx.x / LG;
    if (item >= a.tokens * a.slabs) return;                  // (whole groups leave)
    const int c = threadIdx.x % LG, i0 = c * E;              // this lane's values: i0 .. i0 + E - 1
    const int token = item / a.slabs, slab = item - token * a.slabs;
    const int b = token / a.T, t = token - b * a.T;
    const int pos = a.positions[token];
    const bool mine = i0 < a.D;

    // cosines and sines of this lane's values; a value outside the rotated part turns by nothing
    float cs[E], sn[E];
    int face = i0;                                           // first value of the chunk that this one pairs with
#pragma unroll
    for (int e = 0; e < E; ++e) {
        cs[e] = 1.0f;
        sn[e] = 0.0f;
        const int i = i0 + e, half = a.R / 2;
        if (i >= a.R || pos < 0) continue;
        const int pair = PAIRS ? i / 2 : (i < half ? i : i - half);
        const bool second = PAIRS ? (i & 1) : i >= half;
        const unsigned int top = (unsigned int)(((unsigned long long)(unsigned int)pos * a.turns[pair]) >> 32);
        const float turn = (float)(int)top * 0x1p-32f;       // [-1/2, 1/2]
        float s, co;
        sincospif(2.0f * turn, &s, &co);
        cs[e] = a.magnitude * co;
        sn[e] = a.magnitude * (second ? s : -s);             // partner's factor
    }
    const bool turned = i0 < a.R;
    if (!PAIRS && FACE && turned) face = i0 < a.R / 2 ? i0 + a.R / 2 : i0 - a.R / 2;

    int64_t slot = -1;
    if (a.Hk && pos >= 0) {
        if (a.slots) slot = a.slots[token];
        else slot = a.ring == 0 || pos < a.n_sink ? pos : a.n_sink + (pos - a.n_sink) % a.ring;
        if (slot >= a.capacity) slot = -1;
    }

    const int heads = a.Hq + 2 * a.Hk;
    for (int h = slab; h < heads; h += a.slabs) {
        const char *src;
        char *dst;
        const char *w;
        const bool value = h >= a.Hq + a.Hk;
        if (h < a.Hq) {
            src = a.q + b * a.q_s[0] + t * a.q_s[1] + h * a.q_s[2];
            dst = a.q_out + b * a.o_s[0] + t * a.o_s[1] + h * a.o_s[2];
            w = (const char *)a.qw;
        } else {
            if (slot < 0) break;
            const int hk = value ? h - a.Hq - a.Hk : h - a.Hq;
            src = value ? a.v + b * a.v_s[0] + t * a.v_s[1] + hk * a.v_s[2] : a.k + b * a.k_s[0] + t * a.k_s[1] + hk * a.k_s[2];
            dst = (value ? a.vc : a.kc) + b * a.c_s[0] + slot * a.c_s[1] + hk * a.c_s[2];
            w = (const char *)a.kw;
        }
        u32x4 raw = {0, 0, 0, 0};
        if (mine) raw = *reinterpret_cast<const u32x4 *>(src + c * 16);
        if (value) {                                         // values go to the cache as they are
            if (mine) *reinterpret_cast<u32x4 *>(dst + c * 16) = raw;
            continue;
        }
        if (pos < 0) {                                       // padding: a query of zeros
            if (mine) *reinterpret_cast<u32x4 *>(dst + c * 16) = u32x4{0, 0, 0, 0};
            continue;
        }
        float x[E], y[E];                                    // own values, and those that they pair with
        unpack_row16(raw, x);
        if (PAIRS) {
#pragma unroll
            for (int e = 0; e < E; ++e) y[e] = x[e ^ 1];
        } else if (FACE) {
            u32x4 other = raw;
            if (turned && mine) other = *reinterpret_cast<const u32x4 *>(src + face * ES);
            unpack_row16(other, y);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int i = i0 + e, half = a.R / 2;
                y[e] = mine && i < a.R ? load_value<ES>(src, i < half ? i + half : i - half) : x[e];
            }
        }
        if (a.norm) {
            float ss = 0.0f;
#pragma unroll
            for (int e = 0; e < E; ++e) ss = fmaf(x[e], x[e], ss);
#pragma unroll
            for (int o = LG / 2; o >= 1; o >>= 1) ss += __shfl_xor(ss, o);
            const float r = 1.0f / sqrtf(ss / (float)a.D + a.eps);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                x[e] *= r;
                y[e] *= r;
            }
            if (w && mine) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const int i = i0 + e, half = a.R / 2;
                    const int p = i >= a.R ? i : PAIRS ? i ^ 1 : i < half ? i + half : i - half;
                    x[e] *= load_value<ES>(w, i) + a.offset;
                    y[e] *= load_value<ES>(w, p) + a.offset;
                }
            }
        }
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (i0 + e < a.R) x[e] = fmaf(x[e], cs[e], y[e] * sn[e]);
        if (mine) *reinterpret_cast<u32x4 *>(dst + c * 16) = pack_row16<ES>(x);
    }
}

template <int ES, int LG>
void launch_rope(const RopeArgs &a, bool pairs, hipStream_t stream)
{
    const int per = 256 / LG;
    const dim3 grid((unsigned int)(((int64_t)a.tokens * a.slabs + per - 1) / per)), block(256);
    if (pairs)
        hipLaunchKernelGGL((k_qk_rope<ES, LG, true, false>), grid, block, 0, stream, a);
    else if ((a.R / 2) % (16 / ES) == 0)
        hipLaunchKernelGGL((k_qk_rope<ES, LG, false, true>), grid, block, 0, stream, a);
    else
        hipLaunchKernelGGL((k_qk_rope<ES, LG, false, false>), grid, block, 0, stream, a);
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

extern "C" clada_status clada_qk_rope(clada_ctx *ctx, const clada_rope *rope, const clada_head_norm *norm, int32_t B, int32_t T, int32_t Hq,
                                      const clada_heads *q, const clada_heads *k, const clada_heads *v, const int32_t *positions,
                                      const int32_t *slots, const clada_heads *q_out, const clada_kv_cache *cache, void *hip_stream)
{
    if (!ctx) return CLADA_ERR_NULL;
    if (!rope || !positions || !cache) return clada_fail(ctx, CLADA_ERR_NULL, "rope, positions or cache is NULL");
    if (!q && !k) return clada_fail(ctx, CLADA_ERR_NULL, "neither queries nor keys are given");
    if ((q && !q_out) || (!k != !v)) return clada_fail(ctx, CLADA_ERR_NULL, "queries need q_out, keys need values");
    clada_status st = clada_check_kv(ctx, cache, "cache", k != nullptr);
    if (st != CLADA_OK) return st;
    if (B < 1 || T < 1 || B > CLADA_ATTN_MAX_BATCH || (int64_t)B * T > CLADA_ATTN_MAX_ROWS)
        return clada_fail(ctx, CLADA_ERR_SHAPE, "B=%d, T=%d: need B in [1,%d], T >= 1 and B*T <= %d", B, T, CLADA_ATTN_MAX_BATCH, CLADA_ATTN_MAX_ROWS);
    if (q && (Hq < 1 || Hq > CLADA_ATTN_MAX_HEADS)) return clada_fail(ctx, CLADA_ERR_SHAPE, "Hq=%d outside [1,%d]", Hq, CLADA_ATTN_MAX_HEADS);
    if (k && cache->batch < B) return clada_fail(ctx, CLADA_ERR_SHAPE, "the cache holds %d sequences, the call has %d", cache->batch, B);
    if (k && !slots && cache->ring && T > cache->ring)
        return clada_fail(ctx, CLADA_ERR_SHAPE, "%d tokens a sequence do not fit a ring of %d rows", T, cache->ring);
    const int R = rope->rotary_dim;
    if (R < 0 || R > cache->d || R % 2) return clada_fail(ctx, CLADA_ERR_SHAPE, "rotary_dim=%d is not an even number in [0,%d]", R, cache->d);
    if (R && !rope->turns) return clada_fail(ctx, CLADA_ERR_NULL, "rope->turns is NULL");
    if (rope->layout != CLADA_ROPE_HALF && rope->layout != CLADA_ROPE_PAIRS) return clada_fail(ctx, CLADA_ERR_VALUE, "unknown rotary layout %d", (int)rope->layout);
    if (!isfinite(rope->magnitude)) return clada_fail(ctx, CLADA_ERR_VALUE, "magnitude is not finite");
    if (norm && (!(norm->eps >= 0.0f) || !isfinite(norm->eps) || !isfinite(norm->offset))) return clada_fail(ctx, CLADA_ERR_VALUE, "eps or offset out of range");
    if (((uintptr_t)rope->turns & 7u) || ((uintptr_t)positions & 3u) || ((uintptr_t)slots & 3u) ||
        (norm && (((uintptr_t)norm->q_weight | (uintptr_t)norm->k_weight) & (dtype_size(cache->dtype) - 1))))
        return clada_fail(ctx, CLADA_ERR_ALIGN, "an array is not aligned to its type");
    if (q && (st = clada_check_heads(ctx, q, cache->dtype, "q")) != CLADA_OK) return st;
    if (q && (st = clada_check_heads(ctx, q_out, cache->dtype, "q_out")) != CLADA_OK) return st;
    if (k && (st = clada_check_heads(ctx, k, cache->dtype, "k")) != CLADA_OK) return st;
    if (k && (st = clada_check_heads(ctx, v, cache->dtype, "v")) != CLADA_OK) return st;
    if (ctx->ws_bytes == 0) return clada_fail(ctx, CLADA_ERR_WORKSPACE, "context has no device");

    const int es = (int)dtype_size(cache->dtype);
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
        a.kc = (char *)cache->k;
        a.vc = (char *)cache->v;
        a.c_s[0] = cache->stride_b * es;
        a.c_s[1] = cache->stride_n * es;
        a.c_s[2] = cache->stride_h * es;
        a.Hk = cache->heads;
    }
    a.positions = positions;
    a.slots = slots;
    a.turns = (const unsigned long long *)rope->turns;
    a.T = T;
    a.tokens = B * T;
    a.D = cache->d;
    a.R = R;
    a.capacity = cache->capacity;
    a.n_sink = cache->n_sink;
    a.ring = cache->ring;
    a.magnitude = rope->magnitude;
    if (norm) {
        a.norm = 1;
        a.qw = norm->q_weight;
        a.kw = norm->k_weight;
        a.eps = norm->eps;
        a.offset = norm->offset;
    }
    // A group takes up to eight heads of a token once that leaves groups enough for the chip; fewer tokens spread over more groups.
    const int heads = a.Hq + 2 * a.Hk, chunks = a.D * es / 16;
    int lg = 8;
    while (lg < chunks) lg *= 2;
    int per = 8;
    while (per > 1 && (int64_t)a.tokens * ((heads + per - 1) / per) * lg < (int64_t)ctx->num_cu * 2048) per /= 2;
    a.slabs = (heads + per - 1) / per;
    const bool pairs = rope->layout == CLADA_ROPE_PAIRS;
    hipStream_t s = (hipStream_t)hip_stream;
    if (es == 2) {
        if (lg == 8) launch_rope<2, 8>(a, pairs, s);
        else if (lg == 16) launch_rope<2, 16>(a, pairs, s);
        else launch_rope<2, 32>(a, pairs, s);
    } else {
        if (lg == 8) launch_rope<4, 8>(a, pairs, s);
        else if (lg == 16) launch_rope<4, 16>(a, pairs, s);
        else if (lg == 32) launch_rope<4, 32>(a, pairs, s);
        else launch_rope<4, 64>(a, pairs, s);
    }
    CLADA_CHECK_HIP(ctx, hipGetLastError());
    return CLADA_OK;
}
