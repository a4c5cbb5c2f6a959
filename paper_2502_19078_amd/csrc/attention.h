// Shared by the attention sources of libclada: what the kernels are told about a call, and how rows and keys are counted.
#pragma once
#include "clada_internal.h"

// Keys and values of one kind of row: strides in bytes.
struct AttnKV {
    const char *k, *v;
    int64_t sb, sh, sn;      // of a sequence, a head, a cache row
    int capacity, n_sink, ring;
};

// A launch works on row tiles.  A row is one query head of one query, r = i * G + g: token i of a sequence and head g of the group that
// shares a key head; with a shared prefix, i counts the sequences.  Partial results of split s of row R (R = (b T + t) Hq + hq) lie at
// [R * splits + s]: their maximum and sum (log2 units), and D unnormalised outputs.
struct AttnArgs {
    const char *q;
    char *out;
    float *lse;              // [B][T][Hq] or nullptr
    int64_t q_sb, q_st, q_sh, o_sb, o_st, o_sh;
    AttnKV kv, pre;          // pre: the shared prefix (pre_n rows), unused otherwise
    const int32_t *lens, *q_lens;
    int B, T, Hq, Hkv, G, D;
    int window, sinks;       // window 0: everything
    float scale2;            // scale * log2(e)
    int splits, pre_splits;  // splits of a sequence's own keys, and of the prefix in front of them
    int pre_n;
    int own_tiles, pre_tiles;// row tiles of one (sequence, head) / of one head's prefix
    float2 *part_ml;
    float *part_o;
};

// Which kernel: tiles of 16 rows, of 128 rows, or a shared prefix in tiles of 128 rows with the sequences' own keys in tiles of 16.  Partial
// results are joined where there are any.
enum AttnPath { ATTN_ROWS, ATTN_TILES, ATTN_PREFIX };
hipError_t clada_attn_launch(const AttnArgs &a, int es, AttnPath path, int num_cu, hipStream_t stream);

#ifdef __HIPCC__
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((address_space(3))) char lds_char;

constexpr float NEG_INF = -__builtin_inff();

__device__ __forceinline__ unsigned int pack_bf16(float lo, float hi)      // rounded to nearest even
{
    typedef __attribute__((ext_vector_type(2))) float f32x2;
    return __builtin_bit_cast(unsigned int, __builtin_convertvector((f32x2{lo, hi}), bf16x2_t));
}

// Where a row's query and output lie.
struct RowAt { int64_t q, o, lse; };
__device__ __forceinline__ RowAt row_at(const AttnArgs &a, bool pre, int b, int h, int r, int i)      // i = r / G
{
    const int hq = h * a.G + (r - i * a.G);
    const int bb = pre ? i : b, t = pre ? 0 : i;
    return {bb * a.q_sb + t * a.q_st + hq * a.q_sh, bb * a.o_sb + t * a.o_st + hq * a.o_sh, ((int64_t)bb * a.T + t) * a.Hq + hq};
}

// Four columns of a transposed read: the 16 lanes of a group name four rows of four values each (lane t: row t / 4, values 4 (t % 4) on) and
// lane t receives value t of the four rows.
__device__ __forceinline__ uint2 read_tr16(const char *p)
{
    return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3))) *)p));
}

// The keys that a tile's rows may see, in order: `head` sinks from position 0 on, then the positions from `lo` on.
struct KeyRange {
    int n, head, lo;         // keys in all
    int pos_a, pos_b;        // positions of the tile's first and last query
    int ring_base;           // position of the ring's first row at or before lo

    __device__ __forceinline__ int pos(int i) const { return i < head ? i : lo + (i - head); }
    __device__ __forceinline__ int64_t row(int p, const AttnKV &kv) const
    {
        if (kv.ring == 0 || p < kv.n_sink) return p;
        int s = p - ring_base;                               // the range is no longer than the ring: it wraps once at most
        if (s >= kv.ring) s -= kv.ring;
        return kv.n_sink + s;
    }
};

__device__ __forceinline__ KeyRange key_range(const AttnKV &kv, int first_pos, int i0, int i1, int window, int sinks)
{
    KeyRange k;
    k.pos_a = max(first_pos + i0, 0);
    k.pos_b = first_pos + i1;
    k.n = k.head = k.lo = 0;
    k.ring_base = kv.n_sink;
    if (i1 < i0 || k.pos_b < 0) return k;
    k.lo = window ? max(0, k.pos_a - window + 1) : 0;
    k.head = min(sinks, k.lo);
    k.n = k.head + (k.pos_b - k.lo + 1);
    if (kv.ring && k.lo > kv.n_sink) k.ring_base = kv.n_sink + (k.lo - kv.n_sink) / kv.ring * kv.ring;
    return k;
}

// Which of the keys base, base + 1, ... of a range, up to `end`, the row at position row_pos sees: comparisons of small constants with a few
// numbers.  Keys below kr.head are sinks that all rows of the range see (rows at negative positions see nothing, whatever this says).
struct Sight {
    int end, head, causal, recent, sink;
    __device__ __forceinline__ bool operator()(int c) const
    {
        return (c < end) & ((c < head) | ((c <= causal) & ((c > recent) | (c < sink))));
    }
};
__device__ __forceinline__ Sight sight(const KeyRange &kr, int base, int end, int row_pos, int window, int sinks)
{
    const int p0 = kr.lo - kr.head + base;                   // position of key `base` if it is no sink
    return {end - base, kr.head - base, row_pos - p0, window ? row_pos - window - p0 : INT32_MIN, sinks - p0};
}

// Tokens that a sequence holds and queries that the call brings for it, whatever the arrays say.
__device__ __forceinline__ void sequence_lens(const AttnArgs &a, int len_b, int qlen_b, int &len, int &qlen)
{
    len = max(len_b, 0);
    if (a.kv.ring == 0) len = min(len, a.kv.capacity);
    qlen = min(max(qlen_b, 0), a.T);
}

// A product over a tile gives every row every key of it, and a weight of zero (or the lower half of a weight) times a value that is not finite
// is no zero.  A row whose outputs are not finite is therefore computed a second time by one wave, key by key as it sees them: 64 keys'
// scores at once, a lane each, then their values one after the other, a lane for every 64th dimension.  It also serves a row whose weights
// have outgrown fp32 (attention_tiles.h).  Any other row whose sum is NaN stays: a NaN score makes every output NaN.
struct RowAgain { float m, l, o[CLADA_ATTN_MAX_D / 64]; };

template <int ES>
__device__ __forceinline__ float attn_value(const char *row, int d)
{
    return ES == 2 ? __uint_as_float((unsigned int)reinterpret_cast<const unsigned short *>(row)[d] << 16) : reinterpret_cast<const float *>(row)[d];
}

template <int ES>
__device__ __forceinline__ RowAgain attn_row_again(const AttnArgs &a, const KeyRange &kr, const AttnKV &kv, const char *kp, const char *vp, const char *q,
                                                   int row_pos, int k0, int k1)
{
    const int lane = threadIdx.x & 63;
    RowAgain r;
    r.m = NEG_INF;
    r.l = 0.0f;
    for (int j = 0; j < CLADA_ATTN_MAX_D / 64; ++j) r.o[j] = 0.0f;
    for (int base = k0; base < k1; base += 64) {
        const int key = base + lane, p = kr.pos(min(key, k1 - 1));
        const bool see = key < k1 && p <= row_pos && (a.window == 0 || p > row_pos - a.window || p < a.sinks);
        const int64_t off = kr.row(p, kv) * kv.sn;
        float x = NEG_INF;
        if (see) {
            float s = 0.0f;
            for (int d = 0; d < a.D; ++d) s = fmaf(attn_value<ES>(kp + off, d), attn_value<ES>(q, d), s);
            x = s * a.scale2;
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
            const int64_t row = __shfl(off, t);
            for (int j = 0; j < CLADA_ATTN_MAX_D / 64; ++j)
                if (lane + 64 * j < a.D) r.o[j] = fmaf(wt, attn_value<ES>(vp + row, lane + 64 * j), r.o[j]);
        }
    }
    return r;
}

// What a row of a split, or of a call without splits, leaves behind: by a wave that holds it as above.
template <int ES>
__device__ __forceinline__ void attn_store_again(const AttnArgs &a, const RowAgain &r, const RowAt &at, int part)
{
    const int lane = threadIdx.x & 63, splits = a.splits + a.pre_splits;
    if (splits > 1) {
        if (lane == 0) a.part_ml[at.lse * splits + part] = make_float2(r.m, r.l);
    } else if (a.lse && lane == 0)
        a.lse[at.lse] = r.m * 0.69314718055994531f + logf(r.l);
    for (int j = 0; j < CLADA_ATTN_MAX_D / 64; ++j) {
        const int d = lane + 64 * j;
        if (d >= a.D) continue;
        if (splits > 1) a.part_o[(at.lse * splits + part) * a.D + d] = r.o[j];
        else if (ES == 2) reinterpret_cast<unsigned short *>(a.out + at.o)[d] = (unsigned short)f32_to_bf16_bits(r.o[j] / r.l);
        else reinterpret_cast<float *>(a.out + at.o)[d] = r.o[j] / r.l;
    }
}
#endif
