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

// Which kernel: tiles of 16 rows (both types), 32 rows (fp32), 128 rows (bf16); a shared prefix in tiles of 128 rows with the
// sequences' own keys in tiles of 16 (bf16).  Partial results are joined where there are any.
enum AttnPath { ATTN_ROWS16, ATTN_ROWS32, ATTN_TILES, ATTN_PREFIX };
hipError_t clada_attn_launch(const AttnArgs &a, int es, AttnPath path, hipStream_t stream);

#ifdef __HIPCC__
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) short s16x4;

constexpr float NEG_INF = -__builtin_inff();

__device__ __forceinline__ unsigned int pack_bf16(float lo, float hi)      // rounded to nearest even
{
    typedef __attribute__((ext_vector_type(2))) float f32x2;
    return __builtin_bit_cast(unsigned int, __builtin_convertvector((f32x2{lo, hi}), bf16x2_t));
}

// Where a row's query and output lie.
struct RowAt { int64_t q, o, lse; };
__device__ __forceinline__ RowAt row_at(const AttnArgs &a, bool pre, int b, int h, int r)
{
    const int i = r / a.G, hq = h * a.G + (r - i * a.G);
    const int bb = pre ? i : b, t = pre ? 0 : i;
    return {bb * a.q_sb + t * a.q_st + hq * a.q_sh, bb * a.o_sb + t * a.o_st + hq * a.o_sh, ((int64_t)bb * a.T + t) * a.Hq + hq};
}

// Four columns of a transposed read: the 16 lanes of a group name four rows of four values each (lane t: row t / 4, values 4 (t % 4) on) and
// lane t receives value t of the four rows.
__device__ __forceinline__ uint2 read_tr16(const char *p)
{
    return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3))) *)p));
}

// Values that are not finite.  A weight of zero times such a value is no zero, so a product over a tile would hand it to rows that do not see
// its key.  A pass whose outputs are not all finite is therefore followed by three more over the same keys: the weights 1 for every
// key that a row sees, and V with 1 where a value is +inf or NaN (PASS_UP), then -inf or NaN (PASS_DOWN), which count such values for each
// output; then the plain weights with those values taken out (PASS_REST).  An output with a count is that infinity, or NaN with both.
enum { PASS_PLAIN = 0, PASS_UP = 1, PASS_DOWN = 2, PASS_REST = 3 };
template <int ES>
__device__ __forceinline__ void values_for_pass(u32x4 &v, int pass)
{
    if (pass == PASS_PLAIN) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const unsigned int w = v[e];
        if (ES == 4) {
            const bool odd = (w & 0x7f800000u) == 0x7f800000u, counts = odd && (w << 9 || (w >> 31) == (unsigned int)(pass == PASS_DOWN));
            v[e] = pass == PASS_REST ? (odd ? 0u : w) : (counts ? 0x3f800000u : 0u);
        } else {
            unsigned int r = 0;
#pragma unroll
            for (int s = 0; s < 32; s += 16) {
                const unsigned int x = w >> s & 0xffffu;
                const bool odd = (x & 0x7f80u) == 0x7f80u, counts = odd && ((x & 0x7fu) || (x >> 15) == (unsigned int)(pass == PASS_DOWN));
                r |= (pass == PASS_REST ? (odd ? 0u : x) : (counts ? 0x3f80u : 0u)) << s;
            }
            v[e] = r;
        }
    }
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

// Tokens that a sequence holds and queries that the call brings for it, whatever the arrays say.
__device__ __forceinline__ void sequence_lens(const AttnArgs &a, int b, int &len, int &qlen)
{
    len = max(a.lens[b], 0);
    if (a.kv.ring == 0) len = min(len, a.kv.capacity);
    qlen = a.q_lens ? min(max(a.q_lens[b], 0), a.T) : a.T;
}
#endif
