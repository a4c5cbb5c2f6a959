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

hipError_t clada_attn_rows(const AttnArgs &a, int es, hipStream_t stream);
hipError_t clada_attn_join(const AttnArgs &a, int es, hipStream_t stream);
int clada_attn_rows_tile(int rows);                          // rows of a tile of k_attn_rows for so many rows

#ifdef __HIPCC__
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
