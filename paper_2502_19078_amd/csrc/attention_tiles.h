// The many-row body of the attention kernels (attention.hip): prompts, chunks, and a shared prefix read for a batch.
//
// The same sums as in attention_rows.h.  bf16, bound by the matrix cores and the vector units: 32 rows by 64 keys of 128 values are 32 products
// of 32x32x16 (1024 clocks of a SIMD) beside 32 exponentials, sums and conversions a lane (about 800).  A workgroup of four waves takes 128
// rows, 32 a wave; K and V tiles go through registers into one of two LDS buffers while the other is multiplied, one barrier a
// tile.  Two workgroups share a compute unit, so that one's products can run under the other's exponentials.  fp32: the same with
// 32x32x2 products, tiles of 32 keys and weights in fp32.
//
// Measured (us): 8192 tokens, 32 query and 8 key heads of 128 values, window of 4096, bf16: 427 to 465 over several runs, 887 to 965 TFLOP/s on the
// visible pairs, where a library
// product of 8192^3 runs at 1168; a wave's tile takes 2100 clocks of its SIMD (all products together 1024; the matrix cores are busy 49 % of the
// time): two waves do not keep them busy through each other's exponentials, LDS reads and barriers.  On the way: rows of attention_rows.h 2710; these tiles 554;
// one base address a tile 490; fragments read six products ahead and exponentials between the products 472; no maxima, steady tiles in a
// loop of their own 460; staging between the products another 3 %.  256 rows a workgroup of eight waves, wave priorities, 32 rows with
// deeper reads ahead: within 2 % or slower.  fp32, 2 x 1000 tokens, 32 heads of 80 values, window 256: 96 (rows of 32 in attention_rows.h: 221).
//
// Scores are formed transposed (S^T = K Q^T): a lane holds scores of one row only, keys 8 (i / 4) + 4 (lane / 32) + i % 4 of each 32, and the same
// registers are the second operand of O^T = V^T P^T when its keys are counted in that order (bf16 V is turned by ds_read_tr16).  Weights are
// rounded to bf16 there (2^-8 at most, to nearest: the size of the output's own rounding); their sum is taken before it.  With weights as two
// bf16 (FINE) the prompt above takes 570 for 460, chunks of 64 tokens over windows of 2048 with heads of 64 values 21.3 for 20.0, and the error
// against 64 bits is 0.00165 in place of 0.0018 (all in fp32: 0.0016 to 0.0017).  Behind a prefix, which waits for its loads, they cost 3 % and
// the error is 0.00167 in place of 0.0023.
#pragma once
#include <type_traits>

#include "attention.h"

namespace {

template <int ES, int DP>
struct TilesShape {
    static constexpr int KT = ES == 2 && DP <= 128 ? 64 : 32;        // keys of a tile
    static constexpr int KP = DP * ES + 16, VP = DP * ES + (ES == 2 ? 32 : 16);      // row pitches: K rows 4 banks apart, bf16 V rows 8
    static constexpr int BUF = KT * (KP + VP), LDS = 2 * BUF;
};

// FINE: the weights of a bf16 call enter the second product as two bf16, 16 bits, in two products.
template <int ES, int DP, bool FULL, bool FINE>
__device__ __forceinline__ void attn_tiles(const AttnArgs &a, const bool pre, const int id, char *lds)
{
    using S = TilesShape<ES, DP>;
    constexpr int KT = S::KT, KB = KT / 32, KP = S::KP, VP = S::VP, BUF = S::BUF;
    constexpr int KD = DP * ES / 32, DB = DP / 32;           // 32-byte chunks of a row, 16 bytes a lane; tiles of 32 output dimensions
    constexpr int CPR = DP == 96 ? 128 / (16 / ES) : DP * ES / 16, ROWS = KT * CPR / 256;    // threads a row, 16 bytes each; rows of K (and of V) a thread stages
    constexpr bool WHOLE = FULL && CPR * 16 == DP * ES;      // every thread has a chunk of the row
    static_assert(KT * CPR % 256 == 0 && 256 % CPR == 0, "whole passes");

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n32 = lane & 31, hh = lane >> 5, t16 = lane & 15, g = lane >> 4;
    const int Dd = FULL ? DP : a.D;

    // Units (sequence, key head) fastest: consecutive workgroups go to different XCDs, so a unit's tiles share an L2.  The last row tiles see the
    // most keys and come first.
    const int units = pre ? a.Hkv : a.B * a.Hkv, tiles = pre ? a.pre_tiles : a.own_tiles, splits = pre ? a.pre_splits : a.splits;
    const int unit = id % units, rest = id / units;
    const int split = rest % splits, tile = tiles - 1 - rest / splits;
    const int h = unit % a.Hkv, b = unit / a.Hkv;
    const int rows = (pre ? a.B : a.T) * a.G, r0 = tile * 128;
    const AttnKV &kv = pre ? a.pre : a.kv;
    KeyRange kr;
    int first_pos = 0, qlen = a.T;
    if (pre) {
        kr.n = a.pre_n;
        kr.head = kr.lo = kr.ring_base = 0;
        kr.pos_a = kr.pos_b = a.pre_n;
    } else {
        int len;
        sequence_lens(a, a.lens[b], a.q_lens ? a.q_lens[b] : a.T, len, qlen);
        first_pos = len - qlen;
        kr = key_range(kv, first_pos, r0 / a.G, min(min(r0 + 127, rows - 1) / a.G, qlen - 1), a.window, a.sinks);
    }
    int chunk = (kr.n + splits - 1) / splits;
    chunk = (chunk + KT - 1) / KT * KT;
    const int k0 = min(split * chunk, kr.n), k1 = min(k0 + chunk, kr.n);

    // this lane's row
    const int r = r0 + wave * 32 + n32, rc = min(r, rows - 1);
    const int row_pos = pre ? a.pre_n : rc / a.G < qlen ? first_pos + rc / a.G : -1;
    // positions of the wave's first and last row, for tiles that all or none of its rows see
    const bool idle = r0 + wave * 32 >= rows;
    const int wr0 = min(r0 + wave * 32, rows - 1), wr1 = min(r0 + wave * 32 + 31, rows - 1);
    const int wave_a = pre ? a.pre_n : wr0 / a.G < qlen ? first_pos + wr0 / a.G : -1;
    const int wave_b = pre ? a.pre_n : min(wr1 / a.G, qlen - 1) + first_pos;
    const bool ragged = !pre && wr1 / a.G >= qlen;           // rows of padding among them

    const unsigned int flip = a.scale2 < 0.0f ? (ES == 2 ? 0x80008000u : 0x80000000u) : 0u;      // a negative scale is the queries' sign
    const float scale2 = fmaxf(fabsf(a.scale2), 0x1p-149f);  // positive, so that -inf stays what it is (2^128, the largest product, counts 2^-21)
    u32x4 qf[KD];
#pragma unroll
    for (int c = 0; c < KD; ++c) {
        const int off = 32 * c + 16 * hh;
        const bool in = FULL || off < Dd * ES;
        qf[c] = *reinterpret_cast<const u32x4 *>(a.q + row_at(a, pre, b, h, rc, rc / a.G).q + (in ? off : 0));
#pragma unroll
        for (int e = 0; e < 4; ++e) qf[c][e] = in ? qf[c][e] ^ flip : 0u;
    }

    const char *kp = kv.k + b * kv.sb + h * kv.sh, *vp = kv.v + b * kv.sb + h * kv.sh;
    const int first_key = tid / CPR, col = tid % CPR * 16;   // of the chunks that this thread stages: keys first_key + j * (256 / CPR)
    const bool in = WHOLE || col < Dd * ES;
    const unsigned int lane_off = (unsigned int)first_key * (unsigned int)kv.sn + (in ? col : 0), step_off = 256 / CPR * (unsigned int)kv.sn;
    u32x4 sk[ROWS], sv[ROWS];                                // the tile on its way into LDS
    // A whole tile of consecutive cache rows has one base for all lanes (offsets in 32 bits: no row further than 32 MiB from the next).  Its first
    // and last row tell, except where the key behind the last sink lies elsewhere than in the row behind it: the ring may then wrap just as many
    // rows short as the seam skips.  A tile across such a seam is never regular.
    const int seam = kr.n > kr.head && kr.row(kr.lo, kv) != kr.head ? kr.head : 0;
    auto regular = [&](int i) {
        return i + KT <= k1 && (i >= seam || i + KT <= seam) && kv.sn < (1 << 25) && kr.row(kr.pos(i + KT - 1), kv) - kr.row(kr.pos(i), kv) == KT - 1;
    };
    __amdgpu_buffer_rsrc_t k_tile, v_tile;
    auto aim = [&](int i) {                                  // at a regular tile
        const int64_t at = kr.row(kr.pos(i), kv) * kv.sn;
        k_tile = __builtin_amdgcn_make_buffer_rsrc((void *)(kp + at), 0, -1, 0x00027000);
        v_tile = __builtin_amdgcn_make_buffer_rsrc((void *)(vp + at), 0, -1, 0x00027000);
    };
    auto take = [&](int q) {                                 // transfer q of 2 ROWS of that tile: K, V, K, ..
        const int j = q / 2;
        if (q & 1) sv[j] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(v_tile, lane_off, j * step_off, 0));
        else sk[j] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(k_tile, lane_off, j * step_off, 0));
    };
    auto fetch = [&](int i) {
        if (regular(i)) {
            aim(i);
#pragma unroll
            for (int q = 0; q < 2 * ROWS; ++q) take(q);
        } else {
            int key0 = i + first_key;
            asm volatile("" : "+v"(key0));                   // (nothing of this is kept in registers across the loop)
#pragma unroll
            for (int j = 0; j < ROWS; ++j) {
                const int key = key0 + j * (256 / CPR);
                const int64_t off = kr.row(kr.pos(min(key, k1 - 1)), kv) * kv.sn + (in ? col : 0);
                sk[j] = *reinterpret_cast<const u32x4 *>(kp + off);
                sv[j] = *reinterpret_cast<const u32x4 *>(vp + off);
                if (key >= k1) sv[j] = u32x4{0, 0, 0, 0};
            }
        }
    };
    // (threads without a chunk write into the row's padding)
    const unsigned int put_k = first_key * KP + min(col, DP * ES), put_v = KT * KP + first_key * VP + min(col, DP * ES);
    auto put_one = [&](int buf, int q) {                     // transfer q into LDS
        const int j = q / 2;
        u32x4 x = q & 1 ? sv[j] : sk[j];
        if (!WHOLE && !in) x = u32x4{0, 0, 0, 0};
        char *to = lds + ((q & 1 ? put_v : put_k) + buf * BUF) + j * (256 / CPR) * (q & 1 ? VP : KP);
        *reinterpret_cast<u32x4 *>(to) = x;
    };
    auto put = [&](int buf) {
#pragma unroll
        for (int q = 0; q < 2 * ROWS; ++q) put_one(buf, q);
    };

    // A row's maximum is that of the first tile that it sees; its weights grow past 1 from there on (as floats they lose nothing) and are
    // scaled down where a sum passes 2^60: no maxima in the loop.  A row whose sum has passed 2^100 by then (scores of 94 powers of two and more above
    // those that its maximum was taken from, within a tile) is computed again below: a factor below 2^-126 is zero in the scaling and in the join of
    // splits, which costs a sum of 2^100 a part of 2^-26 at most, but a larger one parts that count, and an infinite one is NaN behind it.
    f32x16 o[DB];
    float m = row_pos < 0 || r >= rows ? 0.0f : NEG_INF;     // (a row that sees nothing does not wait for its first key)
    float l = 0.0f;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[d][e] = 0.0f;
    bool steady = false;                                     // every row has its maximum, and no sum has passed 2^60
    bool outgrown = false;                                   // this row's sum passed 2^100
    // One tile for this wave's rows.  EDGE: some of them do not see all of it, or a maximum has to be set or moved.  Otherwise the next tile goes
    // into LDS, and the one after it (regular, aimed at) is taken, transfer by transfer between the products: the loads of all waves pass one
    // address unit, and in one place they would hold up the waves for 800 clocks of a tile.
    auto multiply = [&](auto edge, int i, int buf, bool all) {
        constexpr bool EDGE = decltype(edge)::value;
        const char *kb = lds + buf * BUF, *vb = kb + KT * KP;
        auto stage = [&](int x, int of) {                    // behind product x of `of`
            if constexpr (!EDGE) {
#pragma unroll
                for (int q = 2 * ROWS * x / of; q < 2 * ROWS * (x + 1) / of; ++q) {
                    put_one(buf ^ 1, q);
                    take(q);
                }
            }
        };
        f32x16 s[KB];
        const f32x16 zero = {};
#pragma unroll
        for (int c = 0; c < KD; ++c)
#pragma unroll
            for (int k = 0; k < KB; ++k) {
                const u32x4 kf = *reinterpret_cast<const u32x4 *>(kb + (k * 32 + n32) * KP + 32 * c + 16 * hh);
                if constexpr (ES == 2)
                    s[k] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf), __builtin_bit_cast(bf16x8, qf[c]), c ? s[k] : zero, 0, 0, 0);
                else
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const unsigned int ka = kf[e], qb = qf[c][e];
                        s[k] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(ka), __uint_as_float(qb), c || e ? s[k] : zero, 0, 0, 0);
                    }
            }
        if constexpr (ES == 2) {                             // six fragments ahead of the products
            __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
#pragma unroll
            for (int x = 0; x < KD * KB - 6; ++x) {
                __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x8, 6, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (EDGE) {
            if (!all) {
                const Sight see = sight(kr, i + 4 * hh, k1, row_pos, pre ? 0 : a.window, a.sinks);
#pragma unroll
                for (int k = 0; k < KB; ++k)
#pragma unroll
                    for (int e = 0; e < 16; ++e) s[k][e] = see(k * 32 + 8 * (e >> 2) + (e & 3)) ? s[k][e] : NEG_INF;
            }
            float top = NEG_INF;
#pragma unroll
            for (int k = 0; k < KB; ++k)
#pragma unroll
                for (int e = 0; e < 16; ++e) top = fmaxf(top, s[k][e]);
            top = fmaxf(top, __shfl_xor(top, 32)) * scale2;
            const float grown = fmaxf(l, __shfl_xor(l, 32)), mn = top > m + 8.0f ? top : grown > 0x1p60f ? m + 60.0f : m;
            if (__any(mn != m)) {
                outgrown = outgrown || grown > 0x1p100f;
                const float f = mn == m ? 1.0f : __builtin_amdgcn_exp2f(m - mn);
                m = mn;
                l *= f;
#pragma unroll
                for (int d = 0; d < DB; ++d) o[d] *= f;
            }
        }
        const float base = EDGE && m == NEG_INF ? 0.0f : m;
        if constexpr (ES == 2) {
            // Sixteen keys are a step of the second product.  Between the products of one step stand the exponentials of the next one and the
            // reads of V four products ahead.
            constexpr int STEPS = 2 * KB, AHEAD = 4;
            u32x4 vt[AHEAD], pk[2], lo[FINE ? 2 : 1];
            auto weight = [&](auto step, int e) {                // the e-th of the step's eight weights of this lane
                constexpr int st = decltype(step)::value, k = st / 2, c = st % 2;
                const float p = __builtin_amdgcn_exp2f(fmaf(s[k][8 * c + e], scale2, -base));
                l += p;
                s[k][8 * c + e] = p;
                if (e & 1) {
                    const float p0 = s[k][8 * c + e - 1];
                    const unsigned int u = pack_bf16(p0, p);
                    pk[st & 1][e >> 1] = u;
                    if (FINE) lo[FINE ? st & 1 : 0][e >> 1] = pack_bf16(p0 - __uint_as_float(u << 16), p - __uint_as_float(u & 0xffff0000u));
                }
            };
            const char *src = vb + (4 * hh + (t16 >> 2)) * VP + (g & 1) * 32 + (t16 & 3) * 8;
            auto read_v = [&](int x) {
                const char *from = src + x / DB * 16 * VP + x % DB * 64;
                const uint2 u0 = read_tr16(from), u1 = read_tr16(from + 8 * VP);
                vt[x % AHEAD] = u32x4{u0.x, u0.y, u1.x, u1.y};
            };
#pragma unroll
            for (int x = 0; x < AHEAD; ++x) read_v(x);
#pragma unroll
            for (int e = 0; e < 8; ++e) weight(std::integral_constant<int, 0>{}, e);
            unrolled<STEPS>([&](auto step) {
                constexpr int st = decltype(step)::value;
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    __builtin_amdgcn_sched_barrier(0);
                    const int x = st * DB + d;
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vt[x % AHEAD]), __builtin_bit_cast(bf16x8, pk[st & 1]), o[d], 0, 0, 0);
                    if constexpr (FINE)
                        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vt[x % AHEAD]), __builtin_bit_cast(bf16x8, lo[st & 1]), o[d], 0, 0, 0);
                    if (x + AHEAD < STEPS * DB) read_v(x + AHEAD);
                    stage(x, STEPS * DB);
                    if constexpr (st + 1 < STEPS) {
#pragma unroll
                        for (int e = 8 * d / DB; e < 8 * (d + 1) / DB; ++e) weight(std::integral_constant<int, st + 1>{}, e);
                    }
                }
            });
            __builtin_amdgcn_sched_barrier(0);
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                s[0][e] = __builtin_amdgcn_exp2f(fmaf(s[0][e], scale2, -base));
                l += s[0][e];
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) {                   // keys 8 (e / 4) + 4 hh + e % 4
                const char *src = vb + (8 * (e >> 2) + 4 * hh + (e & 3)) * VP + n32 * 4;
#pragma unroll
                for (int d = 0; d < DB; ++d)
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(*reinterpret_cast<const float *>(src + d * 128), s[0][e], o[d], 0, 0, 0);
                stage(e, 16);
            }
        }
        steady = !__any(l > 0x1p60f || (EDGE && m == NEG_INF));
    };

    if (k0 < k1) {
        fetch(k0);
        put(0);
        if (k0 + KT < k1) fetch(k0 + KT);
    }
    tile_barrier();
    int buf = 0, i = k0;
    bool none = false, all = false;
    auto look = [&]() {                                      // how the tile at i lies for this wave's rows
        const int last = min(i + KT, k1) - 1, p_first = kr.pos(i), p_last = kr.pos(last);
        // (a tile that begins among the sinks is looked at key by key)
        none = idle || p_first > wave_b || (a.window && p_first >= a.sinks && p_last <= wave_a - a.window && wave_a >= 0);
        all = last == i + KT - 1 && !ragged && (pre || (p_last <= wave_a && (a.window == 0 || p_first > wave_b - a.window || p_last < a.sinks)));
    };
    auto step = [&]() {
        tile_barrier();
        buf ^= 1;
        i += KT;
    };
    // The waves of a workgroup may be in different loops; every tile is one barrier in both.
    while (i < k1) {
        look();
        if (!none) multiply(std::true_type{}, i, buf, all);
        if (i + KT < k1) {
            put(buf ^ 1);
            if (i + 2 * KT < k1) fetch(i + 2 * KT);
        }
        step();
        for (; i < k1; step()) {
            look();
            if (none || !all || !steady || !regular(i + 2 * KT)) break;
            aim(i + 2 * KT);
            multiply(std::false_type{}, i, buf, true);
        }
    }
    l += __shfl_xor(l, 32);
    outgrown = outgrown || l > 0x1p100f;                     // (an l that is NaN without it is a NaN score's)
    bool fine = true;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) fine = fine && fabsf(o[d][e]) < INFINITY;
    const bool nothing = kr.n == 0 || row_pos < 0;
    const unsigned long long odd = __ballot((outgrown || (!fine && l == l)) && !nothing && r < rows);
    const unsigned int again = (unsigned int)odd | (unsigned int)(odd >> 32);      // a bit for every row of the wave
    for (unsigned int left = again; left; left &= left - 1) {
        const int t = __builtin_ctz(left);
        const RowAt at = row_at(a, pre, b, h, r0 + wave * 32 + t, (r0 + wave * 32 + t) / a.G);
        attn_store_again<ES>(a, attn_row_again<ES>(a, kr, kv, kp, vp, a.q + at.q, __shfl(row_pos, t), k0, k1), at, split);
    }
    if (r >= rows || (again >> n32 & 1)) return;
    const RowAt to_row = row_at(a, pre, b, h, r, r / a.G);

    const int all_splits = a.splits + a.pre_splits;
    if (all_splits > 1) {
        const int64_t part = to_row.lse * all_splits + split;
        if (hh == 0) a.part_ml[part] = make_float2(m, l);
        if (k0 == k1) return;
        float *to = a.part_o + part * Dd;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const int dim = 32 * d + 2 * e + 4 * hh;
                if (FULL || dim < Dd) *reinterpret_cast<f32x4 *>(to + dim) = f32x4{o[d][e], o[d][e + 1], o[d][e + 2], o[d][e + 3]};
            }
        return;
    }
    if (a.lse && hh == 0) a.lse[to_row.lse] = nothing ? NEG_INF : (m == NEG_INF ? NEG_INF : m * 0.69314718055994531f) + logf(l);
    const float inv = 1.0f / l;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            const int dim = 32 * d + 2 * e + 4 * hh;
            if (!FULL && dim >= Dd) continue;
            f32x4 y = f32x4{o[d][e], o[d][e + 1], o[d][e + 2], o[d][e + 3]} * inv;
            if (nothing) y = f32x4{0, 0, 0, 0};
            if (ES == 2)
                *reinterpret_cast<uint2 *>(a.out + to_row.o + dim * 2) = make_uint2(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]));
            else
                *reinterpret_cast<f32x4 *>(a.out + to_row.o + dim * 4) = y;
        }
}

}  // namespace
