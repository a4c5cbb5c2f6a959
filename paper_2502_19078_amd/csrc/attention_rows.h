// The few-row body of the attention kernels (attention.hip).
//
// For a row r and the keys p that it may see:  o_r = sum_p exp(s_rp - lse_r) v_p,  s_rp = scale q_r . k_p,  lse_r = log sum_p exp(s_rp).
// One pass over the keys with a running maximum and sum per row, in base 2.
//
// Bound by the cache's bytes (HBM): a key head's rows of the cache are read once for all query heads of its group.  A workgroup takes a tile
// of 16 rows and one split of their keys; its four waves take 32 or 16 keys in turn, each with a running softmax of its own, so
// nothing waits inside the loop; the waves' results are joined through LDS, those of the splits by k_attn_join.
//
// Scores are formed transposed, S^T = K Q^T: a lane then holds scores of one row only, keys 4 (lane / 16) + i of each 16, and the same
// registers are the operand of O^T = V^T P^T when its keys are counted in that order.  K goes from memory into the operand registers as it
// lies; bf16 V goes through LDS, where ds_read_tr16 turns it; fp32 V needs no turning.  The weights enter the second product as two bf16, 16
// bits: the matrix cores have time to spare here.
//
// Measured, bf16, with the join of the splits (us): one token over 131071 rows of 8 key heads of 128 values 96 (5.6 TB/s); 8 tokens, each over a
// window of 4096 and 4 sinks, 33 (4.1; 27 without the join's launch); 64 x 4096 rows of 32 key heads 705 (6.1); 513 rows of one head
// of 256 values 14, of which a step of the loads is 2 and the chain of launches, lengths, first keys and join the rest.
#pragma once
#include "attention.h"

namespace {

// ES: bytes a value.  DP: D rounded up to the products' tiles; FULL: D == DP.
// Keys of a step of a wave.  bf16: 32; 16 for 256 values (registers for one wave a SIMD otherwise: 8 sequences of 8192 rows, 8 key heads, 177 us
// with 32 keys, 98 with 16) and whole heads of 96 (52 and 44 us; 80 values in the same kernel 40 and 43).
template <int ES, int DP, bool FULL>
struct RowsShape {
    static constexpr int KB = ES == 4 || DP == 256 || (DP == 96 && FULL) ? 1 : 2, KS = 16 * KB;
    static constexpr int PITCH = DP * 2 + 32;                // V in LDS: rows 8 banks apart modulo 64
    static constexpr int V_LDS = ES == 2 ? 4 * KS * PITCH : 0, J_LDS = DP * 256 + 512 + 16;     // of the join: outputs and maxima of four waves
    static constexpr int LDS = V_LDS > J_LDS ? V_LDS : J_LDS;
};

template <int ES, int DP, bool FULL>
__device__ __forceinline__ void attn_rows(const AttnArgs &a, const bool pre, const int block, char *lds)
{
    using S = RowsShape<ES, DP, FULL>;
    constexpr int CH = DP * ES / 64;                         // chunks of 64 bytes in a row: lane group g holds 16 bytes of each
    constexpr int KB = S::KB, KS = S::KS, PITCH = S::PITCH;
    constexpr int DB = DP / 16;                              // tiles of 16 output dimensions
    constexpr int CPR = DP * ES / 16;                        // 16-byte chunks of a row
    constexpr int VL = KS * CPR / 64;                        // 16-byte loads of V a lane and step

    static_assert(ES == 2 || DP % 64 == 0, "whole loads of V");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n16 = lane & 15, g = lane >> 4;
    const int Dd = FULL ? DP : a.D;

    // which tile of which keys
    int id = block, split, b = 0, h, tile, splits, rows;
    if (pre) {
        split = id % a.pre_splits;
        id /= a.pre_splits;
        tile = id % a.pre_tiles;
        h = id / a.pre_tiles;
        splits = a.pre_splits;
        rows = a.B * a.G;
    } else {
        split = id % a.splits;
        id /= a.splits;
        tile = id % a.own_tiles;
        id /= a.own_tiles;
        h = id % a.Hkv;
        b = id / a.Hkv;
        splits = a.splits;
        rows = a.T * a.G;
    }
    const int all_splits = a.splits + a.pre_splits, part = pre ? split : a.pre_splits + split;
    const int r0 = tile * 16;
    const AttnKV &kv = pre ? a.pre : a.kv;

    // this lane's row: its query as the second operand.  (Loaded ahead of the lengths, which the keys wait for.)
    const int len_b = pre ? 0 : a.lens[b], qlen_b = pre || !a.q_lens ? a.T : a.q_lens[b];
    u32x4 qf[CH];
    const int row = min(r0 + n16, rows - 1), token = !pre && a.T == 1 ? 0 : row / a.G;
    const RowAt at = row_at(a, pre, b, h, row, token);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int off = 64 * c + 16 * g;
        const bool in = FULL || off < Dd * ES;
        qf[c] = *reinterpret_cast<const u32x4 *>(a.q + at.q + (in ? off : 0));
        if (!in) qf[c] = u32x4{0, 0, 0, 0};
    }
    KeyRange kr;
    int first_pos = 0, qlen = a.T;
    if (pre) {
        kr.n = a.pre_n;
        kr.head = kr.lo = kr.ring_base = 0;
        kr.pos_a = kr.pos_b = a.pre_n;
    } else {
        int len;
        sequence_lens(a, len_b, qlen_b, len, qlen);
        first_pos = len - qlen;
        if (a.pre_splits)                                    // behind a prefix: all of the sequence's rows
            kr = key_range(kv, len - 1, 0, 0, 0, 0);
        else if (a.T == 1)
            kr = key_range(kv, first_pos, 0, qlen - 1, a.window, a.sinks);
        else
            kr = key_range(kv, first_pos, r0 / a.G, min(min(r0 + 15, rows - 1) / a.G, qlen - 1), a.window, a.sinks);
    }
    const int row_pos = pre || a.pre_splits ? 0 : token < qlen ? first_pos + token : -1;
    const bool one_pos = pre || a.pre_splits || kr.pos_a == kr.pos_b;      // all rows see the same keys
    int chunk = (kr.n + splits - 1) / splits;
    chunk = (chunk + 31) & ~31;
    const int k0 = min(split * chunk, kr.n), k1 = min(k0 + chunk, kr.n);

    const char *kp = kv.k + b * kv.sb + h * kv.sh, *vp = kv.v + b * kv.sb + h * kv.sh;
    char *my_v = lds + wave * KS * PITCH;

    f32x4 o[DB];
    float m = NEG_INF, l = 0.0f;
#pragma unroll
    for (int d = 0; d < DB; ++d) o[d] = f32x4{0, 0, 0, 0};
    u32x4 kf[KB][CH], vf[VL];
    auto load_k = [&](int i) {                               // keys i .. i + KS - 1; past the end the last one again
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            const char *p = kp + kr.row(kr.pos(min(i + kb * 16 + n16, k1 - 1)), kv) * kv.sn;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int off = 64 * c + 16 * g;
                const bool in = FULL || off < Dd * ES;
                kf[kb][c] = *reinterpret_cast<const u32x4 *>(p + (in ? off : 0));
                if (!in) kf[kb][c] = u32x4{0, 0, 0, 0};
            }
        }
    };
    auto load_v = [&](int i) {
#pragma unroll
        for (int j = 0; j < VL; ++j) {
            int key, col;                                    // bf16: chunks in order of the rows, for LDS; fp32: key 4 g + j % 4, 64 values a load
            if (ES == 2) {
                const int id = lane + 64 * j;
                key = id / CPR;
                col = id % CPR;
            } else {
                key = 4 * g + j % 4;
                col = 16 * (j / 4) + n16;
            }
            const bool in = FULL || col * 16 < Dd * ES;
            const char *p = vp + kr.row(kr.pos(min(i + key, k1 - 1)), kv) * kv.sn;
            vf[j] = *reinterpret_cast<const u32x4 *>(p + (in ? col * 16 : 0));
            if (!in || i + key >= k1) vf[j] = u32x4{0, 0, 0, 0};
        }
    };

    int i = k0 + wave * KS;
    if (i < k1) {
        load_k(i);
        load_v(i);
    }
    for (; i < k1; i += 4 * KS) {
        // scores of KS keys: lane holds keys 16 kb + 4 g + e of its row
        f32x4 s[KB];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            s[kb] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                if (ES == 2)
                    s[kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf[kb][c]), __builtin_bit_cast(bf16x8, qf[c]), s[kb], 0, 0, 0);
                else
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const unsigned int ka = kf[kb][c][e], qb = qf[c][e];
                        s[kb] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(ka), __uint_as_float(qb), s[kb], 0, 0, 0);
                    }
            }
        }
        const int p_first = kr.pos(i), p_last = kr.pos(min(i + KS, k1) - 1);
        const bool mixed = !one_pos && !(p_last <= kr.pos_a && (a.window == 0 || p_first > kr.pos_b - a.window || p_last < a.sinks));
        if (ES == 2) {
#pragma unroll
            for (int j = 0; j < VL; ++j) {
                const int id = lane + 64 * j;
                *reinterpret_cast<u32x4 *>(my_v + id / CPR * PITCH + id % CPR * 16) = vf[j];
            }
        }
        const int next = i + 4 * KS;
        if (next < k1) {
            load_k(next);
            if (ES == 2) load_v(next);                       // (in LDS by now)
        }
        __builtin_amdgcn_wave_barrier();

        float top = NEG_INF;
        const Sight see = sight(kr, i + 4 * g, k1, row_pos, a.window, a.sinks);
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int key = kb * 16 + e;
                float x = s[kb][e] * a.scale2;
                const bool seen = mixed ? see(key) : key < see.end;
                x = seen ? x : NEG_INF;
                s[kb][e] = x;
                top = fmaxf(top, x);
            }
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        if (__any(top > m + 8.0f)) {                         // (weights up to 2^8 lose nothing)
            const float mn = top > m + 8.0f ? top : m;
            const float f = mn == m ? 1.0f : __builtin_amdgcn_exp2f(m - mn);
            m = mn;
            l *= f;
#pragma unroll
            for (int d = 0; d < DB; ++d) o[d] *= f;
        }
        const float base = m == NEG_INF ? 0.0f : m;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float p = __builtin_amdgcn_exp2f(s[kb][e] - base);
                s[kb][e] = p;
                l += p;
            }

        if (ES == 2) {
            u32x4 hi = {}, lo = {};
#pragma unroll
            for (int w = 0; w < 2 * KB; ++w) {
                const float p0 = s[(w >> 1) % KB][2 * (w & 1)], p1 = s[(w >> 1) % KB][2 * (w & 1) + 1];
                const unsigned int u = pack_bf16(p0, p1);
                hi[w] = u;
                lo[w] = pack_bf16(p0 - __uint_as_float(u << 16), p1 - __uint_as_float(u & 0xffff0000u));
            }
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                const char *src = my_v + (4 * g + (n16 >> 2)) * PITCH + d * 32 + (n16 & 3) * 8;
                if constexpr (KB == 1) {
                    const s16x4 vt = __builtin_bit_cast(s16x4, read_tr16(src));
                    o[d] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(vt, __builtin_bit_cast(s16x4, make_uint2(hi[0], hi[1])), o[d], 0, 0, 0);
                    o[d] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(vt, __builtin_bit_cast(s16x4, make_uint2(lo[0], lo[1])), o[d], 0, 0, 0);
                    continue;
                }
                const uint2 u0 = read_tr16(src), u1 = read_tr16(src + 16 * PITCH);
                const bf16x8 vt = __builtin_bit_cast(bf16x8, u32x4{u0.x, u0.y, u1.x, u1.y});
                o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, __builtin_bit_cast(bf16x8, hi), o[d], 0, 0, 0);
                o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, __builtin_bit_cast(bf16x8, lo), o[d], 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int j = 0; j < VL; ++j)                     // keys 4 g + j % 4, dimensions 64 (j / 4) + 4 n16 + e
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const unsigned int vv = vf[j][e];
                    f32x4 &to = o[(j / 4 * 4 + e) % DB];
                    to = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vv), s[0][j % 4], to, 0, 0, 0);
                }
            if (next < k1) load_v(next);
        }
    }

    // The waves' results side by side in LDS; then every wave joins a part of each row's outputs: v[x] are the four from dim(x) on.
    constexpr int OUT = (DB + 3) / 4;
    auto dim = [&](int x) { return ES == 2 ? 16 * (wave + 4 * x) + 4 * g : 64 * x + 16 * g + 4 * wave; };
    float2 *s_ml = reinterpret_cast<float2 *>(lds + DP * 256);
    unsigned int *s_again = reinterpret_cast<unsigned int *>(lds + DP * 256 + 512);
    f32x4 v[OUT];
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    __syncthreads();
#pragma unroll
    for (int d = 0; d < DB; ++d) reinterpret_cast<f32x4 *>(lds)[(wave * DB + d) * 64 + lane] = o[d];
    if (g == 0) s_ml[wave * 16 + n16] = make_float2(m, l);
    if (threadIdx.x == 0) *s_again = 0;
    __syncthreads();
    float2 ml[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) ml[w] = s_ml[w * 16 + n16];
    m = fmaxf(fmaxf(ml[0].x, ml[1].x), fmaxf(ml[2].x, ml[3].x));
    l = 0.0f;
#pragma unroll
    for (int x = 0; x < OUT; ++x) v[x] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const float f = ml[w].x == NEG_INF ? 0.0f : __builtin_amdgcn_exp2f(ml[w].x - m);
        l += ml[w].y * f;
#pragma unroll
        for (int x = 0; x < OUT; ++x) {
            if (ES == 2) {
                if (DB % 4 == 0 || wave + 4 * x < DB) v[x] += reinterpret_cast<const f32x4 *>(lds)[(w * DB + wave + 4 * x) * 64 + lane] * f;
            } else
#pragma unroll
                for (int e = 0; e < 4; ++e) v[x][e] += reinterpret_cast<const float *>(lds)[((w * DB + 4 * x + e) * 64 + lane) * 4 + wave] * f;
        }
    }
    bool fine = l < INFINITY;
#pragma unroll
    for (int x = 0; x < OUT; ++x)
#pragma unroll
        for (int e = 0; e < 4; ++e) fine = fine && fabsf(v[x][e]) < INFINITY;
    unsigned long long odd = __ballot(!fine && !(l != l) && row_pos >= 0 && r0 + n16 < rows);
    if (odd) {
        odd |= odd >> 32;
        if (lane == 0) atomicOr(s_again, (unsigned int)((odd | odd >> 16) & 0xffff));
    }
    __syncthreads();
    const unsigned int again = kr.n ? __builtin_amdgcn_readfirstlane(*s_again) : 0u;
    if (again) {
        for (int t = wave; t < 16; t += 4) {
            if (!(again >> t & 1)) continue;
            const int i = (r0 + t) / a.G;
            const RowAt to = row_at(a, pre, b, h, r0 + t, i);
            attn_store_again<ES>(a, attn_row_again<ES>(a, kr, kv, kp, vp, a.q + to.q, pre || a.pre_splits ? INT32_MAX : first_pos + i, k0, k1), to, part);
        }
    }

    if (r0 + n16 >= rows || (again >> n16 & 1)) return;
    if (all_splits > 1) {
        const int64_t at_part = at.lse * all_splits + part;
        if (g == 0 && wave == 0) a.part_ml[at_part] = make_float2(m, l);
        if (k0 == k1) return;                                // nothing to read for this split
        float *to = a.part_o + at_part * Dd;
#pragma unroll
        for (int x = 0; x < OUT; ++x)
            if (dim(x) < Dd) *reinterpret_cast<f32x4 *>(to + dim(x)) = v[x];
        return;
    }
    const bool none = kr.n == 0 || row_pos < 0;
    if (a.lse && g == 0 && wave == 0) a.lse[at.lse] = none ? NEG_INF : (m == NEG_INF ? NEG_INF : m * 0.69314718055994531f) + logf(l);
    const float inv = 1.0f / l;
#pragma unroll
    for (int x = 0; x < OUT; ++x) {
        if (dim(x) >= Dd) continue;
        const f32x4 y = none ? f32x4{0, 0, 0, 0} : v[x] * inv;
        if (ES == 2)
            *reinterpret_cast<uint2 *>(a.out + at.o + dim(x) * 2) = make_uint2(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]));
        else
            *reinterpret_cast<f32x4 *>(a.out + at.o + dim(x) * 4) = y;
    }
}

}  // namespace
