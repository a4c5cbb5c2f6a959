// The few-row body of clada_paged_attn: single tokens, and calls of at most 16 rows a key head.
//
// For a row r and the keys p that it sees:  o_r = sum_p exp(s_rp - lse_r) v_p,  lse_r = log sum_p exp(s_rp), s as paged_score says.  One pass over
// the keys with a running maximum and sum per row, in base 2.
//
// Bound by the pages' bytes (HBM): a key head's rows are read once for all query heads of its group.  A workgroup takes a tile of 8 or 16 rows and
// one split of their keys; its four waves (eight for rows of 4 bits) take steps of 16 or 32 keys in turn, each with a running softmax of its
// own, so nothing waits inside the loop; the waves' results are joined through LDS, those of the splits by the last workgroup to arrive.
// Rows of 4 bits come at 2.9 to 4.6 TB/s: 41 to 47 % of a wave's time is a wait for the step on its way, and the vector units are busy for 43 to 52 % of the busy cycles (about 160
// instructions for 32 keys of 64 values).  Two steps on their way, or each weight formed once for tiles of 4 rows (a third fewer
// instructions), changed the time by less than 3 %; twice the workgroups cost 6 us, the time in which the last one reads the others' results.
//
// The range of keys begins at a multiple of a step, so each 16 keys lie in one page: its number is one scalar load (one for the step where pages are as
// long), made two steps ahead of the rows' use and looked at when the rows are loaded, and the rows have one base.
//
// Scores are formed transposed, S^T = K Q^T: a lane then holds scores of one row only, keys 4 (lane / 16) + i of each 16, and the same
// registers are the operand of O^T = V^T P^T when its keys are counted in that order.  K goes from memory into the operand registers as it
// lies; 16-bit V goes through LDS, where ds_read_tr16 turns it; fp32 V needs no turning.  The weights enter the second product as two bf16, 16
// bits.  4 bits: a lane group holds a quarter of a row, its codes become bf16 under their power of two in one instruction for two (exact),
// K in registers in the order in which the query is taken too, V on its way into LDS.
#pragma once
#include "paged.h"

namespace {

// DP: D rounded up to the products' tiles (4 bits: D itself); FULL: D == DP.  KB: 16-key blocks of a step of a wave.
template <PagedType TY, int DP, bool FULL>
struct PagedRowsShape {
    static constexpr int KB = TY == PAGED_F32 ? 1 : TY == PAGED_4BIT ? 2 : DP == 256 || (DP == 96 && FULL) ? 1 : 2;
    static constexpr int KS = 16 * KB, KS_BITS = KB == 1 ? 4 : 5;
    static constexpr int WAVES = TY == PAGED_4BIT && DP <= 128 ? 8 : 4;
    static constexpr int PITCH = DP * 2 + 32;                // V in LDS
    static constexpr int V_LDS = TY == PAGED_F32 ? 0 : WAVES * KS * PITCH, J_LDS = WAVES * (DP * 64 + 128) + 16;     // of the join: outputs and maxima of the waves
    static constexpr int LDS = V_LDS > J_LDS ? V_LDS : J_LDS;
};

typedef const __attribute__((address_space(4))) int32_t *scalar_i32;         // read by scalar loads

template <int N> struct Words;
template <> struct Words<1> { typedef unsigned int type; };
#define CLADA_WORDS(N) template <> struct Words<N> { typedef __attribute__((ext_vector_type(N), aligned(4))) unsigned int type; };
CLADA_WORDS(2) CLADA_WORDS(3) CLADA_WORDS(4) CLADA_WORDS(5) CLADA_WORDS(6) CLADA_WORDS(7) CLADA_WORDS(8)
#undef CLADA_WORDS

// The last of a tile's splits to arrive joins the partial results of all, in the order of the splits: a launch of its own for that costs 4 to 6 us and
// its start.  Rows r0 .. r0 + R - 1 of (b, h); TPR threads hold four values each of a row, and the groups of one row take the splits in turn.
template <int ES, int THREADS>
__device__ __forceinline__ void paged_join(const PagedArgs &a, const int unit, const int b, const int h, const int r0, const int R, char *lds)
{
    f32x4 *s_o = reinterpret_cast<f32x4 *>(lds);
    float2 *s_ml = reinterpret_cast<float2 *>(lds + THREADS * 16);
    int *s_last = reinterpret_cast<int *>(lds + THREADS * 16 + THREADS / 16 * 8);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");         // this wave's results are where every workgroup reads them
    __syncthreads();
    if (threadIdx.x == 0) {
        const int before = __hip_atomic_fetch_add(&a.arrived[unit], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        *s_last = before == a.splits - 1;
        if (*s_last) __hip_atomic_store(&a.arrived[unit], 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);      // ready for the next call
    }
    __syncthreads();
    if (!__builtin_amdgcn_readfirstlane(*s_last)) return;
    const int tpr = a.D <= 64 ? 16 : a.D <= 128 ? 32 : 64, groups = THREADS / tpr;
    int pass = 1;                                            // rows at once
    while (pass < R && pass < groups) pass *= 2;
    const int subs = groups / pass;                          // groups of a row
    const int tid = threadIdx.x, group = tid / tpr, sub = group / pass, dim = tid % tpr * 4;
    for (int x = 0; x < R; x += pass) {                      // (once where a row has several groups)
        const int r = min(x + group % pass, R - 1), i = (r0 + r) / a.G;
        const RowAt at = row_at(a, false, b, h, r0 + r, i);
        const float2 *ml = a.part_ml + at.lse * a.splits;
        const unsigned int po = (unsigned int)at.lse * a.splits * a.D + (dim < a.D ? dim : 0);
        float m = NEG_INF, l = 0.0f;
        f32x4 o = {0, 0, 0, 0};
        constexpr int N = 4;                                 // loads in flight
        for (int s0 = sub; s0 < a.splits; s0 += N * subs) {
            float2 v[N];
            f32x4 part[N];
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const int s = min(s0 + j * subs, a.splits - 1);
                v[j] = load_past(ml + s);
                part[j] = load_past4(a.part_o, po + (unsigned int)s * a.D);
            }
#pragma unroll
            for (int j = 0; j < N; ++j) {
                if (s0 + j * subs >= a.splits || v[j].y == 0.0f) continue;      // (one without keys has written no values)
                const float mn = fmaxf(m, v[j].x), f = v[j].x == NEG_INF ? 0.0f : __builtin_amdgcn_exp2f(v[j].x - mn);
                const float k = m == NEG_INF ? 0.0f : __builtin_amdgcn_exp2f(m - mn);
                l = l * k + (v[j].x == NEG_INF ? v[j].y : v[j].y * f);
                o = o * k + part[j] * f;
                m = mn;
            }
        }
        if (subs > 1) {
            s_o[tid] = o;
            if (dim == 0) s_ml[group] = make_float2(m, l);
            __syncthreads();
            if (sub == 0) {
                for (int j = 1; j < subs; ++j) {
                    const float2 v = s_ml[group + j * pass];
                    if (v.y == 0.0f) continue;
                    const f32x4 part = s_o[tid + j * pass * tpr];
                    const float mn = fmaxf(m, v.x), f = v.x == NEG_INF ? 0.0f : __builtin_amdgcn_exp2f(v.x - mn);
                    const float k = m == NEG_INF ? 0.0f : __builtin_amdgcn_exp2f(m - mn);
                    l = l * k + (v.x == NEG_INF ? v.y : v.y * f);
                    o = o * k + part * f;
                    m = mn;
                }
            }
        }
        const bool mine = sub == 0 && x + group % pass < R;
        const bool none = l == 0.0f;
        if (mine && a.lse && dim == 0) a.lse[at.lse] = none ? NEG_INF : (m == NEG_INF ? NEG_INF : m * 0.69314718055994531f) + logf(l);
        if (mine && dim < a.D) {
            o = none ? f32x4{0, 0, 0, 0} : o * (1.0f / l);
            if (ES == 2)
                *reinterpret_cast<uint2 *>(a.out + at.o + dim * 2) = make_uint2(pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3]));
            else
                *reinterpret_cast<f32x4 *>(a.out + at.o + dim * 4) = o;
        }
    }
}

// Rows that one tile of their sequence alone reads pass by the caches: 32 sequences of 593 to 4096 tokens, 32 key heads of 128 bf16 values 187 us (6.6 TB/s), 212 by
// ordinary loads; one of 131071 tokens, 8 key heads in 4 bits 31.2, 33.6.  Rows that several tiles read do not (64 heads on one key head,
// 8 x 32000 tokens in bf16: 64 us so, 52 by ordinary loads), nor rows shorter than half a cache line, whose line is another head's too (24 x 9000
// tokens in 4 bits, 16 key heads of 64 values, a window of 4096: 27.8, 25.2).
// Sequences that share their pages read the same rows all the same, and lose by it: 32 over one set of 4000 positions, 8 key heads of bf16 44.2 us, 39.4 by
// ordinary loads, 32 key heads 220 and 143, in 4 bits both 23.2 (80.3 and 90.7 with pages of their own).  The tables, which say so, are on the device.
template <bool ONCE, class T>
__device__ __forceinline__ T read_row(const T *p)
{
    if constexpr (ONCE) return __builtin_nontemporal_load(p);
    else return *p;
}

// EIGHT: tiles of 8 rows.  The other 8 columns of the products hold the same rows, with the lower halves of the weights in the second one.
// ALONE: one tile holds all rows of a key head.
template <PagedType TY, int DP, bool FULL, bool EIGHT, bool ALONE>
__device__ __forceinline__ void paged_rows(const PagedArgs &a, const int block, char *lds)
{
    using S = PagedRowsShape<TY, DP, FULL>;
    constexpr int ES = paged_es(TY);
    constexpr bool FOUR = TY == PAGED_4BIT;
    constexpr bool ONCE = ALONE && (!FOUR || DP >= 128);
    constexpr int KB = S::KB, KS = S::KS, PITCH = S::PITCH, WAVES = S::WAVES, TILE = EIGHT ? 8 : 16;
    constexpr int NW = DP / 32;                              // 4 bits: words of a quarter of a row; also its chunks of 8 values
    constexpr int CH = FOUR ? NW : DP * ES / 64;             // operand chunks of a row: 16 bytes of every lane group each
    constexpr int DB = DP / 16;                              // tiles of 16 output dimensions
    constexpr int CPR = DP * ES / 16;                        // 16-byte chunks of a row of bf16 or fp32
    constexpr int VL = FOUR ? 1 : KS * CPR / 64;             // 16-byte loads of V a lane and step
    constexpr int NU = NW == 7 ? 3 : NW == 1 || NW == 2 || NW == 4 ? 1 : 2;     // blocks of 32 values that a quarter of a row touches, at most
    static_assert(ES == 2 || DP % 64 == 0, "whole loads of V");
    static_assert(DP % 16 == 0, "whole tiles");

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n16 = lane & 15, g = lane >> 4, n = n16 % TILE;     // n: the lane's row of the tile
    const int Dd = FULL ? DP : a.D;
    const PagedKV &pg = a.pg;

    int id = block;
    const int split = id % a.splits;
    id /= a.splits;
    const int tile = id % a.own_tiles;
    id /= a.own_tiles;
    const int h = id % a.Hkv, b = id / a.Hkv;
    const int rows = a.T * a.G, r0 = tile * TILE;

    // this lane's row: its query as the second operand.  (Loaded ahead of the lengths, which the keys wait for.)
    const int len_b = a.lens[b], qlen_b = a.q_lens ? a.q_lens[b] : a.T;
    const int row = min(r0 + n, rows - 1), token = a.T == 1 ? 0 : row / a.G;
    const RowAt at = row_at(a, false, b, h, row, token);
    u32x4 qf[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int off = FOUR ? g * (DP / 2) + 16 * c : 64 * c + 16 * g;
        const bool in = FULL || off < Dd * ES;
        qf[c] = *reinterpret_cast<const u32x4 *>(a.q + at.q + (in ? off : 0));
        if (!in) qf[c] = u32x4{0, 0, 0, 0};
    }
    int len, qlen;
    sequence_lens(a, len_b, qlen_b, len, qlen);
    const RowSpan span = paged_span(a, b, token, len, qlen);
    const float slope2 = paged_slope2(a, h * a.G + row - token * a.G);
    // keys that any row sees, and those that all see
    int any0 = span.begin < span.end ? span.begin : INT32_MAX, any1 = span.end, all0 = span.begin, all1 = span.end;
    if (a.T > 1) {
#pragma unroll
        for (int o = TILE / 2; o >= 1; o >>= 1) {
            any0 = min(any0, __shfl_xor(any0, o));
            any1 = max(any1, __shfl_xor(any1, o));
            all0 = max(all0, __shfl_xor(all0, o));
            all1 = min(all1, __shfl_xor(all1, o));
        }
    }
    any0 = __builtin_amdgcn_readfirstlane(any0);
    any1 = __builtin_amdgcn_readfirstlane(any1);
    all0 = __builtin_amdgcn_readfirstlane(all0);
    all1 = __builtin_amdgcn_readfirstlane(all1);
    const int begin = any1 > 0 ? any0 & ~(KS - 1) : 0, keys = any1 - begin;
    int chunk = (keys + a.splits - 1) / a.splits;
    chunk = (chunk + KS - 1) / KS * KS;
    const int64_t from = (int64_t)split * chunk;
    const int k0 = from < keys ? begin + (int)from : any1, k1 = min(k0 + min(chunk, keys), any1);
    const int last16 = k1 > k0 ? (k1 - 1) & ~15 : 0, last = last16 & ~(KS - 1);

    const char *kp = pg.k + h * pg.sh * 16, *vp = pg.v + h * pg.sh * 16;
    const unsigned char *ksp = pg.ks + h * pg.sh, *vsp = pg.vs + h * pg.sh;
    const scalar_i32 table = (scalar_i32)(uintptr_t)(pg.table + b * pg.table_stride);
    char *my_v = lds + wave * KS * PITCH;

    f32x4 o[DB];
    float m = NEG_INF, l = 0.0f;
#pragma unroll
    for (int d = 0; d < DB; ++d) o[d] = f32x4{0, 0, 0, 0};

    // The step's pages, and rows on their way.  A page that is not there is read as page 0 (and not used).
    const bool one_page = pg.shift >= S::KS_BITS;            // of a step
    int entry[KB];                                           // of the table, as it stands there: nothing waits for it before it is used
    int there = 0, there_next = 0;                           // a bit for every block that has a page: of the step, and of the one behind it
    auto look = [&](int i) {
        entry[0] = table[min(i, one_page ? last : last16) >> pg.shift];
        if (!one_page) {
#pragma unroll
            for (int kb = 1; kb < KB; ++kb) entry[kb] = table[min(i + 16 * kb, last16) >> pg.shift];
        }
    };
    int64_t unit[KB];                                        // where the blocks of the step that is loaded lie
    auto aim = [&](int i) {
        const int in_page = (1 << pg.shift) - 1;
        const bool ok = (unsigned int)entry[0] < (unsigned int)pg.pages;
        unit[0] = paged_unit_at(pg, ok ? entry[0] : 0, min(i, one_page ? last : last16) & in_page);
        if (one_page) {
            there_next = ok ? (1 << KB) - 1 : 0;
#pragma unroll
            for (int kb = 1; kb < KB; ++kb) unit[kb] = unit[0] + kb * 16 * (int64_t)pg.sn;
        } else {
            there_next = ok;
#pragma unroll
            for (int kb = 1; kb < KB; ++kb) {
                const bool ok_kb = (unsigned int)entry[kb] < (unsigned int)pg.pages;
                unit[kb] = paged_unit_at(pg, ok_kb ? entry[kb] : 0, min(i + 16 * kb, last16) & in_page);
                there_next |= ok_kb ? 1 << kb : 0;
            }
        }
    };
    u32x4 kf[FOUR ? 1 : KB][CH], vf[VL];
    typename Words<NW>::type kc[FOUR ? KB : 1], vc[FOUR ? KB : 1];
    unsigned char ku[FOUR ? KB : 1][NU], vu[FOUR ? KB : 1][NU];
    const unsigned int lane_row = (unsigned int)n16 * pg.sn;
    const int scale0 = g * NW >> 2;                          // first block of 32 of this lane's quarter
    auto load_k = [&]() {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            const char *p = kp + unit[kb] * 16;
            if constexpr (FOUR) {
                kc[kb] = read_row<ONCE>(reinterpret_cast<const typename Words<NW>::type *>(p + (lane_row * 16 + (unsigned int)(g * (DP / 8)))));
#pragma unroll
                for (int j = 0; j < NU; ++j) ku[kb][j] = (ksp + unit[kb])[lane_row + (unsigned int)min(scale0 + j, NW - 1)];
            } else
#pragma unroll
                for (int c = 0; c < CH; ++c) {
                    const int off = 64 * c + 16 * g;
                    const bool in = FULL || off < Dd * ES;
                    kf[kb][c] = read_row<ONCE>(reinterpret_cast<const u32x4 *>(p + (lane_row * 16 + (unsigned int)(in ? off : 0))));
                    if (!in) kf[kb][c] = u32x4{0, 0, 0, 0};
                }
        }
    };
    auto load_v = [&]() {
        if constexpr (FOUR) {
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
                vc[kb] = read_row<ONCE>(reinterpret_cast<const typename Words<NW>::type *>(vp + unit[kb] * 16 + (lane_row * 16 + (unsigned int)(g * (DP / 8)))));
#pragma unroll
                for (int j = 0; j < NU; ++j) vu[kb][j] = (vsp + unit[kb])[lane_row + (unsigned int)min(scale0 + j, NW - 1)];
            }
        } else
#pragma unroll
            for (int j = 0; j < VL; ++j) {                   // bf16: chunks in order of the rows, for LDS; fp32: key 4 g + j % 4, 64 values a load
                constexpr int PER = 16 * CPR / 64;           // loads of a block
                const int kb = ES == 2 ? j / PER : 0, x = ES == 2 ? lane + 64 * (j % PER) : 0;
                const int key = ES == 2 ? x / CPR : 4 * g + j % 4, col = ES == 2 ? x % CPR : 16 * (j / 4) + n16;
                const bool in = FULL || col * 16 < Dd * ES;
                vf[j] = read_row<ONCE>(reinterpret_cast<const u32x4 *>(vp + unit[kb] * 16 + ((unsigned int)key * pg.sn * 16 + (unsigned int)(in ? col * 16 : 0))));
                if (!in) vf[j] = u32x4{0, 0, 0, 0};
            }
    };
    // Rows of V that no row sees may hold anything: zeros for them.
    auto clean_v = [&](int i) {
        auto dead = [&](int kb, int key) { return !(there >> kb & 1) || i + 16 * kb + key < any0 || i + 16 * kb + key >= any1; };
        if constexpr (FOUR) {
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
                if (dead(kb, n16)) {
                    vc[kb] = 0;
#pragma unroll
                    for (int j = 0; j < NU; ++j) vu[kb][j] = 127;
                }
        } else
#pragma unroll
            for (int j = 0; j < VL; ++j) {
                constexpr int PER = 16 * CPR / 64;
                const int kb = ES == 2 ? j / PER : 0, key = ES == 2 ? (lane + 64 * (j % PER)) / CPR : 4 * g + j % 4;
                if (dead(kb, key)) vf[j] = u32x4{0, 0, 0, 0};
            }
    };
    auto scale_of = [&](const unsigned char (&u)[NU], int c) {     // of word c
        const int j = NU == 1 ? 0 : NW == 8 ? c >> 2 : ((g * NW + c) >> 2) - scale0;
        unsigned int v = u[0];
#pragma unroll
        for (int x = 1; x < NU; ++x) v = j == x ? u[x] : v;
        return paged_scale(v);
    };
    auto word = [](const typename Words<NW>::type &w, int c) {
        if constexpr (NW == 1) return w;
        else return w[c];
    };

    int i = k0 + wave * KS;
    if (i < k1) {
        look(i);
        aim(i);
        look(i + WAVES * KS);
        load_k();
        load_v();
    }
    for (; i < k1; i += WAVES * KS) {
        const int next = i + WAVES * KS;
        there = there_next;
        aim(next);
        look(next + WAVES * KS);
        const bool edge = i < all0 || i + KS > all1 || i + KS > k1 || there != (1 << KB) - 1;
        // scores of KS keys: lane holds keys 16 kb + 4 g + e of its row
        f32x4 s[KB];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            s[kb] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                if constexpr (TY == PAGED_F32) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const unsigned int ka = kf[kb][c][e], qb = qf[c][e];
                        s[kb] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(ka), __uint_as_float(qb), s[kb], 0, 0, 0);
                    }
                } else {
                    u32x4 k;
                    if constexpr (FOUR) k = paged_bf16x8(word(kc[kb], c), scale_of(ku[kb], c));
                    else k = kf[kb][c];
                    s[kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k), __builtin_bit_cast(bf16x8, qf[c]), s[kb], 0, 0, 0);
                }
            }
        }
        if (edge) clean_v(i);
        if constexpr (FOUR) {
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int c = 0; c < NW; ++c)
                    *reinterpret_cast<u32x4 *>(my_v + (16 * kb + n16) * PITCH + g * (DP / 2) + 16 * c) = paged_bf16x8(word(vc[kb], c), scale_of(vu[kb], c));
        } else if constexpr (ES == 2) {
#pragma unroll
            for (int j = 0; j < VL; ++j) {
                const int x = lane + 64 * j;
                *reinterpret_cast<u32x4 *>(my_v + x / CPR * PITCH + x % CPR * 16) = vf[j];
            }
        }
        if (next < k1) {
            load_k();
            if (ES == 2) load_v();                           // (in LDS by now)
        }
        __builtin_amdgcn_wave_barrier();

        paged_scores<TY, 4>(a, s, slope2, (float)(i + 4 * g - span.pos), [](int kb, int e) { return 16 * kb + e; });
        if (edge) {
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int key = i + 16 * kb + 4 * g + e;
                    if (!((there >> kb & 1) && key < k1 && key >= span.begin && key < span.end)) s[kb][e] = NEG_INF;
                }
        }
        float top = NEG_INF;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int e = 0; e < 4; ++e) top = fmaxf(top, s[kb][e]);
        if (__any(top > m + 8.0f)) {                         // (weights up to 2^8 lose nothing)
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
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

        if constexpr (ES == 2) {
#pragma unroll
            for (int k2 = 0; k2 < (KB + 1) / 2; ++k2) {      // 32 keys a product (or 16)
                u32x4 hi = {}, lo = {};
#pragma unroll
                for (int w = 0; w < (KB == 1 ? 2 : 4); ++w) {
                    const float p0 = s[2 * k2 + (w >> 1)][2 * (w & 1)], p1 = s[2 * k2 + (w >> 1)][2 * (w & 1) + 1];
                    const unsigned int u = pack_bf16(p0, p1);
                    const unsigned int rest = pack_bf16(p0 - __uint_as_float(u << 16), p1 - __uint_as_float(u & 0xffff0000u));
                    hi[w] = EIGHT && n16 >= 8 ? rest : u;
                    lo[w] = rest;
                }
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    const char *src = my_v + (32 * k2 + 4 * g + (n16 >> 2)) * PITCH + d * 32 + (n16 & 3) * 8;
                    if constexpr (KB == 1) {
                        const s16x4 vt = __builtin_bit_cast(s16x4, read_tr16(src));
                        o[d] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(vt, __builtin_bit_cast(s16x4, make_uint2(hi[0], hi[1])), o[d], 0, 0, 0);
                        if (!EIGHT) o[d] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(vt, __builtin_bit_cast(s16x4, make_uint2(lo[0], lo[1])), o[d], 0, 0, 0);
                    } else {
                        const uint2 u0 = read_tr16(src), u1 = read_tr16(src + 16 * PITCH);
                        const bf16x8 vt = __builtin_bit_cast(bf16x8, u32x4{u0.x, u0.y, u1.x, u1.y});
                        o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, __builtin_bit_cast(bf16x8, hi), o[d], 0, 0, 0);
                        if (!EIGHT) o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, __builtin_bit_cast(bf16x8, lo), o[d], 0, 0, 0);
                    }
                }
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
            if (next < k1) load_v();
        }
    }

    // The waves' results side by side in LDS; then every wave joins a part of each row's outputs: v[x] are the four from dim(x) on.
    constexpr int OUT = (DB + WAVES - 1) / WAVES;
    static_assert(ES == 2 || WAVES == 4, "an fp32 output tile has a value for each of four waves");
    auto dim = [&](int x) { return ES == 2 ? 16 * (wave + WAVES * x) + 4 * g : 64 * x + 16 * g + 4 * wave; };
    float2 *s_ml = reinterpret_cast<float2 *>(lds + WAVES * DP * 64);
    unsigned int *s_again = reinterpret_cast<unsigned int *>(lds + WAVES * (DP * 64 + 128));
    if constexpr (EIGHT && ES == 2) {
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[d][e] += dpp_move<0x128, 0xf>(o[d][e]);      // row_ror:8
    }
    f32x4 v[OUT];
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    __syncthreads();
#pragma unroll
    for (int d = 0; d < DB; ++d) reinterpret_cast<f32x4 *>(lds)[(wave * DB + d) * 64 + lane] = o[d];
    if (g == 0) s_ml[wave * 16 + n16] = make_float2(m, l);
    if (threadIdx.x == 0) *s_again = 0;
    __syncthreads();
    float2 ml[WAVES];
    m = NEG_INF;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        ml[w] = s_ml[w * 16 + n16];
        m = fmaxf(m, ml[w].x);
    }
    l = 0.0f;
#pragma unroll
    for (int x = 0; x < OUT; ++x) v[x] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        const float f = ml[w].x == NEG_INF ? 0.0f : __builtin_amdgcn_exp2f(ml[w].x - m);
        l += ml[w].y * f;
#pragma unroll
        for (int x = 0; x < OUT; ++x) {
            if (ES == 2) {
                if (DB % WAVES == 0 || wave + WAVES * x < DB) v[x] += reinterpret_cast<const f32x4 *>(lds)[(w * DB + wave + WAVES * x) * 64 + lane] * f;
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
    unsigned long long odd = __ballot(!fine && !(l != l) && r0 + n < rows);
    if (odd) {
        odd |= odd >> 32;
        if (lane == 0) atomicOr(s_again, (unsigned int)((odd | odd >> 16) & (EIGHT ? 0xff : 0xffff)));
    }
    __syncthreads();
    const unsigned int again = __builtin_amdgcn_readfirstlane(*s_again);
    if (again) {
        for (int t = wave; t < TILE; t += WAVES) {
            if (!(again >> t & 1)) continue;
            const int i2 = (r0 + t) / a.G;
            const RowAt to = row_at(a, false, b, h, r0 + t, i2);
            paged_store_row<ES>(a, paged_row<TY>(a, b, h, a.q + to.q, paged_span(a, b, i2, len, qlen), paged_slope2(a, h * a.G + r0 + t - i2 * a.G), k0, k1), to, split);
        }
    }

    const bool mine = n == n16 && r0 + n < rows && !(again >> n & 1);
    if (a.splits > 1) {
        if (mine) {
            const int64_t part = at.lse * a.splits + split;
            if (g == 0 && wave == 0) store_past(&a.part_ml[part], make_float2(m, l));
#pragma unroll
            for (int x = 0; x < OUT; ++x)
                if (dim(x) < Dd && k0 < k1) store_past4(a.part_o, (unsigned int)part * Dd + dim(x), v[x]);      // (nothing for a split that has no keys)
        }
        paged_join<ES, 64 * WAVES>(a, block / a.splits, b, h, r0, min(rows - r0, TILE), lds);
        return;
    }
    if (!mine) return;
    const bool none = l == 0.0f;                             // sees nothing, or only scores of -inf
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
