// The many-row body of clada_paged_attn: prompts and chunks.
//
// The same sums as in paged_rows.h.  A workgroup of four waves takes 128 rows, 32 a wave; K and V tiles go through registers into one of two LDS
// buffers while the other is multiplied, one barrier a tile.  Two workgroups share a compute unit, so that one's products can run under the
// other's exponentials.  bf16: 32x32x16 products and tiles of 64 keys (32 for more than 128 values); fp32: 32x32x2 and 32 keys, weights in fp32.
//
// Rows of 4 bits become bf16 on their way into LDS, 32 values a thread, so that the products are those of bf16 pages.
//
// Scores are formed transposed (S^T = K Q^T): a lane holds scores of one row only, keys 8 (i / 4) + 4 (lane / 32) + i % 4 of each 32, and the same
// registers are the second operand of O^T = V^T P^T when its keys are counted in that order (16-bit V is turned by ds_read_tr16).  Weights are
// rounded to bf16 there (2^-8 at most, to nearest: the size of the output's own rounding); their sum is taken before it.  Outputs are 0.0021 to 0.0023 off then,
// 0.0016 by two bf16 a weight, which take the three cases below to 726, 219 and 184 us.
//
// Every row sees an interval of keys, so a tile is looked at key by key only where an interval begins or ends, or a page is missing.  Tiles are taken
// from the last one down: a row's own key, and with a slope the least of its bias, comes first, so that its maximum is set once and a
// steady loop without a scaling of the sums does for the rest (one inside the loop costs a second set of registers for all of them).
//
// Bound by the matrix and vector units in turn and the clock that they leave (of 2.4 GHz): 8192 tokens, 32 heads on 8 of 128 bf16 values: 556 us, 0.99 PFLOP/s,
// matrix units 49 %, vector units 43 % of the cycles, at 1.80 GHz; of 5 documents, capped: 183 us, 0.60 PFLOP/s of useful pairs, 26 and 49 % at 2.08; 2 x 512
// tokens behind 8000 and 6766 in 4 bits 148 us, 0.81, 35 and 37 % at 2.19.  1000 and 737 tokens of 32 fp32 heads of 80: 152 us, 58 TFLOP/s, the compute units
// busy for 66 % of it (equal tiles, unequal lengths), the matrix units for 42 %, a sixth of that for the padding of 80 to 96.  Scores of the next tile between the products of this one need
// twice the registers: spilled at two waves a SIMD (chunk 249 us), 192 us at one; 64 rows a wave 185.
#pragma once
#include <type_traits>

#include "paged_rows.h"

namespace {

template <PagedType TY, int DP>
struct PagedTilesShape {
    static constexpr int ES = paged_es(TY);
    static constexpr int KT = ES == 2 && DP <= 128 ? 64 : 32, KT_BITS = KT == 64 ? 6 : 5;        // keys of a tile
    static constexpr int KP = DP * ES + 16, VP = DP * ES + (ES == 4 ? 16 : DP % 64 ? 0 : 64);      // row pitches: K rows 4 banks apart, bf16 V rows 16 or 48
    static constexpr int BUF = KT * (KP + VP), LDS = 2 * BUF;
};

// What the scores have beside a scale: nothing, a cap alone (not in fp32), anything.
enum PagedMods { MODS_NONE, MODS_CAP, MODS_ANY };

template <PagedType TY, int DP, bool FULL, PagedMods MODS>
__device__ __forceinline__ void paged_tiles(const PagedArgs &a, const int id, char *lds)
{
    using S = PagedTilesShape<TY, DP>;
    constexpr int ES = S::ES, KT = S::KT, KB = KT / 32, KP = S::KP, VP = S::VP, BUF = S::BUF, NB = KT / 16;
    constexpr bool FOUR = TY == PAGED_4BIT;
    constexpr int KD = DP * ES / 32, DB = DP / 32;           // 32-byte chunks of a row, 16 bytes a lane; tiles of 32 output dimensions
    constexpr int CPR = DP == 96 ? 128 / (16 / ES) : DP * ES / 16;       // threads a row, 16 bytes each
    constexpr int ROWS = FOUR ? 1 : KT * CPR / 256, RPP = FOUR ? 1 : 256 / CPR;      // rows of K (and of V) a thread stages; rows of a pass
    constexpr bool WHOLE = FULL && CPR * 16 == DP * ES;      // every thread has a chunk of the row
    constexpr int NG = DP / 32;                              // 4 bits: blocks of a row, a thread each
    constexpr int PUTS = FOUR ? 8 : 2 * ROWS;                // 16-byte writes into LDS a thread and tile
    static_assert(FOUR ? KT * NG <= 256 : KT * CPR % 256 == 0 && 256 % CPR == 0, "whole passes");

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6) & 3;
    const int n32 = lane & 31, hh = lane >> 5, t16 = lane & 15, g = lane >> 4;
    const int Dd = FULL ? DP : a.D;
    const PagedKV &pg = a.pg;

    // Units (sequence, key head) fastest: consecutive workgroups go to different XCDs, so a unit's tiles share an L2.  The last row tiles see the
    // most keys and come first; where all workgroups are resident at once, two on a compute unit, the second half comes in the other order, so that a long
    // one shares its unit with a short one.
    const int units = a.B * a.Hkv;
    const int unit = id % units, rest = id / units;
    const int split = rest % a.splits, order = rest / a.splits, half = (a.own_tiles + 1) / 2;
    const int tile = !a.snake || order < half ? a.own_tiles - 1 - order : order - half;
    const int h = unit % a.Hkv, b = unit / a.Hkv;
    const int rows = a.T * a.G, r0 = tile * 128;

    // this lane's row, and the keys that it, its wave's and all rows see
    const int r = r0 + wave * 32 + n32, rc = min(r, rows - 1), token = rc / a.G;
    const bool idle = r0 + wave * 32 >= rows;
    int len, qlen;
    sequence_lens(a, a.lens[b], a.q_lens ? a.q_lens[b] : a.T, len, qlen);
    const RowSpan span = paged_span(a, b, token, len, qlen);
    const float slope2 = MODS == MODS_ANY ? paged_slope2(a, h * a.G + rc - token * a.G) : 0.0f;
    int any0 = !idle && span.begin < span.end ? span.begin : INT32_MAX, any1 = idle ? 0 : span.end, all0 = span.begin, all1 = span.end;
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) {
        any0 = min(any0, __shfl_xor(any0, o));
        any1 = max(any1, __shfl_xor(any1, o));
        all0 = max(all0, __shfl_xor(all0, o));
        all1 = min(all1, __shfl_xor(all1, o));
    }
    const int wave0 = __builtin_amdgcn_readfirstlane(any0), wave1 = __builtin_amdgcn_readfirstlane(any1);
    all0 = __builtin_amdgcn_readfirstlane(all0);
    all1 = __builtin_amdgcn_readfirstlane(all1);
    int *s_range = reinterpret_cast<int *>(lds);
    if (lane == 0) {
        s_range[wave] = wave0;
        s_range[4 + wave] = wave1;
    }
    __syncthreads();
    const int low = __builtin_amdgcn_readfirstlane(min(min(s_range[0], s_range[1]), min(s_range[2], s_range[3])));
    const int high = __builtin_amdgcn_readfirstlane(max(max(s_range[4], s_range[5]), max(s_range[6], s_range[7])));
    __syncthreads();
    const int begin = high > 0 ? low & ~(KT - 1) : 0, n = high - begin;
    int chunk = (n + a.splits - 1) / a.splits;
    chunk = (chunk + KT - 1) / KT * KT;
    const int64_t from = (int64_t)split * chunk;
    const int k0 = from < n ? begin + (int)from : high, k1 = min(k0 + min(chunk, n), high);
    const int last16 = k1 > k0 ? (k1 - 1) & ~15 : 0, last = last16 & ~(KT - 1);

    const unsigned int flip = MODS == MODS_NONE && a.scale2 < 0.0f ? (ES == 2 ? 0x80008000u : 0x80000000u) : 0u;     // a negative scale is the queries' sign
    const float scale2 = fmaxf(fabsf(a.scale2), 0x1p-149f);  // positive, so that -inf stays what it is
    u32x4 qf[KD];
#pragma unroll
    for (int c = 0; c < KD; ++c) {
        const int off = 32 * c + 16 * hh;
        const bool in = FULL || off < Dd * ES;
        qf[c] = *reinterpret_cast<const u32x4 *>(a.q + row_at(a, false, b, h, rc, token).q + (in ? off : 0));
#pragma unroll
        for (int e = 0; e < 4; ++e) qf[c][e] = in ? qf[c][e] ^ flip : 0u;
    }
    // (here, once: a wait for them inside the loop would be one for the tiles on their way too)
#pragma unroll
    for (int c = 0; c < KD; ++c) asm volatile("" : "+v"(qf[c]));

    // Staging.  16 and 32 bits: a wave's rows of a pass lie in one 16-key block, whose page is a scalar; 4 bits: a thread has one row of K and of V.
    // A page that is not there is read as page 0 (and not used).
    const char *kp = pg.k + h * pg.sh * 16, *vp = pg.v + h * pg.sh * 16;
    const unsigned char *ksp = pg.ks + h * pg.sh, *vsp = pg.vs + h * pg.sh;
    const scalar_i32 table = (scalar_i32)(uintptr_t)(pg.table + b * pg.table_stride);
    const int in_page = (1 << pg.shift) - 1;
    const bool one_page = pg.shift >= S::KT_BITS;            // of a tile
    const int first_key = FOUR ? tid / NG : tid / CPR, col = FOUR ? tid % NG : tid % CPR * 16;
    const bool in = FOUR ? first_key < KT : WHOLE || col < Dd * ES;
    const unsigned int lane_off = FOUR ? 0u : (unsigned int)(lane / CPR) * pg.sn * 16 + (in ? col : 0);
    const unsigned int lane_unit = (unsigned int)(first_key & (KT - 1)) * pg.sn + (in ? col : 0);      // 4 bits
    int64_t step[ROWS];                                      // of a pass, in a tile of one page
#pragma unroll
    for (int j = 0; j < ROWS; ++j) step[j] = (int64_t)(wave * (64 / CPR) + j * RPP) * pg.sn * 16;
    u32x4 sk[ROWS], sv[ROWS];                                // the tile on its way into LDS
    unsigned int uk = 127, uv = 127;
    int entry[NB];                                           // of the table, of the tile that is fetched next, as they stand there: nothing waits for them here
    int there_reg = 0, there = 0;                            // a bit for every block that has a page: of the tile in registers, of the one in LDS
    auto look = [&](int i) {
        entry[0] = table[max(min(i, one_page ? last : last16), k0) >> pg.shift];
        if (!one_page) {
#pragma unroll
            for (int x = 1; x < NB; ++x) entry[x] = table[max(min(i + 16 * x, last16), k0) >> pg.shift];
        }
    };
    int64_t at_j[ROWS], at_u = 0;                            // where the rows of the tile that is taken lie
    auto aim = [&](int i) {
        // (rows past the last block are read as rows of it, and those ahead of the first one as its)
        constexpr int ALL = (1 << NB) - 1;
        if (one_page) {
            const bool ok = (unsigned int)entry[0] < (unsigned int)pg.pages;
            there_reg = ok ? ALL : 0;
            const int64_t unit = paged_unit_at(pg, ok ? entry[0] : 0, max(min(i, last), k0) & in_page);
            if constexpr (FOUR) at_u = unit + (int64_t)lane_unit;
            else
#pragma unroll
                for (int j = 0; j < ROWS; ++j) at_j[j] = (unit << 4) + step[j];
            return;
        }
        int64_t unit[NB];
        there_reg = 0;
#pragma unroll
        for (int x = 0; x < NB; ++x) {
            const bool ok = (unsigned int)entry[x] < (unsigned int)pg.pages;
            unit[x] = paged_unit_at(pg, ok ? entry[x] : 0, max(min(i + 16 * x, last16), k0) & in_page);
            there_reg |= ok ? 1 << x : 0;
        }
        if constexpr (FOUR) {
            const int x = (first_key & (KT - 1)) >> 4;
            at_u = unit[0];
#pragma unroll
            for (int y = 1; y < NB; ++y) at_u = x == y ? unit[y] : at_u;
            at_u += (unsigned int)(first_key & 15) * pg.sn + (in ? col : 0);
        } else
#pragma unroll
            for (int j = 0; j < ROWS; ++j) {
                const int first = wave * (64 / CPR) + j * RPP, x = first / 16;      // the wave's first row of the pass, and its block
                int64_t u = unit[0];
#pragma unroll
                for (int y = 1; y < NB; ++y) u = x == y ? unit[y] : u;
                at_j[j] = (u + (first % 16) * (int64_t)pg.sn) * 16;
            }
    };
    auto take = [&](int q) {                                 // transfer q of that tile: K, V, K, ..
        if constexpr (FOUR) {
            if (q & 1) {
                sv[0] = *reinterpret_cast<const u32x4 *>(vp + at_u * 16);
                uv = vsp[at_u];
            } else {
                sk[0] = *reinterpret_cast<const u32x4 *>(kp + at_u * 16);
                uk = ksp[at_u];
            }
        } else {
            const int j = q / 2;
            if (q & 1) sv[j] = *reinterpret_cast<const u32x4 *>(vp + at_j[j] + lane_off);
            else sk[j] = *reinterpret_cast<const u32x4 *>(kp + at_j[j] + lane_off);
        }
    };
    auto fetch = [&](int i) {
        aim(i);
#pragma unroll
        for (int q = 0; q < 2 * ROWS; ++q) take(q);
    };
    // (threads without a chunk write into the padding of a row of K and no V; 4 bits: threads without a row write nothing)
    // The 16-byte chunks of each 64 bytes of a row of bf16 V change places by the row, so that neither the reads nor the writes of four rows meet in a
    // bank (with bf16 pages no conflicts are counted then; in 4 bits, where a thread writes 64 bytes of a row, 7 million cycles in the chunk).
    const unsigned int put_at = FOUR ? col * 64 : min(col, DP * ES), turn = ES == 2 ? (first_key & 3) * 16 : 0;
    const unsigned int put_k = first_key * KP + put_at, put_v = KT * KP + first_key * VP + (FOUR ? put_at : put_at ^ turn);
    auto put_one = [&](int buf, int q) {                     // write q into LDS
        if constexpr (FOUR) {
            if (KT * NG < 256 && !in) return;
            const int c = q & 3;
            char *to = lds + ((q & 4 ? put_v : put_k) + buf * BUF) + (q & 4 ? c * 16 ^ turn : c * 16);
            *reinterpret_cast<u32x4 *>(to) = q & 4 ? paged_bf16x8(sv[0][c], paged_scale(uv)) : paged_bf16x8(sk[0][c], paged_scale(uk));
        } else {
            if ((q & 1) && CPR * 16 > DP * ES && col >= DP * ES) return;
            const int j = q / 2;
            u32x4 x = q & 1 ? sv[j] : sk[j];
            if (!WHOLE && !in) x = u32x4{0, 0, 0, 0};
            char *to = lds + ((q & 1 ? put_v : put_k) + buf * BUF) + j * RPP * (q & 1 ? VP : KP);
            *reinterpret_cast<u32x4 *>(to) = x;
        }
    };
    auto clean = [&](int i) { return i >= low && i + KT <= k1 && there_reg == (1 << NB) - 1; };     // the tile in registers, at i
    auto put = [&](int buf, int i) {
        if (!clean(i)) {                                     // rows of V that no row sees may hold anything: zeros for them
#pragma unroll
            for (int j = 0; j < ROWS; ++j) {
                const int key = first_key + j * RPP;
                if (i + key < low || i + key >= k1 || !(there_reg >> (key >> 4) & 1)) {
                    sv[j] = u32x4{0, 0, 0, 0};
                    uv = 127;
                }
            }
        }
#pragma unroll
        for (int q = 0; q < PUTS; ++q) put_one(buf, q);
        there = there_reg;
    };

    f32x16 o[DB];
    float m = NEG_INF, l = 0.0f;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[d][e] = 0.0f;
    // MODS_CAP: a steady tile takes cap2 tanh(x kappa) as x times a polynomial of x^2, x the product.
    float cap_k[5] = {};
    if constexpr (MODS == MODS_CAP) {
        constexpr float coeff[5] = {0.99999850f, -0.33326973f, 0.13257454f, -0.05019526f, 0.013194188f};
        float f = a.cap2 * a.inv_cap_scale;
#pragma unroll
        for (int c = 0; c < 5; ++c) {
            cap_k[c] = f * coeff[c];
            f *= a.inv_cap_scale * a.inv_cap_scale;
        }
    }
    // One tile for this wave's rows.  EDGE: some of them do not see all of it, or a maximum has to be set or moved.  Otherwise the next tile goes
    // into LDS, and the one behind it is taken, transfer by transfer between the products; false, and nothing has been done, where a maximum has to be moved.
    auto multiply = [&](auto edge, int i, int buf) -> bool {
        constexpr bool EDGE = decltype(edge)::value;
        const char *kb = lds + buf * BUF, *vb = kb + KT * KP;
        auto stage = [&](int x, int of) {                    // behind product x of `of`
            if constexpr (!EDGE) {
#pragma unroll
                for (int q = PUTS * x / of; q < PUTS * (x + 1) / of; ++q) {
                    put_one(buf ^ 1, q);
                    if (!FOUR) take(q);
                    else if ((q & 3) == 3) take(q >> 2);
                }
            }
        };
        f32x16 s[KB];
        const f32x16 zero = {};
        constexpr int QKS = KD * KB, KA = QKS < 6 ? QKS : 6; // fragments of K ahead of the products
        u32x4 kf[KA];
        const char *k_lane = kb + n32 * KP + 16 * hh;
        auto read_k = [&](int x) { kf[x % KA] = *reinterpret_cast<const u32x4 *>(k_lane + x % KB * (32 * KP) + x / KB * 32); };
#pragma unroll
        for (int x = 0; x < KA; ++x) read_k(x);
#pragma unroll
        for (int x = 0; x < QKS; ++x) {
            const int c = x / KB, k = x % KB;
            if (TY == PAGED_F32 && !FULL && 32 * c >= Dd * ES) continue;      // (fp32: nothing but the products' own time counts)
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (ES == 2)
                s[k] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf[x % KA]), __builtin_bit_cast(bf16x8, qf[c]), c ? s[k] : zero, 0, 0, 0);
            else
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const unsigned int ka = kf[x % KA][e], qb = qf[c][e];
                    s[k] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(ka), __uint_as_float(qb), c || e ? s[k] : zero, 0, 0, 0);
                }
            if (x + KA < QKS) read_k(x + KA);
        }
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (MODS == MODS_ANY || (MODS == MODS_CAP && EDGE)) paged_scores<TY, 16>(a, s, slope2, (float)(i + 4 * hh - span.pos), [](int k, int e) { return k * 32 + 8 * (e >> 2) + (e & 3); });
        if constexpr (EDGE) {
            const int lo = span.begin - i - 4 * hh;
            const unsigned int width = (unsigned int)max(min(span.end, k1) - span.begin, 0);
#pragma unroll
            for (int k = 0; k < KB; ++k)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const bool seen = (unsigned int)(k * 32 + 8 * (e >> 2) + (e & 3) - lo) < width && (there >> (2 * k + (e >> 3)) & 1);
                    s[k][e] = seen ? s[k][e] : NEG_INF;
                }
        }
        constexpr bool BOUND = MODS == MODS_CAP && !EDGE;    // the largest magnitude of a product in place of the largest score
        float top = BOUND ? 0.0f : NEG_INF;
#pragma unroll
        for (int k = 0; k < KB; ++k)
#pragma unroll
            for (int e = 0; e < 16; ++e) top = fmaxf(top, BOUND ? fabsf(s[k][e]) : s[k][e]);
        if (MODS == MODS_NONE) top *= scale2;
        if constexpr (EDGE) {
            if (__any(top > m + 8.0f)) {                     // (weights above 1 lose nothing)
                top = fmaxf(top, __shfl_xor(top, 32));
                const float mn = top > m + 8.0f ? top : m;
                const float f = mn == m ? 1.0f : __builtin_amdgcn_exp2f(m - mn);
                m = mn;
                l *= f;
#pragma unroll
                for (int d = 0; d < DB; ++d) o[d] *= f;
            }
        } else {
            if (BOUND ? __any(top > a.cap_limit || top * fabsf(cap_k[0]) > m + 32.0f) : __any(top > m + 32.0f)) return false;
            there = there_reg;
            aim(i - 2 * KT);
            look(i - 3 * KT);
        }
        const float base = m == NEG_INF ? 0.0f : m;
        auto weight_of = [&](float x) {
            if constexpr (MODS == MODS_NONE) return __builtin_amdgcn_exp2f(fmaf(x, scale2, -base));
            if constexpr (BOUND) {
                const float x2 = x * x;
                float y = fmaf(cap_k[4], x2, cap_k[3]);
                y = fmaf(y, x2, cap_k[2]);
                y = fmaf(y, x2, cap_k[1]);
                y = fmaf(y, x2, cap_k[0]);
                return __builtin_amdgcn_exp2f(fmaf(x, y, -base));
            }
            return __builtin_amdgcn_exp2f(x - base);
        };
        if constexpr (ES == 2) {
            // Sixteen keys are a step of the second product.  Between the products of one step stand the exponentials of the next one and the
            // reads of V four products ahead.
            constexpr int STEPS = 2 * KB, AHEAD = STEPS * DB < 4 ? STEPS * DB : 4;
            u32x4 vt[AHEAD], pk[2];
            auto weight = [&](auto step, int e) {                // the e-th of the step's eight weights of this lane
                constexpr int st = decltype(step)::value, k = st / 2, c = st % 2;
                const float p = weight_of(s[k][8 * c + e]);
                l += p;
                s[k][8 * c + e] = p;
                if (e & 1) pk[st & 1][e >> 1] = pack_bf16(s[k][8 * c + e - 1], p);
            };
            // (row 4 hh + t16 / 4 of each 8, whose chunks are turned by t16 / 4)
            const char *src = vb + (4 * hh + (t16 >> 2)) * VP + ((((g & 1) * 2 + (t16 >> 1 & 1)) ^ (t16 >> 2)) * 16) + (t16 & 1) * 8;
            auto read_v = [&](int x) {
                const char *at = src + x / DB * 16 * VP + x % DB * 64;
                const uint2 u0 = read_tr16(at), u1 = read_tr16(at + 8 * VP);
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
                s[0][e] = weight_of(s[0][e]);
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
        return true;
    };

    int i = k0 + (k1 > k0 ? (k1 - k0 - 1) / KT * KT : -KT), buf = 0;
    if (k0 < k1) {
        look(i);
        fetch(i);
        put(0, i);
        look(i - KT);
        if (i - KT >= k0) fetch(i - KT);
        look(i - 2 * KT);
    }
    tile_barrier();
    // Where a tile is seen by all rows of the wave and the next one has no row that nobody sees.
    const int steady0 = max(all0, max(low, k0) + KT), steady1 = min(all1, k1) - KT;
    // The waves of a workgroup may be in different loops; every tile is one barrier in both.
    while (i >= k0) {
        if (i < wave1 && i + KT > wave0) multiply(std::true_type{}, i, buf);
        if (i - KT >= k0) {
            put(buf ^ 1, i - KT);
            if (i - 2 * KT >= k0) fetch(i - 2 * KT);
            look(i - 3 * KT);
        }
        for (;;) {
            tile_barrier();
            buf ^= 1;
            i -= KT;
            if (i < steady0 || i > steady1 || (there & there_reg) != (1 << NB) - 1) break;
            if (!multiply(std::false_type{}, i, buf)) break;
        }
    }
    l += __shfl_xor(l, 32);
    bool fine = true;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) fine = fine && fabsf(o[d][e]) < INFINITY;
    const unsigned long long odd = __ballot((!fine || !(l < INFINITY)) && l == l && r < rows);
    const unsigned int again = (unsigned int)odd | (unsigned int)(odd >> 32);      // a bit for every row of the wave
    for (unsigned int left = again; left; left &= left - 1) {
        const int t = __builtin_ctz(left), row = r0 + wave * 32 + t, tok = row / a.G;
        const RowAt at = row_at(a, false, b, h, row, tok);
        paged_store_row<ES>(a, paged_row<TY>(a, b, h, a.q + at.q, paged_span(a, b, tok, len, qlen), paged_slope2(a, h * a.G + row - tok * a.G), k0, k1), at, split);
    }
    if (r >= rows || (again >> n32 & 1)) return;
    const RowAt to_row = row_at(a, false, b, h, r, token);
    if (a.splits > 1) {
        const int64_t part = to_row.lse * a.splits + split;
        if (hh == 0) a.part_ml[part] = make_float2(m, l);
        if (k0 >= k1) return;
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
    const bool nothing = l == 0.0f;                          // sees nothing, or only scores of -inf
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
