// Kernels of clada_window_attn and clada_shared_prefix_attn: few rows (single tokens) run attention_rows.h, many attention_tiles.h; where
// a row's keys are split among workgroups, k_attn_join adds their results up in a second launch.
#include <math.h>

#include "attention_rows.h"
#include "attention_tiles.h"

namespace {

template <int ES, int DP, bool FULL>
__global__ void __launch_bounds__(256, ES == 2 || DP <= 128 ? 2 : 1)
k_attn_rows(const AttnArgs a)
{
    __shared__ __align__(16) char lds[RowsShape<ES, DP, FULL>::LDS];
    const int pre_blocks = a.Hkv * a.pre_tiles * a.pre_splits, id = blockIdx.x;
    attn_rows<ES, DP, FULL>(a, id < pre_blocks, id < pre_blocks ? id : id - pre_blocks, lds);
}

template <int ES, int DP, bool FULL>
__global__ void __launch_bounds__(256, DP <= 128 ? 2 : 1)
k_attn_tiles(const AttnArgs a)
{
    __shared__ __align__(16) char lds[TilesShape<ES, DP>::LDS];
    attn_tiles<ES, DP, FULL, false>(a, false, blockIdx.x, lds);
}

// A shared prefix for more than 16 rows: its workgroups first, then those of the sequences' own keys, in one launch.  Bound by the bytes of both:
// 16 sequences behind 8192 rows, 8 key heads of 128 values, 21 us (2.5 TB/s with the join); 48 behind 4095, 32 key heads, 39 (3.3).  Tiles
// of 32 rows in attention_rows.h, which read the prefix once for every 32 rows, took 48 and 93.
template <int ES, int DP, bool FULL>
__global__ void __launch_bounds__(256, DP <= 128 ? 2 : 1)
k_attn_prefix(const AttnArgs a)
{
    constexpr int L0 = TilesShape<ES, DP>::LDS, L1 = RowsShape<ES, DP, FULL>::LDS;
    __shared__ __align__(16) char lds[L0 > L1 ? L0 : L1];
    const int pre_blocks = a.Hkv * a.pre_tiles * a.pre_splits, id = blockIdx.x;
    if (id < pre_blocks) attn_tiles<ES, DP, FULL, ES == 2>(a, true, id, lds);
    else attn_rows<ES, DP, FULL>(a, false, id - pre_blocks, lds);
}

// A joined row: four outputs of a thread, and the log of the sum by the thread that holds dim 0.
template <int ES>
__device__ __forceinline__ void join_store(const AttnArgs &a, const int64_t row, const int dim, f32x4 o, const float l, const float top)
{
    const int hq = (int)(row % a.Hq);
    const int64_t bt = row / a.Hq;
    const int b = a.T == 1 ? (int)bt : (int)(bt / a.T), t = (int)(bt - (int64_t)b * a.T);
    int len, qlen;
    sequence_lens(a, a.lens[b], a.q_lens ? a.q_lens[b] : a.T, len, qlen);
    const bool none = a.pre_splits ? a.pre_n + len == 0 : t >= qlen || len - qlen + t < 0;
    if (a.lse && dim == 0) a.lse[row] = none ? NEG_INF : top * 0.69314718055994531f + logf(l);
    if (dim >= a.D) return;
    o = none ? f32x4{0, 0, 0, 0} : o * (1.0f / l);
    char *to = a.out + b * a.o_sb + t * a.o_st + hq * a.o_sh;
    if (ES == 2)
        *reinterpret_cast<uint2 *>(to + dim * 2) = make_uint2(pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3]));
    else
        *reinterpret_cast<f32x4 *>(to + dim * 4) = o;
}

// One workgroup a row: its splits' partial results joined in a fixed order.  TPR threads hold 4 values each of a row; the 256 / TPR groups take
// splits in turn and are joined through LDS.  A split's factor is computed by one thread for all.
// 4 us for 256 rows of four splits, 5 for 512 rows of 34: latency of a launch and two dependent loads.
template <int ES, int TPR>
__global__ void __launch_bounds__(256)
k_attn_join(const AttnArgs a)
{
    constexpr int GR = 256 / TPR;
    __shared__ float s_f[256], s_red[8];
    __shared__ f32x4 s_o[GR][TPR];
    const int64_t row = blockIdx.x;
    const int splits = a.splits + a.pre_splits, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int gr = tid / TPR, dim = tid % TPR * 4;
    float l = 0.0f, top = NEG_INF;
    f32x4 o = {0, 0, 0, 0};
    const float *po = a.part_o + row * splits * a.D + dim;
    f32x4 first[4];                                          // on their way while the factors are formed
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (gr + j * GR < splits && dim < a.D) first[j] = *reinterpret_cast<const f32x4 *>(po + (int64_t)(gr + j * GR) * a.D);
    for (int s0 = 0; s0 < splits; s0 += 256) {               // (512 splits at most: two rounds)
        const float2 v = s0 + tid < splits ? a.part_ml[row * splits + s0 + tid] : make_float2(NEG_INF, 0.0f);
        const float most = wave_max(v.x);
        __syncthreads();
        if (lane == 0) s_red[wave] = most;
        __syncthreads();
        const float mn = fmaxf(top, fmaxf(fmaxf(s_red[0], s_red[1]), fmaxf(s_red[2], s_red[3])));
        // a split without keys has written no values: none are used for it
        const float f = v.x == NEG_INF ? 0.0f : __builtin_amdgcn_exp2f(v.x - mn), g = top == NEG_INF ? 0.0f : __builtin_amdgcn_exp2f(top - mn);
        s_f[tid] = v.y == 0.0f ? -1.0f : f;
        const float sum = wave_sum(v.x == NEG_INF ? v.y : v.y * f);
        if (lane == 0) s_red[4 + wave] = sum;
        __syncthreads();
        l = l * g + ((s_red[4] + s_red[5]) + (s_red[6] + s_red[7]));
        o *= g;
        top = mn;
        const int n = min(splits - s0, 256);
        if (dim >= a.D) continue;
        int s = gr;
        if (s0 == 0) {
#pragma unroll
            for (int j = 0; j < 4; ++j, s += GR)
                if (s < n && s_f[s] != -1.0f) o += first[j] * s_f[s];
        }
#pragma unroll 4
        for (; s < n; s += GR) {
            const float fs = s_f[s];
            if (fs != -1.0f) o += *reinterpret_cast<const f32x4 *>(po + (int64_t)(s0 + s) * a.D) * fs;
        }
    }
    s_o[gr][tid % TPR] = o;
    __syncthreads();
    if (gr) return;
#pragma unroll
    for (int k = 1; k < GR; ++k) o += s_o[k][tid];
    join_store<ES>(a, row, dim, o, l, top);
}

// The same for at most FEW_SPLITS: TPR threads a row, 256 / TPR rows a workgroup, every thread forms the factors for itself; no LDS, no barriers.
// Loads are not conditional, so that all are in flight together (with conditions 186 registers and slower than a workgroup a row up to 2112 rows).
constexpr int FEW_SPLITS = 8;
template <int ES, int TPR>
__global__ void __launch_bounds__(256)
k_attn_join_few(const AttnArgs a)
{
    const int64_t row = (int64_t)blockIdx.x * (256 / TPR) + threadIdx.x / TPR;
    if (row >= (int64_t)a.B * a.T * a.Hq) return;
    const int splits = a.splits + a.pre_splits, dim = threadIdx.x % TPR * 4;
    const float *po = a.part_o + row * splits * a.D + (dim < a.D ? dim : 0);
    float2 v[FEW_SPLITS];
    f32x4 part[FEW_SPLITS];
#pragma unroll
    for (int s = 0; s < FEW_SPLITS; ++s) {
        const int at = min(s, splits - 1);                   // (those past the last read it again and count for nothing)
        v[s] = a.part_ml[row * splits + at];
        part[s] = *reinterpret_cast<const f32x4 *>(po + at * a.D);
    }
#pragma unroll
    for (int s = 0; s < FEW_SPLITS; ++s) {
        if (s >= splits) v[s] = make_float2(NEG_INF, 0.0f);
        if (v[s].y == 0.0f) part[s] = f32x4{0, 0, 0, 0};     // a split without keys has written no values
    }
    float l = 0.0f, top = NEG_INF;
    f32x4 o = {0, 0, 0, 0};
#pragma unroll
    for (int s = 0; s < FEW_SPLITS; ++s) top = fmaxf(top, v[s].x);
#pragma unroll
    for (int s = 0; s < FEW_SPLITS; ++s) {
        const float f = v[s].x == NEG_INF ? 0.0f : __builtin_amdgcn_exp2f(v[s].x - top);
        l += v[s].x == NEG_INF ? v[s].y : v[s].y * f;
        o += part[s] * f;
    }
    join_store<ES>(a, row, dim, o, l, top);
}

template <int ES, int TPR>
void launch_join(const AttnArgs &a, int num_cu, hipStream_t stream)
{
    const int64_t rows = (int64_t)a.B * a.T * a.Hq;
    constexpr int RW = 256 / TPR;
    // Whole calls, us, a workgroup a row against this: 8 rows 14.3 / 14.9, 256 rows even, 1280 rows of 64 values 16.6 / 15.4, 4096 rows 22.0 / 17.6,
    // 8192 rows of 128 values 43.0 / 36.2, 4096 rows of 256 values 55.7 / 53.1.
    if (rows > 4 * num_cu && a.splits + a.pre_splits <= FEW_SPLITS)
        hipLaunchKernelGGL((k_attn_join_few<ES, TPR>), dim3((unsigned int)((rows + RW - 1) / RW)), dim3(256), 0, stream, a);
    else
        hipLaunchKernelGGL((k_attn_join<ES, TPR>), dim3((unsigned int)rows), dim3(256), 0, stream, a);
}

template <int ES, int DP, bool FULL>
void launch_full(const AttnArgs &a, AttnPath path, dim3 grid, hipStream_t stream)
{
    if (path == ATTN_TILES) hipLaunchKernelGGL((k_attn_tiles<ES, DP, FULL>), grid, dim3(256), 0, stream, a);
    if constexpr (ES == 2 || DP % 64 == 0) {                 // (the rows of the fp32 kernels come in 64 values)
        if (path == ATTN_ROWS) hipLaunchKernelGGL((k_attn_rows<ES, DP, FULL>), grid, dim3(256), 0, stream, a);
        if (path == ATTN_PREFIX) hipLaunchKernelGGL((k_attn_prefix<ES, DP, FULL>), grid, dim3(256), 0, stream, a);
    }
}

template <int ES, int DP>
void launch(const AttnArgs &a, AttnPath path, dim3 grid, hipStream_t stream)
{
    if (a.D == DP) launch_full<ES, DP, true>(a, path, grid, stream);
    else launch_full<ES, DP, false>(a, path, grid, stream);
}

template <int ES>
void launch_type(const AttnArgs &a, AttnPath path, dim3 grid, hipStream_t stream)
{
    if (a.D <= 64) launch<ES, 64>(a, path, grid, stream);
    else if (a.D <= 96 && (ES == 2 || path == ATTN_TILES)) launch<ES, 96>(a, path, grid, stream);
    else if (a.D <= 128) launch<ES, 128>(a, path, grid, stream);
    else launch<ES, 256>(a, path, grid, stream);
}

}  // namespace

hipError_t clada_attn_launch(const AttnArgs &a, int es, AttnPath path, int num_cu, hipStream_t stream)
{
    const dim3 grid((unsigned int)((int64_t)a.Hkv * a.pre_tiles * a.pre_splits + (int64_t)a.B * a.Hkv * a.own_tiles * a.splits));
    if (es == 2) launch_type<2>(a, path, grid, stream);
    else launch_type<4>(a, path, grid, stream);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.splits + a.pre_splits == 1) return e;
    if (es == 2) {
        if (a.D <= 64) launch_join<2, 16>(a, num_cu, stream);
        else if (a.D <= 128) launch_join<2, 32>(a, num_cu, stream);
        else launch_join<2, 64>(a, num_cu, stream);
    } else {
        if (a.D <= 64) launch_join<4, 16>(a, num_cu, stream);
        else if (a.D <= 128) launch_join<4, 32>(a, num_cu, stream);
        else launch_join<4, 64>(a, num_cu, stream);
    }
    return hipGetLastError();
}
