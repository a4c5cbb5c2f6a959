// The second launch of an attention call whose rows' keys are split among workgroups: it joins their partial results.
#pragma once
#include "attention.h"

namespace {

// A joined row: four outputs of a thread, and the log of the sum by the thread that holds dim 0.
template <int ES, class Args>
__device__ __forceinline__ void join_store(const Args &a, const int64_t row, const int dim, f32x4 o, const float l, const float top)
{
    const int hq = (int)(row % a.Hq);
    const int64_t bt = row / a.Hq;
    const int b = a.T == 1 ? (int)bt : (int)(bt / a.T), t = (int)(bt - (int64_t)b * a.T);
    const bool none = joined_none(a, b, t, l);
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
template <int ES, int TPR, class Args>
__global__ void __launch_bounds__(256)
k_attn_join(const Args a)
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
template <int ES, int TPR, class Args>
__global__ void __launch_bounds__(256)
k_attn_join_few(const Args a)
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

template <int ES, int TPR, class Args>
void launch_join_as(const Args &a, int num_cu, hipStream_t stream)
{
    const int64_t rows = (int64_t)a.B * a.T * a.Hq;
    constexpr int RW = 256 / TPR;
    // Whole calls, us, a workgroup a row against this: 8 rows 14.3 / 14.9, 256 rows even, 1280 rows of 64 values 16.6 / 15.4, 4096 rows 22.0 / 17.6,
    // 8192 rows of 128 values 43.0 / 36.2, 4096 rows of 256 values 55.7 / 53.1.
    if (rows > 4 * num_cu && a.splits + a.pre_splits <= FEW_SPLITS)
        hipLaunchKernelGGL((k_attn_join_few<ES, TPR, Args>), dim3((unsigned int)((rows + RW - 1) / RW)), dim3(256), 0, stream, a);
    else
        hipLaunchKernelGGL((k_attn_join<ES, TPR, Args>), dim3((unsigned int)rows), dim3(256), 0, stream, a);
}

template <class Args>
void launch_join(const Args &a, int es, int num_cu, hipStream_t stream)
{
    if (es == 2) {
        if (a.D <= 64) launch_join_as<2, 16>(a, num_cu, stream);
        else if (a.D <= 128) launch_join_as<2, 32>(a, num_cu, stream);
        else launch_join_as<2, 64>(a, num_cu, stream);
    } else {
        if (a.D <= 64) launch_join_as<4, 16>(a, num_cu, stream);
        else if (a.D <= 128) launch_join_as<4, 32>(a, num_cu, stream);
        else launch_join_as<4, 64>(a, num_cu, stream);
    }
}

}  // namespace
