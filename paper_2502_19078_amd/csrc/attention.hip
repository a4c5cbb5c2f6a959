// Kernels of clada_window_attn and clada_shared_prefix_attn: few rows (single tokens) run attention_rows.h, many attention_tiles.h; where
// a row's keys are split among workgroups, k_attn_join adds their results up in a second launch.
#include <math.h>

#include "attention_join.h"
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
    launch_join(a, es, num_cu, stream);
    return hipGetLastError();
}
