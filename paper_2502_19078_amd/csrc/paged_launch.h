// Kernels of clada_paged_attn and their launch for one type of page; each type is compiled in a file of its own.
#pragma once
#include "attention_join.h"
#include "paged_tiles.h"

namespace {

template <PagedType TY, int DP, bool FULL, bool EIGHT, bool ALONE>
__global__ void __launch_bounds__((64 * PagedRowsShape<TY, DP, FULL>::WAVES), TY == PAGED_4BIT && DP <= 128 ? 4 : TY != PAGED_F32 || DP <= 128 ? 2 : 1)
k_paged_rows(const PagedArgs a)
{
    __shared__ __align__(16) char lds[PagedRowsShape<TY, DP, FULL>::LDS];
    paged_rows<TY, DP, FULL, EIGHT, ALONE>(a, blockIdx.x, lds);
}

template <PagedType TY, int DP, bool FULL, PagedMods MODS>
__global__ void __launch_bounds__(256, DP <= 128 ? 2 : 1)
k_paged_tiles(const PagedArgs a)
{
    __shared__ __align__(16) char lds[PagedTilesShape<TY, DP>::LDS];
    paged_tiles<TY, DP, FULL, MODS>(a, blockIdx.x, lds);
}

template <PagedType TY, int DP, bool FULL>
void launch_paged_full(const PagedArgs &a, AttnPath path, dim3 grid, hipStream_t stream)
{
    if (path == ATTN_TILES) {
        if (a.slopes || (TY == PAGED_F32 && a.cap2 != 0.0f)) hipLaunchKernelGGL((k_paged_tiles<TY, DP, FULL, MODS_ANY>), grid, dim3(256), 0, stream, a);
        else if (a.cap2 != 0.0f) hipLaunchKernelGGL((k_paged_tiles<TY, DP, FULL, TY == PAGED_F32 ? MODS_ANY : MODS_CAP>), grid, dim3(256), 0, stream, a);
        else hipLaunchKernelGGL((k_paged_tiles<TY, DP, FULL, MODS_NONE>), grid, dim3(256), 0, stream, a);
    } else if constexpr (TY != PAGED_F32 || DP % 64 == 0) {  // (the rows of the fp32 kernels come in 64 values)
        const dim3 block(64 * PagedRowsShape<TY, DP, FULL>::WAVES);
        if (TY != PAGED_F32 && a.tile_rows == 8) hipLaunchKernelGGL((k_paged_rows<TY, DP, FULL, TY != PAGED_F32, true>), grid, block, 0, stream, a);
        else if (a.own_tiles == 1) hipLaunchKernelGGL((k_paged_rows<TY, DP, FULL, false, true>), grid, block, 0, stream, a);
        else hipLaunchKernelGGL((k_paged_rows<TY, DP, FULL, false, false>), grid, block, 0, stream, a);
    }
}

template <PagedType TY, int DP>
void launch_paged_as(const PagedArgs &a, AttnPath path, dim3 grid, hipStream_t stream)
{
    if (TY == PAGED_4BIT || a.D == DP) launch_paged_full<TY, DP, true>(a, path, grid, stream);
    else if constexpr (TY != PAGED_4BIT) launch_paged_full<TY, DP, false>(a, path, grid, stream);
}

template <PagedType TY>
hipError_t launch_paged(const PagedArgs &a, AttnPath path, int num_cu, hipStream_t stream)
{
    const dim3 grid((unsigned int)((int64_t)a.B * a.Hkv * a.own_tiles * a.splits));
    if constexpr (TY == PAGED_4BIT) {
        switch (a.D / 32) {
        case 1: launch_paged_as<TY, 32>(a, path, grid, stream); break;
        case 2: launch_paged_as<TY, 64>(a, path, grid, stream); break;
        case 3: launch_paged_as<TY, 96>(a, path, grid, stream); break;
        case 4: launch_paged_as<TY, 128>(a, path, grid, stream); break;
        case 5: launch_paged_as<TY, 160>(a, path, grid, stream); break;
        case 6: launch_paged_as<TY, 192>(a, path, grid, stream); break;
        case 7: launch_paged_as<TY, 224>(a, path, grid, stream); break;
        default: launch_paged_as<TY, 256>(a, path, grid, stream);
        }
    } else {
        if (a.D <= 64) launch_paged_as<TY, 64>(a, path, grid, stream);
        else if (a.D <= 96 && (TY == PAGED_BF16 || path == ATTN_TILES)) launch_paged_as<TY, 96>(a, path, grid, stream);
        else if (a.D <= 128) launch_paged_as<TY, 128>(a, path, grid, stream);
        else launch_paged_as<TY, 256>(a, path, grid, stream);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1 || path == ATTN_ROWS) return e;      // (rows are joined by the last split's workgroup)
    launch_join(a, paged_es(TY), num_cu, stream);
    return hipGetLastError();
}

}  // namespace
