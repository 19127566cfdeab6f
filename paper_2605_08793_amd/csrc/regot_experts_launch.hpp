// Products grouped by expert: which kernel a call runs.  One source for each type of numbers includes this.
#pragma once

#include "regot_experts_few.hpp"
#include "regot_experts_tile.hpp"

namespace regot {

enum { kTileStaged, kTileDirect, kTileStagedSmall, kTileDirectSmall, kTileBig, kTileFew };

struct TilePlan {
    int kind, across, tile, out_type, gather;
    int64_t units;  // few rows: what a wave has of a sum
};

struct TileShape {
    int64_t rows, cols;
};
inline TileShape tile_shape(int tile)
{
    if (tile == kTileBig) return {256, 256};
    if (tile == kTileStagedSmall || tile == kTileDirectSmall) return {64, 128};
    if (tile == kTileFew) return {16, 32};
    return {128, 128};
}

template <int TYPE, bool ACROSS, int KIND, int OUT, bool GATHER>
void launch_tile(const GroupArgs &A, int tile, hipStream_t s)
{
    const dim3 grid(A.tiles), threads(256);
    if (tile == kTileBig) {
        if constexpr (TYPE != REGOT_F32) hipLaunchKernelGGL((expert_tile_kernel<TYPE, 256, 256, 2, 2, ACROSS, KIND, true, OUT, GATHER>), grid, threads, 0, s, A);
    } else if (tile == kTileDirect) {
        hipLaunchKernelGGL((expert_tile_kernel<TYPE, 128, 128, 2, 2, ACROSS, KIND, true, OUT, GATHER>), grid, threads, 0, s, A);
    } else if (tile == kTileDirectSmall) {
        hipLaunchKernelGGL((expert_tile_kernel<TYPE, 64, 128, 2, 2, ACROSS, KIND, true, OUT, GATHER>), grid, threads, 0, s, A);
    } else if (tile == kTileStaged) {
        hipLaunchKernelGGL((expert_tile_kernel<TYPE, 128, 128, 2, 2, ACROSS, KIND, false, OUT, GATHER>), grid, threads, 0, s, A);
    } else {
        hipLaunchKernelGGL((expert_tile_kernel<TYPE, 64, 128, 2, 2, ACROSS, KIND, false, OUT, GATHER>), grid, threads, 0, s, A);
    }
}

template <int TYPE>
void launch_tiles(const GroupArgs &A, const TilePlan &P, hipStream_t s)
{
    if (P.tile == kTileFew) {
        const dim3 grid(A.tiles), threads(kFewWaves * kLanes);
        if (P.units <= 4) {
            if (P.kind == kGate) hipLaunchKernelGGL((expert_few_kernel<TYPE, true, 4>), grid, threads, 0, s, A);
            else hipLaunchKernelGGL((expert_few_kernel<TYPE, false, 4>), grid, threads, 0, s, A);
        } else {
            if (P.kind == kGate) hipLaunchKernelGGL((expert_few_kernel<TYPE, true, kFewUnits>), grid, threads, 0, s, A);
            else hipLaunchKernelGGL((expert_few_kernel<TYPE, false, kFewUnits>), grid, threads, 0, s, A);
        }
    } else if (P.kind == kWeightGrad) {
        if (P.out_type == REGOT_F32) P.gather ? launch_tile<TYPE, true, kWeightGrad, REGOT_F32, true>(A, P.tile, s) : launch_tile<TYPE, true, kWeightGrad, REGOT_F32, false>(A, P.tile, s);
        else P.gather ? launch_tile<TYPE, true, kWeightGrad, TYPE, true>(A, P.tile, s) : launch_tile<TYPE, true, kWeightGrad, TYPE, false>(A, P.tile, s);
    } else if (P.across) {
        if (P.kind == kPlain) launch_tile<TYPE, true, kPlain, TYPE, false>(A, P.tile, s);
        else if (P.kind == kGate) launch_tile<TYPE, true, kGate, TYPE, false>(A, P.tile, s);
        else launch_tile<TYPE, true, kGateGrad, TYPE, false>(A, P.tile, s);
    } else {
        if (P.kind == kPlain) launch_tile<TYPE, false, kPlain, TYPE, false>(A, P.tile, s);
        else if (P.kind == kGate) launch_tile<TYPE, false, kGate, TYPE, false>(A, P.tile, s);
        else launch_tile<TYPE, false, kGateGrad, TYPE, false>(A, P.tile, s);
    }
}

}  // namespace regot
