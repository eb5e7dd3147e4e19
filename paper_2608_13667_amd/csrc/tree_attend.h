// Attention of drafted trees: the kernels of prefill_tiles.h with a mask of nodes to each row.
#pragma once

#include "prefill_tiles.h"

namespace fka {
namespace {

using tiles::kHalves;
using tiles::kPhases;
using tiles::kStream;

template <bool PAGED, int KIND>  // head_dim 128
__global__ __launch_bounds__(64 * tiles::NW) __attribute__((amdgpu_waves_per_eu(2))) void tree_tiles_kernel(TreeArgs a)
{
    tiles::prefill_tiles<128, PAGED, KIND>(a);
}

template <bool PAGED, int KIND>  // head_dim 64
__global__ __launch_bounds__(64 * tiles::NW) __attribute__((amdgpu_waves_per_eu(2))) void tree_tiles_d64_kernel(TreeArgs a)
{
    tiles::prefill_tiles<64, PAGED, KIND>(a);
}

template <int KIND>
hipError_t launch_tree_kind(const TreeArgs &a, int n_blocks, int head_dim, hipStream_t s)
{
    if (head_dim == 128) {
        if (a.paged)
            tree_tiles_kernel<true, KIND><<<n_blocks, 64 * tiles::NW, 0, s>>>(a);
        else
            tree_tiles_kernel<false, KIND><<<n_blocks, 64 * tiles::NW, 0, s>>>(a);
    } else if (head_dim == 64) {
        if (a.paged)
            tree_tiles_d64_kernel<true, KIND><<<n_blocks, 64 * tiles::NW, 0, s>>>(a);
        else
            tree_tiles_d64_kernel<false, KIND><<<n_blocks, 64 * tiles::NW, 0, s>>>(a);
    } else {
        return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

}  // namespace

inline hipError_t launch_tree_kernels(const TreeArgs &a, TreeKind kind, int n_blocks, int head_dim, hipStream_t s)
{
    if (n_blocks <= 0) return hipSuccess;
    return kind == TreeKind::kHalves   ? launch_tree_kind<kHalves>(a, n_blocks, head_dim, s)
           : kind == TreeKind::kStream ? launch_tree_kind<kStream>(a, n_blocks, head_dim, s)
                                       : launch_tree_kind<kPhases>(a, n_blocks, head_dim, s);
}

}  // namespace fka
