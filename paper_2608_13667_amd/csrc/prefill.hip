// Instruction prefill at the fork: the kernels of prefill_tiles.h over the instruction's tokens.
#include "prefill_tiles.h"

namespace fka {
namespace {

using tiles::kPhases;
using tiles::NW;
using tiles::prefill_tiles;

template <bool PAGED>  // head_dim 128
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(2))) void prefill_tiles_kernel(PrefillArgs a)
{
    prefill_tiles<128, PAGED, kPhases>(a);
}

template <bool PAGED>  // head_dim 64
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(2))) void prefill_tiles_d64_kernel(PrefillArgs a)
{
    prefill_tiles<64, PAGED, kPhases>(a);
}

}  // namespace

int prefill_tiles_unit_rows() { return 32; }
int prefill_tiles_waves() { return NW; }

int prefill_tiles_blocks_per_cu(int head_dim, bool paged)
{
    const void *f = nullptr;
    if (head_dim == 128)
        f = paged ? reinterpret_cast<const void *>(&prefill_tiles_kernel<true>)
                  : reinterpret_cast<const void *>(&prefill_tiles_kernel<false>);
    else if (head_dim == 64)
        f = paged ? reinterpret_cast<const void *>(&prefill_tiles_d64_kernel<true>)
                  : reinterpret_cast<const void *>(&prefill_tiles_d64_kernel<false>);
    int n = 0;
    if (!f || hipOccupancyMaxActiveBlocksPerMultiprocessor(&n, f, 64 * NW, 0) != hipSuccess) return 0;
    return n;
}

hipError_t launch_prefill_tiles(const PrefillArgs &a, int n_blocks, int head_dim, hipStream_t s)
{
    if (n_blocks <= 0) return hipSuccess;
    if (head_dim == 128) {
        if (a.paged)
            prefill_tiles_kernel<true><<<n_blocks, 64 * NW, 0, s>>>(a);
        else
            prefill_tiles_kernel<false><<<n_blocks, 64 * NW, 0, s>>>(a);
    } else if (head_dim == 64) {
        if (a.paged)
            prefill_tiles_d64_kernel<true><<<n_blocks, 64 * NW, 0, s>>>(a);
        else
            prefill_tiles_d64_kernel<false><<<n_blocks, 64 * NW, 0, s>>>(a);
    } else {
        return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

}  // namespace fka
