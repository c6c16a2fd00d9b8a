// The tile kernel for microscaled products with activations in E4M3.  (The two formats are compiled by themselves, side by side.)
#include "mx_tile.h"

namespace quest {

// (mx_tile.h has the hipLaunchKernelGGL of this file's kernels)
hipError_t prepare_mx_tiles_e4m3_kernels()
{
    static OncePerDevice once;
    return once([] { return prepare_mx_tiles<QUEST_MX_E4M3>(); });
}

hipError_t launch_mx_tiles_e4m3(const MxGemmArgs &a, int block, hipStream_t stream)
{
    const hipError_t err = prepare_mx_tiles_e4m3_kernels();
    return err != hipSuccess ? err : launch_mx_tiles<QUEST_MX_E4M3>(a, block, stream);
}

}  // namespace quest
