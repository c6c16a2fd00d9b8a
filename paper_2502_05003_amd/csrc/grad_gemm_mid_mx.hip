// The gradient products for outputs of few tiles with microscaled operands: the kernels of grad_gemm_mid.h.  (A file of their own,
// compiled beside the others.)
// (grad_gemm_mid.h has the hipLaunchKernelGGL of this file's kernels.)
#include "grad_gemm_mid.h"

namespace quest {
namespace {

constexpr int kE2M1 = kGridMx + QUEST_MX_E2M1, kE4M3 = kGridMx + QUEST_MX_E4M3;

template <int MODE>
hipError_t launch_mode(const GradMidArgs &a, int shape, hipStream_t stream)
{
    return a.grid == kE4M3 ? launch_shape<MODE, kE4M3>(a, shape, stream) : launch_shape<MODE, kE2M1>(a, shape, stream);
}

}  // namespace

hipError_t prepare_grad_gemm_mid_mx_kernels()
{
    hipError_t err = prepare_grid<0, kE2M1>();
    if (err == hipSuccess)
        err = prepare_grid<0, kE4M3>();
    if (err == hipSuccess)
        err = prepare_grid<1, kE2M1>();
    if (err == hipSuccess)
        err = prepare_grid<1, kE4M3>();
    return err;
}

hipError_t launch_grad_gemm_mid_mx(const GradMidArgs &a, int shape, hipStream_t stream)
{
    return a.mode == 0   ? launch_mode<0>(a, shape, stream)
           : a.mode == 1 ? launch_mode<1>(a, shape, stream)
                         : hipErrorInvalidValue;
}

}  // namespace quest
