// The 16-bit products with a code-packed operand for outputs of few tiles: the kernels of grad_gemm_mid.h for operands with a
// scale for each row, and the choice of a block.
// (grad_gemm_mid.h has the hipLaunchKernelGGL of this file's kernels.)
#include "grad_gemm_mid.h"

namespace quest {
namespace {

template <int MODE>
hipError_t launch_mode(const GradMidArgs &a, int shape, hipStream_t stream)
{
    switch (a.grid) {
    case 0:
        if constexpr (MODE != 2)
            return launch_shape<MODE, 0>(a, shape, stream);
        return hipErrorInvalidValue;   // no weight-only product on E2M1 codes
    case 1: return launch_shape<MODE, 1>(a, shape, stream);
    case 2: return launch_shape<MODE, 2>(a, shape, stream);
    case 3: return launch_shape<MODE, 3>(a, shape, stream);
    default: return launch_shape<MODE, 4>(a, shape, stream);
    }
}

template <int MODE>
hipError_t prepare_mode()
{
    hipError_t err = prepare_grid<MODE, 1>();
    if (err == hipSuccess)
        err = prepare_grid<MODE, 2>();
    if (err == hipSuccess)
        err = prepare_grid<MODE, 3>();
    if (err == hipSuccess)
        err = prepare_grid<MODE, 4>();
    if constexpr (MODE != 2) {
        if (err == hipSuccess)
            err = prepare_grid<MODE, 0>();
    }
    return err;
}

}  // namespace

quest_plan grad_gemm_mid_plan(int grid, int64_t C, int64_t R, int64_t K, int cus)
{
    const Shape &s = kShapes[cheapest_shape(grid, C, R, K, cus)];
    return {QUEST_PLAN_MID, 64 * s.wi, 64 * s.wj, s.groups};
}

double grad_gemm_mid_cost(int grid, int64_t C, int64_t R, int64_t K, int cus)
{
    return shape_cost(kShapes[cheapest_shape(grid, C, R, K, cus)], grid, C, R, K, cus);
}

hipError_t prepare_grad_gemm_mid_kernels()
{
    hipError_t err = prepare_mode<0>();
    if (err == hipSuccess)
        err = prepare_mode<1>();
    if (err == hipSuccess)
        err = prepare_mode<2>();
    return err;
}

hipError_t launch_grad_gemm_mid(const GradMidArgs &a, hipStream_t stream)
{
    const int shape = cheapest_shape(a.grid, a.C, a.R, a.K, device_compute_units());
    if (a.grid >= kGridMx)
        return launch_grad_gemm_mid_mx(a, shape, stream);
    return a.mode == 0   ? launch_mode<0>(a, shape, stream)
           : a.mode == 1 ? launch_mode<1>(a, shape, stream)
                         : launch_mode<2>(a, shape, stream);
}

}  // namespace quest
