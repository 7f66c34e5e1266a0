// Host build of the plans of the 8-bit products with block scales and of their gradients, for tests/test_scaled_plan_host.py.  Compiled for the host only;
// nothing here touches a GPU.
#include "../paper_2605_19269_amd/csrc/scaled_launch.hpp"

extern "C" {

// plan[0..3] = coda::ScaledPlan: tile rows and columns, ranges (0: tile and program in one kernel), few rows in one kernel
__attribute__((visibility("default"))) void host_plan_scaled(int64_t M, int64_t N, int64_t K, int workspace, int narrow, int *plan)
{
    const coda::ScaledPlan pl = coda::plan_scaled(M, N, K, workspace != 0, narrow != 0);
    plan[0] = pl.bm; plan[1] = pl.bn; plan[2] = pl.nsplit; plan[3] = pl.few;
}

// plan[0..1] = coda::GradPlan: tile, ranges of the tokens
__attribute__((visibility("default"))) void host_plan_grad(int64_t M, int64_t N, int64_t K, int workspace, int *plan)
{
    const coda::GradPlan pl = coda::plan_grad(M, N, K, workspace != 0);
    plan[0] = pl.tile; plan[1] = pl.nsplit;
}

}
