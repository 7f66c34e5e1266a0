// grad_scaled_inst.hip -- instantiations and host launcher of grad_scaled.hpp.
#include "grad_scaled.hpp"
#include "scaled_launch.hpp"
#include "small_launch.hpp"

namespace coda {

template <class C, int H>
static hipError_t launch_grad_tile(bool b8, const GemmParams &g, GradParams p, hipStream_t s)
{
    p.tiles_m = (p.M + C::BM - 1) / C::BM;
    p.tiles_n = (p.N + C::BN - 1) / C::BN;
    const dim3 grid((unsigned)(p.tiles_m * p.tiles_n * p.nsplit));
    if (b8) hipLaunchKernelGGL((grad_scaled_kernel<C, H, true>), grid, dim3(C::NT), 0, s, g, p);
    else hipLaunchKernelGGL((grad_scaled_kernel<C, H, false>), grid, dim3(C::NT), 0, s, g, p);
    return hipGetLastError();
}

hipError_t launch_grad_scaled(const GradPlan &pl, bool b8, const GemmParams &g, const GradParams &p_in, hipStream_t s)
{
    GradParams p = p_in;
    p.nsplit = pl.nsplit;
    const hipError_t e = pl.tile == 256 ? launch_grad_tile<TileCfg<256, 256, 32, 2, 4>, 2>(b8, g, p, s) : launch_grad_tile<TileCfg<128, 128, 32, 2, 2>, 2>(b8, g, p, s);
    return e != hipSuccess || pl.nsplit == 1 ? e : launch_program_rows(EPI_ACCUM, g, p.part, pl.nsplit, s);
}

}  // namespace coda
