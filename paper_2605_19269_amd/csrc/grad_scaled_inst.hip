// grad_scaled_inst.hip -- instantiations and host launcher of grad_scaled.hpp.
#include "grad_scaled.hpp"
#include "scaled_launch.hpp"
#include "small_launch.hpp"

namespace coda {

hipError_t launch_grad_scaled(int nsplit, bool b8, const GemmParams &g, const GradParams &p_in, hipStream_t s)
{
    using C = TileCfg<256, 256, 32, 2, 4>;
    GradParams p = p_in;
    p.tiles_m = (p.M + 255) / 256;
    p.tiles_n = (p.N + 255) / 256;
    p.nsplit = nsplit;
    const dim3 grid((unsigned)(p.tiles_m * p.tiles_n * nsplit));
    if (b8) hipLaunchKernelGGL((grad_scaled_kernel<C, true>), grid, dim3(C::NT), 0, s, g, p);
    else hipLaunchKernelGGL((grad_scaled_kernel<C, false>), grid, dim3(C::NT), 0, s, g, p);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess || nsplit == 1 ? e : launch_program_rows(EPI_ACCUM, g, p.part, nsplit, s);
}

}  // namespace coda
