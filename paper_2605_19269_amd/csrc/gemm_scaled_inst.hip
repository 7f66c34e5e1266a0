// gemm_scaled_inst.hip -- host launcher of gemm_scaled.hpp and its divided contractions; tiles with their programs: gemm_scaled_tile_*.hip.
#include "gemm_scaled.hpp"
#include "scaled_launch.hpp"
#include "small_launch.hpp"

namespace coda {

template <class C>
static hipError_t launch_partial(bool bkc, const ScaledParams &p, hipStream_t s)
{
    const dim3 grid((unsigned)(p.tiles_m * p.tiles_n * p.nsplit));
    if (bkc) hipLaunchKernelGGL((gemm_scaled_partial<C, true>), grid, dim3(C::NT), 0, s, p);
    else hipLaunchKernelGGL((gemm_scaled_partial<C, false>), grid, dim3(C::NT), 0, s, p);
    return hipGetLastError();
}

template <int MODE>
static hipError_t launch_rows_q8(const GemmParams &g, const Q8Params &q, const ScaledParams &p, hipStream_t s)
{
    hipLaunchKernelGGL((epi_rows_q8_kernel<MODE>), dim3((unsigned)((p.N + 255) / 256), (unsigned)((p.M + EPI_ROWS - 1) / EPI_ROWS)), dim3(256), 0, s, g, q,
                       p.part, p.nsplit);
    return hipGetLastError();
}

template <int RB, int CB>
static hipError_t launch_few(int mode, const GemmParams &g, const ScaledParams &p, hipStream_t s)
{
    const dim3 grid((unsigned)((p.N + CB * 16 - 1) / (CB * 16)));
    if (mode == EPI_LINEAR) hipLaunchKernelGGL((gemm_scaled_few<RB, CB, EPI_LINEAR>), grid, dim3(512), 0, s, g, p);
    else hipLaunchKernelGGL((gemm_scaled_few<RB, CB, EPI_SWIGLU_FWD>), grid, dim3(512), 0, s, g, p);
    return hipGetLastError();
}

hipError_t launch_gemm_scaled(const ScaledPlan &pl, int mode, bool q8, bool bkc, const GemmParams &g, const Q8Params &q, const ScaledParams &p_in,
                              hipStream_t s)
{
    ScaledParams p = p_in;
    if (pl.few) {
        // 32 columns a workgroup where that leaves one for more than half of the CUs (us, 16 and 32 columns: one row of K = 4096, N = 4096 5.9 and 7.1, 4112 7.1 and 7.1,
        // 4608 7.6 and 7.2, 6144 8.2 and 7.4, 8192 9.4 and 8.7; 16 rows, 4096 6.7 and 8.3, 4608 10.3 and 8.4; 32 rows of K = 2048, 4096 5.4 and 6.3, 4608 9.1 and 6.5)
        const int cb = p.N > 4096 ? 2 : 1;
        if (p.M <= 16) return cb == 2 ? launch_few<1, 2>(mode, g, p, s) : launch_few<1, 1>(mode, g, p, s);
        return cb == 2 ? launch_few<2, 2>(mode, g, p, s) : launch_few<2, 1>(mode, g, p, s);
    }
    p.tiles_m = (p.M + pl.bm - 1) / pl.bm;
    p.tiles_n = (p.N + pl.bn - 1) / pl.bn;
    p.nsplit = pl.nsplit;
    if (pl.nsplit == 0) {
        if (pl.bm == 256) return bkc ? launch_scaled_256<true>(mode, q8, g, q, p, s) : launch_scaled_256<false>(mode, q8, g, q, p, s);
        return bkc ? launch_scaled_128<true>(mode, q8, g, q, p, s) : launch_scaled_128<false>(mode, q8, g, q, p, s);
    }
    const hipError_t e = pl.bm == 32   ? launch_partial<ScaledCfg<32, 128, 1, 4, 3>>(bkc, p, s)
                         : pl.bm == 64 ? launch_partial<ScaledCfg<64, 128, 1, 4, 3>>(bkc, p, s)
                                       : launch_partial<ScaledCfg<128, 128, 2, 4, 4>>(bkc, p, s);
    if (e != hipSuccess) return e;
    if (q8) {
        if (mode == Q8_LINEAR) return launch_rows_q8<Q8_LINEAR>(g, q, p, s);
        if (mode == Q8_SWIGLU_FWD) return launch_rows_q8<Q8_SWIGLU_FWD>(g, q, p, s);
        return launch_rows_q8<Q8_SWIGLU_BWD>(g, q, p, s);
    }
    return launch_program_rows(mode, g, p.part, p.nsplit, s);
}

}  // namespace coda
