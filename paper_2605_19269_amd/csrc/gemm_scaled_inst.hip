// gemm_scaled_inst.hip -- instantiations and host launchers of gemm_scaled.hpp.
#include "gemm_scaled.hpp"
#include "scaled_launch.hpp"
#include "small_launch.hpp"

namespace coda {

template <class C, bool BKC, int EPI, bool Q8>
static hipError_t launch_tile(const GemmParams &g, const Q8Params &q, const ScaledParams &p, hipStream_t s)
{
    hipLaunchKernelGGL((gemm_scaled_tile<C, BKC, EPI, Q8>), dim3((unsigned)(p.tiles_m * p.tiles_n)), dim3(C::NT), 0, s, g, q, p);
    return hipGetLastError();
}
template <class C, bool BKC>
static hipError_t launch_program(int mode, bool q8, const GemmParams &g, const Q8Params &q, const ScaledParams &p, hipStream_t s)
{
    if (q8) {
        if (mode == Q8_LINEAR) return launch_tile<C, BKC, Q8_LINEAR, true>(g, q, p, s);
        if (mode == Q8_SWIGLU_FWD) return launch_tile<C, BKC, Q8_SWIGLU_FWD, true>(g, q, p, s);
        return launch_tile<C, BKC, Q8_SWIGLU_BWD, true>(g, q, p, s);
    }
    if (mode == EPI_LINEAR) return launch_tile<C, BKC, EPI_LINEAR, false>(g, q, p, s);
    if (mode == EPI_SWIGLU_FWD) return launch_tile<C, BKC, EPI_SWIGLU_FWD, false>(g, q, p, s);
    if (mode == EPI_SWIGLU_BWD) return launch_tile<C, BKC, EPI_SWIGLU_BWD, false>(g, q, p, s);
    if constexpr (C::BM == 256)                      // column partials are per 256 rows
        if (mode == EPI_RMSNORM_BWD) return launch_tile<C, BKC, EPI_RMSNORM_BWD, false>(g, q, p, s);
    return hipErrorInvalidConfiguration;
}

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

hipError_t launch_gemm_scaled(const ScaledPlan &pl, int mode, bool q8, bool bkc, const GemmParams &g, const Q8Params &q, const ScaledParams &p_in,
                              hipStream_t s)
{
    ScaledParams p = p_in;
    p.tiles_m = (p.M + pl.bm - 1) / pl.bm;
    p.tiles_n = (p.N + pl.bn - 1) / pl.bn;
    p.nsplit = pl.nsplit;
    if (pl.nsplit == 0) {
        using C256 = ScaledCfg<256, 256, 2, 4, 2>;
        using C128 = ScaledCfg<128, 256, 2, 4, 3>;
        if (pl.bm == 256) return bkc ? launch_program<C256, true>(mode, q8, g, q, p, s) : launch_program<C256, false>(mode, q8, g, q, p, s);
        return bkc ? launch_program<C128, true>(mode, q8, g, q, p, s) : launch_program<C128, false>(mode, q8, g, q, p, s);
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
