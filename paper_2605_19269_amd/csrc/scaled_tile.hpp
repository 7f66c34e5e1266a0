// scaled_tile.hpp -- launchers of a tile with its program (gemm_scaled.hpp), instantiated per tile and layout of B in gemm_scaled_tile_*.hip.
#pragma once
#include "gemm_scaled.hpp"

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
    return hipErrorInvalidConfiguration;             // RMSNORM_BWD: its column partials are per 256 rows
}

// 256 x 256 tiles
template <bool BKC, int EPI, bool Q8>
static hipError_t launch_large(const GemmParams &g, const Q8Params &q, const ScaledParams &p, hipStream_t s)
{
    const dim3 grid((unsigned)(p.tiles_m * p.tiles_n)), block(ScaledLargeCfg::NT);
    if (p.M % 256 || p.N % 256 || p.K % 128 || p.K == 0) hipLaunchKernelGGL((gemm_scaled_large<BKC, EPI, Q8, true>), grid, block, 0, s, g, q, p);
    else hipLaunchKernelGGL((gemm_scaled_large<BKC, EPI, Q8, false>), grid, block, 0, s, g, q, p);
    return hipGetLastError();
}
template <bool BKC>
static hipError_t launch_large_program(int mode, bool q8, const GemmParams &g, const Q8Params &q, const ScaledParams &p, hipStream_t s)
{
    if (q8) {
        if (mode == Q8_LINEAR) return launch_large<BKC, Q8_LINEAR, true>(g, q, p, s);
        if (mode == Q8_SWIGLU_FWD) return launch_large<BKC, Q8_SWIGLU_FWD, true>(g, q, p, s);
        return launch_large<BKC, Q8_SWIGLU_BWD, true>(g, q, p, s);
    }
    if (mode == EPI_LINEAR) return launch_large<BKC, EPI_LINEAR, false>(g, q, p, s);
    if (mode == EPI_SWIGLU_FWD) return launch_large<BKC, EPI_SWIGLU_FWD, false>(g, q, p, s);
    if (mode == EPI_SWIGLU_BWD) return launch_large<BKC, EPI_SWIGLU_BWD, false>(g, q, p, s);
    return launch_large<BKC, EPI_RMSNORM_BWD, false>(g, q, p, s);
}

}  // namespace coda
