// scaled_launch.hpp -- plan and host launchers of the products of 8-bit operands with block scales.
#pragma once
#include "gemm_kernel.hpp"

namespace coda {

struct ScaledParams {
    const unsigned char *A, *B, *sa, *sb;
    int64_t lda, ldb, ld_sa, ld_sb;      // bytes
    int M, N, K;
    int tiles_m, tiles_n, nsplit;
    float *part;                         // [nsplit][M][N]
};

// Programs that end in STORE_Q8
enum Q8Mode : int { Q8_LINEAR = 0, Q8_SWIGLU_FWD = 1, Q8_SWIGLU_BWD = 2 };
struct Q8Params {
    uint8_t *out; int64_t ld_out;        // codes [M x W]
    uint8_t *out_s; int64_t ld_out_s;    // scales [blocks of W][M]
    uint8_t *z; int64_t ldz;             // pre-activation: SWIGLU_FWD writes it (null: not wanted), SWIGLU_BWD reads it
    uint8_t *z_s; int64_t ld_z_s;
};

struct GradParams {
    const unsigned char *A, *B;          // [K x M] codes; [K x N] codes or bf16
    const unsigned char *sa, *sb;        // [ceil(M / 128)][K], [ceil(N / 128)][K]
    int64_t lda, ldb, ld_sa, ld_sb;      // bytes
    int M, N, K;                         // K: tokens
    int tiles_m, tiles_n, nsplit;
    float *part;                         // [nsplit][M][N] where nsplit > 1
};

// bm x bn tiles; nsplit = 0: tile and program in one kernel, else every tile is cut along the contraction into nsplit ranges whose fp32
// partials lie in the workspace, and the program runs over those
struct ScaledPlan {
    int bm, bn, nsplit;
};
inline ScaledPlan plan_scaled(int64_t M, int64_t N, int64_t K, bool workspace)
{
    const int64_t blocks = (K + 127) / 128, large = ((M + 255) / 256) * ((N + 255) / 256);
    if (workspace && blocks > 0 && (M <= 64 || large < 64)) {
        const int bm = M <= 32 ? 32 : (M <= 64 ? 64 : 128);
        const int64_t tiles = ((M + bm - 1) / bm) * ((N + 127) / 128);
        int64_t n = tiles >= 192 ? 1 : (256 + tiles / 2) / tiles;
        if (n > 16) n = 16;
        if (n > blocks / 4) n = blocks / 4 > 0 ? blocks / 4 : 1;
        return ScaledPlan{bm, 128, (int)n};
    }
    return ScaledPlan{large >= 192 ? 256 : 128, 256, 0};
}
inline size_t scaled_bytes(const ScaledPlan &pl, int64_t M, int64_t N) { return (size_t)pl.nsplit * (size_t)M * (size_t)N * sizeof(float); }

// mode: an EpiMode of `g`, or with q8 a Q8Mode
hipError_t launch_gemm_scaled(const ScaledPlan &pl, int mode, bool q8, bool bkc, const GemmParams &g, const Q8Params &q, const ScaledParams &p,
                              hipStream_t s);

// a tile and its program in one kernel, per layout of B (true: [N x K])
template <bool BKC>
hipError_t launch_scaled_256(int mode, bool q8, const GemmParams &g, const Q8Params &q, const ScaledParams &p, hipStream_t s);
template <bool BKC>
hipError_t launch_scaled_128(int mode, bool q8, const GemmParams &g, const Q8Params &q, const ScaledParams &p, hipStream_t s);
template <> hipError_t launch_scaled_256<true>(int, bool, const GemmParams &, const Q8Params &, const ScaledParams &, hipStream_t);
template <> hipError_t launch_scaled_256<false>(int, bool, const GemmParams &, const Q8Params &, const ScaledParams &, hipStream_t);
template <> hipError_t launch_scaled_128<true>(int, bool, const GemmParams &, const Q8Params &, const ScaledParams &, hipStream_t);
template <> hipError_t launch_scaled_128<false>(int, bool, const GemmParams &, const Q8Params &, const ScaledParams &, hipStream_t);

// Ranges of the tokens of a gradient, so that its 256 x 256 tiles fill the chip; 1: G is added to by the tiles' own kernel
inline int plan_grad(int64_t M, int64_t N, int64_t K, bool workspace)
{
    const int64_t tiles = ((M + 255) / 256) * ((N + 255) / 256), stages = (K + 63) / 64;
    if (!workspace || tiles >= 128 || tiles <= 0) return 1;
    int64_t n = 256 / tiles;
    if (n > 16) n = 16;
    if (n > stages / 4) n = stages / 4;
    return n > 1 ? (int)n : 1;
}
inline size_t grad_bytes(int nsplit, int64_t M, int64_t N) { return nsplit > 1 ? (size_t)nsplit * (size_t)M * (size_t)N * sizeof(float) : 0; }
hipError_t launch_grad_scaled(int nsplit, bool b8, const GemmParams &g, const GradParams &p, hipStream_t s);

}  // namespace coda
