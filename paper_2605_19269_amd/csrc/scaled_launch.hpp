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

// few: up to 32 rows in one kernel.  Else bm x bn tiles; nsplit = 0: tile and program in one kernel, else every tile is cut along the contraction into
// nsplit ranges whose fp32 partials lie in the workspace, and the program runs over those.
struct ScaledPlan {
    int bm, bn, nsplit;
    bool few;
};
// `narrow`: a program without row reductions and 8-bit outputs, on a B stored [N x K]
inline ScaledPlan plan_scaled(int64_t M, int64_t N, int64_t K, bool workspace, bool narrow)
{
    // Against partials and a second kernel (us): 6144 x 4096, 1 / 8 / 16 / 32 rows 7.6 / 8.1 / 8.7 / 10.6 and 9.2 / 9.5 / 9.9 / 10.9; 4096 x 14336, 1 / 8 / 24 rows
    // 12.5 / 13.4 / 19.7 and 13.4 / 13.8 / 14.2; 16384 x 2048, one row 9.6 and 10.1; 4096 x 4096, 24 rows 8.0 and 9.5; 28672 x 4096, one row 27.4 and 21.0 (many
    // workgroups one after the other, each with its own start; every one fetches the rows of A anew).  Without a workspace against 128-row tiles: 4096 x 14336,
    // 32 rows 22.6 and 72.8.
    const bool small = (M <= 8 && N <= 8192) || (M <= 16 && N * K <= (int64_t)1 << 25) || N * K <= (int64_t)1 << 24;
    if (narrow && M <= 32 && (!workspace || small)) return ScaledPlan{0, 0, 0, true};
    // What the choices take, in microseconds, as fitted.  A round of 256 tiles of 128 x 256 takes 6 and 0.8 for a block of the contraction, one of 256 x 256, which
    // reads less for what it computes, 8 and 1.43; with few of the CUs at work a block takes 0.63 and 1.05.  Tiles of 128 and 256 rows: 1000 x 4096 x 14336 78 and 126,
    // 1039 x 14336 x 4096 66 and 95 (two rounds and 1.1), 2048 x 4096 x 4096 34.5 and 45.4, 4608 x 4608 x 4096 92 and 95; 2500 x 4608 x 2048 35.7 and 30.8,
    // 2048 x 8192 x 4096 66 and 56, 8192 x 16384 x 2048 300 and 254.
    const int64_t blocks = (K + 127) / 128, half = ((M + 127) / 128) * ((N + 255) / 256), large = ((M + 255) / 256) * ((N + 255) / 256);
    auto rounds = [blocks](int64_t count, double start, double few, double all) {
        const double rest = (double)(count % 256) / 256;
        return (double)(count / 256) * (start + all * (double)blocks) + (rest > 0 ? start + (few + (all - few) * rest) * (double)blocks : 0);
    };
    const double t128 = rounds(half, 6, 0.63, 0.8), t256 = rounds(large, 8, 1.05, 1.43);
    const ScaledPlan direct{t128 <= t256 ? 128 : 256, 256, 0, false};
    if (!workspace || blocks == 0) return direct;
    // Partials: a block takes 0.33, 0.36 and 0.5 in tiles of 32, 64 and 128 x 128; partials are written and read at 6.5 TB/s; 9 for two launches.  No more than a
    // workgroup a CU: 215 x 4224 x 10416, 66 tiles in 3 ranges 26.4, in 4 38.3; 33 x 11264 x 2048, 88 tiles in 2 ranges 10.9, in 3 12.9.  Against the
    // direct tiles: 1000 x 2048 x 5632 24.8 and 33.9, 300 x 2048 x 2048 14.3 and 16.1, 96 x 2048 x 1024 8.7 and 11.4; 614 x 5600 x 1584 23.0 and 18.7.  Level:
    // 300 x 2048 x 256 7.1 and 7.4 (direct: a launch less for the host), 1000 x 4096 x 14336 in one range, 256 tiles for 128, 77.1 and 77.8 (partials).
    const int bm = M <= 32 ? 32 : (M <= 64 ? 64 : 128);
    const int64_t tiles = ((M + bm - 1) / bm) * ((N + 127) / 128);
    const double stage = bm == 32 ? 0.33 : (bm == 64 ? 0.36 : 0.5), join = (double)M * (double)N * 8 / 6.5e6;
    double best = t128 < t256 ? t128 : t256;
    int n = 0;
    for (int i = 1; i <= 16 && i <= blocks && (tiles * i <= 256 || (i == 1 && bm < 128)); ++i) {
        const double t = 9 + stage * (double)((blocks + i - 1) / i) * (double)((tiles * i + 255) / 256) + join * i;
        if (t < best) {
            best = t;
            n = i;
        }
    }
    return n ? ScaledPlan{bm, 128, n, false} : direct;
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

// tile x tile of a gradient, and ranges of its tokens (1: G is added to by the tiles' own kernel).
// 256: one workgroup a CU, bound by the matrix cores and LDS.  128: two a CU, four waves of 64 x 64, which read a third more from LDS for what they
// compute but fill the chip with a quarter of the output, end a tile while the other computes, and need fewer partials where the tokens
// are divided.  So 128 up to the 512 tiles of one round of them, and where there is little to contract (us, 256 / 128): 512 tiles, 1000 x (2048 x 4096) 39.6 / 30.6,
// 4096 x (2048 x 4096) 114 / 86, 320 x (1024 x 8192) 22.9 / 18.6; 544 and more, 1000 x (256 x 34816) 40.1 / 45.0, 4096 x (2304 x 4096) 114 / 137, 320 x (2304 x 4096)
// 23.8 / 24.3, 1000 x (5632 x 2048) 43.6 / 48.8, 4096 x (4096 x 4096) 127 / 157, 8192 x (2048 x 16384) 470 / 608; few tokens, 256 x (4096 x 14336) 126 / 115,
// 64 x (4096 x 14336) 107 / 102, 64 x (2048 x 8192) 25.2 / 26.3.  With few tiles, in ranges: 8192 x (512 x 1024) 208 / 116, in 16 ranges 26.9;
// 300 x (4800 x 752) 21.4 / 12.1, 2048 x (2048 x 2048) 62 / 38.5.
struct GradPlan {
    int tile, nsplit;
};
inline GradPlan plan_grad(int64_t M, int64_t N, int64_t K, bool workspace)
{
    const int64_t small = ((M + 127) / 128) * ((N + 127) / 128), stages = (K + 63) / 64;
    if (small > 512 && K > 256) return GradPlan{256, 1};
    int64_t n = workspace && small > 0 && small < 256 ? 512 / small : 1;
    if (n > 16) n = 16;
    if (n > stages / 4) n = stages / 4;
    return GradPlan{128, n > 1 ? (int)n : 1};
}
inline size_t grad_bytes(const GradPlan &pl, int64_t M, int64_t N) { return pl.nsplit > 1 ? (size_t)pl.nsplit * (size_t)M * (size_t)N * sizeof(float) : 0; }
hipError_t launch_grad_scaled(const GradPlan &pl, bool b8, const GemmParams &g, const GradParams &p, hipStream_t s);

}  // namespace coda
