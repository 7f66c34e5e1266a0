// grad_scaled.hpp -- the weight gradient from 8-bit checkpoints: G[i][j] += sum over tokens t of a[t][i] b[t][j], in fp32.
//
// a[t][i] = code 2^(sa[i / 128][t] - 127): the blocks of 128 run along the features, the contraction along the tokens, so every element of
// the contraction has a scale of its own and none factors out of a matrix instruction.  Codes are widened to bf16 with their scale, which is
// exact, on the way from memory to LDS, once for a workgroup, and the bf16 instruction contracts.  That keeps the sums exact to fp32 as
// well: those of the 8-bit instructions are off by 1.3e-5 (2-norm, any K), of the bf16 ones by 2e-7.  Against codes that are
// widened to memory first, a gradient reads 1 byte an element instead of 1 + 2 (written) + 2.
//
// Bound by the bf16 matrix cores and what LDS feeds them, like the other bf16 products.
#pragma once
#include "gemm_kernel.hpp"
#include "q8.hpp"
#include "scaled_launch.hpp"

namespace coda {

// Sixteen codes with their scale as bf16
__device__ __forceinline__ void widen16(u32x4 (&o)[2], u32x4 w, float s)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        o[e >> 1][(e & 1) * 2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[e], s, false));
        o[e >> 1][(e & 1) * 2 + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[e], s, true));
    }
}

// C: 256 x 256 tiles, eight waves of 128 x 64.  A stage is 64 tokens: four [32][256] bf16 tiles (A and B, two halves) of 16 KB in the layout
// of lds_mn, two slots of them.  A thread widens two granules of sixteen columns of each operand per stage.
template <class C, bool B8>
__global__ __launch_bounds__(C::NT) __attribute__((amdgpu_waves_per_eu(2, 2), amdgpu_num_vgpr(256))) void grad_scaled_kernel(const GemmParams g, const GradParams p)
{
    constexpr int TILE = 32 * 256 * 2, SLOT = 4 * TILE, NB = C::WTM / 16, NU = C::WTN / 16;
    static_assert(C::BM == 256 && C::BN == 256 && C::NT == 512, "thread -> granule");
    __shared__ __attribute__((aligned(1024))) unsigned char smem[2 * SLOT];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave % C::WGM, wn = wave / C::WGM;
    const int tiles = p.tiles_m * p.tiles_n, split = (int)blockIdx.x / tiles;
    int tm, tn;
    tile_coords((int)blockIdx.x - split * tiles, tiles, p.tiles_m, p.tiles_n, tm, tn);
    const int m0 = tm * 256, n0 = tn * 256;
    const int stages = (p.K + 63) / 64;
    const int s0 = (int)((int64_t)split * stages / p.nsplit), s1 = (int)((int64_t)(split + 1) * stages / p.nsplit);

    const int k = tid >> 4, gr = tid & 15;           // the thread's token (and k + 32) and granule
    const bool in_a = m0 + gr * 16 < p.M, in_b = n0 + gr * 16 < p.N;             // M, N: multiples of 16 (bf16 B: of 8)
    const bool half_b = !B8 && n0 + gr * 16 + 8 >= p.N;
    const unsigned char *pa = p.A + m0 + gr * 16, *pb = p.B + (int64_t)(n0 + gr * 16) * (B8 ? 1 : 2);
    const unsigned char *psa = p.sa + (int64_t)((m0 + gr * 16) >> 7) * p.ld_sa;
    const unsigned char *psb = B8 ? p.sb + (int64_t)((n0 + gr * 16) >> 7) * p.ld_sb : nullptr;
    u32x4 ra[2], rb[2][B8 ? 1 : 2];
    uint32_t ba[2], bb[2];
    auto fetch = [&](int s) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t t = (int64_t)s * 64 + h * 32 + k;
            const bool in = t < p.K;
            ra[h] = rb[h][0] = u32x4{0u, 0u, 0u, 0u};
            ba[h] = bb[h] = 127u;
            if constexpr (!B8) rb[h][1] = u32x4{0u, 0u, 0u, 0u};
            if (in && in_a) {
                ra[h] = *reinterpret_cast<const u32x4 *>(pa + t * p.lda);
                ba[h] = psa[t];
            }
            if (in && in_b) {
                rb[h][0] = *reinterpret_cast<const u32x4 *>(pb + t * p.ldb);
                if constexpr (B8) bb[h] = psb[t];
                else if (!half_b) rb[h][1] = *reinterpret_cast<const u32x4 *>(pb + t * p.ldb + 16);
            }
        }
    };
    const uint32_t spot = lds_mn<256>(k, gr);
    auto put = [&](int slot) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            u32x4 w[2];
            widen16(w, ra[h], q8_scale(ba[h]));
            u32x4 *at = reinterpret_cast<u32x4 *>(smem + slot * SLOT + h * TILE + spot);
            at[0] = w[0];
            at[1] = w[1];
            if constexpr (B8) {
                widen16(w, rb[h][0], q8_scale(bb[h]));
            } else {
                w[0] = rb[h][0];
                w[1] = rb[h][1];
            }
            u32x4 *bt = reinterpret_cast<u32x4 *>(smem + slot * SLOT + (2 + h) * TILE + spot);
            bt[0] = w[0];
            bt[1] = w[1];
        }
    };
    Acc16<C> acc;
    acc_zero(acc);
    auto contract = [&](int slot) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const unsigned char *ta = smem + slot * SLOT + h * TILE, *tb = ta + 2 * TILE;
            bf16x8 fb[NU];
#pragma unroll
            for (int u = 0; u < NU; ++u) fb[u] = dl_frag16<256, false>(tb, wn * C::WTN + u * 16, lane);
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                const bf16x8 fa = dl_frag16<256, false>(ta, wm * C::WTM + i * 16, lane);
#pragma unroll
                for (int u = 0; u < NU; ++u) acc.a[i][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[u], fa, acc.a[i][u], 0, 0, 0);
            }
        }
    };
    if (s0 < s1) {
        fetch(s0);
        put(0);
        if (s0 + 1 < s1) fetch(s0 + 1);
        __syncthreads();
        for (int s = s0; s < s1; ++s) {
            const int slot = (s - s0) & 1;
            contract(slot);
            if (s + 1 < s1) put(slot ^ 1);
            if (s + 2 < s1) fetch(s + 2);
            __syncthreads();
        }
    }
    if (p.nsplit > 1) {
        const int m = m0 + wm * C::WTM + (lane & 15), n = n0 + wn * C::WTN + (lane >> 4) * 4;
        float *out = p.part + (int64_t)split * p.M * p.N;
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int u = 0; u < NU; ++u)
                if (m + i * 16 < p.M && n + u * 16 < p.N) *reinterpret_cast<f32x4 *>(out + (int64_t)(m + i * 16) * p.N + n + u * 16) = acc.get(i, u);
        return;
    }
    if (m0 + 256 > p.M || n0 + 256 > p.N) run_epilogue<C, Acc16<C>, EPI_ACCUM, true, 2 * SLOT>(acc, g, m0, n0, tn, smem, nullptr, tid);
    else run_epilogue<C, Acc16<C>, EPI_ACCUM, false, 2 * SLOT>(acc, g, m0, n0, tn, smem, nullptr, tid);
}

}  // namespace coda
