// grad_scaled.hpp -- the weight gradient from 8-bit checkpoints: G[i][j] += sum over tokens t of a[t][i] b[t][j], in fp32.
//
// a[t][i] = code 2^(sa[i / 128][t] - 127): the blocks of 128 run along the features, the contraction along the tokens, so every element of
// the contraction has a scale of its own and none factors out of a matrix instruction.  Codes are widened to bf16 with their scale, which is
// exact, on the way from memory to LDS, once for a workgroup, and the bf16 instruction contracts.  That keeps the sums exact to fp32 as
// well: those of the 8-bit instructions are off by 0.9e-5 to 1.6e-5 (2-norm, any K), of the bf16 ones by 2e-7 over 1000 tokens, 6e-7 over 8192.  Against codes that are
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

// C: 256 x 256 tiles in eight waves of 128 x 64, or 128 x 128 in four of 64 x 64, two workgroups a CU.  A stage is 32 H tokens: H bf16 tiles of 32 tokens of either operand in the layout of lds_mn, two slots of them.  A
// thread widens granules of sixteen columns, a few of each operand, for the next stage while this one is multiplied.
template <class C, int H, bool B8>
__global__ __launch_bounds__(C::NT) __attribute__((amdgpu_waves_per_eu(2, 2), amdgpu_num_vgpr(256))) void grad_scaled_kernel(const GemmParams g, const GradParams p)
{
    constexpr int GRA = C::BM / 16, GRB = C::BN / 16, QA = 32 * H * GRA / C::NT, QB = 32 * H * GRB / C::NT;       // granules a token, a thread
    constexpr int TA = 32 * C::BM * 2, TB = 32 * C::BN * 2, SLOT = H * (TA + TB), NB = C::WTM / 16, NU = C::WTN / 16;
    static_assert(32 * H * GRA % C::NT == 0 && 32 * H * GRB % C::NT == 0 && C::NT % GRA == 0 && C::NT % GRB == 0, "thread -> granule");
    __shared__ __attribute__((aligned(1024))) unsigned char smem[2 * SLOT];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave % C::WGM, wn = wave / C::WGM;
    const int tiles = p.tiles_m * p.tiles_n, split = (int)blockIdx.x / tiles;
    int tm, tn;
    tile_coords((int)blockIdx.x - split * tiles, tiles, p.tiles_m, p.tiles_n, tm, tn);
    const int m0 = tm * C::BM, n0 = tn * C::BN;
    const int stages = (p.K + 32 * H - 1) / (32 * H);
    const int s0 = (int)((int64_t)split * stages / p.nsplit), s1 = (int)((int64_t)(split + 1) * stages / p.nsplit);

    // the thread's granule columns, and its token in a stage; further granules are NT / GR tokens on
    const int ka = tid / GRA, ca = tid % GRA * 16, kb = tid / GRB, cb = tid % GRB * 16;
    const bool in_a = m0 + ca < p.M, in_b = n0 + cb < p.N;                       // M, N: multiples of 16 (bf16 B: of 8)
    const bool half_b = !B8 && n0 + cb + 8 >= p.N;
    const unsigned char *pa = p.A + m0 + ca, *pb = p.B + (int64_t)(n0 + cb) * (B8 ? 1 : 2);
    const unsigned char *psa = p.sa + (int64_t)((m0 + ca) >> 7) * p.ld_sa;
    const unsigned char *psb = B8 ? p.sb + (int64_t)((n0 + cb) >> 7) * p.ld_sb : nullptr;
    u32x4 ra[QA], rb[QB][B8 ? 1 : 2];
    uint32_t ba[QA], bb[QB];
    auto fetch = [&](int s) {
#pragma unroll
        for (int q = 0; q < QA; ++q) {
            const int64_t t = (int64_t)s * (32 * H) + ka + q * (C::NT / GRA);
            ra[q] = u32x4{0u, 0u, 0u, 0u};
            ba[q] = 127u;
            if (t < p.K && in_a) {
                ra[q] = *reinterpret_cast<const u32x4 *>(pa + t * p.lda);
                ba[q] = psa[t];
            }
        }
#pragma unroll
        for (int q = 0; q < QB; ++q) {
            const int64_t t = (int64_t)s * (32 * H) + kb + q * (C::NT / GRB);
            rb[q][0] = u32x4{0u, 0u, 0u, 0u};
            bb[q] = 127u;
            if constexpr (!B8) rb[q][1] = u32x4{0u, 0u, 0u, 0u};
            if (t < p.K && in_b) {
                rb[q][0] = *reinterpret_cast<const u32x4 *>(pb + t * p.ldb);
                if constexpr (B8) bb[q] = psb[t];
                else if (!half_b) rb[q][1] = *reinterpret_cast<const u32x4 *>(pb + t * p.ldb + 16);
            }
        }
    };
    auto put = [&](int slot) {
        u32x4 w[2];
#pragma unroll
        for (int q = 0; q < QA; ++q) {
            const int k = ka + q * (C::NT / GRA);
            widen16(w, ra[q], q8_scale(ba[q]));
            u32x4 *at = reinterpret_cast<u32x4 *>(smem + slot * SLOT + (k >> 5) * TA + lds_mn<C::BM>(k & 31, ca >> 4));
            at[0] = w[0];
            at[1] = w[1];
        }
#pragma unroll
        for (int q = 0; q < QB; ++q) {
            const int k = kb + q * (C::NT / GRB);
            if constexpr (B8) {
                widen16(w, rb[q][0], q8_scale(bb[q]));
            } else {
                w[0] = rb[q][0];
                w[1] = rb[q][1];
            }
            u32x4 *at = reinterpret_cast<u32x4 *>(smem + slot * SLOT + H * TA + (k >> 5) * TB + lds_mn<C::BN>(k & 31, cb >> 4));
            at[0] = w[0];
            at[1] = w[1];
        }
    };
    Acc16<C> acc;
    acc_zero(acc);
    auto contract = [&](int slot) {
#pragma unroll
        for (int h = 0; h < H; ++h) {
            const unsigned char *ta = smem + slot * SLOT + h * TA, *tb = smem + slot * SLOT + H * TA + h * TB;
            bf16x8 fb[NU];
#pragma unroll
            for (int u = 0; u < NU; ++u) fb[u] = dl_frag16<C::BN, false>(tb, wn * C::WTN + u * 16, lane);
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                const bf16x8 fa = dl_frag16<C::BM, false>(ta, wm * C::WTM + i * 16, lane);
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
        // Of eight waves, two on a SIMD, one widens the next stage before it multiplies this one and the other after it, so that the SIMD's
        // vector and matrix unit work at the same time; raised priority keeps the multiplying one fed (8192 x 2048 x 16384: 529 us
        // without either, 512 with the order alone, 498 with both; 477 with the tokens of a stage indexed as here).
        const bool first = C::NT == 512 && wave >= 4;
        for (int s = s0; s < s1; ++s) {
            const int slot = (s - s0) & 1;
            auto next = [&]() {
                if (s + 1 < s1) put(slot ^ 1);
                if (s + 2 < s1) fetch(s + 2);
            };
            if (first) next();
            __builtin_amdgcn_s_setprio(1);
            contract(slot);
            __builtin_amdgcn_s_setprio(0);
            // the MFMAs stay ahead of the branch
#pragma unroll
            for (int i = 0; i < NB; ++i)
#pragma unroll
                for (int u = 0; u < NU; ++u) asm volatile("" : "+v"(acc.a[i][u]));
            if (!first) next();
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
    if (m0 + C::BM > p.M || n0 + C::BN > p.N) run_epilogue<C, Acc16<C>, EPI_ACCUM, true, 2 * SLOT>(acc, g, m0, n0, tn, smem, nullptr, tid);
    else run_epilogue<C, Acc16<C>, EPI_ACCUM, false, 2 * SLOT>(acc, g, m0, n0, tn, smem, nullptr, tid);
}

}  // namespace coda
