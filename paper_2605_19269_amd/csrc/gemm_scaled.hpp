// gemm_scaled.hpp -- the product of 8-bit operands with a scale for each block of 128 of the contraction.
//
//   D[i][j] = sum over blocks b of 2^(sa[b][i] - 127) 2^(sb[b][j] - 127) sum over k in b of A[i][k] B[k][j]
//
// A stage of the contraction is one block: 128 bytes of every row.  Its scales travel with it -- BM + BN bytes behind the operand tiles
// of the stage's LDS slot, fetched by the first and the last wave -- and go into the matrix instruction with the fragments, a
// byte for the lane's row of A and one for its column of B.  So the sums stay in one set of fp32 accumulators and a block costs
// a few byte reads.  Scales lie [block][row]: the rows of a tile are BM consecutive bytes.
//
// The ring, its loads and waits are those of the small tiles (gemm_small.hpp).  The fragments of A are read in place: the row of
// blocks i of the next half stage follows the MFMAs of row i of this one, which leaves 256 x 256 tiles the registers that they need
// (two waves a SIMD, 256 registers: 128 accumulators, 32 + 32 fragments).
#pragma once
#include "gemm_small.hpp"
#include "epi_rows.hpp"
#include "q8.hpp"
#include "scaled_launch.hpp"

namespace coda {

template <int BM_, int BN_, int WGM_, int WGN_, int S_>
struct ScaledCfg : SmallCfg<BM_, BN_, WGM_, WGN_, S_, true> {
    using Base = SmallCfg<BM_, BN_, WGM_, WGN_, S_, true>;
    static constexpr int TILES = Base::A_BYTES + Base::B_BYTES, STAGE = TILES + 1024, LDS = S_ * STAGE, RED = 2 * WGN_ * BM_ * 4;
    static_assert(BM_ + BN_ <= 1024 && Base::NW >= 2 && LDS + RED <= 160 * 1024, "LDS");
};

// The contraction of one tile over the blocks [kbeg, kbeg + KT), KT >= 1.  On return no wave reads or fills the ring any more.
template <class C, bool BKC>
__device__ __forceinline__ void scaled_contract(Acc32<C> &acc, const ScaledParams &p, int m0, int n0, int kbeg, int KT, unsigned char *smem)
{
    constexpr int NB = C::WTM / 32, NU = C::WTN / 32, S = C::S, L = C::LA + C::LB;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % C::WGM, wn = wave / C::WGM;
    acc_zero(acc);
    uint32_t offa[C::LA], offb[C::LB];
    int cka[C::LA], ckb[C::LB];
    const int valid_m = p.M - m0 < C::BM ? p.M - m0 : C::BM, valid_n = p.N - n0 < C::BN ? p.N - n0 : C::BN;
#pragma unroll
    for (int i = 0; i < C::LA; ++i) offa[i] = small_goffset<C, true, C::BM>(wave * C::LA + i, lane, p.lda, valid_m, cka[i]);
#pragma unroll
    for (int i = 0; i < C::LB; ++i) offb[i] = small_goffset<C, BKC, C::BN>(wave * C::LB + i, lane, p.ldb, valid_n, ckb[i]);
    const int64_t stepb = BKC ? (int64_t)128 : 128 * p.ldb;
    const unsigned char *ga = p.A + (int64_t)m0 * p.lda + (int64_t)kbeg * 128;
    const unsigned char *gb = p.B + (BKC ? (int64_t)n0 * p.ldb : (int64_t)n0) + kbeg * stepb;
    // scales: sixteen rows a lane; chunks past the last row's fetch that one again (pitches are multiples of 16 and hold it)
    const bool scales_a = wave == 0, scales_b = wave == C::NW - 1;
    const int chunk = lane < (((scales_a ? valid_m : valid_n) - 1) >> 4) ? lane : ((scales_a ? valid_m : valid_n) - 1) >> 4;
    const uint32_t offs = (uint32_t)chunk * 16;
    const int64_t steps = scales_a ? p.ld_sa : p.ld_sb;
    const unsigned char *gs = (scales_a ? p.sa + m0 : p.sb + n0) + kbeg * steps;
    const uint32_t lds0 = (uint32_t)(uintptr_t)smem;
    const bool ragged = (kbeg + KT) * 128 > p.K;     // the last stage reaches past K, see small_contract
    int next = 0;
    uint32_t slot_in = 0;
    auto issue_scales = [&]() {
        if (scales_a) {
            if (lane < C::BM / 16) dl_load16(offs, gs + next * steps, lds0 + slot_in + (uint32_t)C::TILES);
        } else if (scales_b) {
            if (lane < C::BN / 16) dl_load16(offs, gs + next * steps, lds0 + slot_in + (uint32_t)(C::TILES + C::BM));
        }
    };
    auto advance = [&]() {
        ++next;
        slot_in = slot_in + C::STAGE == C::LDS ? 0u : slot_in + C::STAGE;
    };
    // part q of Q of the stage's loads; the last part moves on to the next stage
    auto issue_part = [&](int q, int Q) {
        const unsigned char *sa = ga + (int64_t)next * 128, *sb = gb + (int64_t)next * stepb;
        const uint32_t la = lds0 + slot_in + (uint32_t)(wave * C::LA * 1024), lb = lds0 + slot_in + (uint32_t)(C::A_BYTES + wave * C::LB * 1024);
#pragma unroll
        for (int i = 0; i < L; ++i) {
            if (i < q * L / Q || i >= (q + 1) * L / Q) continue;
            if (i < C::LA) dl_load16(offa[i < C::LA ? i : 0], sa, la + (uint32_t)(i * 1024));
            else dl_load16(offb[i < C::LA ? 0 : i - C::LA], sb, lb + (uint32_t)((i - C::LA) * 1024));
        }
        if (q == Q - 1) {
            issue_scales();
            advance();
        }
    };
    auto issue_last = [&]() {                        // the stage that reaches past K: zeros there
        const int have = p.K - (kbeg + KT - 1) * 128;
        const unsigned char *sa = ga + (int64_t)next * 128, *sb = gb + (int64_t)next * stepb;
        unsigned char *slot = smem + slot_in + lane * 16;
#pragma unroll
        for (int i = 0; i < C::LA; ++i) {
            const int at = (wave * C::LA + i) * 1024;
            if (cka[i] < have) dl_load16(offa[i], sa, lds0 + slot_in + (uint32_t)at);
            else *reinterpret_cast<u32x4 *>(slot + at) = u32x4{0u, 0u, 0u, 0u};
        }
#pragma unroll
        for (int i = 0; i < C::LB; ++i) {
            const int at = C::A_BYTES + (wave * C::LB + i) * 1024;
            if (ckb[i] < have) dl_load16(offb[i], sb, lds0 + slot_in + (uint32_t)at);
            else *reinterpret_cast<u32x4 *>(slot + at) = u32x4{0u, 0u, 0u, 0u};
        }
        issue_scales();
    };
    // loads of `ahead` stages (at most MAX) may be in flight; the waves that fetch scales have one more each
    auto wait_ahead = [&](auto n) {
        constexpr int AHEAD = decltype(n)::value;
        if (scales_a || scales_b) wait_loads<AHEAD *(L + 1)>();
        else wait_loads<AHEAD * L>();
    };
    auto wait_up_to = [&](int ahead) {
        if (ahead <= 0) wait_loads<0>();
        else if (ahead == 1 || S <= 3) wait_ahead(std::integral_constant<int, S >= 3 ? 1 : 0>{});
        else wait_ahead(std::integral_constant<int, S >= 4 ? 2 : 0>{});
    };
    static_assert(S >= 2 && S <= 4, "wait_up_to");

    SmallFrag<C> fa[NB], fb[NU], fn[NU];
    int sa[NB], sb[NU], na[NB], nb[NU];
    uint32_t slot_out = 0;
    auto read_a = [&](int i, int h) { fa[i] = small_frag<C, true, C::BM>(smem + slot_out, wm * C::WTM + i * 32, lane, h); };
    auto read_b = [&](SmallFrag<C>(&f)[NU], int h) {
#pragma unroll
        for (int u = 0; u < NU; ++u) f[u] = small_frag<C, BKC, C::BN>(smem + slot_out + C::A_BYTES, wn * C::WTN + u * 32, lane, h);
    };
    auto read_scales = [&](int(&a)[NB], int(&b)[NU]) {
        const unsigned char *s = smem + slot_out + C::TILES + (lane & 31);
#pragma unroll
        for (int i = 0; i < NB; ++i) a[i] = s[wm * C::WTM + i * 32];
#pragma unroll
        for (int u = 0; u < NU; ++u) b[u] = s[C::BM + wn * C::WTN + u * 32];
    };
    // one MFMA step of half a stage; `beside(i)` follows the MFMAs of row i
    auto mma = [&](const SmallFrag<C>(&f)[NU], auto beside) {
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int u = 0; u < NU; ++u)
                acc.a[i][u] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(f[u], fa[i], acc.a[i][u], 0, 0, 0, sb[u], 0, sa[i]);
            __builtin_amdgcn_sched_barrier(0);
            beside(i);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    auto meet = [&]() {                              // see small_contract
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0xC07F);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("" ::: "memory");
    };
    auto stage = [&](int t, bool steady) {
        mma(fb, [&](int i) {
            if (i == 0) read_b(fn, 1);
            read_a(i, 1);
        });
        const bool more = steady || t + 1 < KT;
        bool fill = steady;
        if (more) {
            const int ahead = KT - 2 - t;            // stages behind t + 1
            if (steady) wait_ahead(std::integral_constant<int, S - 2>{});
            else if (ragged && ahead <= S - 1) wait_loads<0>();
            else wait_up_to(ahead < S - 2 ? ahead : S - 2);
            meet();
            slot_out = slot_out + C::STAGE == C::LDS ? 0u : slot_out + C::STAGE;
            if (!steady) {
                fill = t + S < KT;
                if (ragged && t + S == KT - 1) {
                    issue_last();
                    fill = false;
                }
            }
        }
        mma(fn, [&](int i) {
            if (fill) issue_part(i, NB);
            if (!more) return;
            if (i == 0) {
                read_b(fb, 0);
                read_scales(na, nb);
            }
            read_a(i, 0);
        });
        if (more) {
#pragma unroll
            for (int i = 0; i < NB; ++i) sa[i] = na[i];
#pragma unroll
            for (int u = 0; u < NU; ++u) sb[u] = nb[u];
        }
    };
#pragma unroll
    for (int t = 0; t < S; ++t)
        if (t < KT) {
            if (ragged && t == KT - 1) issue_last();
            else issue_part(0, 1);
        }
    if (KT >= S && !(ragged && KT == S)) wait_ahead(std::integral_constant<int, S - 1>{});
    else wait_loads<0>();
    meet();
    read_b(fb, 0);
    read_scales(sa, sb);
#pragma unroll
    for (int i = 0; i < NB; ++i) read_a(i, 0);
    int t = 0;
    for (; t + S + (ragged ? 1 : 0) < KT; ++t) stage(t, true);
    for (; t < KT; ++t) stage(t, false);
    __syncthreads();
}

// ---------------------------------------------------------------------------------
// Programs that end in STORE_Q8 on the accumulators of a tile of 256 columns, waves of 64 (layout: Acc32).
// The scale of a block is the largest magnitude of 128 columns of a row, which lie in two waves (four for the halved width of SwiGLU
// forward, one for the doubled width of its backward): the waves meet in `red`.  Codes go to LDS, [BM rows][row bytes] with the
// chunks of 16 swizzled by the row, and leave from there in whole rows.
// ---------------------------------------------------------------------------------
template <int RB>
__device__ __forceinline__ uint32_t q8_spot(int r, int byte)
{
    constexpr int NCH = RB / 16;
    const int sw = RB == 128 ? r >> 1 : r;
    return (uint32_t)(r * RB + ((((byte >> 4) ^ sw) & (NCH - 1)) << 4) + (byte & 15));
}
// rows of RB bytes from LDS to global memory; bytes_ok: a multiple of 16
template <class C, int RB, bool EDGE>
__device__ __forceinline__ void q8_store_rows(const unsigned char *ring, uint8_t *out, int64_t ld, int rows_ok, int bytes_ok, int tid)
{
    constexpr int NCH = RB / 16;
#pragma unroll 4
    for (int idx = tid; idx < C::BM * NCH; idx += C::NT) {
        const int r = idx / NCH, c = idx % NCH;
        if (!EDGE || (r < rows_ok && c * 16 < bytes_ok))
            *reinterpret_cast<u32x4 *>(out + r * ld + c * 16) = *reinterpret_cast<const u32x4 *>(ring + q8_spot<RB>(r, c * 16));
    }
}

template <class C, int MODE, bool EDGE>
__device__ __forceinline__ void run_epilogue_q8(Acc32<C> &acc, const GemmParams &p, const Q8Params &q, int m0, int n0, int tn, unsigned char *ring,
                                                float *red, int tid)
{
    constexpr int BM = C::BM, NB = C::WTM / 32, NU = C::WTN / 8;
    static_assert(C::BN == 256 && C::WTN == 64 && C::WGN == 4 && BM * 512 <= C::LDS, "tile");
    const int lane = tid & 63, wave = tid >> 6, lrow = lane & 31, half = lane >> 5;
    const int wm = wave % C::WGM, wn = wave / C::WGM, rw = wm * C::WTM, nw = n0 + wn * 64;
    const int rows_ok = EDGE ? clampi(p.M - m0, 0, BM) : BM, cols_ok = EDGE ? clampi(p.N - n0, 0, 256) : 256;
    auto there = [&](int u) { return !EDGE || nw + u * 8 + half * 4 < p.N; };
    auto either_half = [&](float m) { return fmaxf(m, __shfl_xor(m, 32, 64)); };

    if constexpr (MODE == Q8_SWIGLU_BWD) {
        constexpr int NCH = 32, STEPS = BM * NCH / C::NT, BATCH = 8;
        static_assert(STEPS % BATCH == 0, "whole batches");
        const uint8_t *z = q.z + (int64_t)m0 * q.ldz + 2 * n0;
#pragma unroll
        for (int b = 0; b < STEPS; b += BATCH) {
            u32x4 t[BATCH];
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
                const int idx = (b + k) * C::NT + tid, r = idx / NCH, c = idx % NCH;
                t[k] = u32x4{0u, 0u, 0u, 0u};
                if (!EDGE || (r < rows_ok && c * 8 < cols_ok)) t[k] = *reinterpret_cast<const u32x4 *>(z + r * q.ldz + c * 16);
            }
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
                const int idx = (b + k) * C::NT + tid, r = idx / NCH, c = idx % NCH;
                *reinterpret_cast<u32x4 *>(ring + q8_spot<512>(r, c * 16)) = t[k];
            }
        }
        const int64_t kb = n0 / 64 + wn;             // the wave's block of 128 of the doubled width
        uint32_t zb[NB];
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            const int r = rw + i * 32 + lrow;
            zb[i] = !EDGE || (r < rows_ok && nw < p.N) ? q.z_s[kb * q.ld_z_s + m0 + r] : 127u;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            const int r = rw + i * 32 + lrow;
            const float s = q8_scale(zb[i]);
            float dz[NU][8], largest = 0.0f, stat = 0.0f;
#pragma unroll
            for (int u = 0; u < NU; ++u) {
                const u32x2 w = *reinterpret_cast<const u32x2 *>(ring + q8_spot<512>(r, wn * 128 + u * 16 + half * 8));
                const f32x4 d = acc.get(i, u);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const f32x2 gu = e & 1 ? __builtin_amdgcn_cvt_pk_f32_fp8((int)w[e >> 1], true) : __builtin_amdgcn_cvt_pk_f32_fp8((int)w[e >> 1], false);
                    const float g = gu[0] * s, up = gu[1] * s, sg = fast_sigmoid(g), sl = g * sg;
                    const float dU = d[e] * sl, dG = d[e] * up * (sg + sl * (1.0f - sg));
                    dz[u][2 * e] = dG;
                    dz[u][2 * e + 1] = dU;
                    if (there(u)) {
                        largest = fmaxf(largest, fmaxf(q8_magnitude(dG), q8_magnitude(dU)));
                        stat += g * dG + up * dU;
                    }
                }
            }
            const uint32_t byte = q8_scale_byte(either_half(largest));
            const float inv = q8_inverse(byte);
#pragma unroll
            for (int u = 0; u < NU; ++u)
                *reinterpret_cast<u32x2 *>(ring + q8_spot<512>(r, wn * 128 + u * 16 + half * 8)) =
                    u32x2{q8_codes(dz[u][0], dz[u][1], dz[u][2], dz[u][3], inv), q8_codes(dz[u][4], dz[u][5], dz[u][6], dz[u][7], inv)};
            if (half == 0 && (!EDGE || (r < rows_ok && nw < p.N))) q.out_s[kb * q.ld_out_s + m0 + r] = (uint8_t)byte;
            if (p.rowred_mode != ROWRED_NONE) {
                stat += __shfl_xor(stat, 32, 64);
                if (half == 0) red[wn * BM + r] = stat;
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        __syncthreads();
        q8_store_rows<C, 512, EDGE>(ring, q.out + (int64_t)m0 * q.ld_out + 2 * n0, q.ld_out, rows_ok, 2 * cols_ok, tid);
        if (p.rowred_mode != ROWRED_NONE)
            for (int r = tid; r < BM; r += C::NT) {
                const int m = m0 + r;
                if (EDGE && m >= p.M) continue;
                const float s = (red[r] + red[BM + r]) + (red[2 * BM + r] + red[3 * BM + r]);
                if (p.rowred_mode == ROWRED_PARTIALS) p.rowred[(int64_t)tn * p.M + m] = s;
                else atomicAdd(p.rowred + m, s);
            }
    } else {
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            const int m = m0 + rw + i * 32 + lrow;
            const float rs = p.row_scale && (!EDGE || m < p.M) ? p.row_scale[m] : 1.0f;
#pragma unroll
            for (int u = 0; u < NU; ++u) acc.set(i, u, acc.get(i, u) * rs);
        }
        // codes and scales of the values themselves: the output, or the pre-activation
        auto put_values = [&](uint8_t *out, int64_t ld, uint8_t *scales, int64_t ld_s) {
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                float largest = 0.0f;
#pragma unroll
                for (int u = 0; u < NU; ++u) {
                    const f32x4 v = acc.get(i, u);
                    if (there(u)) largest = fmaxf(fmaxf(fmaxf(largest, q8_magnitude(v[0])), fmaxf(q8_magnitude(v[1]), q8_magnitude(v[2]))), q8_magnitude(v[3]));
                }
                largest = either_half(largest);
                if (half == 0) red[wn * BM + rw + i * 32 + lrow] = largest;
            }
            __syncthreads();
            const int64_t kb = n0 / 128 + (wn >> 1);
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                const int r = rw + i * 32 + lrow;
                const uint32_t byte = q8_scale_byte(fmaxf(red[(wn & 2) * BM + r], red[((wn & 2) + 1) * BM + r]));
                const float inv = q8_inverse(byte);
#pragma unroll
                for (int u = 0; u < NU; ++u) {
                    const f32x4 v = acc.get(i, u);
                    *reinterpret_cast<uint32_t *>(ring + q8_spot<256>(r, wn * 64 + u * 8 + half * 4)) = q8_codes(v[0], v[1], v[2], v[3], inv);
                }
                if ((wn & 1) == 0 && half == 0 && (!EDGE || (r < rows_ok && nw < p.N))) scales[kb * ld_s + m0 + r] = (uint8_t)byte;
            }
            __syncthreads();
            q8_store_rows<C, 256, EDGE>(ring, out + (int64_t)m0 * ld + n0, ld, rows_ok, cols_ok, tid);
        };
        if constexpr (MODE == Q8_LINEAR) {
            put_values(q.out, q.ld_out, q.out_s, q.ld_out_s);
        } else {
            if (q.z) put_values(q.z, q.ldz, q.z_s, q.ld_z_s);
            // silu(g) u takes the place of its pair; the row's 128 of them are the tile's
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                float largest = 0.0f;
#pragma unroll
                for (int u = 0; u < NU; ++u) {
                    const f32x4 v = acc.get(i, u);
                    const float h0 = v[0] * fast_sigmoid(v[0]) * v[1], h1 = v[2] * fast_sigmoid(v[2]) * v[3];
                    acc.set(i, u, f32x4{h0, h1, 0.0f, 0.0f});
                    if (there(u)) largest = fmaxf(largest, fmaxf(q8_magnitude(h0), q8_magnitude(h1)));
                }
                largest = either_half(largest);
                if (half == 0) red[wn * BM + rw + i * 32 + lrow] = largest;
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                const int r = rw + i * 32 + lrow;
                const uint32_t byte = q8_scale_byte(fmaxf(fmaxf(red[r], red[BM + r]), fmaxf(red[2 * BM + r], red[3 * BM + r])));
                const float inv = q8_inverse(byte);
#pragma unroll
                for (int u = 0; u < NU; ++u) {
                    const f32x4 v = acc.get(i, u);
                    *reinterpret_cast<uint16_t *>(ring + q8_spot<128>(r, wn * 32 + u * 4 + half * 2)) =
                        (uint16_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[0] * inv, v[1] * inv, 0, false);
                }
                if (wn == 0 && half == 0 && (!EDGE || r < rows_ok)) q.out_s[(int64_t)tn * q.ld_out_s + m0 + r] = (uint8_t)byte;
            }
            __syncthreads();
            q8_store_rows<C, 128, EDGE>(ring, q.out + (int64_t)m0 * q.ld_out + n0 / 2, q.ld_out, rows_ok, cols_ok / 2, tid);
        }
    }
}

// The same programs on fp32 partials, a wave a row of 256 columns (see epi_rows.hpp).
template <int W>
__device__ __forceinline__ float lanes_max(float v)
{
#pragma unroll
    for (int off = 1; off < W; off <<= 1) v = fmaxf(v, __shfl_xor(v, off, 64));
    return v;
}
template <int MODE>
__global__ __launch_bounds__(256) void epi_rows_q8_kernel(const GemmParams p, const Q8Params q, const float *__restrict__ part, const int nsplit)
{
    const int lane = threadIdx.x & 63;
    const int m = blockIdx.y * EPI_ROWS + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), tn = blockIdx.x, n = tn * 256 + lane * 4;
    if (m >= p.M) return;
    const bool ok = n < p.N;
    float rs = 1.0f;
    u32x2 zc = {0u, 0u};
    uint32_t zb = 127u;
    if (MODE != Q8_SWIGLU_BWD && p.row_scale) rs = p.row_scale[m];
    if (MODE == Q8_SWIGLU_BWD && ok) {
        zc = *reinterpret_cast<const u32x2 *>(q.z + (int64_t)m * q.ldz + 2 * n);
        zb = q.z_s[(int64_t)(n >> 6) * q.ld_z_s + m];
    }
    f32x4 sum[1] = {{0.f, 0.f, 0.f, 0.f}};
    if (ok) sum_parts(sum, {part + (int64_t)m * p.N + n}, nsplit, (int64_t)p.M * p.N);
    f32x4 v = sum[0];
    if constexpr (MODE == Q8_SWIGLU_BWD) {
        const float s = q8_scale(zb);
        float dz[8], largest = 0.0f, stat = 0.0f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const f32x2 gu = e & 1 ? __builtin_amdgcn_cvt_pk_f32_fp8((int)zc[e >> 1], true) : __builtin_amdgcn_cvt_pk_f32_fp8((int)zc[e >> 1], false);
            const float g = gu[0] * s, up = gu[1] * s, sg = fast_sigmoid(g), sl = g * sg;
            const float dU = v[e] * sl, dG = v[e] * up * (sg + sl * (1.0f - sg));
            dz[2 * e] = dG;
            dz[2 * e + 1] = dU;
            largest = fmaxf(largest, fmaxf(q8_magnitude(dG), q8_magnitude(dU)));
            stat += g * dG + up * dU;
        }
        const uint32_t byte = q8_scale_byte(lanes_max<16>(ok ? largest : 0.0f));
        if (ok) {
            const float inv = q8_inverse(byte);
            *reinterpret_cast<u32x2 *>(q.out + (int64_t)m * q.ld_out + 2 * n) = u32x2{q8_codes(dz[0], dz[1], dz[2], dz[3], inv), q8_codes(dz[4], dz[5], dz[6], dz[7], inv)};
            if ((lane & 15) == 0) q.out_s[(int64_t)(n >> 6) * q.ld_out_s + m] = (uint8_t)byte;
        }
        if (p.rowred_mode != ROWRED_NONE) {
            stat = wave_sum(ok ? stat : 0.0f);
            if (lane == 0) {
                if (p.rowred_mode == ROWRED_PARTIALS) p.rowred[(int64_t)tn * p.M + m] = stat;
                else atomicAdd(p.rowred + m, stat);
            }
        }
    } else {
        v *= rs;
        auto put_values = [&](uint8_t *out, int64_t ld, uint8_t *scales, int64_t ld_s) {
            const float largest = fmaxf(fmaxf(q8_magnitude(v[0]), q8_magnitude(v[1])), fmaxf(q8_magnitude(v[2]), q8_magnitude(v[3])));
            const uint32_t byte = q8_scale_byte(lanes_max<32>(ok ? largest : 0.0f));
            if (!ok) return;
            *reinterpret_cast<uint32_t *>(out + (int64_t)m * ld + n) = q8_codes(v[0], v[1], v[2], v[3], q8_inverse(byte));
            if ((lane & 31) == 0) scales[(int64_t)(n >> 7) * ld_s + m] = (uint8_t)byte;
        };
        if constexpr (MODE == Q8_LINEAR) {
            put_values(q.out, q.ld_out, q.out_s, q.ld_out_s);
        } else {
            if (q.z) put_values(q.z, q.ldz, q.z_s, q.ld_z_s);
            const float h0 = v[0] * fast_sigmoid(v[0]) * v[1], h1 = v[2] * fast_sigmoid(v[2]) * v[3];
            const uint32_t byte = q8_scale_byte(lanes_max<64>(ok ? fmaxf(q8_magnitude(h0), q8_magnitude(h1)) : 0.0f));
            const float inv = q8_inverse(byte);
            if (ok) *reinterpret_cast<uint16_t *>(q.out + (int64_t)m * q.ld_out + (n >> 1)) = (uint16_t)__builtin_amdgcn_cvt_pk_fp8_f32(h0 * inv, h1 * inv, 0, false);
            if (lane == 0) q.out_s[(int64_t)tn * q.ld_out_s + m] = (uint8_t)byte;
        }
    }
}

// Kernels: a tile and its program (EPI of GemmParams, or with Q8 a Q8Mode), and the partials of a divided contraction.
template <class C, bool BKC, int EPI, bool Q8>
__global__ __launch_bounds__(C::NT) __attribute__((amdgpu_waves_per_eu(2, 2), amdgpu_num_vgpr(256))) void gemm_scaled_tile(const GemmParams g, const Q8Params q,
                                                                                                                         const ScaledParams p)
{
    __shared__ __attribute__((aligned(1024))) unsigned char smem[C::LDS + C::RED];
    int tm, tn, split;
    small_coords((int)blockIdx.x, p.tiles_m, p.tiles_n, 1, tm, tn, split);
    const int m0 = tm * C::BM, n0 = tn * C::BN, stages = (p.K + 127) / 128;
    Acc32<C> acc;
    if (stages > 0) scaled_contract<C, BKC>(acc, p, m0, n0, 0, stages, smem);
    else acc_zero(acc);
    float *red = reinterpret_cast<float *>(smem + C::LDS);
    const bool edge = m0 + C::BM > p.M || n0 + C::BN > p.N;
    if constexpr (Q8) {
        if (edge) run_epilogue_q8<C, EPI, true>(acc, g, q, m0, n0, tn, smem, red, (int)threadIdx.x);
        else run_epilogue_q8<C, EPI, false>(acc, g, q, m0, n0, tn, smem, red, (int)threadIdx.x);
    } else {
        if (edge) run_epilogue<C, Acc32<C>, EPI, true, C::S * C::TILES>(acc, g, m0, n0, tn, smem, red, (int)threadIdx.x);
        else run_epilogue<C, Acc32<C>, EPI, false, C::S * C::TILES>(acc, g, m0, n0, tn, smem, red, (int)threadIdx.x);
    }
}

template <class C, bool BKC>
__global__ __launch_bounds__(C::NT) __attribute__((amdgpu_waves_per_eu(2, 2), amdgpu_num_vgpr(256))) void gemm_scaled_partial(const ScaledParams p)
{
    __shared__ __attribute__((aligned(1024))) unsigned char smem[C::LDS];
    int tm, tn, split;
    small_coords((int)blockIdx.x, p.tiles_m, p.tiles_n, p.nsplit, tm, tn, split);
    const int stages = (p.K + 127) / 128;
    const int k0 = __builtin_amdgcn_readfirstlane((int)((int64_t)split * stages / p.nsplit));
    const int k1 = __builtin_amdgcn_readfirstlane((int)((int64_t)(split + 1) * stages / p.nsplit));   // k1 > k0: nsplit <= stages
    Acc32<C> acc;
    const int m0 = tm * C::BM, n0 = tn * C::BN;
    scaled_contract<C, BKC>(acc, p, m0, n0, k0, k1 - k0, smem);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int mw = m0 + wave % C::WGM * C::WTM, nw = n0 + wave / C::WGM * C::WTN;
    float *out = p.part + (int64_t)split * p.M * p.N;
    constexpr int RB = C::WTN * 4, UB = 32;
    unsigned char *reg = smem + wave * 32 * RB;
    const uint32_t ulane = Stage<RB>::template unit_lane<16, 32>(lane);
#pragma unroll
    for (int i = 0; i < Acc32<C>::NB; ++i) {
#pragma unroll
        for (int u = 0; u < Acc32<C>::NU; ++u) *reinterpret_cast<f32x4 *>(reg + Stage<RB>::template unit_addr<32>(ulane, 0, u * UB)) = acc.get(i, u);
        stage_fence();
        stage_store<RB, 32, true, false>(reg, reinterpret_cast<unsigned char *>(out + (int64_t)(mw + i * 32) * p.N + nw), (int64_t)p.N * 4, p.M - mw - i * 32,
                                         (p.N - nw) * 4, lane);
        stage_fence();
    }
}

}  // namespace coda
