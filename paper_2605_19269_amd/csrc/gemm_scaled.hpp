// gemm_scaled.hpp -- the product of 8-bit operands with a scale for each block of 128 of the contraction.
//
//   D[i][j] = sum over blocks b of 2^(sa[b][i] - 127) 2^(sb[b][j] - 127) sum over k in b of A[i][k] B[k][j]
//
// A stage of the contraction is one block: 128 bytes of every row.  Its scales travel with it -- BM + BN bytes behind the operand tiles
// of the stage's LDS slot, fetched by the first and the last wave -- and go into the matrix instruction with the fragments, a
// byte for the lane's row of A and one for its column of B.  So the sums stay in one set of fp32 accumulators and a block costs
// a few byte reads.  Scales lie [block][row]: the rows of a tile are BM consecutive bytes.
//
// Tiles of up to 128 rows: the ring and its waits are those of the small tiles (gemm_small.hpp).  The loads of a stage are spread over a whole one: half of
// them in the second half of the stage whose slot they refill, half in the first of the next, between the MFMAs of each row.  All in one half the waves queue
// up behind them (1000 x 4096 x 14336 in 128 x 256 tiles 93.4 us, spread 76; 2048 x 4096 x 4096 36.1 and 34.0).  256 x 256: see scaled_contract_large.
#pragma once
#include "gemm_small.hpp"
#include "epi_rows.hpp"
#include "q8.hpp"
#include "scaled_launch.hpp"

namespace coda {

// 4 bytes a lane, straight to LDS
__device__ __forceinline__ void dl_load4(uint32_t voff, const void *sbase, uint32_t lds_addr)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" : : "v"(voff), "s"(sbase), "s"(lds_addr) : "memory", "m0");
}
// The same by all lanes or, where `mask` is 0 (else -1), none.  Without a branch: the compiler sinks MFMAs from in front of one into the
// block behind it, and with them a compute phase into the memory phase.
__device__ __forceinline__ void dl_load4_if(int mask, uint32_t voff, const void *sbase, uint32_t lds_addr)
{
    uint64_t keep;
    asm volatile("s_mov_b64 %0, exec\n\ts_mov_b32 exec_lo, %1\n\ts_mov_b32 exec_hi, %1\n\ts_mov_b32 m0, %4\n\ts_nop 0\n\tglobal_load_lds_dword %2, %3\n\ts_mov_b64 exec, %0"
                 : "=&s"(keep)
                 : "s"(mask), "v"(voff), "s"(sbase), "s"(lds_addr)
                 : "memory", "m0");
}

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
    // part q of Q of a stage's loads; the last part moves on to the next stage
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
    bool pending = false;                            // the second half of a stage's loads is still to come
    auto stage = [&](int t, bool steady, bool pend) {
        mma(fb, [&](int i) {
            if (pend) issue_part(NB + i, 2 * NB);
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
            if (fill) issue_part(i, 2 * NB);
            if (!more) return;
            if (i == 0) {
                read_b(fb, 0);
                read_scales(na, nb);
            }
            read_a(i, 0);
        });
        pending = fill;
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
    if (S + (ragged ? 1 : 0) < KT) {
        stage(t++, true, false);
        for (; t + S + (ragged ? 1 : 0) < KT; ++t) stage(t, true, true);
    }
    for (; t < KT; ++t) stage(t, false, pending);
    __syncthreads();
}

// ---------------------------------------------------------------------------------
// 256 x 256 tiles: eight waves of 128 x 64, two on a SIMD and one phase apart, as in the large kernel of unscaled 8-bit operands
// (gemm_item_dl_f8).  That one's ring fills LDS: three pair slots of A (a pair of K-steps is 128 bytes of the contraction, one block)
// and two of B, 160 KB.  The scales need room, and A's third slot is only ever half in use: the upper rows of a pair are fetched when the
// lower rows of the pair two before have been read for good.  So A has five half slots of 16 KB -- half h of pair T at (2 T + h) mod 5 --
// and there are 16 KB for the scales of eight pairs and for the programs' exchange.
//   M1  even step: fetch A's lower rows of pair T+2 (over the upper rows of T-1), odd step: its upper rows (over the lower rows of T).
//       Read the upper row fragments, odd step: the scales of pair T+1 as well, and wait for all loads but those of pair T+2
//   C1  MFMAs of the lower rows
//   M2  odd step: fetch B of pair T+2.  Read the lower row and the column fragments of the next step
//   C2  MFMAs of the upper rows
// The wave that runs a phase behind is done with what a load overwrites: its reads of the upper rows of T-1 and of B were waited for two
// phases before; those of the lower rows of T, one phase before, are waited for in the phase that issues them (even M2).
// Scales come for four pairs at once, a load of 256 bytes from every wave: two waves that fetched them for every pair, under a mask and out
// of step with the others, cost 5 %.
// 16384 x 4096 x 28672, B [K x N]: 1376 us, 2.80 PFLOP/s (unscaled 8-bit operands, in turn with it, 1276).  Four waves of 256 x 64 with two whole slots: 1750 (their loads are in flight for half to one
// stage, which is less than what memory takes, and one wave on a SIMD has no other to compute while it issues them).
// ---------------------------------------------------------------------------------
struct ScaledLargeCfg : DlCfg<256, 256, 2, 4, 4> {
    static constexpr int HALF = 128 * 128, A_REGION = 5 * HALF, PAIR_B = 256 * 128, B_REGION = 2 * PAIR_B, TILES = A_REGION + B_REGION;
    static constexpr int SCALES = 512, LDS = TILES + 8 * SCALES, RED = 2 * WGN * BM * 4, EPI_RING = 128 * 1024;
    static_assert(LDS + RED <= 160 * 1024 && EPI_RING <= TILES, "LDS");
};

// RAGGED: tiles on the edges of M and N, and K that is no whole number of blocks.
template <class C, bool BKC, bool RAGGED>
__device__ __forceinline__ void scaled_contract_large(Acc32<C> &acc, const ScaledParams &p, int m0, int n0, unsigned char *smem)
{
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave & 1, wn = wave >> 1;
    const int P = RAGGED ? (p.K + 127) / 128 : p.K / 128;            // pairs of K-steps
    const int valid_m = RAGGED ? (p.M - m0 < 256 ? p.M - m0 : 256) : 256, valid_n = RAGGED ? (p.N - n0 < 256 ? p.N - n0 : 256) : 256;
    acc_zero(acc);
    // A: two wave-loads of a half slot per wave.  Local row q of half h is row (q / 64) * 128 + 64 h + q % 64 of the tile.
    uint32_t offa[2][2], offb[4];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int q = (wave * 2 + i) * 8 + (lane >> 3), r = (q >> 6) * 128 + h * 64 + (q & 63);
            offa[h][i] = (uint32_t)((int64_t)(r < valid_m ? r : valid_m - 1) * p.lda + (((lane & 7) ^ ((q >> 1) & 7)) << 4));
        }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        offb[i] = BKC ? dl_goffset_pair_f8(wave * 4 + i, lane, p.ldb, valid_n) : dl_goffset_mn_f8(wave * 4 + i, lane, p.ldb, valid_n);
    const int64_t stepb = BKC ? (int64_t)128 : 128 * p.ldb;
    const unsigned char *ga = p.A + (int64_t)m0 * p.lda, *gb = p.B + (BKC ? (int64_t)n0 * p.ldb : (int64_t)n0);
    const uint32_t lds0 = (uint32_t)(uintptr_t)smem;
    // scales: wave w < 4 fetches A's of pair w of four, wave 4 + w B's, four rows a lane (past the last row: its chunk again; past the last
    // pair: that one's again)
    const bool scales_b = wave >= 4;
    const int last = ((scales_b ? valid_n : valid_m) - 1) & ~3;
    const uint32_t offs = (uint32_t)(lane * 4 < last ? lane * 4 : last);
    const int64_t steps = scales_b ? p.ld_sb : p.ld_sa;
    const unsigned char *gs = scales_b ? p.sb + n0 : p.sa + m0;

    auto a_half = [&](int T, int h) { return (2 * T + h) % 5 * C::HALF; };
    auto b_slot = [&](int T) { return C::A_REGION + (T & 1) * C::PAIR_B; };
    auto scale_slot = [&](int T) { return C::TILES + (T & 7) * C::SCALES; };
    auto load_or_zero = [&](bool there, uint32_t off, const unsigned char *from, int to) {
        if (there) dl_load16(off, from, lds0 + (uint32_t)to);
        else *reinterpret_cast<u32x4 *>(smem + to + lane * 16) = u32x4{0u, 0u, 0u, 0u};
    };
    // `inside`: the caller knows that the pair lies within K
    auto issue_a = [&](int T, int h, bool inside) {
        const int to = a_half(T, h) + wave * 2048;
        const unsigned char *from = ga + (int64_t)T * 128;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int q = (wave * 2 + i) * 8 + (lane >> 3);
            if (RAGGED && !inside) load_or_zero(T * 128 + (((lane & 7) ^ ((q >> 1) & 7)) << 4) < p.K, offa[h][i], from, to + i * 1024);
            else dl_load16(offa[h][i], from, lds0 + (uint32_t)(to + i * 1024));
        }
    };
    auto issue_b = [&](int T, bool inside) {
        const int to = b_slot(T) + wave * 4096;
        const unsigned char *from = gb + (int64_t)T * stepb;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int at = BKC ? dl_chunk_k_pair_f8(wave * 4 + i, lane) : dl_chunk_k_mn_f8(wave * 4 + i, lane);
            if (RAGGED && !inside) load_or_zero(T * 128 + at < p.K, offb[i], from, to + i * 1024);
            else dl_load16(offb[i], from, lds0 + (uint32_t)(to + i * 1024));
        }
    };
    auto issue_scales = [&](int T, bool now) {       // of pairs T .. T + 3, T a multiple of four
        const int w = T + (wave & 3);
        dl_load4_if(__builtin_amdgcn_readfirstlane(now ? -1 : 0), offs, gs + (w < P ? w : P - 1) * steps, lds0 + (uint32_t)(scale_slot(w) + (scales_b ? 256 : 0)));
    };

    // Fragment addresses: loop-invariant lane parts, the slot's scalar offset added in a compute phase (as in gemm_item_dl_f8).
    constexpr int NXB = 2;
    auto pin = [](uint32_t &x) { asm volatile("" : "+v"(x)); };
    uint32_t la[2], lb[NXB];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const int r = wm * 64 + (lane & 31), sw = (r >> 1) & 7;
        la[c] = (uint32_t)(r * 128 + (((2 * (lane >> 5) + c) ^ sw) << 4));
        pin(la[c]);
        if (BKC) {
            const int rb = wn * 64 + (lane & 31), sb = (rb >> 1) & 7;
            lb[c] = (uint32_t)(rb * 128 + (((2 * (lane >> 5) + c) ^ sb) << 4));
        } else {
            const int i = lane & 15, g = lane >> 4, chunk = ((wn * 64 + c * 32) >> 4) + (g & 1), k0 = 32 * (g >> 1) + (i >> 1);
            lb[c] = (uint32_t)(k0 * 256 + ((chunk ^ (2 * (k0 & 7))) << 4) + ((i & 1) << 3));
        }
        pin(lb[c]);
    }
    auto prep_a = [&](uint32_t(&x)[2], int T, int step, int h) {
        uint32_t so = (uint32_t)a_half(T, h);
        asm volatile("" : "+s"(so));
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            x[c] = (la[c] ^ (uint32_t)(step * 64)) + so;
            pin(x[c]);
        }
    };
    auto prep_b = [&](uint32_t(&x)[NXB], int T, int step) {
        uint32_t so = (uint32_t)(b_slot(T) + (BKC ? 0 : step * 64 * 256));
        asm volatile("" : "+s"(so));
#pragma unroll
        for (int c = 0; c < NXB; ++c) {
            x[c] = (BKC ? lb[c] ^ (uint32_t)(step * 64) : lb[c]) + so;
            pin(x[c]);
        }
    };
    auto two_chunks = [&](uint32_t lo, uint32_t hi) -> i32x8 {
        const u32x4 a = *reinterpret_cast<const u32x4 *>(smem + lo), b = *reinterpret_cast<const u32x4 *>(smem + hi);
        return i32x8{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]};
    };
    auto load_a = [&](i32x8(&f)[2], const uint32_t(&x)[2]) {
#pragma unroll
        for (int i = 0; i < 2; ++i) f[i] = two_chunks(x[0] + (uint32_t)(i * 32 * 128), x[1] + (uint32_t)(i * 32 * 128));
    };
    auto load_b = [&](i32x8(&f)[2], const uint32_t(&x)[NXB]) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            if constexpr (BKC) {
                f[j] = two_chunks(x[0] + (uint32_t)(j * 32 * 128), x[1] + (uint32_t)(j * 32 * 128));
            } else {
                typedef int v2i __attribute__((ext_vector_type(2)));
                typedef __attribute__((address_space(3))) v2i lds_v2i;
                const unsigned char *a = smem + x[j];
                const v2i r0 = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_v2i *)(a));
                const v2i r1 = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_v2i *)(a + 8 * 256));
                const v2i r2 = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_v2i *)(a + 16 * 256));
                const v2i r3 = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_v2i *)(a + 24 * 256));
                f[j] = i32x8{r0[0], r0[1], r1[0], r1[1], r2[0], r2[1], r3[0], r3[1]};
            }
        }
    };
    // The scales of a wave's four row blocks in one register and of its two column blocks in another: the instruction selects the byte.
    struct Scales {
        uint32_t a[4], b[2];
    };
    auto load_scales = [&](Scales &s, int T) {
        const unsigned char *at = smem + scale_slot(T) + (lane & 31);
#pragma unroll
        for (int i = 0; i < 4; ++i) s.a[i] = at[wm * 128 + i * 32];
#pragma unroll
        for (int j = 0; j < 2; ++j) s.b[j] = at[256 + wn * 64 + j * 32];
    };
    int sa = 0, sb = 0, na = 0, nb = 0;
    auto pack_scales = [&](const Scales &s) {
        na = (int)(s.a[0] | s.a[1] << 8 | s.a[2] << 16 | s.a[3] << 24);
        nb = (int)(s.b[0] | s.b[1] << 8);
    };
    auto mma = [&](const i32x8(&fa)[2], const i32x8(&fb)[2], auto half) {
        constexpr int H = decltype(half)::value;
        acc.a[2 * H][0] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fb[0], fa[0], acc.a[2 * H][0], 0, 0, 0, sb, 2 * H, sa);
        acc.a[2 * H][1] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fb[1], fa[0], acc.a[2 * H][1], 0, 0, 1, sb, 2 * H, sa);
        acc.a[2 * H + 1][0] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fb[0], fa[1], acc.a[2 * H + 1][0], 0, 0, 0, sb, 2 * H + 1, sa);
        acc.a[2 * H + 1][1] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fb[1], fa[1], acc.a[2 * H + 1][1], 0, 0, 1, sb, 2 * H + 1, sa);
    };
    // MFMAs stay in their phase: sunk over a branch, to where their result is used, they keep the fragments alive
    auto pin_sums = [&](int h) {
#pragma unroll
        for (int i = 0; i < 2; ++i) asm volatile("" : "+v"(acc.a[2 * h + i][0]), "+v"(acc.a[2 * h + i][1]));
    };
    auto phase_barrier = [&]() {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    const std::integral_constant<int, 0> LOWER{};
    const std::integral_constant<int, 1> UPPER{};
    i32x8 fal[2], fah[2], fb0[2], fb1[2];
    uint32_t xal[2], xah[2], xb[NXB];
    Scales ns;
    // One K-step, `odd` of pair T: steady: pair T + 2 exists, and lies within K.
    auto step = [&](int T, auto odd, const i32x8(&fbc)[2], i32x8(&fbn)[2], bool last, bool steady) {
        constexpr int O = decltype(odd)::value;
        if (steady || T + 2 < P) issue_a(T + 2, O, steady);                       // memory phase 1
        load_a(fah, xah);
        if (O == 1 && !last) {
            load_scales(ns, T + 1);
            if (steady) wait_loads<4>();
            else wait_loads<0>();
        }
        phase_barrier();
        __builtin_amdgcn_s_setprio(1);                                           // compute phase 1
        mma(fal, fbc, LOWER);
        if (!steady) pin_sums(0);
        if (!last) {
            prep_b(xb, T + O, 1 - O);
            prep_a(xal, T + O, 1 - O, 0);
        }
        __builtin_amdgcn_s_setprio(0);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (O == 1 && !last) pack_scales(ns);
        phase_barrier();
        if (!last) {                                                             // memory phase 2
            if (O == 1 && (steady || T + 2 < P)) issue_b(T + 2, steady);
            if (O == 1) issue_scales(T + 4, (T & 3) == 0 && T + 4 < P);
            load_b(fbn, xb);
            load_a(fal, xal);
            if (O == 0) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // the lower rows of T have been read
        }
        phase_barrier();
        __builtin_amdgcn_s_setprio(1);                                           // compute phase 2
        mma(fah, fbc, UPPER);
        if (!steady) pin_sums(1);
        if (!last) prep_a(xah, T + O, 1 - O, 1);
        __builtin_amdgcn_s_setprio(0);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (O == 1 && !last) {
            sa = na;
            sb = nb;
        }
        phase_barrier();
    };
    const std::integral_constant<int, 0> EVEN{};
    const std::integral_constant<int, 1> ODD{};

    issue_scales(0, true);
    issue_a(0, 0, false);
    issue_a(0, 1, false);
    issue_b(0, false);
    if (P > 1) {
        issue_a(1, 0, false);
        issue_a(1, 1, false);
        issue_b(1, false);
    }
    if (P > 1 && (!RAGGED || 256 <= p.K)) wait_loads<8>();
    else wait_loads<0>();
    __syncthreads();
    prep_a(xal, 0, 0, 0);
    prep_b(xb, 0, 0);
    prep_a(xah, 0, 0, 1);
    load_a(fal, xal);
    load_b(fb0, xb);
    load_scales(ns, 0);
    pack_scales(ns);
    sa = na;
    sb = nb;
    if (wave >= 4) phase_barrier();                     // the second wave of every SIMD runs one phase behind
    int T = 0;
    for (; T + 2 < P && (!RAGGED || (T + 3) * 128 <= p.K); ++T) {
        step(T, EVEN, fb0, fb1, false, true);
        step(T, ODD, fb1, fb0, false, true);
    }
    for (; T + 1 < P; ++T) {                            // the ring runs dry, or the last pair reaches past K
        step(T, EVEN, fb0, fb1, false, false);
        step(T, ODD, fb1, fb0, false, false);
    }
    step(T, EVEN, fb0, fb1, false, false);
    step(T, ODD, fb1, fb0, true, false);
    if (wave < 4) phase_barrier();                      // every wave passes the same number of barriers
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
    static_assert(C::BN == 256 && C::WTN == 64 && C::WGN == 4 && BM * 512 + 1024 <= C::LDS, "tile");
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lrow = lane & 31, half = lane >> 5;
    const int wm = wave % C::WGM, wn = wave / C::WGM, rw = wm * C::WTM, nw = n0 + wn * 64;
    const int rows_ok = EDGE ? clampi(p.M - m0, 0, BM) : BM, cols_ok = EDGE ? clampi(p.N - n0, 0, 256) : 256;
    auto there = [&](int u) { return !EDGE || nw + u * 8 + half * 4 < p.N; };
    auto either_half = [&](float m) { return fmaxf(m, __shfl_xor(m, 32, 64)); };

    if constexpr (MODE == Q8_SWIGLU_BWD) {
        // A wave's 64 columns are one block of the doubled width, so it works by itself.  Its rows of Z, 128 bytes each, go straight to
        // a region of its own, in the layout of Stage (a chunk's place is its lane's, so the swizzle is in what the lane fetches), 32
        // rows are computed while the next are on their way, and the codes of dZ take the place of Z's.  No register holds Z ahead of
        // time: 128 accumulators and the 64 values of a lane's row leave none (fetched to registers: 120 spilled; 8192 x 8192 x 2048 290 us, so 167).
        constexpr int RB = 128, P = 32;
        using St = Stage<RB>;
        unsigned char *reg = ring + wave * (C::WTM * RB), *zs = ring + BM * 512 + wave * 128;
        const bool want_stat = p.rowred_mode != ROWRED_NONE;
        const int wave_rows = EDGE ? clampi(rows_ok - rw, 0, C::WTM) : C::WTM, wave_bytes = EDGE ? clampi(2 * (p.N - nw), 0, RB) : RB;
        const int64_t kb = n0 / 64 + wn;
        if (!EDGE || (wave_rows > 0 && wave_bytes > 0)) {
            const int last = (wave_rows - 1) & ~3;
            if (lane < 32) dl_load4(lane * 4 < last ? lane * 4 : last, q.z_s + kb * q.ld_z_s + m0 + rw, (uint32_t)(uintptr_t)zs);
            const uint8_t *z = q.z + (int64_t)(m0 + rw) * q.ldz + 2 * nw;
#pragma unroll
            for (int it = 0; it < C::WTM / St::RPI; ++it) {
                const int r = it * St::RPI + (lane >> 3), c = ((lane & 7) ^ ((r >> 1) & 7)) << 4;
                const int rr = EDGE && r >= wave_rows ? wave_rows - 1 : r, cc = EDGE && c >= wave_bytes ? wave_bytes - 16 : c;
                dl_load16((uint32_t)((int64_t)rr * q.ldz + cc), z, (uint32_t)(uintptr_t)reg + (uint32_t)(it * 1024));
            }
            auto block = [&](auto ic) {
                constexpr int i = decltype(ic)::value;
                wait_loads<(NB - 1 - i) * (P / St::RPI)>();
                const int r = rw + i * 32 + lrow;
                const float s = q8_scale(zs[i * 32 + lrow]);
                uint32_t ulane = St::template unit_lane<8, 32>(lane);
                asm volatile("" : "+v"(ulane));
                float dz[NU][8], stat = 0.0f;
#pragma unroll
                for (int u = 0; u < NU; ++u) {
                    const u32x2 w = *reinterpret_cast<const u32x2 *>(reg + St::template unit_addr<32>(ulane, i, u * 16));
                    const f32x4 d = acc.get(i, u);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const f32x2 gu = e & 1 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[e >> 1], s, true) : __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[e >> 1], s, false);
                        const float g = gu[0], up = gu[1], sg = fast_sigmoid(g), sl = g * sg;
                        dz[u][2 * e] = d[e] * up * (sg + sl * (1.0f - sg));
                        dz[u][2 * e + 1] = d[e] * sl;
                        if (want_stat && there(u)) stat += g * dz[u][2 * e] + up * dz[u][2 * e + 1];
                    }
                    if (u & 1) __builtin_amdgcn_sched_barrier(0);
                }
                const float largest = q8_largest([&](auto take) {
#pragma unroll
                    for (int u = 0; u < NU; ++u)
                        if (there(u)) {
                            take(dz[u][0], dz[u][1]);
                            take(dz[u][2], dz[u][3]);
                            take(dz[u][4], dz[u][5]);
                            take(dz[u][6], dz[u][7]);
                        }
                });
                const uint32_t byte = q8_scale_byte(either_half(largest));
                const float scale = q8_scale(byte);
                uint32_t ulane2 = St::template unit_lane<8, 32>(lane);
                asm volatile("" : "+v"(ulane2));
#pragma unroll
                for (int u = 0; u < NU; ++u)
                    *reinterpret_cast<u32x2 *>(reg + St::template unit_addr<32>(ulane2, i, u * 16)) =
                        u32x2{q8_codes(dz[u][0], dz[u][1], dz[u][2], dz[u][3], scale), q8_codes(dz[u][4], dz[u][5], dz[u][6], dz[u][7], scale)};
                zs[i * 32 + lrow] = (unsigned char)byte;
                if (want_stat) {
                    stat += __shfl_xor(stat, 32, 64);
                    if (half == 0) red[wn * BM + r] = stat;
                }
                stage_fence();
            };
            block(std::integral_constant<int, 0>{});
            block(std::integral_constant<int, 1>{});
            if constexpr (NB > 2) {
                block(std::integral_constant<int, 2>{});
                block(std::integral_constant<int, 3>{});
            }
            static_assert(NB == 2 || NB == 4, "blocks");
            // stores after the last wait for loads
            stage_store<RB, C::WTM, EDGE, false>(reg, q.out + (int64_t)(m0 + rw) * q.ld_out + 2 * nw, q.ld_out, wave_rows, wave_bytes, lane);
            uint8_t *to = q.out_s + kb * q.ld_out_s + m0 + rw;
#pragma unroll
            for (int r = lane; r < C::WTM; r += 64)
                if (!EDGE || r < wave_rows) to[r] = zs[r];
        } else if (want_stat) {
            for (int r = lane; r < C::WTM; r += 64) red[wn * BM + rw + r] = 0.0f;
        }
        if (want_stat) {
            __syncthreads();
            for (int r = tid; r < BM; r += C::NT) {
                const int m = m0 + r;
                if (EDGE && m >= p.M) continue;
                const float s = (red[r] + red[BM + r]) + (red[2 * BM + r] + red[3 * BM + r]);
                if (p.rowred_mode == ROWRED_PARTIALS) p.rowred[(int64_t)tn * p.M + m] = s;
                else atomicAdd(p.rowred + m, s);
            }
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
                const float largest = either_half(q8_largest([&](auto take) {
#pragma unroll
                    for (int u = 0; u < NU; ++u)
                        if (there(u)) {
                            const f32x4 v = acc.get(i, u);
                            take(v[0], v[1]);
                            take(v[2], v[3]);
                        }
                }));
                if (half == 0) red[wn * BM + rw + i * 32 + lrow] = largest;
            }
            __syncthreads();
            const int64_t kb = n0 / 128 + (wn >> 1);
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                const int r = rw + i * 32 + lrow;
                const uint32_t byte = q8_scale_byte(fmaxf(red[(wn & 2) * BM + r], red[((wn & 2) + 1) * BM + r]));
                const float scale = q8_scale(byte);
#pragma unroll
                for (int u = 0; u < NU; ++u) {
                    const f32x4 v = acc.get(i, u);
                    *reinterpret_cast<uint32_t *>(ring + q8_spot<256>(r, wn * 64 + u * 8 + half * 4)) = q8_codes(v[0], v[1], v[2], v[3], scale);
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
#pragma unroll
                for (int u = 0; u < NU; ++u) {
                    const f32x4 v = acc.get(i, u);
                    acc.set(i, u, f32x4{v[0] * fast_sigmoid(v[0]) * v[1], v[2] * fast_sigmoid(v[2]) * v[3], 0.0f, 0.0f});
                }
                const float largest = either_half(q8_largest([&](auto take) {
#pragma unroll
                    for (int u = 0; u < NU; ++u)
                        if (there(u)) take(acc.get(i, u)[0], acc.get(i, u)[1]);
                }));
                if (half == 0) red[wn * BM + rw + i * 32 + lrow] = largest;
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                const int r = rw + i * 32 + lrow;
                const uint32_t byte = q8_scale_byte(fmaxf(fmaxf(red[r], red[BM + r]), fmaxf(red[2 * BM + r], red[3 * BM + r])));
                const float scale = q8_scale(byte);
#pragma unroll
                for (int u = 0; u < NU; ++u) {
                    const f32x4 v = acc.get(i, u);
                    *reinterpret_cast<uint16_t *>(ring + q8_spot<128>(r, wn * 32 + u * 4 + half * 2)) = q8_codes2(v[0], v[1], scale);
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
            const f32x2 gu = e & 1 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(zc[e >> 1], s, true) : __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(zc[e >> 1], s, false);
            const float g = gu[0], up = gu[1], sg = fast_sigmoid(g), sl = g * sg;
            dz[2 * e] = v[e] * up * (sg + sl * (1.0f - sg));
            dz[2 * e + 1] = v[e] * sl;
            largest = fmaxf(largest, fmaxf(q8_magnitude(dz[2 * e]), q8_magnitude(dz[2 * e + 1])));
            stat += g * dz[2 * e] + up * dz[2 * e + 1];
        }
        const uint32_t byte = q8_scale_byte(lanes_max<16>(ok ? largest : 0.0f));
        if (ok) {
            const float scale = q8_scale(byte);
            *reinterpret_cast<u32x2 *>(q.out + (int64_t)m * q.ld_out + 2 * n) = u32x2{q8_codes(dz[0], dz[1], dz[2], dz[3], scale), q8_codes(dz[4], dz[5], dz[6], dz[7], scale)};
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
            *reinterpret_cast<uint32_t *>(out + (int64_t)m * ld + n) = q8_codes(v[0], v[1], v[2], v[3], q8_scale(byte));
            if ((lane & 31) == 0) scales[(int64_t)(n >> 7) * ld_s + m] = (uint8_t)byte;
        };
        if constexpr (MODE == Q8_LINEAR) {
            put_values(q.out, q.ld_out, q.out_s, q.ld_out_s);
        } else {
            if (q.z) put_values(q.z, q.ldz, q.z_s, q.ld_z_s);
            const float h0 = v[0] * fast_sigmoid(v[0]) * v[1], h1 = v[2] * fast_sigmoid(v[2]) * v[3];
            const uint32_t byte = q8_scale_byte(lanes_max<64>(ok ? fmaxf(q8_magnitude(h0), q8_magnitude(h1)) : 0.0f));
            if (ok) *reinterpret_cast<uint16_t *>(q.out + (int64_t)m * q.ld_out + (n >> 1)) = q8_codes2(h0, h1, q8_scale(byte));
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

template <bool BKC, int EPI, bool Q8, bool RAGGED>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) void gemm_scaled_large(const GemmParams g, const Q8Params q, const ScaledParams p)
{
    using C = ScaledLargeCfg;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[C::LDS + C::RED];
    int tm, tn;
    tile_coords((int)blockIdx.x, p.tiles_m * p.tiles_n, p.tiles_m, p.tiles_n, tm, tn);
    const int m0 = tm * 256, n0 = tn * 256;
    Acc32<C> acc;
    if (RAGGED && p.K == 0) acc_zero(acc);
    else scaled_contract_large<C, BKC, RAGGED>(acc, p, m0, n0, smem);
    float *red = reinterpret_cast<float *>(smem + C::LDS);
    if constexpr (Q8) run_epilogue_q8<C, EPI, RAGGED>(acc, g, q, m0, n0, tn, smem, red, (int)threadIdx.x);
    else run_epilogue<C, Acc32<C>, EPI, RAGGED, C::EPI_RING>(acc, g, m0, n0, tn, smem, red, (int)threadIdx.x);
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


// ---------------------------------------------------------------------------------
// Up to 32 rows against a B stored [N x K], in one kernel and without a workspace: a workgroup owns 16 or 32 columns, its eight waves take
// every eighth block of the contraction and add up in LDS, in wave order.  A block is one v_mfma_scale_f32_16x16x128_f8f6f4, whose fragments
// come straight from memory: lane l holds bytes 16 (l / 16) .. and 64 + 16 (l / 16) .. of its row's 128, for both operands (which k meets which
// is free within a block), so that a load takes 64 consecutive bytes of a row.  Four blocks of a wave are in flight.  Bound by HBM and, with
// few weights, by the launch.  For programs without row reductions, whose partials are per 256 columns.
// ---------------------------------------------------------------------------------
template <int EPI>
__device__ __forceinline__ void few_program(const GemmParams &p, int m, int n, f32x4 v)
{
    static_assert(EPI == EPI_LINEAR || EPI == EPI_SWIGLU_FWD, "programs without row reductions");
    if (p.row_scale) v *= p.row_scale[m];
    if constexpr (EPI == EPI_SWIGLU_FWD) {
        const float h0 = v[0] * fast_sigmoid(v[0]) * v[1], h1 = v[2] * fast_sigmoid(v[2]) * v[3];
        *reinterpret_cast<uint32_t *>(reinterpret_cast<uint16_t *>(p.out) + (int64_t)m * p.ld_out + (n >> 1)) = pack_bf16x2(h0, h1);
        if (p.out2) *reinterpret_cast<u32x2 *>(p.out2 + (int64_t)m * p.ld_out2 + n) = pack4(v);
    } else {
        if (p.rope_cos && n < p.rope_cols)
            rope_unit(v, p, (int64_t)clampi(p.rope_pos[m], 0, p.rope_T - 1) * p.rope_half, (n >> 1) % p.rope_half);
        if (p.add) v += unpack4(*reinterpret_cast<const u32x2 *>(p.add + (int64_t)m * p.ld_add + n));
        if (p.side) *reinterpret_cast<u32x2 *>(p.side + (int64_t)m * p.ld_side + n) = pack4(v * *reinterpret_cast<const f32x4 *>(p.col_scale + n));
        if (p.out_f32) *reinterpret_cast<f32x4 *>(reinterpret_cast<float *>(p.out) + (int64_t)m * p.ld_out + n) = v;
        else *reinterpret_cast<u32x2 *>(reinterpret_cast<uint16_t *>(p.out) + (int64_t)m * p.ld_out + n) = pack4(v);
    }
}

template <int RB, int CB, int EPI>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(RB + CB > 2 ? 2 : 4, RB + CB > 2 ? 2 : 4))) void gemm_scaled_few(const GemmParams g, const ScaledParams p)
{
    constexpr int W = 8, DEPTH = RB + CB > 3 ? 3 : 4, ROWS = RB * 16, COLS = CB * 16;
    __shared__ f32x4 sums[W][ROWS][COLS / 4 + 1];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lr = lane & 15, q = lane >> 4;
    const int n0 = (int)blockIdx.x * COLS, blocks = (p.K + 127) / 128;
    struct Block {
        u32x4 a[RB][2], b[CB][2];
        int sa[RB], sb[CB];
    };
    // rows and columns past the end: the last one's again
    const unsigned char *ga[RB], *gb[CB], *gsa[RB], *gsb[CB];
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        const int m = r * 16 + lr < p.M ? r * 16 + lr : p.M - 1;
        ga[r] = p.A + (int64_t)m * p.lda + q * 16;
        gsa[r] = p.sa + m;
    }
#pragma unroll
    for (int c = 0; c < CB; ++c) {
        const int n = n0 + c * 16 + lr < p.N ? n0 + c * 16 + lr : p.N - 1;
        gb[c] = p.B + (int64_t)n * p.ldb + q * 16;
        gsb[c] = p.sb + n;
    }
    auto load = [&](Block &s, int blk) {
        const int64_t at = (int64_t)blk * 128;
        const bool lo = at + q * 16 < p.K, hi = at + 64 + q * 16 < p.K;          // K is a multiple of 16
        auto two = [&](u32x4(&v)[2], const unsigned char *from) {
            v[0] = v[1] = u32x4{0u, 0u, 0u, 0u};
            if (lo) v[0] = *reinterpret_cast<const u32x4 *>(from + at);
            if (hi) v[1] = *reinterpret_cast<const u32x4 *>(from + at + 64);
        };
#pragma unroll
        for (int c = 0; c < CB; ++c) {
            two(s.b[c], gb[c]);
            s.sb[c] = gsb[c][blk * p.ld_sb];
        }
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            two(s.a[r], ga[r]);
            s.sa[r] = gsa[r][blk * p.ld_sa];
        }
    };
    f32x4 acc[RB][CB];
#pragma unroll
    for (int r = 0; r < RB; ++r)
#pragma unroll
        for (int c = 0; c < CB; ++c) acc[r][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto join = [](const u32x4(&v)[2]) {
        return i32x8{(int)v[0][0], (int)v[0][1], (int)v[0][2], (int)v[0][3], (int)v[1][0], (int)v[1][1], (int)v[1][2], (int)v[1][3]};
    };
    Block ring[DEPTH];
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
        if (wave + d * W < blocks) load(ring[d], wave + d * W);
    for (int b0 = wave; b0 < blocks; b0 += DEPTH * W) {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            const int blk = b0 + d * W;
            if (blk >= blocks) break;
#pragma unroll
            for (int r = 0; r < RB; ++r)
#pragma unroll
                for (int c = 0; c < CB; ++c)
                    acc[r][c] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(join(ring[d].b[c]), join(ring[d].a[r]), acc[r][c], 0, 0, 0, ring[d].sb[c], 0,
                                                                                 ring[d].sa[r]);
            if (blk + DEPTH * W < blocks) load(ring[d], blk + DEPTH * W);
        }
    }
#pragma unroll
    for (int r = 0; r < RB; ++r)
#pragma unroll
        for (int c = 0; c < CB; ++c) sums[wave][r * 16 + lr][c * 4 + q] = acc[r][c];
    __syncthreads();
    const int m = tid / (COLS / 4), u = tid % (COLS / 4), n = n0 + u * 4;
    if (tid >= ROWS * (COLS / 4) || m >= p.M || n >= p.N) return;
    f32x4 v = sums[0][m][u];
#pragma unroll
    for (int w = 1; w < W; ++w) v += sums[w][m][u];
    few_program<EPI>(g, m, n, v);
}

}  // namespace coda
