// attention.hip -- attention of packed sequences, forward.
//
//   S_ij = scale q_i . k_j,  lse_i = log sum_j exp S_ij,  o_i = sum_j exp(S_ij - lse_i) v_j   over the keys j that row i sees
//
// in one pass over the keys with the running maximum and sum of each row (attn_tile.hpp).  Bound by exponentials and products, which share a wave's issue: a workgroup of four waves has 128 rows and tiles of 64
// keys, K and V doubly buffered in 64 KB of LDS at 128 columns, two workgroups a CU.  32 heads over 8 of 128 columns: 16384 rows 1980 us (1110 TFLOP/s) once the clock has settled, up to 2150 before; 8192 in six
// sequences 195 to 204 (880 to 920).
#include "attn_launch.hpp"
#include "attn_tile.hpp"

namespace coda {

constexpr int FWD_WAVES = 4;

// SPLIT waves share 32 rows, each with every SPLIT-th tile of KEYS keys (a stream), and their sums are joined at the end
template <int DP, bool PAD, int SPLIT, int KEYS>
__global__ __launch_bounds__(256, DP == 128 && SPLIT == 4 ? 1 : 2) void attention_kernel(AttnParams p, float c)
{
    constexpr int NW = FWD_WAVES / SPLIT, ROWS = NW * 32, TILE = KEYS * DP * 2, ROUND = SPLIT * KEYS;
    constexpr int UNITS = DP / 32 * 4, PARTS_AT_END = SPLIT > 1 ? (FWD_WAVES * UNITS + 2) * 1024 : 0;      // UNITS: of four registers of O, 1 KB each
    __shared__ __attribute__((aligned(1024))) unsigned char smem[4 * SPLIT * TILE > PARTS_AT_END ? 4 * SPLIT * TILE : PARTS_AT_END];
    __shared__ int dirty;                                  // a masked tile of V held something that is not finite
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    const int block = wave % NW, stream = wave / NW;       // which 32 rows, which tiles
    // The last tiles of rows, which see the most keys, come first.  Workgroups go round the XCDs: the heads of one group are kept on one XCD, whose L2 then
    // serves their keys and values.
    const int64_t tiles = (int64_t)gridDim.x / p.heads;
    const int64_t t = tiles - 1 - blockIdx.x / p.heads;
    int head = blockIdx.x % p.heads;
    if (p.heads % 8 == 0) head = head % 8 * (p.heads / 8) + head / 8;
    const int s = attn_find(p.seq_q, p.n_seqs, ROWS, t, lane);
    const AttnSpan q = attn_span_of_wave(p.seq_q, s, p.Tq), k = attn_span_of_wave(p.seq_k, s, p.Tk);
    const int64_t first = (t - (max(p.seq_q[s], 0) / ROWS + s)) * ROWS;
    if (first < 0 || first >= q.count) return;
    const int row0 = (int)first, ahead = k.count - q.count;
    const int kv = head / (p.heads / p.kv_heads);
    const uint16_t *K = p.K + (int64_t)k.begin * p.ldk + (int64_t)kv * p.D, *V = p.V + (int64_t)k.begin * p.ldv + (int64_t)kv * p.D;

    const int row = row0 + block * 32 + (lane & 31), last = min(row, q.count - 1);
    const uint16_t *Q = p.Q + (q.begin + (int64_t)last) * p.ldq + (int64_t)head * p.D;
    bf16x8 qf[DP / 16];
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) {
        const int d = 16 * i + 8 * h;
        qf[i] = !PAD || d < p.D ? *reinterpret_cast<const bf16x8 *>(Q + d) : bf16x8{};
    }
    // keys that the lane's row sees, and those that the wave's first and last and the workgroup's last do
    const auto sees = [&](int r) { return p.causal ? min(max(r + ahead + 1, 0), k.count) : k.count; };
    const int mine = sees(last), low = sees(min(row0 + block * 32, q.count - 1)), high = row0 + block * 32 < q.count ? sees(min(row0 + block * 32 + 31, q.count - 1)) : 0;
    const int keys = sees(min(row0 + ROWS - 1, q.count - 1)), whole = sees(row0);
    const AttnLane<DP> in(lane);
    AttnRows<DP> acc;
    acc.clear();
    if (threadIdx.x == 0) dirty = 0;
    if (PAD) attn_zero(smem, sizeof(smem), 256);
    const int n = (keys + ROUND - 1) / ROUND;
    AttnLoad<DP, PAD, KEYS, NW> load_k(K, p.ldk, block, lane, p.D), load_v(V, p.ldv, block, lane, p.D);
    const auto stage = [&](int j) { return smem + ((j & 1) * SPLIT + stream) * 2 * TILE; };
    // The stream's tile of round j in parts, that a step issues among its products: all waves' at once after the barrier would hold each other up
    constexpr int PARTS = 2 * load_k.LOADS, PRODUCTS = DP / 16 * (KEYS / 32);
    const auto load = [&](int j, int part) {
        unsigned char *at = stage(j);
        if (part == 0) {
            load_k.begin(j * ROUND + stream * KEYS, k.count, attn_lds(at));
            load_v.begin(j * ROUND + stream * KEYS, k.count, attn_lds(at + TILE));
        }
        if (part < PARTS / 2) load_k.next(part);
        else load_v.next(part - PARTS / 2);
    };
    const auto load_all = [&](int j) {
#pragma unroll
        for (int i = 0; i < PARTS; ++i) load(j, i);
    };
    if (n > 0) load_all(0);
    if (NW == 1) {                                         // `dirty` is cleared before anyone sets it
        attn_reads_done();
        attn_barrier();
    }
    attn_arrived(qf);
    for (int j = 0; j < n; ++j) {
        attn_wait();
        if (NW > 1) attn_barrier();                        // the tiles of round j are there, and nobody reads those of j - 1 any more; a lone wave's are its own
        const int k0 = j * ROUND + stream * KEYS;
        unsigned char *at = stage(j);
        if ((j + 1) * ROUND > whole) {
            constexpr int PART = TILE / NW;
            if (attn_clean(at + TILE + block * PART, PART, min(k.count - k0, KEYS) * (DP * 2) - block * PART, lane)) dirty = 1;
            attn_reads_done();
            if (NW > 1) attn_barrier();
        }
        if (k0 < high) {
            const int lim = mine - k0;
            static_assert(PRODUCTS % PARTS == 0 || PARTS % PRODUCTS == 0, "a place for every load");
            attn_step<DP, KEYS / 32>(attn_lds(at) + in.rows, attn_lds(at + TILE) + in.cols, qf, acc, c, lane, k0 + KEYS > low, [&](int key) { return key < lim; },
                                     [&](int i) {                                          // past the last key there is nothing to load
                                         if constexpr (PARTS > PRODUCTS) {
#pragma unroll
                                             for (int e = 0; e < PARTS / PRODUCTS; ++e) load(j + 1, i * (PARTS / PRODUCTS) + e);
                                         } else if (i % (PRODUCTS / PARTS) == 0)
                                             load(j + 1, i / (PRODUCTS / PARTS));
                                     });
        } else
            load_all(j + 1);
    }
    f32x2 halves = attn_halves(acc.l);
    float l = halves[0] + halves[1], m = acc.m;
    if constexpr (SPLIT > 1) {
        // Every stream's part goes to LDS, and stream s finishes the blocks of 32 columns s, s + SPLIT, ..
        f32x4 *parts = reinterpret_cast<f32x4 *>(smem) + lane;
        float *stats = reinterpret_cast<float *>(smem + FWD_WAVES * UNITS * 1024) + lane;
        attn_wait();
        __syncthreads();
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            const int g = u % 4 * 4;
            const f32x16 &v = acc.o[u / 4];
            parts[(wave * UNITS + u) * 64] = f32x4{v[g], v[g + 1], v[g + 2], v[g + 3]};
        }
        stats[wave * 128] = m;
        stats[wave * 128 + 64] = l;
        __syncthreads();
        float ms[SPLIT], ls[SPLIT];
#pragma unroll
        for (int j = 0; j < SPLIT; ++j) {
            ms[j] = stats[(j * NW + block) * 128];
            ls[j] = stats[(j * NW + block) * 128 + 64];
            m = fmaxf(m, ms[j]);
        }
        l = 0.0f;
#pragma unroll
        for (int j = 0; j < SPLIT; ++j) {
            ms[j] = ms[j] == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f((ms[j] - m) * c);       // the stream's weight
            l += ms[j] * ls[j];
        }
#pragma unroll
        for (int b = 0; b < DP / 32; ++b) {
            if (b % SPLIT != stream) continue;
            f32x16 sum = {};
#pragma unroll
            for (int j = 0; j < SPLIT; ++j)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const f32x4 v = parts[((j * NW + block) * UNITS + b * 4 + g) * 64];
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[4 * g + e] += ms[j] * v[e];
                }
            acc.o[b] = sum;
        }
    }
    if (n * ROUND > whole) {
        attn_wait();                                       // the last round's loads for the next
        __syncthreads();
        if (dirty)
            for (int j = whole / ROUND * SPLIT; j < n * SPLIT; ++j) {
                AttnLoad<DP, PAD, KEYS, FWD_WAVES>(V, p.ldv, wave, lane, p.D)(j * KEYS, k.count, smem);
                attn_wait();
                attn_barrier();
                const int lim = mine - j * KEYS;
                attn_add_marks<DP, KEYS / 16>(attn_lds(smem) + in.cols, acc.o, lane, [&](int key) { return key < lim; }, attn_marked);
                __syncthreads();
            }
    }
    const bool none = mine == 0;                           // sees nothing: zeros, and a log-sum-exp of -inf
    const float inv = none ? 0.0f : 1.0f / l;
    const bool there = row < q.count;
    if (there && p.lse && h == 0 && stream == 0) p.lse[(int64_t)head * p.Tq + q.begin + row] = none ? -__builtin_inff() : m * p.scale + LN2 * __builtin_amdgcn_logf(l);
    uint16_t *out = p.out + ((int64_t)q.begin + row) * p.ldo + (int64_t)head * p.D;
#pragma unroll
    for (int b = 0; b < DP / 32; ++b) {
        if (b % SPLIT != stream) continue;
#pragma unroll
        for (int g = 0; g < 4; g += 2) {
            float lo[4], hi[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                lo[e] = acc.o[b][4 * g + e] * inv;
                hi[e] = acc.o[b][4 * g + 4 + e] * inv;
            }
            const u32x4 v = attn_store_unit(lo, hi);
            const int d = 32 * b + 8 * (g + h);
            if (there && (!PAD || d < p.D)) *reinterpret_cast<u32x4 *>(out + d) = v;
        }
    }
}

// How many waves share 32 rows.  A wave's time is that of its steps one after the other (0.9 us for 64 keys where nothing else runs on its SIMD), so while the
// card has room for all workgroups at once (by their registers and LDS: SPLIT 4 one a CU, SPLIT 2 two, D <= 64 twice as many), splitting rows' keys cuts the longest
// one's steps; past that, shared tiles count.  Tiles are estimated, half a tile a sequence on average, and an eighth more than fits at once is still
// worth it.  Measured, us with SPLIT 1 / 2 / 4, 32 heads over 8: D = 64, a sequence of 128: 6.0 / 5.1 / 5.0, 509: 11.5 / 8.7 / 7.5, 1024: 18.9 / 13.7 / 16.1,
// 2048: 33.3 / 28.9 / 39, 4096: 88 / 91 / 122; 4 x 512: 16.0 / 15.9 / 24.6.  D = 128: 128: 8.0 / 6.8 / 6.6, 509: 15.1 / 11.5 / 15.1, 1024: 24.3 / 19.9 / 34.5, 2048: 48.9 / 51.6 / 90.
// 8 heads over 2: D = 64, 1024: 18.2 / 12.8 / 8.6, 4096: 61 / 39 / 36; D = 128, 1024: 23.2 / 17.0 / 12.1.  33 keys, one tile: 4.3 / 4.3 / 4.9.
static int fwd_split(const AttnParams &p)
{
    if (p.Tk <= 64) return 1;
    const int64_t room = p.D > 64 ? 288 : 576;
    return attn_about(p.Tq, p.n_seqs, 32) * p.heads <= room ? 4 : attn_about(p.Tq, p.n_seqs, 64) * p.heads <= 2 * room ? 2 : 1;
}
int64_t attn_workgroups(const AttnParams &p) { return ((int64_t)p.Tq * fwd_split(p) / (32 * FWD_WAVES) + p.n_seqs) * p.heads; }

template <int DP, bool PAD>
static hipError_t launch_fwd(const AttnParams &p, hipStream_t s)
{
    const float c = p.scale * LOG2E;
    const dim3 grid((unsigned)attn_workgroups(p));
    switch (fwd_split(p)) {
    case 4: hipLaunchKernelGGL((attention_kernel<DP, PAD, 4, 32>), grid, dim3(256), 0, s, p, c); break;
    case 2: hipLaunchKernelGGL((attention_kernel<DP, PAD, 2, 32>), grid, dim3(256), 0, s, p, c); break;
    default: hipLaunchKernelGGL((attention_kernel<DP, PAD, 1, 64>), grid, dim3(256), 0, s, p, c);
    }
    return hipGetLastError();
}

hipError_t launch_attention(const AttnParams &p, hipStream_t s)
{
    if (p.D == 128) return launch_fwd<128, false>(p, s);
    if (p.D > 64) return launch_fwd<128, true>(p, s);
    if (p.D == 64) return launch_fwd<64, false>(p, s);
    return launch_fwd<64, true>(p, s);
}

}  // namespace coda
