// attention_bwd.hip -- backward pass of attention.hip.
//
//   P = exp(S - lse),  delta_i = sum_d dO_id O_id,  dS = P (dO V^T - delta)
//   dV = P^T dO,  dQ = scale dS K,  dK = scale dS^T Q
//
// Two kernels, no atomics: dQ, a workgroup for 128 rows, over the keys, which also leaves the row statistics; dK and dV, a workgroup for 64 keys of a key / value
// head, over all rows of all heads of the group.  S and dO V^T are formed in both (eight products, with dS in two parts, where five would do): the
// alternative, dQ added up in fp32 across workgroups, is either of no fixed order or a partial of every row for every tile of keys.  dQ is bound by vector instructions and
// products, which take the time of a SIMD in turn (53 and 44 % of it at 64 columns, 38 and 53 % at 128); dK and dV at 64 columns by neither (34 and 33 %) but by waiting for each other, two barriers of eight waves for 32 rows, at 128
// columns by products, LDS and vector instructions in turn (41, 33 and 29 %): 4 x 2048 rows, 32 heads over 8 of 64 columns, 146 + 169 us (870 TFLOP/s over the eight products), 8192 rows in six
// sequences of 128 columns 327 + 395 (990), once the clock has settled; 152 + 192 and 345 + 414 from idle, as all further figures here are.
#include "attn_launch.hpp"
#include "attn_tile.hpp"

#include <type_traits>

namespace coda {

constexpr int BWD_WAVES = 4;

// Columns 32 b .. of 32 rows of dQ, dK or dV out of their accumulators: times `scale`, turned back by the angle of table row `at` where there are tables
template <bool PAD>
__device__ __forceinline__ void bwd_store(const f32x16 &acc, int b, float scale, const BwdParams &p, const float *cos, int64_t at, uint16_t *out, bool there, int h)
{
#pragma unroll
    for (int g = 0; g < 4; g += 2) {
        float v[2][4];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[i][e] = acc[4 * (g + i) + e] * scale;
            const int d = 32 * b + 8 * (g + i) + 4 * h;
            if (cos && there && (!PAD || d < p.f.D)) {
                const f32x2 c = *reinterpret_cast<const f32x2 *>(cos + at + d / 2), s = *reinterpret_cast<const f32x2 *>(p.sin + at + d / 2);
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float x = v[i][2 * e], y = v[i][2 * e + 1];
                    v[i][2 * e] = x * c[e] + y * s[e];
                    v[i][2 * e + 1] = y * c[e] - x * s[e];
                }
            }
        }
        const u32x4 u = attn_store_unit(v[0], v[1]);
        const int d = 32 * b + 8 * (g + h);
        if (there && (!PAD || d < p.f.D)) *reinterpret_cast<u32x4 *>(out + d) = u;
    }
}

// The table row of a token, times D / 2
__device__ __forceinline__ int64_t bwd_angle(const BwdParams &p, const int32_t *pos, bool there)
{
    return p.cos && there ? (int64_t)min(max(*pos, 0), p.rope_rows - 1) * (p.f.D / 2) : 0;
}

// A row of dO (in memory) whose elements that are not finite were cleared for the products: added to the accumulators of dV^T of the lane's key, if it is seen.  Its weight is positive, so that
// an infinity stays one, and the order of additions does not matter to what comes of it.
template <int DP, bool PAD>
__device__ __forceinline__ void bwd_add_infinities(const uint16_t *x, int D, int lane, bool seen, f32x16 (&acc)[DP / 32])
{
    typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
#pragma unroll
    for (int b = 0; b < DP / 32; ++b)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int d = 32 * b + 8 * g + 4 * (lane >> 5);
            const u32x2 v = !PAD || d < D ? *reinterpret_cast<const u32x2 *>(x + d) : u32x2{};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t w = e & 1 ? v[e / 2] & 0xffff0000u : v[e / 2] << 16;
                if (seen && (w & 0x7f800000u) == 0x7f800000u) acc[b][4 * g + e] += __builtin_bit_cast(float, w);
            }
            __builtin_amdgcn_sched_barrier(0);             // one after the other: all at once would not find registers
        }
}

// dK and dV.  The waves are KB blocks of 32 keys times NS streams: a stream takes every NS-th of the (32 rows, head of the group) pairs that see the keys, and the
// streams are added up at the end.  S = Q K^T and dP = dO V^T have the lane's key in their columns, so P and dS are operands of dV^T += dO^T P and
// dK^T += Q^T dS as they stand.  K, and V where D is at most 64, stay in registers; Q and dO are read from LDS twice, by rows and by columns: at D = 128, 40 KB of LDS
// for 2 MFLOP a wave and round, 2560 of the CU's cycles for its 8 waves against 2048 of products.
template <int DP, bool PAD, int KB, int NS>
__global__ __launch_bounds__(KB * NS * 64, KB * NS / 4) void attention_dkv_kernel(BwdParams p, float c)
{
    constexpr bool VLDS = DP == 128;                       // 32 registers that there are not
    constexpr int ROWS = 32, TILE = ROWS * DP * 2, STAGE = 2 * TILE + 256, KEYS = KB * 32;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[2 * NS * STAGE + (VLDS ? KEYS * DP * 2 : 0)];
    __shared__ int found[NS][KB];                          // what the waves of a stream found in its masked tile
    unsigned char *const v_tile = smem + 2 * NS * STAGE;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    const int kb = wave % KB, stream = wave / KB;
    const int64_t t = blockIdx.x / p.f.kv_heads;
    const int kv = blockIdx.x % p.f.kv_heads;
    const int s = attn_find(p.f.seq_k, p.f.n_seqs, KEYS, t, lane);
    const AttnSpan q = attn_span_of_wave(p.f.seq_q, s, p.f.Tq), k = attn_span_of_wave(p.f.seq_k, s, p.f.Tk);
    const int64_t first = (t - (max(p.f.seq_k[s], 0) / KEYS + s)) * KEYS;
    if (first < 0 || first >= k.count) return;
    const int key0 = (int)first, ahead = k.count - q.count, group = p.f.heads / p.f.kv_heads;
    const int key = key0 + kb * 32 + (lane & 31), last = min(key, k.count - 1);
    bf16x8 kf[DP / 16], vf[VLDS ? 1 : DP / 16];
    {
        const uint16_t *K = p.f.K + ((int64_t)k.begin + last) * p.f.ldk + (int64_t)kv * p.f.D, *V = p.f.V + ((int64_t)k.begin + last) * p.f.ldv + (int64_t)kv * p.f.D;
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) {
            const int d = 16 * i + 8 * h;
            kf[i] = !PAD || d < p.f.D ? *reinterpret_cast<const bf16x8 *>(K + d) : bf16x8{};
            if constexpr (!VLDS) vf[i] = !PAD || d < p.f.D ? *reinterpret_cast<const bf16x8 *>(V + d) : bf16x8{};
        }
    }
    f32x16 dk[DP / 32], dv[DP / 32];
#pragma unroll
    for (int b = 0; b < DP / 32; ++b) dk[b] = dv[b] = f32x16{};
    if (PAD) attn_zero(smem, sizeof(smem), KB * NS * 64);
    // A stream's places are (tile of rows, head of the group), tiles from the first that sees key0
    const int t0 = p.f.causal ? max(0, key0 - ahead) / ROWS : 0, tiles = (q.count + ROWS - 1) / ROWS;
    const int rounds = tiles > t0 ? ((tiles - t0) * group + NS - 1) / NS : 0;
    struct Place {
        int tile, head;
    };
    const auto place = [&](int x) { return Place{t0 + x / group, x % group}; };
    const int step_tile = NS / group, step_head = NS % group;
    const auto step = [&](Place &x) {
        x.tile += step_tile;
        x.head += step_head;
        if (x.head >= group) {
            x.head -= group;
            ++x.tile;
        }
    };
    AttnLoad<DP, PAD, ROWS, KB> load_q(p.f.Q + (int64_t)q.begin * p.f.ldq + (int64_t)kv * group * p.f.D, p.f.ldq, kb, lane, p.f.D),
        load_do(p.dO + (int64_t)q.begin * p.lddo + (int64_t)kv * group * p.f.D, p.lddo, kb, lane, p.f.D);
    const uint16_t *const q_base = load_q.base, *const do_base = load_do.base;
    const float *const stats_base = p.stats + ((int64_t)kb * p.f.heads + (int64_t)kv * group) * p.f.Tq + q.begin;
    // In parts, that a round issues among its products: all waves' at once after the barrier would hold each other up
    constexpr int PARTS = ROWS * DP * 2 / 1024 / KB;       // 1 KB loads of Q, and of dO, of a wave
    const auto load = [&](const Place &x, int buf, int part) {
        const uint32_t at = attn_lds(smem) + (buf * NS + stream) * STAGE;
        const int row0 = x.tile * ROWS;                    // past the last row where there is no such place
        if (part == 0) {
            load_q.base = q_base + x.head * p.f.D;
            load_q.begin(row0, q.count, at);
        }
        if (part == PARTS) {
            load_do.base = do_base + x.head * p.f.D;
            load_do.begin(row0, q.count, at + TILE);
        }
        if (part < PARTS) load_q.next(part);
        else if (part < 2 * PARTS) load_do.next(part - PARTS);
        else                                               // one wave has lse, the other delta, or the only one both
#pragma unroll
            for (int i = 0; i < 2 / KB; ++i)
                attn_load4(stats_base + ((int64_t)i * p.f.heads + x.head) * p.f.Tq + row0, lane * 4, __builtin_amdgcn_readfirstlane(at + 2 * TILE + (kb + i) * ROWS * 4),
                           attn_first_lanes(max(0, min(q.count - row0, ROWS))));
    };
    // some of the tile's rows do not see all of the workgroup's keys, or are none
    const auto ahead_of_keys = [&](int tile) { return p.f.causal && tile * ROWS + ahead < key0 + KEYS - 1; };
    const auto ragged = [&](int tile) { return tile * ROWS + ROWS > q.count; };
    if constexpr (VLDS) AttnLoad<DP, PAD, KEYS, KB * NS>(p.f.V + (int64_t)k.begin * p.f.ldv + (int64_t)kv * p.f.D, p.f.ldv, wave, lane, p.f.D)(key0, k.count, v_tile);
    const AttnLane<DP> in(lane);
    const uint32_t v_rows = attn_lds(v_tile) + kb * 32 * DP * 2 + in.rows;
    Place here = place(stream);
    if (rounds)
#pragma unroll
        for (int i = 0; i <= 2 * PARTS; ++i) load(here, 0, i);
    attn_arrived(kf);
    if constexpr (!VLDS) attn_arrived(vf);
    // Half of the streams are half a round behind the others, and there is one of each on every SIMD: the products of S and dP of one run beside the
    // exponentials of the other.  A barrier each half keeps them so.  With KB = 1 nobody shares a tile, and waves that go their own way take a tenth to a fifth less (1024 rows,
    // 32 heads over 8 of 64 columns 26 -> 24 us, of 128 columns 58 -> 48).
    const bool behind = stream >= NS / 2;
    if (KB == 1 ? VLDS : behind) {                         // the first barrier of every wave comes behind its part of V's tile, which all read from then on: here, or in the first round
        if (VLDS) attn_wait();
        attn_barrier();
    }
    for (int i = 0; i < rounds; ++i) {
        attn_wait();
        if (KB > 1) attn_barrier();
        unsigned char *at = smem + ((i & 1) * NS + stream) * STAGE;
        const Place now = here;
        step(here);
        const bool mine = ahead_of_keys(now.tile) || ragged(now.tile);     // a place behind the last is masked altogether
        const int row0 = now.tile * ROWS;
        const uint32_t rows = attn_lds(at) + in.rows, cols = attn_lds(at) + in.cols;      // of Q; dO's tile is behind it
        const float *stats = reinterpret_cast<const float *>(at + 2 * TILE);
        const auto issue = [&](int product) {              // a load behind every product of S and dP, or every second
            if (product % KB == 0) load(here, (i + 1) & 1, product / KB);
            if (product == DP / 8 - 1) load(here, (i + 1) & 1, 2 * PARTS);
        };
        static_assert(2 * PARTS * KB == DP / 8, "a place for every load");
        // S, and dO V^T - delta: those accumulators begin with -delta
        f32x16 sc = {}, dp;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const f32x4 delta = *reinterpret_cast<const f32x4 *>(stats + 32 + 8 * g + 4 * h);
#pragma unroll
            for (int e = 0; e < 4; ++e) dp[4 * g + e] = delta[e];
        }
        constexpr int B = VLDS ? 2 : 4;                    // batches; two operands a product where V is in LDS
        if constexpr (VLDS) {
            bf16x8 v[2][B];
            const auto read_v = [&](int n) {
#pragma unroll
                for (int j = 0; j < B; ++j) v[n & 1][j] = attn_rows<DP>(v_rows, 0, n * B + j);
            };
            read_v(0);
            attn_products<DP / 16, B>([&](int i) { return attn_rows<DP>(rows, 0, i); }, [&](int u, bf16x8 a) {
                sc = attn_mfma(a, kf[u], sc);
                issue(u);
            });
            attn_products<DP / 16, B>(
                [&](int i) {
                    if (i % B == 0 && i) read_v(i / B);
                    return attn_rows<DP>(rows, ROWS, i);
                },
                [&](int u, bf16x8 a) {
                    dp = attn_mfma(a, v[u / B & 1][u % B], dp);
                    issue(DP / 16 + u);
                });
        } else {
            attn_products<DP / 16, B>([&](int i) { return attn_rows<DP>(rows, 0, i); }, [&](int u, bf16x8 a) {
                sc = attn_mfma(a, kf[u], sc);
                issue(u);
            });
            attn_products<DP / 16, B>([&](int i) { return attn_rows<DP>(rows, ROWS, i); }, [&](int u, bf16x8 a) {
                dp = attn_mfma(a, vf[VLDS ? 0 : u], dp);
                issue(DP / 16 + u);
            });
        }
        // S and dP are masked by selection, but for the products with the rows' columns Q and dO have to be finite.  The tiles are only looked at here, where the other wave of a pair may still
        // read them for S or dP; where something was found, each wave clears all of both behind the barrier, ahead of its own reads: whoever comes second finds what it would have written.
        int bad = 0;
        if (mine) {
            const int bytes = max(0, min(q.count - row0, ROWS)) * (DP * 2);
            for (int j = kb; j < 2; j += KB) bad |= (int)attn_check<TILE>(at + j * TILE, bytes, lane) << j;
            if (KB > 1) found[stream][kb] = bad;
        }
        attn_reads_done();
        if (KB > 1) attn_barrier();
        bf16x8 first[VLDS ? 1 : 4];                        // of dO's columns, to arrive behind the exponentials
        const auto read_do = [&](int i) { return attn_cols<DP>(cols + TILE, i / (DP / 32), i % (DP / 32)); };
        f32x4 l2[4];                                       // of the lane's rows, ahead of the columns: the exponentials wait for them
        const auto read_l2 = [&](int g) { l2[g] = *reinterpret_cast<const f32x4 *>(stats + 8 * g + 4 * h); };
        if constexpr (!VLDS) {
#pragma unroll
            for (int g = 0; g < 4; ++g) read_l2(g);
            __builtin_amdgcn_sched_barrier(0);
            attn_read<4>(first, read_do);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            if (VLDS) read_l2(g);                          // no registers to do so there
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int r = 4 * g + e;
                sc[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[r], c, -l2[g][e]));
            }
        }
        if (mine) {
            if (KB > 1) bad = __builtin_amdgcn_readfirstlane(found[stream][0] | found[stream][KB - 1]);
            const int lim = p.f.causal ? key - ahead - row0 : 0;
            if (bad) {
                int own = lane;
                asm volatile("" : "+v"(own));              // no addresses of this are kept in registers all the way
                // What is cleared of dO reaches its columns of dV for the keys that the row sees (of Q it needs nothing: lse and dS are not finite then, in all columns)
                if (bad & 2)
                    for (int row = 0; row < ROWS && row0 + row < q.count; ++row)
                        bwd_add_infinities<DP, PAD>(do_base + (int64_t)now.head * p.f.D + (int64_t)(row0 + row) * p.lddo, p.f.D, own, row >= lim, dv);
                attn_clean(at, 2 * TILE, 0, own);
                attn_reads_done();
                if constexpr (!VLDS) attn_read<4>(first, read_do);
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int row = attn_acc_row(r, h);
                const bool sees = bool((int)(row >= lim) & (int)(row0 + row < q.count));
                sc[r] = sees ? sc[r] : 0.0f;
                dp[r] = sees ? dp[r] : 0.0f;
            }
        }
        bf16x8 w[2], x[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) w[u] = attn_operand(sc, u);
        constexpr int B32 = DP / 32, N = 2 * B32;          // products of dV; dS is formed among them
        const auto add_dv = [&](int i, bf16x8 a) {
            dv[i % B32] = attn_mfma(a, w[i / B32], dv[i % B32]);
#pragma unroll
            for (int r = i * 16 / N; r < (i + 1) * 16 / N; ++r) dp[r] *= sc[r];
        };
        if constexpr (VLDS) attn_products<N, 4>(read_do, add_dv);
        else attn_products<N, 4>(first, read_do, add_dv, [] {});
#pragma unroll
        for (int u = 0; u < 2; ++u) x[u] = attn_operand(dp, u);
        attn_values<DP, 1, 4>(cols, x, dk);
    }
    attn_wait();                                           // the last round's loads for the next, which go where the parts come
    if (KB > 1 && !behind) attn_barrier();
    // The streams' parts are added up in their order: all of dK, then all of dV through LDS, and a stream finishes every NS-th 32 columns
    const int64_t row = (int64_t)k.begin + key;
    const bool there = key < k.count;
    const int64_t angle = bwd_angle(p, p.pos_k + row, there);
    f32x4 *parts = reinterpret_cast<f32x4 *>(smem) + lane;
    constexpr int UNITS = DP / 32 * 4;                     // of four registers, 1 KB each
    static_assert(KB * NS * UNITS * 1024 <= 2 * NS * STAGE, "the parts take the place of the tiles");
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        __syncthreads();
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            const f32x16 &v = which ? dv[u / 4] : dk[u / 4];
            const int g = u % 4 * 4;
            parts[(wave * UNITS + u) * 64] = f32x4{v[g], v[g + 1], v[g + 2], v[g + 3]};
        }
        __syncthreads();
        for (int b = stream; b < DP / 32; b += NS) {
            f32x16 sum = {};
#pragma unroll
            for (int j = 0; j < NS; ++j)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const f32x4 v = parts[((j * KB + kb) * UNITS + b * 4 + g) * 64];
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[4 * g + e] += v[e];
                }
            if (which) bwd_store<PAD>(sum, b, 1.0f, p, nullptr, 0, p.dV + row * p.lddv + (int64_t)kv * p.f.D, there, h);
            else bwd_store<PAD>(sum, b, p.f.scale, p, p.cos, angle, p.dK + row * p.lddk + (int64_t)kv * p.f.D, there, h);
        }
    }
}

// dQ, as the forward kernel goes, SPLIT waves for 32 rows with every SPLIT-th tile of KEYS keys each: S^T = K Q^T and dP^T = V dO^T with the lane's row in their columns, dQ^T += K^T dS^T
template <int DP, bool PAD, int SPLIT, int KEYS>
__global__ __launch_bounds__(256, DP == 64 && SPLIT < 4 ? 3 : 2) void attention_dq_kernel(BwdParams p, float c)
{
    constexpr int NW = BWD_WAVES / SPLIT, ROWS = NW * 32, TILE = KEYS * DP * 2, ROUND = SPLIT * KEYS;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[4 * SPLIT * TILE];
    __shared__ int dirty;                                  // a masked tile of K held something that is not finite
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    const int block = wave % NW, stream = wave / NW;
    const int64_t tiles = (int64_t)gridDim.x / p.f.heads;
    const int64_t t = tiles - 1 - blockIdx.x / p.f.heads;
    int head = blockIdx.x % p.f.heads;
    if (p.f.heads % 8 == 0) head = head % 8 * (p.f.heads / 8) + head / 8;
    const int s = attn_find(p.f.seq_q, p.f.n_seqs, ROWS, t, lane);
    const AttnSpan q = attn_span_of_wave(p.f.seq_q, s, p.f.Tq), k = attn_span_of_wave(p.f.seq_k, s, p.f.Tk);
    const int64_t first = (t - (max(p.f.seq_q[s], 0) / ROWS + s)) * ROWS;
    if (first < 0 || first >= q.count) return;
    const int row0 = (int)first, ahead = k.count - q.count, kv = head / (p.f.heads / p.f.kv_heads);
    const uint16_t *K = p.f.K + (int64_t)k.begin * p.f.ldk + (int64_t)kv * p.f.D, *V = p.f.V + (int64_t)k.begin * p.f.ldv + (int64_t)kv * p.f.D;
    const int row = row0 + block * 32 + (lane & 31), last = min(row, q.count - 1);
    bf16x8 qf[DP / 16], of[DP / 16];
    {
        const uint16_t *Q = p.f.Q + ((int64_t)q.begin + last) * p.f.ldq + (int64_t)head * p.f.D, *dO = p.dO + ((int64_t)q.begin + last) * p.lddo + (int64_t)head * p.f.D;
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) {
            const int d = 16 * i + 8 * h;
            qf[i] = !PAD || d < p.f.D ? *reinterpret_cast<const bf16x8 *>(Q + d) : bf16x8{};
            of[i] = !PAD || d < p.f.D ? *reinterpret_cast<const bf16x8 *>(dO + d) : bf16x8{};
        }
    }
    // The row's statistics, for this kernel and the next: lse * log2(e), and -delta, which the accumulators of dO V^T begin with
    float l2 = p.f.lse[(int64_t)head * p.f.Tq + q.begin + last] * LOG2E, delta = 0.0f;
    {
        const uint16_t *O = p.O + ((int64_t)q.begin + last) * p.ldo + (int64_t)head * p.f.D;
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) {
            const int d = 16 * i + 8 * h;
            const bf16x8 o = !PAD || d < p.f.D ? *reinterpret_cast<const bf16x8 *>(O + d) : bf16x8{};
#pragma unroll
            for (int e = 0; e < 8; ++e) delta -= (float)o[e] * (float)of[i][e];
        }
        const f32x2 both = attn_halves(delta);
        delta = both[0] + both[1];
        if (h == 0 && stream == 0 && row < q.count) {
            float *stats = p.stats + (int64_t)head * p.f.Tq + q.begin + row;
            stats[0] = l2;
            stats[(int64_t)p.f.heads * p.f.Tq] = delta;
        }
    }
    const auto sees = [&](int r) { return p.f.causal ? min(max(r + ahead + 1, 0), k.count) : k.count; };
    const int mine = sees(last), low = sees(min(row0 + block * 32, q.count - 1)), high = row0 + block * 32 < q.count ? sees(min(row0 + block * 32 + 31, q.count - 1)) : 0;
    const int keys = sees(min(row0 + ROWS - 1, q.count - 1)), whole = sees(row0);
    const AttnLane<DP> in(lane);
    f32x16 dq[DP / 32];
#pragma unroll
    for (int b = 0; b < DP / 32; ++b) dq[b] = f32x16{};
    if (threadIdx.x == 0) dirty = 0;
    if (PAD) attn_zero(smem, sizeof(smem), 256);
    const int n = (keys + ROUND - 1) / ROUND;
    AttnLoad<DP, PAD, KEYS, NW> load_k(K, p.f.ldk, block, lane, p.f.D), load_v(V, p.f.ldv, block, lane, p.f.D);
    constexpr int PARTS = 2 * load_k.LOADS, EVERY = DP / 8 / PARTS;
    const auto stage = [&](int j) { return smem + ((j & 1) * SPLIT + stream) * 2 * TILE; };
    const auto load = [&](int j, int part) {               // as in the forward kernel
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
    attn_arrived(of);
    asm volatile("" : "+v"(l2), "+v"(delta));
    // A weight of zero times an infinity of K is NaN, so K is cleaned where rows do not see all of it, but for the product with dS alone: S takes K as it is (a weight of zero may come
    // of an infinity).  Nearly always there is nothing to clean, so the tile is only looked at ahead of S, and cleaned behind S, with barriers, where something was found.
    bool slow = false;
    for (int j = 0; j < n; ++j) {
        attn_wait();
        if (NW > 1) attn_barrier();                        // else a wave's tiles are its own
        const int k0 = j * ROUND + stream * KEYS;
        unsigned char *at = stage(j);
        if ((j + 1) * ROUND > whole) {
            constexpr int PART = TILE / NW;
            if (attn_check<PART>(at + block * PART, min(k.count - k0, KEYS) * (DP * 2) - block * PART, lane)) dirty = 1;
            attn_reads_done();
            if (NW > 1) attn_barrier();
            slow = __builtin_amdgcn_readfirstlane(dirty) != 0;
        }
        const auto clean = [&](int b) {                    // the keys of block b, by all waves that share them
            constexpr int PART = 32 * DP * 2 / NW;
            int own = lane;
            asm volatile("" : "+v"(own));                  // no addresses of this are kept in registers all the way
            if (NW > 1) attn_barrier();
            attn_clean(at + b * 32 * DP * 2 + block * PART, PART, 0, own);
            attn_reads_done();
            if (NW > 1) attn_barrier();
        };
        if (k0 >= high) {
            load_all(j + 1);
            if (slow)
                for (int b = 0; b < KEYS / 32; ++b) clean(b);
            continue;
        }
        const int lim = mine - k0;
        const bool masked = k0 + KEYS > low;
        const uint32_t rows = attn_lds(at) + in.rows;      // of K; V's tile is behind it
        static_assert(DP / 8 == EVERY * PARTS, "a place for every load");
#pragma unroll
        for (int b = 0; b < KEYS / 32; ++b) {
            f32x16 sc = {}, dp;                            // dP - delta: the accumulators begin with -delta
#pragma unroll
            for (int r = 0; r < 16; ++r) dp[r] = delta;
            attn_products<DP / 16, 4>([&](int i) { return attn_rows<DP>(rows, b * 32, i); },
                                      [&](int i, bf16x8 a) {
                                          sc = attn_mfma(a, qf[i], sc);
                                          if (b == 0 && i % EVERY == 0) load(j + 1, i / EVERY);
                                      });
            attn_products<DP / 16, 4>([&](int i) { return attn_rows<DP>(rows, KEYS + b * 32, i); },
                                      [&](int i, bf16x8 a) {
                                          dp = attn_mfma(a, of[i], dp);
                                          if (b == 0 && i % EVERY == 0) load(j + 1, PARTS / 2 + i / EVERY);
                                      });
            if (slow) clean(b);
#pragma unroll
            for (int r = 0; r < 16; ++r) dp[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[r], c, -l2)) * dp[r];
            if (masked) {
#pragma unroll
                for (int r = 0; r < 16; ++r) dp[r] = b * 32 + attn_acc_row(r, h) < lim ? dp[r] : 0.0f;
            }
            // dS in two parts: the key channels that a row's weights go by weigh its errors most, and rounded once they came to as much as one and a half roundings of dQ
            // (0.0025 of its norm, against 0.0017 for the rounding of the output alone).  The second product and its operand take a sixth of this kernel's
            // time (with the loads as they were then 130 and 159 us for 4 sequences of 2048, 32 heads over 8 of 64 columns, 308 and 368 for 8192 rows of 128).
            bf16x8 upper[2], lower[2];
            attn_two_parts(dp, upper, lower);
            const uint32_t cols = attn_lds(at) + in.cols + b * 32 * DP * 2;
            attn_products<DP / 16, 4>([&](int i) { return attn_cols<DP>(cols, i / (DP / 32), i % (DP / 32)); },
                                      [&](int i, bf16x8 a) {
                                          f32x16 &sum = dq[i % (DP / 32)];
                                          sum = attn_mfma(a, upper[i / (DP / 32)], sum);
                                          sum = attn_mfma(a, lower[i / (DP / 32)], sum);
                                      });
        }
    }
    if (SPLIT > 1) {
        attn_wait();                                       // the last round's loads for the next, which go where the parts come
        __syncthreads();
        slow = __builtin_amdgcn_readfirstlane(dirty) != 0;
    }
    if (slow) {                                            // what was cleaned, for the rows that see it: whatever their weight, an infinity or a NaN times dS makes NaN of their sum
        attn_wait();
        __syncthreads();
        for (int j = whole / ROUND * SPLIT; j < n * SPLIT; ++j) {
            AttnLoad<DP, PAD, KEYS, BWD_WAVES>(K, p.f.ldk, wave, lane, p.f.D)(j * KEYS, k.count, smem);
            attn_wait();
            attn_barrier();
            const int lim = mine - j * KEYS;
            attn_add_marks<DP, KEYS / 16>(attn_lds(smem) + in.cols, dq, lane, [&](int key) { return key < lim; },
                                          [](float x, float marks) { return marks == 0.0f ? x : __builtin_nanf(""); });
            __syncthreads();
        }
    }
    const int64_t at = (int64_t)q.begin + row;
    const bool there = row < q.count;
    const int64_t angle = bwd_angle(p, p.pos_q + at, there);
    if constexpr (SPLIT > 1) {                             // the streams' parts are added up in their order
        constexpr int UNITS = DP / 32 * 4;                 // of four registers, 1 KB each
        static_assert(BWD_WAVES * UNITS * 1024 <= 4 * SPLIT * TILE, "the parts take the place of the tiles");
        f32x4 *parts = reinterpret_cast<f32x4 *>(smem) + lane;
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            const int g = u % 4 * 4;
            parts[(wave * UNITS + u) * 64] = f32x4{dq[u / 4][g], dq[u / 4][g + 1], dq[u / 4][g + 2], dq[u / 4][g + 3]};
        }
        __syncthreads();
        for (int b = stream; b < DP / 32; b += SPLIT) {
            f32x16 sum = {};
#pragma unroll
            for (int j = 0; j < SPLIT; ++j)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const f32x4 v = parts[((j * NW + block) * UNITS + b * 4 + g) * 64];
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[4 * g + e] += v[e];
                }
            bwd_store<PAD>(sum, b, p.f.scale, p, p.cos, angle, p.dQ + at * p.lddq + (int64_t)head * p.f.D, there, h);
        }
    } else
#pragma unroll
        for (int b = 0; b < DP / 32; ++b) bwd_store<PAD>(dq[b], b, p.f.scale, p, p.cos, angle, p.dQ + at * p.lddq + (int64_t)head * p.f.D, there, h);
}

// How many waves share 32 rows, as in the forward kernel, and for the same reason.  us with SPLIT 1 / 2 / 4, 32 heads over 8: D = 64, a sequence of 256: 10 / 8 / 7,
// 509: 15 / 11 / 10, 1024: 25 / 19 / 22, 2048: 51 / 46 / 56, 4096: 141 / 141 / 181; D = 128, 256: 15 / 11, 1024: 38 / 30, 2048: 81 / 79, 4 x 512: 33 / 37 (SPLIT 4 gains too
// little to be there).
static int dq_split(const BwdParams &p)
{
    const int64_t room = p.f.D > 64 ? 288 : 576;
    return p.f.D <= 64 && attn_about(p.f.Tq, p.f.n_seqs, 32) * p.f.heads <= room ? 4 : attn_about(p.f.Tq, p.f.n_seqs, 64) * p.f.heads <= 2 * room ? 2 : 1;
}
// Keys of a workgroup of dK's kernel: 32, whose waves each have tiles of their own and no barrier, while there are at most two workgroups a CU, or 64, whose pairs of waves share their
// tiles.  us with 64 / 32, 32 heads over 8: D = 64, a sequence of 509: 23 / 15, 1024: 37 / 24, 2048: 69 / 53, 4096: 179 / 192, 4 x 512: 24 / 28; D = 128, 256: 22 / 18,
// 1024: 58 / 49, 2048: 111 / 109, 4096: 297 / 415, 4 x 512: 38 / 50.
static int dkv_keys(const BwdParams &p) { return attn_about(p.f.Tk, p.f.n_seqs, 32) * p.f.kv_heads <= 512 ? 32 : 64; }
static int64_t dkv_workgroups(const BwdParams &p) { return ((int64_t)p.f.Tk / dkv_keys(p) + p.f.n_seqs) * p.f.kv_heads; }
static int64_t dq_workgroups(const BwdParams &p) { return ((int64_t)p.f.Tq * dq_split(p) / 128 + p.f.n_seqs) * p.f.heads; }

int64_t bwd_workgroups(const BwdParams &p)
{
    const int64_t a = 2 * dkv_workgroups(p), b = dq_workgroups(p);       // of 256
    return a > b ? a : b;
}
size_t bwd_bytes(int64_t Tq, int heads) { return (size_t)Tq * heads * 8; }

template <int DP, bool PAD>
static hipError_t launch_bwd(const BwdParams &p, hipStream_t s)
{
    const float c = p.f.scale * LOG2E;
    hipError_t e = hipSuccess;
    if (p.f.Tq > 0) {
        const dim3 grid((unsigned)dq_workgroups(p));
        const int split = dq_split(p);
        if constexpr (DP == 64)
            if (split == 4) hipLaunchKernelGGL((attention_dq_kernel<DP, PAD, 4, 32>), grid, dim3(256), 0, s, p, c);
        if (split == 2) hipLaunchKernelGGL((attention_dq_kernel<DP, PAD, 2, 32>), grid, dim3(256), 0, s, p, c);
        if (split == 1) hipLaunchKernelGGL((attention_dq_kernel<DP, PAD, 1, 64>), grid, dim3(256), 0, s, p, c);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (p.f.Tk > 0) {
        const dim3 grid((unsigned)dkv_workgroups(p));
        constexpr int NS = DP == 64 ? 8 : 4;               // streams that LDS has room for
        if (dkv_keys(p) == 32) hipLaunchKernelGGL((attention_dkv_kernel<DP, PAD, 1, NS>), grid, dim3(NS * 64), 0, s, p, c);
        else hipLaunchKernelGGL((attention_dkv_kernel<DP, PAD, 2, 4>), grid, dim3(512), 0, s, p, c);
        e = hipGetLastError();
    }
    return e;
}

hipError_t launch_attention_bwd(const BwdParams &p, hipStream_t s)
{
    if (p.f.D == 128) return launch_bwd<128, false>(p, s);
    if (p.f.D > 64) return launch_bwd<128, true>(p, s);
    if (p.f.D == 64) return launch_bwd<64, false>(p, s);
    return launch_bwd<64, true>(p, s);
}

}  // namespace coda
