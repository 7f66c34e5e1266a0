// attention_bwd.hip -- backward pass of attention.hip.
//
//   P = exp(S - lse),  delta_i = sum_d dO_id O_id,  dS = P (dO V^T - delta)
//   dV = P^T dO,  dQ = scale dS K,  dK = scale dS^T Q
//
// Three kernels, no atomics: the row statistics; dK and dV, a workgroup for 64 keys of a key / value head, over all rows of all heads of the
// group; dQ, a workgroup for 128 rows, over the keys.  S and dO V^T are formed in both (seven products where five would do): the
// alternative, dQ added up in fp32 across workgroups, is either of no fixed order or a partial of every row for every tile of keys.
#include "attn_launch.hpp"
#include "attn_tile.hpp"

namespace coda {

constexpr int BWD_WAVES = 4;
#ifndef DKV_NS
#define DKV_NS 4
#endif

// stats[0][h][t] = lse * log2(e), stats[1][h][t] = delta.  16 (8) lanes a row of a head.
template <int DP>
__global__ __launch_bounds__(256) void attention_delta_kernel(BwdParams p)
{
    constexpr int CH = DP / 8;
    const int64_t id = ((int64_t)blockIdx.x * 256 + threadIdx.x) / CH;
    const int64_t t = id % p.f.Tq;                          // neighbours share a head: their statistics are neighbours too
    const int head = (int)(id / p.f.Tq), ch = threadIdx.x % CH;
    if (head >= p.f.heads) return;
    float sum = 0.0f;
    if (ch * 8 < p.f.D) {
        const int64_t col = (int64_t)head * p.f.D + ch * 8;
        const bf16x8 a = *reinterpret_cast<const bf16x8 *>(p.O + t * p.ldo + col), b = *reinterpret_cast<const bf16x8 *>(p.dO + t * p.lddo + col);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += (float)a[e] * (float)b[e];
    }
#pragma unroll
    for (int off = CH / 2; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
    if (ch == 0) {
        const int64_t at = (int64_t)head * p.f.Tq + t;
        p.stats[at] = p.f.lse[at] * LOG2E;
        p.stats[(int64_t)p.f.heads * p.f.Tq + at] = sum;
    }
}

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

// dK and dV.  The four waves are two blocks of 32 keys times two streams: a stream takes every second of the (head of the group, 32 rows) pairs that
// see the keys, and the two are added up at the end.  S = Q K^T and dP = dO V^T have the lane's key in their columns, so P and dS are
// operands of dV^T += dO^T P and dK^T += Q^T dS as they stand.
template <int DP, bool PAD, int KB, int NS>
__global__ __launch_bounds__(KB * NS * 64, 2) void attention_dkv_kernel(BwdParams p, float c)
{
    constexpr int ROWS = 32, TILE = ROWS * DP * 2, STAGE = 2 * TILE + 256, KEYS = KB * 32;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[2 * NS * STAGE];
    int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    const int kb = wave % KB, stream = wave / KB;
    const int64_t t = blockIdx.x / p.f.kv_heads;
    const int kv = blockIdx.x % p.f.kv_heads;
    const int s = attn_find(p.f.seq_k, p.f.n_seqs, 1, KEYS, t, lane);
    const AttnSpan q = attn_span(p.f.seq_q, s, p.f.Tq), k = attn_span(p.f.seq_k, s, p.f.Tk);
    const int64_t first = (t - (max(p.f.seq_k[s], 0) / KEYS + s)) * KEYS;
    if (first < 0 || first >= k.count) return;
    const int key0 = (int)first, ahead = k.count - q.count, group = p.f.heads / p.f.kv_heads;
    const int key = key0 + kb * 32 + (lane & 31), last = min(key, k.count - 1);
    bf16x8 kf[DP / 16], vf[DP / 16];
    {
        const uint16_t *K = p.f.K + ((int64_t)k.begin + last) * p.f.ldk + (int64_t)kv * p.f.D, *V = p.f.V + ((int64_t)k.begin + last) * p.f.ldv + (int64_t)kv * p.f.D;
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) {
            const int d = 16 * i + 8 * h;
            kf[i] = !PAD || d < p.f.D ? *reinterpret_cast<const bf16x8 *>(K + d) : bf16x8{};
            vf[i] = !PAD || d < p.f.D ? *reinterpret_cast<const bf16x8 *>(V + d) : bf16x8{};
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
    const float *const stats_base = p.stats + (int64_t)kv * group * p.f.Tq + q.begin;
    const auto load = [&](const Place &x, int buf) {
        if (x.tile >= tiles) return;
        unsigned char *at = smem + (buf * NS + stream) * STAGE;
        load_q.base = q_base + x.head * p.f.D;
        load_do.base = do_base + x.head * p.f.D;
        load_q(x.tile * ROWS, q.count, at, lane);
        load_do(x.tile * ROWS, q.count, at + TILE, lane);
        if (kb == 0)
            attn_load4(stats_base + (int64_t)x.head * p.f.Tq + ((int64_t)h * p.f.heads * p.f.Tq + min(x.tile * ROWS + (lane & 31), q.count - 1)),
                       __builtin_amdgcn_readfirstlane(attn_lds(at + 2 * TILE)));
    };
    // some of the tile's rows do not see all of the workgroup's keys, or are none
    const auto ahead_of_keys = [&](int tile) { return p.f.causal && tile * ROWS + ahead < key0 + KEYS - 1; };
    const auto ragged = [&](int tile) { return tile * ROWS + ROWS > q.count; };
    Place lead = place(0), x = place(stream), next = x;   // the first stream's and this one's
    if (rounds) load(x, 0);
    for (int i = 0; i < rounds; ++i) {
        attn_wait();
        attn_barrier();
        step(next);
        if (i + 1 < rounds) load(next, (i + 1) & 1);
        unsigned char *at = smem + ((i & 1) * NS + stream) * STAGE;
        const Place now = x;
        x = next;
        const bool mine = now.tile < tiles && (ahead_of_keys(now.tile) || ragged(now.tile));
        // where any stream has a masked tile all wait while it is cleaned: theirs are tiles lead.tile to (NS - 1) / group + 1 further
        if (ahead_of_keys(lead.tile) || ragged(lead.tile + (NS - 1) / group + 1)) {
            if (mine) {
                for (int j = kb; j < 2; j += KB) attn_clean(at + j * TILE, TILE, lane);
                attn_reads_done();
            }
            attn_barrier();
        }
        step(lead);
        if (DP == 128) asm volatile("" : "+v"(lane));      // the addresses of the LDS reads are formed again each round: 16 registers that the kernel has not
        const int row0 = now.tile * ROWS;
        if (now.tile >= tiles || (p.f.causal && row0 + ROWS - 1 + ahead < key0 + kb * 32)) continue;
        f32x16 sc = {}, dp = {};
#pragma unroll
        for (int u = 0; u < DP / 16; ++u) sc = attn_mfma(attn_rows<DP>(at, 0, u, lane), kf[u], sc);
#pragma unroll
        for (int u = 0; u < DP / 16; ++u) dp = attn_mfma(attn_rows<DP>(at + TILE, 0, u, lane), vf[u], dp);
        const float *stats = reinterpret_cast<const float *>(at + 2 * TILE);
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const f32x4 l2 = *reinterpret_cast<const f32x4 *>(stats + 8 * g + 4 * h), delta = *reinterpret_cast<const f32x4 *>(stats + 32 + 8 * g + 4 * h);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int r = 4 * g + e;
                sc[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[r], c, -l2[e]));
                dp[r] = sc[r] * (dp[r] - delta[e]);
            }
            if (mine) {
                // a row of dO that is not finite was cleaned above; delta - delta hands what it was on
                const int lim = p.f.causal ? key - ahead - row0 : 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int r = 4 * g + e, row = attn_acc_row(r, h);
                    const bool sees = bool((int)(row >= lim) & (int)(row0 + row < q.count));
                    sc[r] = sees ? sc[r] + (delta[e] - delta[e]) : 0.0f;
                    dp[r] = sees ? dp[r] : 0.0f;
                }
            }
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const bf16x8 w = attn_operand(sc, u);
#pragma unroll
            for (int b = 0; b < DP / 32; ++b) dv[b] = attn_mfma(attn_cols<DP>(at + TILE, u, b, lane), w, dv[b]);
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const bf16x8 w = attn_operand(dp, u);
#pragma unroll
            for (int b = 0; b < DP / 32; ++b) dk[b] = attn_mfma(attn_cols<DP>(at, u, b, lane), w, dk[b]);
        }
    }
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

// dQ, as the forward kernel goes: S^T = K Q^T and dP^T = V dO^T with the lane's row in their columns, dQ^T += K^T dS^T
template <int DP, bool PAD>
__global__ __launch_bounds__(256, 2) void attention_dq_kernel(BwdParams p, float c)
{
    constexpr int ROWS = 128, KEYS = 64, TILE = KEYS * DP * 2;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[4 * TILE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    const int64_t tiles = (int64_t)gridDim.x / p.f.heads;
    const int64_t t = tiles - 1 - blockIdx.x / p.f.heads;
    int head = blockIdx.x % p.f.heads;
    if (p.f.heads % 8 == 0) head = head % 8 * (p.f.heads / 8) + head / 8;
    const int s = attn_find(p.f.seq_q, p.f.n_seqs, 1, ROWS, t, lane);
    const AttnSpan q = attn_span(p.f.seq_q, s, p.f.Tq), k = attn_span(p.f.seq_k, s, p.f.Tk);
    const int64_t first = (t - (max(p.f.seq_q[s], 0) / ROWS + s)) * ROWS;
    if (first < 0 || first >= q.count) return;
    const int row0 = (int)first, ahead = k.count - q.count, kv = head / (p.f.heads / p.f.kv_heads);
    const uint16_t *K = p.f.K + (int64_t)k.begin * p.f.ldk + (int64_t)kv * p.f.D, *V = p.f.V + (int64_t)k.begin * p.f.ldv + (int64_t)kv * p.f.D;
    const int row = row0 + wave * 32 + (lane & 31), last = min(row, q.count - 1);
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
    const float *stats = p.stats + (int64_t)head * p.f.Tq + q.begin + last;
    const float l2 = stats[0], delta = stats[(int64_t)p.f.heads * p.f.Tq];
    const auto sees = [&](int r) { return p.f.causal ? min(max(r + ahead + 1, 0), k.count) : k.count; };
    const int mine = sees(last), low = sees(min(row0 + wave * 32, q.count - 1)), high = row0 + wave * 32 < q.count ? sees(min(row0 + wave * 32 + 31, q.count - 1)) : 0;
    const int keys = sees(min(row0 + ROWS - 1, q.count - 1)), whole = sees(row0);
    f32x16 dq[DP / 32];
#pragma unroll
    for (int b = 0; b < DP / 32; ++b) dq[b] = f32x16{};
    if (PAD) attn_zero(smem, sizeof(smem), 256);
    const int n = (keys + KEYS - 1) / KEYS;
    const AttnLoad<DP, PAD, KEYS, BWD_WAVES> load_k(K, p.f.ldk, wave, lane, p.f.D), load_v(V, p.f.ldv, wave, lane, p.f.D);
    const auto load = [&](int j) {
        unsigned char *at = smem + (j & 1) * 2 * TILE;
        load_k(j * KEYS, k.count, at, lane);
        load_v(j * KEYS, k.count, at + TILE, lane);
    };
    if (n > 0) load(0);
    for (int j = 0; j < n; ++j) {
        attn_wait();
        attn_barrier();
        if (j + 1 < n) load(j + 1);
        const int k0 = j * KEYS;
        unsigned char *at = smem + (j & 1) * 2 * TILE;
        if (k0 + KEYS > whole) {
            attn_clean(at + wave * (TILE / BWD_WAVES), TILE / BWD_WAVES, lane);
            attn_reads_done();
            attn_barrier();
        }
        if (k0 >= high) continue;
        const int lim = mine - k0;
        const bool masked = k0 + KEYS > low;
#pragma unroll
        for (int b = 0; b < KEYS / 32; ++b) {
            f32x16 sc = {}, dp = {};
#pragma unroll
            for (int u = 0; u < DP / 16; ++u) {
                sc = attn_mfma(attn_rows<DP>(at, b * 32, u, lane), qf[u], sc);
                dp = attn_mfma(attn_rows<DP>(at + TILE, b * 32, u, lane), of[u], dp);
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) dp[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[r], c, -l2)) * (dp[r] - delta);
            if (masked) {
#pragma unroll
                for (int r = 0; r < 16; ++r) dp[r] = b * 32 + attn_acc_row(r, h) < lim ? dp[r] : 0.0f;
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const bf16x8 w = attn_operand(dp, u);
#pragma unroll
                for (int d = 0; d < DP / 32; ++d) dq[d] = attn_mfma(attn_cols<DP>(at, 2 * b + u, d, lane), w, dq[d]);
            }
        }
    }
    const int64_t at = (int64_t)q.begin + row;
    const bool there = row < q.count;
    const int64_t angle = bwd_angle(p, p.pos_q + at, there);
#pragma unroll
    for (int b = 0; b < DP / 32; ++b) bwd_store<PAD>(dq[b], b, p.f.scale, p, p.cos, angle, p.dQ + at * p.lddq + (int64_t)head * p.f.D, there, h);
}

static int64_t delta_workgroups(const BwdParams &p) { return ((int64_t)p.f.Tq * p.f.heads * (p.f.D > 64 ? 16 : 8) + 255) / 256; }
static int64_t dkv_workgroups(const BwdParams &p) { return ((int64_t)p.f.Tk / 64 + p.f.n_seqs) * p.f.kv_heads; }
static int64_t dq_workgroups(const BwdParams &p) { return ((int64_t)p.f.Tq / 128 + p.f.n_seqs) * p.f.heads; }

int64_t bwd_workgroups(const BwdParams &p)
{
    const int64_t a = delta_workgroups(p), b = dkv_workgroups(p), d = dq_workgroups(p);
    return a > b ? (a > d ? a : d) : b > d ? b : d;
}
size_t bwd_bytes(int64_t Tq, int heads) { return (size_t)Tq * heads * 8; }

template <int DP, bool PAD>
static hipError_t launch_bwd(const BwdParams &p, hipStream_t s)
{
    const float c = p.f.scale * LOG2E;
    hipError_t e = hipSuccess;
    if (p.f.Tq > 0) {
        hipLaunchKernelGGL((attention_delta_kernel<DP>), dim3((unsigned)delta_workgroups(p)), dim3(256), 0, s, p);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (p.f.Tk > 0) {
        hipLaunchKernelGGL((attention_dkv_kernel<DP, PAD, 2, DKV_NS>), dim3((unsigned)dkv_workgroups(p)), dim3(128 * DKV_NS), 0, s, p, c);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (p.f.Tq > 0) {
        hipLaunchKernelGGL((attention_dq_kernel<DP, PAD>), dim3((unsigned)dq_workgroups(p)), dim3(256), 0, s, p, c);
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
