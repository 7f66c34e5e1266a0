// attention.hip -- attention of packed sequences, forward.
//
//   S_ij = scale q_i . k_j,  lse_i = log sum_j exp S_ij,  o_i = sum_j exp(S_ij - lse_i) v_j   over the keys j that row i sees
//
// in one pass over the keys with the running maximum and sum of each row (attn_tile.hpp).
#include "attn_launch.hpp"
#include "attn_tile.hpp"

namespace coda {

constexpr int FWD_ROWS = 128, FWD_KEYS = 64, FWD_WAVES = 4;

template <int DP, bool PAD>
__global__ __launch_bounds__(256, 2) void attention_kernel(AttnParams p, float c)
{
    constexpr int TILE = FWD_KEYS * DP * 2;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[4 * TILE];
    __shared__ int dirty;                                  // a masked tile of V held something that is not finite
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    // The last tiles of rows, which see the most keys, come first.  Workgroups go round the XCDs: the heads of one group are kept on one XCD, whose L2 then
    // serves their keys and values.
    const int64_t tiles = (int64_t)gridDim.x / p.heads;
    const int64_t t = tiles - 1 - blockIdx.x / p.heads;
    int head = blockIdx.x % p.heads;
    if (p.heads % 8 == 0) head = head % 8 * (p.heads / 8) + head / 8;
    const int s = attn_find(p.seq_q, p.n_seqs, 1, FWD_ROWS, t, lane);
    const AttnSpan q = attn_span(p.seq_q, s, p.Tq), k = attn_span(p.seq_k, s, p.Tk);
    const int64_t first = (t - (max(p.seq_q[s], 0) / FWD_ROWS + s)) * FWD_ROWS;
    if (first < 0 || first >= q.count) return;
    const int row0 = (int)first, ahead = k.count - q.count;
    const int kv = head / (p.heads / p.kv_heads);
    const uint16_t *K = p.K + (int64_t)k.begin * p.ldk + (int64_t)kv * p.D, *V = p.V + (int64_t)k.begin * p.ldv + (int64_t)kv * p.D;

    const int row = row0 + wave * 32 + (lane & 31), last = min(row, q.count - 1);
    const uint16_t *Q = p.Q + (q.begin + (int64_t)last) * p.ldq + (int64_t)head * p.D;
    bf16x8 qf[DP / 16];
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) {
        const int d = 16 * i + 8 * h;
        qf[i] = !PAD || d < p.D ? *reinterpret_cast<const bf16x8 *>(Q + d) : bf16x8{};
    }
    // keys that the lane's row sees, and those that the wave's first and last and the workgroup's last do
    const auto sees = [&](int r) { return p.causal ? min(max(r + ahead + 1, 0), k.count) : k.count; };
    const int mine = sees(last), low = sees(min(row0 + wave * 32, q.count - 1)), high = row0 + wave * 32 < q.count ? sees(min(row0 + wave * 32 + 31, q.count - 1)) : 0;
    const int keys = sees(min(row0 + FWD_ROWS - 1, q.count - 1)), whole = sees(row0);
    const AttnLane<DP> in(lane);
    AttnRows<DP> acc;
    acc.clear();
    if (threadIdx.x == 0) dirty = 0;
    if (PAD) attn_zero(smem, sizeof(smem), 256);
    const int n = (keys + FWD_KEYS - 1) / FWD_KEYS;
    AttnLoad<DP, PAD, FWD_KEYS, FWD_WAVES> load_k(K, p.ldk, wave, lane, p.D), load_v(V, p.ldv, wave, lane, p.D);
    // Tile j in parts, that a step issues among its products: all waves' at once after the barrier would hold each other up
    constexpr int PARTS = 2 * load_k.LOADS;
    const auto load = [&](int j, int part) {
        unsigned char *at = smem + (j & 1) * 2 * TILE;
        if (part == 0) {
            load_k.begin(j * FWD_KEYS, k.count, attn_lds(at));
            load_v.begin(j * FWD_KEYS, k.count, attn_lds(at + TILE));
        }
        if (part < PARTS / 2) load_k.next(part);
        else load_v.next(part - PARTS / 2);
    };
    const auto load_all = [&](int j) {
#pragma unroll
        for (int i = 0; i < PARTS; ++i) load(j, i);
    };
    if (n > 0) load_all(0);
    attn_arrived(qf);
    for (int j = 0; j < n; ++j) {
        attn_wait();
        attn_barrier();                                    // tile j is there, and nobody reads tile j - 1 any more
        const int k0 = j * FWD_KEYS;
        unsigned char *at = smem + (j & 1) * 2 * TILE;
        if (k0 + FWD_KEYS > whole) {
            if (attn_clean(at + TILE + wave * (TILE / FWD_WAVES), TILE / FWD_WAVES, lane)) dirty = 1;
            attn_reads_done();
            attn_barrier();
        }
        if (k0 < high) {
            const int lim = mine - k0;
            static_assert(DP / 16 * (FWD_KEYS / 32) == 2 * PARTS, "a place for every load");
            attn_step<DP, FWD_KEYS / 32>(attn_lds(at) + in.rows, attn_lds(at + TILE) + in.cols, qf, acc, c, lane, k0 + FWD_KEYS > low, [&](int key) { return key < lim; },
                                         [&](int i) {
                                             if (i % 2 == 0) load(j + 1, i / 2);           // past the last key there is nothing to load
                                         });
        } else
            load_all(j + 1);
    }
    if (n * FWD_KEYS > whole) {
        __syncthreads();
        if (dirty)
            for (int j = whole / FWD_KEYS; j < n; ++j) {
                load_v(j * FWD_KEYS, k.count, smem);
                attn_wait();
                attn_barrier();
                const int lim = mine - j * FWD_KEYS;
                attn_add_marks<DP, FWD_KEYS / 16>(attn_lds(smem) + in.cols, acc.o, lane, [&](int key) { return key < lim; });
                __syncthreads();
            }
    }
    const f32x2 halves = attn_halves(acc.l);
    const float l = halves[0] + halves[1];
    const bool none = mine == 0;                           // sees nothing: zeros, and a log-sum-exp of -inf
    const float inv = none ? 0.0f : 1.0f / l;
    const bool there = row < q.count;
    if (there && p.lse && h == 0) p.lse[(int64_t)head * p.Tq + q.begin + row] = none ? -__builtin_inff() : acc.m * p.scale + LN2 * __builtin_amdgcn_logf(l);
    uint16_t *out = p.out + ((int64_t)q.begin + row) * p.ldo + (int64_t)head * p.D;
#pragma unroll
    for (int b = 0; b < DP / 32; ++b)
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

int64_t attn_workgroups(const AttnParams &p) { return ((int64_t)p.Tq / FWD_ROWS + p.n_seqs) * p.heads; }

hipError_t launch_attention(const AttnParams &p, hipStream_t s)
{
    const dim3 grid((unsigned)attn_workgroups(p));
    const float c = p.scale * LOG2E;
    if (p.D == 128) hipLaunchKernelGGL((attention_kernel<128, false>), grid, dim3(256), 0, s, p, c);
    else if (p.D > 64) hipLaunchKernelGGL((attention_kernel<128, true>), grid, dim3(256), 0, s, p, c);
    else if (p.D == 64) hipLaunchKernelGGL((attention_kernel<64, false>), grid, dim3(256), 0, s, p, c);
    else hipLaunchKernelGGL((attention_kernel<64, true>), grid, dim3(256), 0, s, p, c);
    return hipGetLastError();
}

}  // namespace coda
