// attention_cached.hip -- attention of new tokens over a paged cache, and storing into it.
//
// The rows of one key / value head are the tokens of a sequence times the query heads of the group, so that every key is read once for all of
// them.  Bound by HBM for few rows: 4 D bytes a key and key / value head, and 4 D operations a key and row.
//
//  * Rows are cut into tiles of 32 (the workgroup's four waves take a quarter of the keys of a tile each, from LDS of their own, without a
//    barrier, and are joined in LDS at the end) or of 128 (a wave has 32 rows, the keys are shared).
//  * The tiles of keys of all tiles of rows, laid end to end, are cut into equal ranges, a workgroup each: lengths may differ as they like and
//    the host needs to know none of them.  A range that covers a tile of rows whole writes its outputs; otherwise fp32 partials go to slot
//    (range + number of the tile of rows), which no other pair has, since both only grow, and a second kernel joins them in order.
#include "attn_launch.hpp"
#include "attn_tile.hpp"

namespace coda {

constexpr int CACHED_WAVES = 4;

template <int DP, bool SHARED>
struct CachedTile {
    static constexpr int ROWS = SHARED ? 128 : 32;
    static constexpr int WAVE_KEYS = SHARED ? 64 : DP == 128 ? 32 : 64;             // keys of a wave's step
    static constexpr int KEYS = SHARED ? 64 : CACHED_WAVES * WAVE_KEYS;             // of the workgroup's
    static constexpr int TILE = WAVE_KEYS * DP * 2;                                // bytes of K, or of V
    static constexpr int LDS = (SHARED ? 1 : CACHED_WAVES) * 4 * TILE;
    static constexpr int LOAD_WAVES = SHARED ? CACHED_WAVES : 1;
    static constexpr int LOADS = TILE / 1024 / LOAD_WAVES;
};

struct CachedSeq {
    int q0, nq, len, tiles, steps;     // first row, rows, keys, tiles of rows, tiles of keys
};
__device__ __forceinline__ CachedSeq cached_seq(const CachedParams &p, int s, int rows, int keys)
{
    const AttnSpan q = attn_span(p.seq_q, s, p.Tq);
    const int len = min(max(p.lens[s], 0), p.capacity);
    const int tiles = (int)(((int64_t)q.count * p.group + rows - 1) / rows);
    return {q.begin, q.count, len, tiles, max(1, (len + keys - 1) / keys)};
}
__device__ __forceinline__ int64_t cached_item(const CachedParams &p, const CachedSeq &q, int s, int rows) { return (int64_t)q.q0 * p.group / rows + s; }

// Sum over the workgroup's 256 threads of each one's value, and of those before it
__device__ __forceinline__ int64_t cached_scan(int64_t v, int64_t *part, int64_t &before)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t run = v;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int64_t o = __shfl_up(run, off, 64);
        if (lane >= off) run += o;
    }
    __syncthreads();
    if (lane == 63) part[wave] = run;
    __syncthreads();
    int64_t total = 0;
    before = run - v;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if (w < wave) before += part[w];
        total += part[w];
    }
    return total;
}

template <int DP, bool PAD, bool SHARED>
__global__ __launch_bounds__(256, SHARED ? 2 : 1) void attention_cached_kernel(CachedParams p, float c)
{
    typedef CachedTile<DP, SHARED> C;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[C::LDS];
    __shared__ float stats[2][CACHED_WAVES][32];
    __shared__ int64_t part[4], found[2];
    __shared__ int dirty;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    const int kv = blockIdx.x % p.kv_heads, range = blockIdx.x / p.kv_heads;

    // This workgroup's range, and the sequence that it begins in
    int64_t mine = 0, before;
    const int each = (p.n_seqs + 255) / 256, s0 = min((int)threadIdx.x * each, p.n_seqs), s1 = min(s0 + each, p.n_seqs);
    for (int s = s0; s < s1; ++s) {
        const CachedSeq q = cached_seq(p, s, C::ROWS, C::KEYS);
        mine += (int64_t)q.tiles * q.steps;
    }
    const int64_t total = cached_scan(mine, part, before);
    const int64_t ranges = min((int64_t)p.ranges, total);
    if (range >= ranges) return;
    int64_t at = range * total / ranges;
    const int64_t end = (range + 1) * total / ranges;
    if (before <= at && at < before + mine) {
        int s = s0;
        for (;; ++s) {
            const CachedSeq q = cached_seq(p, s, C::ROWS, C::KEYS);
            const int64_t cost = (int64_t)q.tiles * q.steps;
            if (at < before + cost) break;
            before += cost;
        }
        found[0] = s;
        found[1] = before;
    }
    __syncthreads();
    int s = (int)found[0];
    int64_t base = found[1];

    while (at < end) {
        const CachedSeq seq = cached_seq(p, s, C::ROWS, C::KEYS);
        const int64_t cost = (int64_t)seq.tiles * seq.steps;
        if (at >= base + cost) {
            base += cost;
            ++s;
            continue;
        }
        const int tile = (int)((at - base) / seq.steps), j0 = (int)((at - base) % seq.steps), j1 = (int)min((int64_t)seq.steps, j0 + (end - at));
        at += j1 - j0;
        __syncthreads();                                   // the LDS of the range's last piece is free
        if (threadIdx.x == 0) dirty = 0;
        if (PAD) attn_zero(smem, sizeof(smem), 256);

        const int nrows = seq.nq * p.group, row0 = tile * C::ROWS + (SHARED ? wave * 32 : 0);
        const int row = row0 + (lane & 31), last = min(row, nrows - 1);
        const int token = last / p.group, head = kv * p.group + last % p.group;
        const uint16_t *Q = p.Q + (int64_t)(seq.q0 + token) * p.ldq + (int64_t)head * p.D;
        bf16x8 qf[DP / 16];
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) {
            const int d = 16 * i + 8 * h;
            qf[i] = !PAD || d < p.D ? *reinterpret_cast<const bf16x8 *>(Q + d) : bf16x8{};
        }
        // Keys below `lim` are seen, and draft j (key drafts + j) where bit j is set
        const int drafts = seq.len - seq.nq;
        const int lim = p.tree ? max(drafts, 0) : drafts + token + 1;
        uint64_t bits = 0;
        if (p.tree) bits = p.tree[seq.q0 + token] & (seq.nq >= 64 ? ~0ull : (1ull << seq.nq) - 1);
        const int whole = max(0, p.tree ? drafts : drafts + 1);                    // keys that all rows see
        const uint32_t bits0 = (uint32_t)bits, bits1 = (uint32_t)(bits >> 32);
        // without branches: each of 32 scores a lane would have one
        const auto sees = [&](int k) {
            const uint32_t d = (uint32_t)(k - drafts), word = d < 32u ? bits0 : bits1;
            return bool((int)(k < lim) | (int)((word >> (d & 31)) & (uint32_t)(d < 64u)));
        };

        unsigned char *own = smem + (SHARED ? 0 : wave * 4 * C::TILE);
        const int32_t *table = p.table + (int64_t)s * p.ld_table;
        const auto first_key = [&](int j) { return j * C::KEYS + (SHARED ? 0 : wave * C::WAVE_KEYS); };
        constexpr int CH = DP / 8, RPL = 64 / CH;
        const auto tile_row = [&](int i) { return (i * C::LOAD_WAVES + (SHARED ? wave : 0)) * RPL + lane / CH; };
        // The pages of the rows that this lane loads, a step ahead of the loads
        int32_t page[C::LOADS];
        const auto look_up = [&](int j) {
#pragma unroll
            for (int i = 0; i < C::LOADS; ++i) {
                const int key = max(0, min(first_key(j) + tile_row(i), seq.len - 1));
                page[i] = table[key >> p.page_bits];
            }
        };
        const auto load = [&](const uint16_t *cache, int j, unsigned char *to) {
#pragma unroll
            for (int i = 0; i < C::LOADS; ++i) {
                const int r = tile_row(i), ch = (lane % CH) ^ attn_swizzle<DP>(r);
                const int key = max(0, min(first_key(j) + r, seq.len - 1));
                const int64_t pg = min(max(page[i], 0), p.pages - 1);
                const uint16_t *from = cache + ((((pg * p.kv_heads + kv) << p.page_bits) + (key & ((1 << p.page_bits) - 1))) * p.D + ch * 8);
                if (!PAD || ch * 8 < p.D) attn_load16(from, __builtin_amdgcn_readfirstlane(attn_lds(to) + (i * C::LOAD_WAVES + (SHARED ? wave : 0)) * 1024));
            }
        };
        AttnRows<DP> acc;
        acc.clear();
        bool bad = false;
        if (seq.len > 0) {
            look_up(j0);
            load(p.K, j0, own);
            load(p.V, j0, own + C::TILE);
            if (j0 + 1 < j1) look_up(j0 + 1);
            for (int j = j0; j < j1; ++j) {
                unsigned char *now = own + ((j - j0) & 1) * 2 * C::TILE, *next = own + ((j - j0 + 1) & 1) * 2 * C::TILE;
                attn_wait();
                if (SHARED) attn_barrier();
                if (j + 1 < j1) {
                    load(p.K, j + 1, next);
                    load(p.V, j + 1, next + C::TILE);
                    if (j + 2 < j1) look_up(j + 2);
                }
                const int k0 = first_key(j);
                const bool masked = k0 + C::WAVE_KEYS > whole;
                if (masked) {
                    constexpr int PART = C::TILE / C::LOAD_WAVES;
                    if (attn_clean(now + C::TILE + (SHARED ? wave * PART : 0), PART, lane)) {
                        bad = true;
                        if (SHARED) dirty = 1;
                    }
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                    if (SHARED) attn_barrier();
                }
                if (k0 >= seq.len || row0 >= nrows) continue;
                attn_step<DP, C::WAVE_KEYS / 32>(now, now + C::TILE, qf, acc, c, lane, masked, [&](int k) { return sees(k0 + k); });
            }
            attn_wait();
            if (SHARED) {
                __syncthreads();
                bad = dirty != 0;
            }
            if (bad)
                for (int j = max(j0, (whole - (SHARED ? 0 : wave * C::WAVE_KEYS)) / C::KEYS); j < j1; ++j) {
                    const int k0 = first_key(j);
                    if (k0 + C::WAVE_KEYS <= whole) continue;
                    look_up(j);
                    load(p.V, j, own);
                    attn_wait();
                    if (SHARED) attn_barrier();
                    attn_add_marks<DP, C::WAVE_KEYS / 16>(own, acc.o, lane, [&](int k) { return sees(k0 + k); });
                    attn_wait();
                    if (SHARED) attn_barrier();
                }
        }
        const f32x2 halves = attn_halves(acc.l);
        acc.l = halves[0] + halves[1];
        acc.m *= c;                                        // log2 units from here on
        const bool partial = j0 > 0 || j1 < seq.steps;
        float *to = nullptr;
        if (partial) to = p.part + ((range + cached_item(p, seq, s, C::ROWS) + tile) * p.kv_heads + kv) * (C::ROWS * (DP + 2));
        if (!SHARED) {
            // The four waves' outputs [DP][32] side by side in LDS; then a thread joins DP / 8 columns of one row
            float *o = reinterpret_cast<float *>(own);
#pragma unroll
            for (int b = 0; b < DP / 32; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[(b * 32 + attn_acc_row(r, h)) * 32 + (lane & 31)] = acc.o[b][r];
            if (h == 0) {
                stats[0][wave][lane] = acc.m;
                stats[1][wave][lane] = acc.l;
            }
            __syncthreads();
            const int r = threadIdx.x & 31, d0 = (threadIdx.x >> 5) * (DP / 8);
            float m = stats[0][0][r], l = 0.0f, w[CACHED_WAVES], v[DP / 8];
#pragma unroll
            for (int i = 1; i < CACHED_WAVES; ++i) m = fmaxf(m, stats[0][i][r]);
            const float ms = m == -__builtin_inff() ? 0.0f : m;
#pragma unroll
            for (int i = 0; i < CACHED_WAVES; ++i) {
                w[i] = __builtin_amdgcn_exp2f(stats[0][i][r] - ms);
                l += w[i] * stats[1][i][r];
            }
#pragma unroll
            for (int d = 0; d < DP / 8; ++d) {
                v[d] = 0.0f;
#pragma unroll
                for (int i = 0; i < CACHED_WAVES; ++i) v[d] += w[i] * reinterpret_cast<const float *>(smem + i * 4 * C::TILE)[(d0 + d) * 32 + r];
            }
            const bool there = tile * C::ROWS + r < nrows;
            const bool none = m == -__builtin_inff() && l == 0.0f;
            const float inv = none ? 0.0f : 1.0f / l;
            if (there && partial) {
                if (d0 == 0) {
                    to[r] = m;
                    to[C::ROWS + r] = l;
                }
                float *po = to + 2 * C::ROWS + r * DP + d0;
#pragma unroll
                for (int d = 0; d < DP / 8; d += 4) *reinterpret_cast<f32x4 *>(po + d) = f32x4{v[d], v[d + 1], v[d + 2], v[d + 3]};
            } else if (there) {                            // r is this lane's row as above: token and head are its
                if (d0 == 0 && p.lse) p.lse[(int64_t)head * p.Tq + seq.q0 + token] = none ? -__builtin_inff() : LN2 * (m + __builtin_amdgcn_logf(l));
                uint16_t *out = p.out + (int64_t)(seq.q0 + token) * p.ldo + (int64_t)head * p.D;
#pragma unroll
                for (int d = 0; d < DP / 8; d += 8) {
                    u32x4 u;
#pragma unroll
                    for (int e = 0; e < 4; ++e) u[e] = attn_pack(v[d + 2 * e] * inv, v[d + 2 * e + 1] * inv);
                    if (!PAD || d0 + d < p.D) *reinterpret_cast<u32x4 *>(out + d0 + d) = u;
                }
            }
        } else {
            const bool there = row < nrows;
            const bool none = acc.m == -__builtin_inff() && acc.l == 0.0f;
            const float inv = partial ? 1.0f : none ? 0.0f : 1.0f / acc.l;
            if (there && h == 0) {
                if (partial) {
                    to[wave * 32 + lane] = acc.m;
                    to[C::ROWS + wave * 32 + lane] = acc.l;
                } else if (p.lse)
                    p.lse[(int64_t)head * p.Tq + seq.q0 + token] = none ? -__builtin_inff() : LN2 * (acc.m + __builtin_amdgcn_logf(acc.l));
            }
            uint16_t *out = p.out + (int64_t)(seq.q0 + token) * p.ldo + (int64_t)head * p.D;
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
                    if (partial) {
                        float *po = to + 2 * C::ROWS + (wave * 32 + (lane & 31)) * DP + 32 * b + 8 * g + 4 * h;
                        if (there) {
                            *reinterpret_cast<f32x4 *>(po) = f32x4{lo[0], lo[1], lo[2], lo[3]};
                            *reinterpret_cast<f32x4 *>(po + 8) = f32x4{hi[0], hi[1], hi[2], hi[3]};
                        }
                    } else {
                        const u32x4 u = attn_store_unit(lo, hi);
                        const int d = 32 * b + 8 * (g + h);
                        if (there && (!PAD || d < p.D)) *reinterpret_cast<u32x4 *>(out + d) = u;
                    }
                }
        }
    }
}

// Joins the partials of the tiles of rows that more than one range had a part of.  A wave has a row, a lane DP / 64 columns.
template <int DP, bool SHARED>
__global__ __launch_bounds__(256) void attention_join_kernel(CachedParams p)
{
    typedef CachedTile<DP, SHARED> C;
    __shared__ int64_t part[4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t item = blockIdx.x / p.kv_heads;
    const int kv = blockIdx.x % p.kv_heads;
    const int s = attn_find(p.seq_q, p.n_seqs, p.group, C::ROWS, item, lane);
    const CachedSeq seq = cached_seq(p, s, C::ROWS, C::KEYS);
    const int64_t tile = item - cached_item(p, seq, s, C::ROWS);
    if (tile < 0 || tile >= seq.tiles) return;
    const int r = (int)blockIdx.y * 4 + wave, row = (int)tile * C::ROWS + r;
    if ((int)tile * C::ROWS + (int)blockIdx.y * 4 >= seq.nq * p.group) return;
    int64_t mine = 0, ahead = 0, unused;
    for (int i = threadIdx.x; i < p.n_seqs; i += 256) {
        const CachedSeq q = cached_seq(p, i, C::ROWS, C::KEYS);
        const int64_t cost = (int64_t)q.tiles * q.steps;
        mine += cost;
        if (i < s) ahead += cost;
    }
    const int64_t total = cached_scan(mine, part, unused), ranges = min((int64_t)p.ranges, total);
    const int64_t first = cached_scan(ahead, part, unused) + tile * seq.steps;
    // the range that holds step x is the last that begins at or before it, at floor(range * total / ranges)
    const int64_t w0 = ((first + 1) * ranges - 1) / total, w1 = ((first + seq.steps) * ranges - 1) / total;
    if (w0 == w1 || row >= seq.nq * p.group) return;
    const int64_t stride = (int64_t)p.kv_heads * (C::ROWS * (DP + 2));
    const float *from = p.part + ((w0 + item) * p.kv_heads + kv) * (C::ROWS * (DP + 2));
    const int n = (int)(w1 - w0 + 1);
    float m = -__builtin_inff();
    for (int i = lane; i < n; i += 64) m = fmaxf(m, from[i * stride + r]);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
    const float ms = m == -__builtin_inff() ? 0.0f : m;
    float l = 0.0f, v[DP / 64] = {};
#pragma unroll 4
    for (int i = 0; i < n; ++i) {
        const float w = __builtin_amdgcn_exp2f(from[i * stride + r] - ms);
        l += w * from[i * stride + C::ROWS + r];
#pragma unroll
        for (int d = 0; d < DP / 64; ++d) v[d] += w * from[i * stride + 2 * C::ROWS + r * DP + lane * (DP / 64) + d];
    }
    const bool none = m == -__builtin_inff() && l == 0.0f;
    const float inv = none ? 0.0f : 1.0f / l;
    const int token = seq.q0 + row / p.group, head = kv * p.group + row % p.group, col = lane * (DP / 64);
    if (lane == 0 && p.lse) p.lse[(int64_t)head * p.Tq + token] = none ? -__builtin_inff() : LN2 * (m + __builtin_amdgcn_logf(l));
    if (col >= p.D) return;
    uint16_t *out = p.out + (int64_t)token * p.ldo + (int64_t)head * p.D + col;
    const uint32_t u = attn_pack(v[0] * inv, v[DP / 64 - 1] * inv);
    if (DP == 128) *reinterpret_cast<uint32_t *>(out) = u;
    else *out = (uint16_t)u;
}

// 16 bytes of K and of V a thread
__global__ __launch_bounds__(256) void cache_store_kernel(const uint16_t *K, int64_t ldk, const uint16_t *V, int64_t ldv, int64_t T, int chunks, int D,
                                                          const int32_t *slots, uint16_t *k, uint16_t *v, int64_t slots_there, int page_bits, int kv_heads)
{
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t t = id / chunks;
    const int col = (int)(id % chunks) * 8;
    if (t >= T) return;
    const int64_t slot = slots[t];
    if (slot < 0 || slot >= slots_there) return;
    const int64_t page = slot >> page_bits, place = slot & ((1 << page_bits) - 1);
    const int64_t to = (((page * kv_heads + col / D) << page_bits) + place) * D + col % D;
    *reinterpret_cast<u32x4 *>(k + to) = *reinterpret_cast<const u32x4 *>(K + t * ldk + col);
    *reinterpret_cast<u32x4 *>(v + to) = *reinterpret_cast<const u32x4 *>(V + t * ldv + col);
}

// Tiles of 128 rows once a sequence has more than 32 on average
static bool cached_shared(int64_t Tq, int n_seqs, int group) { return Tq * group > 32 * (int64_t)n_seqs; }
static int cached_ranges(int kv_heads, bool shared) { return ((shared ? 512 : 256) + kv_heads - 1) / kv_heads; }

int64_t cached_items(int64_t Tq, int n_seqs, int group, bool shared) { return Tq * group / (shared ? 128 : 32) + n_seqs; }

size_t cached_bytes(int64_t Tq, int n_seqs, int heads, int kv_heads, int D)
{
    const int group = heads / kv_heads, DP = D > 64 ? 128 : 64;
    const bool shared = cached_shared(Tq, n_seqs, group);
    return (size_t)(cached_items(Tq, n_seqs, group, shared) + cached_ranges(kv_heads, shared)) * kv_heads * ((shared ? 128 : 32) * (DP + 2) * 4);
}

int64_t cached_workgroups(const CachedParams &p)
{
    const bool shared = cached_shared(p.Tq, p.n_seqs, p.group);
    const int64_t join = cached_items(p.Tq, p.n_seqs, p.group, shared) * p.kv_heads * (shared ? 32 : 8);
    const int64_t main = (int64_t)cached_ranges(p.kv_heads, shared) * p.kv_heads;
    return join > main ? join : main;
}

template <int DP, bool PAD>
static hipError_t launch_cached(CachedParams p, hipStream_t s)
{
    const bool shared = cached_shared(p.Tq, p.n_seqs, p.group);
    p.ranges = cached_ranges(p.kv_heads, shared);
    const float c = p.scale * LOG2E;
    const dim3 grid((unsigned)(p.ranges * p.kv_heads)), join((unsigned)(cached_items(p.Tq, p.n_seqs, p.group, shared) * p.kv_heads), shared ? 32 : 8);
    if (shared) {
        hipLaunchKernelGGL((attention_cached_kernel<DP, PAD, true>), grid, dim3(256), 0, s, p, c);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL((attention_join_kernel<DP, true>), join, dim3(256), 0, s, p);
    } else {
        hipLaunchKernelGGL((attention_cached_kernel<DP, PAD, false>), grid, dim3(256), 0, s, p, c);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL((attention_join_kernel<DP, false>), join, dim3(256), 0, s, p);
    }
    return hipGetLastError();
}

hipError_t launch_attention_cached(const CachedParams &p, hipStream_t s)
{
    if (p.D == 128) return launch_cached<128, false>(p, s);
    if (p.D > 64) return launch_cached<128, true>(p, s);
    if (p.D == 64) return launch_cached<64, false>(p, s);
    return launch_cached<64, true>(p, s);
}

int64_t cache_store_workgroups(int64_t T, int cols) { return (T * (cols / 8) + 255) / 256; }

hipError_t launch_cache_store(const uint16_t *K, int64_t ldk, const uint16_t *V, int64_t ldv, int64_t T, int cols, int D, const int32_t *slots, uint16_t *k,
                              uint16_t *v, int64_t slots_there, int page_bits, hipStream_t s)
{
    hipLaunchKernelGGL(cache_store_kernel, dim3((unsigned)cache_store_workgroups(T, cols)), dim3(256), 0, s, K, ldk, V, ldv, T, cols / 8, D, slots, k, v,
                       slots_there, page_bits, cols / D);
    return hipGetLastError();
}

}  // namespace coda
