// attention_cached.hip -- attention of new tokens over a paged cache, and storing into it.
//
// The rows of one key / value head are the tokens of a sequence times the query heads of the group, so that every key is read once for all of
// them.  Bound by HBM for few rows: 4 D bytes a key and key / value head, and 4 D operations a key and row.  32 heads over 8 of 128 columns: 64 sequences of 200000 keys in all 140 us (5.8 TB/s); a
// lone one of 4097 keys 9.3, of which 6 are launch, code and three trips to memory.
//
//  * Rows are cut into tiles of 32 or 128.  With 32 (a few tokens) the workgroup's four waves take a quarter of the keys of a tile each, from LDS of their
//    own without a barrier: four slots of K or V a wave, three of them on their way (24 KB a wave, 96 KB a CU) while one is read.  With 128 (trees) four
//    waves have 32 rows each and share the keys, and the workgroup's two such groups take the halves of a tile of 128 keys, a barrier a step.  Two a step, with V's
//    loads behind K's products and more of them on their way, take 36.4 us where 33.1 are for eight sequences of 31000 keys in all and 32 drafts each (47.5 and 48.0 with the join where nothing of
//    them is cached), and 29.0 where 27.6 are for one of 16411 keys and 61 drafts.  At the end the waves of a row are joined in LDS.
//  * The tiles of keys of all tiles of rows, laid end to end, are cut into equal ranges, a workgroup each: lengths may differ as they like and
//    the host needs to know none of them; a tile of rows counts for two or three steps more than it has, which is what a range loses between two (64 sequences' last workgroups
//    ended 12 us behind the first without).  A range that covers a tile of rows whole writes its outputs; otherwise fp32 partials go to slot
//    (range + number of the tile of rows), which no other pair has, since both only grow, and a second kernel joins them in order.
#include "attn_launch.hpp"
#include "attn_tile.hpp"

namespace coda {

template <int DP, bool MANY>
struct CachedTile {
    static constexpr int GROUP = MANY ? 4 : 1;             // waves that share their keys
    static constexpr int GROUPS = MANY ? 2 : 4;            // of the workgroup
    static constexpr int WAVES = GROUP * GROUPS;
    static constexpr int ROWS = GROUP * 32;
    static constexpr int WAVE_KEYS = MANY || DP == 64 ? 64 : 32;
    static constexpr int KEYS = GROUPS * WAVE_KEYS;        // of a step of the workgroup
    static constexpr int TILE = WAVE_KEYS * DP * 2;        // bytes of K, or of V, of a group
    static constexpr int LDS = GROUPS * 4 * TILE;
    static constexpr int LOADS = TILE / 1024 / GROUP;      // 1 KB each, of a wave
    static constexpr int RESTART = MANY ? 3 : 2;           // steps that a range's next tile of rows costs on top of its own
    static constexpr int UNITS = DP / 8;                   // fours of columns that a lane holds; each wave finishes UNITS / GROUPS of them
    static constexpr int PART = (MANY ? UNITS * 1024 : 4 * TILE) / 16;              // from one wave's part to the next, in fours: a lone wave's takes the place of its tiles
    static_assert(WAVES * PART * 16 <= LDS && UNITS * 64 <= PART, "the parts of all waves take the place of the tiles");
};
constexpr int CACHED_SEQS = 256;                           // sequences kept in LDS

// Numbers of tiles of rows, as attn_find() counts them
__host__ __device__ __forceinline__ int64_t cached_items(int64_t Tq, int n_seqs, int group, bool many) { return Tq * group / (many ? 128 : 32) + n_seqs; }
struct CachedSeq {
    int q0, nq, len, tiles, steps;     // first row, rows, keys, tiles of rows, tiles of keys
};
__device__ __forceinline__ CachedSeq cached_seq_of(const CachedParams &p, int q0, int nq, int len, int rows, int keys)
{
    return {q0, nq, len, (int)(((int64_t)nq * p.group + rows - 1) / rows), max(1, (len + keys - 1) / keys)};
}
__device__ __forceinline__ CachedSeq cached_seq(const CachedParams &p, int s, int rows, int keys)
{
    const AttnSpan q = attn_span(p.seq_q, s, p.Tq);
    return cached_seq_of(p, q.begin, q.count, min(max(p.lens[s], 0), p.capacity), rows, keys);
}
__device__ __forceinline__ int64_t cached_item(const CachedParams &p, const CachedSeq &q, int s, int rows) { return (int64_t)q.q0 * p.group / rows + s; }

// Whether row `token` of a sequence of nq rows from q0 on sees no key at all: asked for rows whose sum of weights is zero, which may also see keys, all with a score of -inf
__device__ __forceinline__ bool cached_sees_nothing(const CachedParams &p, int q0, int nq, int len, int token)
{
    const int drafts = len - nq;
    if (!p.tree) return drafts + token + 1 <= 0;
    if (drafts > 0) return false;
    const uint64_t bits = p.tree[q0 + token] & (nq >= 64 ? ~0ull : (1ull << nq) - 1);
    return drafts <= -64 || (bits >> -drafts) == 0;
}

__device__ __forceinline__ int64_t cached_uniform(int64_t x)
{
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)x));
}
__device__ __forceinline__ int64_t cached_of_lane(int64_t x, int lane)
{
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)x, lane));
}
// Sum over the workgroup's threads of each one's value, and of those before it
template <int WAVES>
__device__ __forceinline__ int64_t cached_scan(int64_t v, int64_t *part, int64_t &before)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t run = v;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int64_t o = __shfl_up(run, off, 64);
        if (lane >= off) run += o;
    }
    if (lane == 63) part[wave] = run;
    __syncthreads();
    int64_t total = 0;
    before = run - v;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        if (w < wave) before += part[w];
        total += part[w];
    }
    return total;
}

template <int DP, bool PAD, bool MANY>
__global__ __launch_bounds__((CachedTile<DP, MANY>::WAVES * 64), MANY ? 2 : 1) void attention_cached_kernel(CachedParams p, float c)
{
    typedef CachedTile<DP, MANY> C;
    constexpr int THREADS = C::WAVES * 64, CH = DP / 8, RPL = 64 / CH, NB = C::WAVE_KEYS / 32;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[C::LDS];
    __shared__ int32_t ids[C::WAVES][4][64];               // pages of the keys of four steps
    __shared__ uint64_t rows_at[C::WAVES][64];
    __shared__ float stats[2][C::GROUPS][C::ROWS];
    __shared__ int32_t seqs[CACHED_SEQS][3];
    __shared__ int64_t part[C::WAVES], found[2];
    __shared__ int dirty;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    const int member = wave % C::GROUP, kg = wave / C::GROUP;
    const int kv = blockIdx.x % p.kv_heads, range = blockIdx.x / p.kv_heads;

    const AttnLane<DP> in(lane);

    // This workgroup's range, and the sequence that it begins in
    const auto cost_of = [](const CachedSeq &q) { return (int64_t)q.tiles * (q.steps + C::RESTART); };
    const int each = (p.n_seqs + THREADS - 1) / THREADS, s0 = min((int)threadIdx.x * each, p.n_seqs), s1 = min(s0 + each, p.n_seqs);
    // Up to 64 sequences a wave looks at by itself (all leave the same in LDS): without barriers, which with the exchange through LDS take 0.5 us of a lone token's 10
    const bool alone = p.n_seqs <= 64;
    const int t0 = alone ? min(lane, p.n_seqs) : s0, t1 = alone ? min(lane + 1, p.n_seqs) : s1;
    int64_t mine = 0, before, total;
    for (int s = t0; s < t1; ++s) {
        const CachedSeq q = cached_seq(p, s, C::ROWS, C::KEYS);
        mine += cost_of(q);
        if (s < CACHED_SEQS) {
            seqs[s][0] = q.q0;
            seqs[s][1] = q.nq;
            seqs[s][2] = q.len;
        }
    }
    if (alone) {
        int64_t run = mine;
        for (int off = 1; off < p.n_seqs; off <<= 1) {
            const int64_t o = __shfl_up(run, off, 64);
            if (lane >= off) run += o;
        }
        before = run - mine;
        total = cached_of_lane(run, p.n_seqs - 1);
    } else
        total = cached_uniform(cached_scan<C::WAVES>(mine, part, before));
    const int64_t ranges = min((int64_t)p.ranges, total);
    if (blockIdx.x == 0) {                                 // numbers that no tile of rows has
        const int64_t items = cached_items(p.Tq, p.n_seqs, p.group, MANY);
        for (int s = s0; s < s1; ++s) {
            const CachedSeq q = cached_seq(p, s, C::ROWS, C::KEYS);
            const int64_t next = s + 1 < p.n_seqs ? min(items, cached_item(p, cached_seq(p, s + 1, C::ROWS, C::KEYS), s + 1, C::ROWS)) : items;
            for (int64_t i = cached_item(p, q, s, C::ROWS) + q.tiles; i < next; ++i) p.spans[i].parts = 0;
            if (s == 0)
                for (int64_t i = 0; i < cached_item(p, q, 0, C::ROWS); ++i) p.spans[i].parts = 0;
        }
    }
    if (range >= ranges) return;
    int64_t at = range * total / ranges;
    const int64_t end = (range + 1) * total / ranges;
    const auto sequence = [&](int s) {
        if (s >= CACHED_SEQS) return cached_seq(p, s, C::ROWS, C::KEYS);
        return cached_seq_of(p, __builtin_amdgcn_readfirstlane(seqs[s][0]), __builtin_amdgcn_readfirstlane(seqs[s][1]), __builtin_amdgcn_readfirstlane(seqs[s][2]),
                             C::ROWS, C::KEYS);
    };
    int s;
    int64_t base;
    const bool here = before <= at && at < before + mine;
    if (alone) {
        s = __builtin_ctzll(__ballot(here));
        base = cached_of_lane(before, s);
    } else {
        if (here) {
            s = s0;
            for (;; ++s) {
                const int64_t cost = cost_of(cached_seq(p, s, C::ROWS, C::KEYS));
                if (at < before + cost) break;
                before += cost;
            }
            found[0] = s;
            found[1] = before;
        }
        __syncthreads();
        s = __builtin_amdgcn_readfirstlane((int)found[0]);
        base = cached_uniform(found[1]);
    }

    while (at < end) {
        const CachedSeq seq = sequence(s);
        if (at >= base + cost_of(seq)) {
            base += cost_of(seq);
            ++s;
            continue;
        }
        const int length = seq.steps + C::RESTART;         // of a tile of rows: its restart, then its steps
        const int tile = __builtin_amdgcn_readfirstlane((int)((at - base) / length)), from = __builtin_amdgcn_readfirstlane((int)(at - base - (int64_t)tile * length));
        const int to_step = __builtin_amdgcn_readfirstlane((int)min((int64_t)length, from + (end - at)));
        const int j0 = max(0, from - C::RESTART), j1 = to_step - C::RESTART;
        at += to_step - from;
        if (j1 <= 0) continue;                             // the range ends ahead of the first step
        const int64_t item = cached_item(p, seq, s, C::ROWS) + tile;
        if (j0 == 0 && kv == 0 && threadIdx.x == 0) {      // the last step's range is the last that begins at or before it, at floor(range * total / ranges)
            const int last = j1 == seq.steps ? range : (int)(((base + (int64_t)(tile + 1) * length) * ranges - 1) / total);
            p.spans[item] = {range, last - range + 1, seq.q0, tile * C::ROWS, seq.nq * p.group, seq.len};
        }
        __syncthreads();                                   // the LDS of the range's last piece is free
        if (threadIdx.x == 0) dirty = 0;
        if (PAD) attn_zero(smem, sizeof(smem), THREADS);

        const int nrows = seq.nq * p.group, row0 = tile * C::ROWS + member * 32;
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

        const int64_t head_at = (((int64_t)kv << p.page_bits) * p.D) * 2;
        const unsigned char *K = reinterpret_cast<const unsigned char *>(p.K) + head_at, *V = reinterpret_cast<const unsigned char *>(p.V) + head_at;
        unsigned char *own = smem + kg * 4 * C::TILE;      // the group's four slots
        const int32_t *table = p.table + (int64_t)s * p.ld_table;
        const auto first_key = [&](int j) { return j * C::KEYS + kg * C::WAVE_KEYS; };
        const auto clamped = [&](int k) { return max(0, min(k, seq.len - 1)); };
        const auto tile_row = [&](int i) { return (i * C::GROUP + member) * RPL + lane / CH; };
        const auto lane_chunk = [&](int i) { return (lane % CH) ^ attn_swizzle<DP>(tile_row(i)); };
        // Where the rows of a step's keys begin in the cache: a lane finds that of one key and leaves it in LDS for the lanes that load
        const auto find_rows = [&](int j) {
            const uint64_t pg = (uint64_t)(uint32_t)min(max(ids[wave][j & 3][lane], 0), p.pages - 1);
            rows_at[wave][lane] = pg * p.page_bytes + ((uint32_t)clamped(first_key(j) + lane) & p.page_mask) * (uint32_t)(p.D * 2);
            __builtin_amdgcn_wave_barrier();               // a wave's LDS operations stay in order
        };
        const auto load = [&](const unsigned char *cache, unsigned char *to) {
#pragma unroll
            for (int i = 0; i < C::LOADS; ++i)
                if (!PAD || lane_chunk(i) * 8 < p.D)
                    attn_load16(cache + lane_chunk(i) * 16 + rows_at[wave][tile_row(i)], __builtin_amdgcn_readfirstlane(attn_lds(to) + (i * C::GROUP + member) * 1024));
        };
        // V's tiles that are cleaned: masked ones, and where groups wait for each other also what lies beside one
        const auto cleaned = [&](int j) { return (MANY ? j * C::KEYS + C::KEYS : first_key(j) + C::WAVE_KEYS) > whole; };
        AttnRows<DP> acc;
        acc.clear();
        bool bad = false;
        if (seq.len > 0) {
            // Four slots: step j has K in slot 2 j % 4 and V in the next.  The pages of a step's keys come to LDS steps ahead.  Loads arrive in order, so a
            // wait says how many of the later ones may be on their way.
            constexpr int L = C::LOADS;
            const auto slot = [&](int j, int v) { return own + ((2 * (j - j0) + v) & 3) * C::TILE; };
            const auto fetch_ids = [&](int j) {
                attn_load4(table + (clamped(first_key(j) + lane) >> p.page_bits), __builtin_amdgcn_readfirstlane(attn_lds(reinterpret_cast<unsigned char *>(ids[wave][j & 3]))));
            };
            const auto fetch = [&](const unsigned char *cache, int j, int v) { load(cache, slot(j, v)); };
            fetch_ids(j0);
            fetch_ids(j0 + 1);
            attn_wait();
            attn_arrived(qf);
            asm volatile("" : : "v"(bits0), "v"(bits1));
            find_rows(j0);
            fetch(K, j0, 0);
            if (!MANY) fetch_ids(j0 + 2);
            fetch(V, j0, 1);
            if (MANY) fetch_ids(j0 + 2);
            if (!MANY && j0 + 1 < j1) {
                find_rows(j0 + 1);
                fetch(K, j0 + 1, 0);
                fetch_ids(j0 + 3);
                fetch(V, j0 + 1, 1);
            }
            for (int j = j0; j < j1; ++j) {
                const int k0 = first_key(j);
                const bool here = k0 < seq.len && row0 < nrows;                    // the last step's keys may leave nothing for this wave
                const bool masked = k0 + C::WAVE_KEYS > whole;
                const auto see = [&](int k) { return sees(k0 + k); };
                if constexpr (MANY) {
                    attn_wait_but<1>();                    // K and V of j and the pages of j + 1 are there; pages are to come
                    attn_reads_done();
                    attn_barrier();                        // for all waves, and K and V of j - 1 are read
                    if (cleaned(j)) {
                        constexpr int PART = C::TILE / C::GROUP;
                        if (attn_clean(slot(j, 1) + member * PART, PART, PART, lane)) dirty = 1;
                        attn_reads_done();
                        attn_barrier();
                    }
                    const bool more = j + 1 < j1;
                    if (more) {
                        find_rows(j + 1);
                        fetch(K, j + 1, 0);
                        fetch(V, j + 1, 1);
                    }
                    if (here)
                        attn_step<DP, NB>(attn_lds(slot(j, 0)) + in.rows, attn_lds(slot(j, 1)) + in.cols, qf, acc, c, lane, masked, see, [](int) {});
                    if (more) fetch_ids(j + 3);
                } else {
                    f32x16 sc[NB];
                    bf16x8 w[2 * NB];
                    if (j + 1 < j1) attn_wait_but<3 * L + 1>();                    // K and the pages of step j + 2 are there; V, K, pages, V are to come
                    else attn_wait_but<L>();
                    attn_scores<DP, NB, 4>(attn_lds(slot(j, 0)) + in.rows, qf, sc, [](int) {});
                    attn_reads_done();
                    if (j + 2 < j1) {
                        find_rows(j + 2);
                        fetch(K, j + 2, 0);
                        fetch_ids(j + 4);
                    }
                    if (here) attn_weights<DP, NB>(sc, w, acc, c, lane, masked, see);
                    if (j + 2 < j1) attn_wait_but<3 * L + 2>();                    // V is there; K, pages, V, K, pages are to come
                    else if (j + 1 < j1) attn_wait_but<2 * L + 1>();
                    else attn_wait_but<0>();
                    if (here) {
                        if (cleaned(j)) {
                            if (attn_clean(slot(j, 1), C::TILE, C::TILE, lane)) bad = true;
                            attn_reads_done();
                        }
                        attn_values<DP, NB, 4>(attn_lds(slot(j, 1)) + in.cols, w, acc.o);
                    }
                    attn_reads_done();
                    if (j + 2 < j1) fetch(V, j + 2, 1);
                }
            }
            if (MANY) {
                __syncthreads();
                bad = dirty != 0;
            }
            if (bad)
                for (int j = j0; j < j1; ++j) {
                    if (!cleaned(j)) continue;
                    const int k0 = first_key(j);
                    fetch_ids(j);
                    attn_wait();
                    find_rows(j);
                    load(V, own);
                    attn_wait();
                    if (MANY) attn_barrier();
                    attn_add_marks<DP, C::WAVE_KEYS / 16>(attn_lds(own) + in.cols, acc.o, lane, [&](int k) { return sees(k0 + k); }, attn_marked);
                    attn_reads_done();
                    if (MANY) attn_barrier();
                }
        }
        // The groups' parts of each row side by side in LDS; then each wave joins UNITS / GROUPS of the fours of columns of its rows
        const f32x2 halves = attn_halves(acc.l);
        f32x4 *parts = reinterpret_cast<f32x4 *>(smem) + lane;
        if (MANY) __syncthreads();                         // tiles are shared
#pragma unroll
        for (int u = 0; u < C::UNITS; ++u) {
            const f32x16 &o = acc.o[u / 4];
            const int g = u % 4 * 4;
            parts[wave * C::PART + u * 64] = f32x4{o[g], o[g + 1], o[g + 2], o[g + 3]};
        }
        if (h == 0) {
            stats[0][kg][member * 32 + lane] = acc.m * c;  // log2 units from here on
            stats[1][kg][member * 32 + lane] = halves[0] + halves[1];
        }
        __syncthreads();
        float m = -__builtin_inff(), l = 0.0f, w[C::GROUPS];
#pragma unroll
        for (int i = 0; i < C::GROUPS; ++i) m = fmaxf(m, stats[0][i][member * 32 + (lane & 31)]);
        const float ms = m == -__builtin_inff() ? 0.0f : m;
#pragma unroll
        for (int i = 0; i < C::GROUPS; ++i) {
            w[i] = __builtin_amdgcn_exp2f(stats[0][i][member * 32 + (lane & 31)] - ms);
            l += w[i] * stats[1][i][member * 32 + (lane & 31)];
        }
        const bool partial = j0 > 0 || j1 < seq.steps, there = row < nrows;
        const bool none = m == -__builtin_inff() && l == 0.0f && cached_sees_nothing(p, seq.q0, seq.nq, seq.len, token);
        const float inv = partial ? 1.0f : none ? 0.0f : 1.0f / l;
        float *to = nullptr;
        if (partial) to = p.part + ((range + item) * p.kv_heads + kv) * (C::ROWS * (DP + 2));
        if (there && h == 0 && kg == 0) {
            if (partial) {
                to[member * 32 + lane] = m;
                to[C::ROWS + member * 32 + lane] = l;
            } else if (p.lse)
                p.lse[(int64_t)head * p.Tq + seq.q0 + token] = none ? -__builtin_inff() : LN2 * (m + __builtin_amdgcn_logf(l));
        }
        uint16_t *out = p.out + (int64_t)(seq.q0 + token) * p.ldo + (int64_t)head * p.D;
        constexpr int OWN = C::UNITS / C::GROUPS;
        static_assert(OWN % 2 == 0, "pairs of fours make 16 bytes of output");
#pragma unroll
        for (int u = 0; u < OWN; u += 2) {
            float v[2][4];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                f32x4 sum = {};
#pragma unroll
                for (int k = 0; k < C::GROUPS; ++k) {
                    const f32x4 x = parts[(k * C::GROUP + member) * C::PART + (kg * OWN + u + i) * 64];
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[e] += w[k] * x[e];
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) v[i][e] = sum[e] * inv;
            }
            const int f = 2 * (kg * OWN + u);              // unit (kg OWN + u), half h: four f + h of the row's columns
            if (partial) {
                f32x4 *po = reinterpret_cast<f32x4 *>(to + 2 * C::ROWS) + (f + h) * C::ROWS + member * 32 + (lane & 31);
                if (there) {
                    po[0] = f32x4{v[0][0], v[0][1], v[0][2], v[0][3]};
                    po[2 * C::ROWS] = f32x4{v[1][0], v[1][1], v[1][2], v[1][3]};
                }
            } else {
                const u32x4 o = attn_store_unit(v[0], v[1]);
                const int d = 4 * f + 8 * h;
                if (there && (!PAD || d < p.D)) *reinterpret_cast<u32x4 *>(out + d) = o;
            }
        }
    }
}

// Joins the partials of the tiles of rows that more than one range had a part of, in the order of the ranges.  They lie [slot][kv head]: the rows' maxima and
// sums, then [DP / 4][rows] fours of columns.  A workgroup has 32 rows and 4 FOURS columns; its eight half waves take every eighth partial, all columns at once, since
// a trip to memory is what this kernel takes its time for, and are added up in LDS four fours at a time.
template <int DP, bool MANY, int FOURS>
__global__ __launch_bounds__(256) void attention_join_kernel(CachedParams p)
{
    typedef CachedTile<DP, MANY> C;
    __shared__ f32x4 sums[8][4][32];
    __shared__ float stats[2][8][32];
    const int r = threadIdx.x & 31, part = threadIdx.x >> 5;
    const int64_t item = blockIdx.x / p.kv_heads;
    const int kv = blockIdx.x % p.kv_heads;
    const CachedSpan span = p.spans[item];
    // within the workspace and the outputs, whatever seq_q holds
    const int w0 = min(max(span.first, 0), p.ranges - 1), n = min(span.parts, p.ranges - w0), q0 = min(max(span.q0, 0), p.Tq);
    const int row0 = max(span.row, 0) + (int)blockIdx.y * 32, row = row0 + r, nrows = (int)min((int64_t)span.rows, ((int64_t)p.Tq - q0) * p.group);
    if (n <= 1 || row0 >= nrows) return;
    const int64_t stride = (int64_t)p.kv_heads * (C::ROWS * (DP + 2));
    const float *from = p.part + ((w0 + item) * p.kv_heads + kv) * (C::ROWS * (DP + 2)) + blockIdx.y * 32 + r;
    float m = -__builtin_inff(), l = 0.0f;
    f32x4 v[FOURS] = {};
    if (row < nrows) {
#pragma unroll 2
        for (int i = part; i < n; i += 8) {
            const float mi = from[i * stride], li = from[i * stride + C::ROWS];
            const f32x4 *o = reinterpret_cast<const f32x4 *>(from - r - blockIdx.y * 32 + i * stride + 2 * C::ROWS) + blockIdx.z * FOURS * C::ROWS + blockIdx.y * 32 + r;
            const float top = fmaxf(m, mi), ms = top == -__builtin_inff() ? 0.0f : top;
            const float a = __builtin_amdgcn_exp2f(m - ms), b = __builtin_amdgcn_exp2f(mi - ms);
            m = top;
            l = l * a + li * b;
#pragma unroll
            for (int u = 0; u < FOURS; ++u) {
                const f32x4 x = o[u * C::ROWS];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[u][e] = v[u][e] * a + x[e] * b;
            }
        }
    }
    stats[0][part][r] = m;
    stats[1][part][r] = l;
    const int token = q0 + row / p.group, head = kv * p.group + row % p.group;
    float w[8], inv = 0.0f;
#pragma unroll
    for (int z = 0; z < FOURS / 4; ++z) {
        if (z) __syncthreads();
#pragma unroll
        for (int u = 0; u < 4; ++u) sums[part][u][r] = v[4 * z + u];
        __syncthreads();
        if (z == 0) {
            m = stats[0][0][r];
#pragma unroll
            for (int i = 1; i < 8; ++i) m = fmaxf(m, stats[0][i][r]);
            const float ms = m == -__builtin_inff() ? 0.0f : m;
            l = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                w[i] = __builtin_amdgcn_exp2f(stats[0][i][r] - ms);
                l += w[i] * stats[1][i][r];
            }
            const bool none = m == -__builtin_inff() && l == 0.0f && row < nrows && cached_sees_nothing(p, q0, span.rows / p.group, span.len, token - q0);
            inv = none ? 0.0f : 1.0f / l;
            if (blockIdx.z == 0 && part == 0 && row < nrows && p.lse)
                p.lse[(int64_t)head * p.Tq + token] = none ? -__builtin_inff() : LN2 * (m + __builtin_amdgcn_logf(l));
        }
        const int col = (blockIdx.z * FOURS + 4 * z + part) * 4;
        if (part < 4 && row < nrows && col < p.D) {        // four half waves finish four columns each
            f32x4 sum = {};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const f32x4 x = sums[i][part][r];
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[e] += w[i] * x[e];
            }
            typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
            *reinterpret_cast<u32x2 *>(p.out + (int64_t)token * p.ldo + (int64_t)head * p.D + col) =
                u32x2{attn_pack(sum[0] * inv, sum[1] * inv), attn_pack(sum[2] * inv, sum[3] * inv)};
        }
    }
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

// Tiles of 128 rows once a sequence has more than 32 on average, which tiles of 32 would go over all keys twice for.  us with 32 / 128, 32 heads over 8, each sequence of 16, 32, 36, 64 and 128 rows (tokens times group): 64
// columns, one sequence of 4096 keys 12.4 / 15.0, 12.6 / 15.2, 13.8 / 15.5, 14.1 / 15.6, 15.0 / 16.5; eight 23.5 / 26.7, 24.0 / 27.0, 26.0 / 27.6, 26.7 / 28.2, 33.2 / 30.6; 32 of 2048 32.5 / 34.8, 32.6 / 35.0, 53.5 / 35.2, 54.0 / 36.1, 92.5 / 40.1.
// 128 columns, one 15.3 / 18.2, 16.0 / 18.5, 15.4 / 19.0, 16.2 / 19.6, 18.0 / 21.6; eight 34.6 / 39.6, 35.8 / 40.3, 37.0 / 41.1, 38.7 / 42.6, 52.6 / 47.5; 32 54.1 / 56.8, 54.8 / 57.4, 93.4 / 57.8, 94.4 / 58.7, 168.8 / 63.7.  A lone sequence loses
// up to a quarter by it, eight a tenth just above 32 rows, and as many as fill the card's time with their keys gain a third or more.
static bool cached_many(int64_t Tq, int n_seqs, int group) { return Tq * group > 32 * (int64_t)n_seqs; }
// One workgroup for each CU
static int cached_ranges(int kv_heads) { return (256 + kv_heads - 1) / kv_heads; }
static int64_t cached_part_floats(int64_t Tq, int n_seqs, int kv_heads, int group, int D)
{
    const bool many = cached_many(Tq, n_seqs, group);
    return (cached_items(Tq, n_seqs, group, many) + cached_ranges(kv_heads)) * kv_heads * ((many ? 128 : 32) * ((D > 64 ? 128 : 64) + 2));
}

size_t cached_bytes(int64_t Tq, int n_seqs, int heads, int kv_heads, int D)
{
    const int group = heads / kv_heads;
    return (size_t)cached_part_floats(Tq, n_seqs, kv_heads, group, D) * 4 + (size_t)cached_items(Tq, n_seqs, group, cached_many(Tq, n_seqs, group)) * sizeof(CachedSpan);
}

int64_t cached_workgroups(const CachedParams &p)
{
    const bool many = cached_many(p.Tq, p.n_seqs, p.group);
    const int64_t join = cached_items(p.Tq, p.n_seqs, p.group, many) * p.kv_heads * (many ? 4 : 1) * 8, main = (int64_t)cached_ranges(p.kv_heads) * p.kv_heads * 2;
    return join > main ? join : main;
}

template <int DP, bool PAD, bool MANY>
static hipError_t launch_cached(CachedParams p, hipStream_t s)
{
    p.ranges = cached_ranges(p.kv_heads);
    p.spans = reinterpret_cast<CachedSpan *>(p.part + cached_part_floats(p.Tq, p.n_seqs, p.kv_heads, p.group, p.D));
    hipLaunchKernelGGL((attention_cached_kernel<DP, PAD, MANY>), dim3((unsigned)(p.ranges * p.kv_heads)), dim3(CachedTile<DP, MANY>::WAVES * 64), 0, s, p, p.scale * LOG2E);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    // 64 columns a workgroup where that leaves one for every CU, else 16
    const int64_t tiles = cached_items(p.Tq, p.n_seqs, p.group, MANY) * p.kv_heads * (MANY ? 4 : 1);
    dim3 join((unsigned)(tiles / (MANY ? 4 : 1)), MANY ? 4 : 1, DP / 16);
    if (tiles >= 256) {
        join.z = DP / 64;
        hipLaunchKernelGGL((attention_join_kernel<DP, MANY, 16>), join, dim3(256), 0, s, p);
    } else
        hipLaunchKernelGGL((attention_join_kernel<DP, MANY, 4>), join, dim3(256), 0, s, p);
    return hipGetLastError();
}

template <int DP, bool PAD>
static hipError_t launch_cached(const CachedParams &p, hipStream_t s)
{
    return cached_many(p.Tq, p.n_seqs, p.group) ? launch_cached<DP, PAD, true>(p, s) : launch_cached<DP, PAD, false>(p, s);
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
