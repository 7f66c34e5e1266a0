// attn_tile.hpp -- tiles, fragments and the softmax step that the attention kernels share (gfx950).
//
// One head's rows of Q, K, V or dO are tiles [rows x DP] of bf16 in LDS, DP = 64 or 128 columns (a head dimension below that leaves the
// chunks behind it zero).  All products are v_mfma_f32_32x32x16_bf16, written so that what one product leaves in the accumulators is an
// operand of the next as it stands: S^T = K Q^T leaves lane l with query l % 32 and, in register r, key (r & 3) + 8 (r >> 2) + 4 (l / 32);
// the contraction of O^T = V^T P^T may run over the keys in any order that both operands share, so eight registers, rounded to bf16, are
// the operand of 16 keys, and the transposing LDS read of V takes its keys in the same order: 4 h .. 4 h + 3 and 8 + 4 h .. 8 + 4 h + 3 for
// the lanes of half h.  No element of P ever moves between lanes, and a row's maximum and sum are in-lane but for one swap of the halves.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace coda {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(8))) short s16x8;

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// Chunk c (16 bytes) of row r lies at chunk position c ^ attn_swizzle(r).  Both reads below are then free of bank conflicts: 16 consecutive
// rows of one chunk, and four rows (r % 4 == 0) of 64 bytes each, cover all 64 banks.
template <int DP>
__device__ __forceinline__ int attn_swizzle(int r)
{
    return DP == 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
}

__device__ __forceinline__ uint32_t attn_lds(const unsigned char *p)
{
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const unsigned char *)p;
}

// 16 bytes a lane from its own address straight to LDS, lane l to lds + 16 l.  Not seen by the compiler's wait counts: attn_wait().
__device__ __forceinline__ void attn_load16(const void *p, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(p), "s"(lds) : "memory", "m0");
}
__device__ __forceinline__ uint64_t attn_uniform(uint64_t a)
{
    return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(a >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)a);
}
// Four bytes a lane
__device__ __forceinline__ void attn_load4(const void *p, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" : : "v"(p), "s"(lds) : "memory", "m0");
}
// The same from a uniform address and a lane's offset, by the lanes of `mask` alone, which need be none; what the others' four bytes of LDS hold stays.  No branch: the
// callers issue these among their products, and a branch would part those.
__device__ __forceinline__ void attn_load4(const void *base, uint32_t off, uint32_t lds, uint64_t mask)
{
    uint64_t all;
    asm volatile("s_mov_b64 %0, exec\n\ts_mov_b64 exec, %4\n\ts_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2\n\ts_mov_b64 exec, %0"
                 : "=&s"(all) : "v"(off), "s"(attn_uniform(reinterpret_cast<uint64_t>(base))), "s"(lds), "s"(attn_uniform(mask)) : "memory", "m0");
}
// The first n of 64 lanes, n from 0 on
__device__ __forceinline__ uint64_t attn_first_lanes(int n) { return n >= 64 ? ~0ull : (1ull << n) - 1; }
// All loads of this wave have arrived, all its LDS reads are done
__device__ __forceinline__ void attn_wait()
{
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xc07f);                    // lgkmcnt(0) that the compiler sees: else it waits for a step's first operand as if scalar loads from ahead of the loop were on their way
    asm volatile("" ::: "memory");
}
// All but the last N of them
template <int N>
__device__ __forceinline__ void attn_wait_but()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void attn_reads_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void attn_barrier()
{
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Tiles of ROWS rows of one head, loaded by NW waves together, 1 KB a load.  Loads go through a buffer descriptor that ends with the last row of the tile that there is, so rows behind it need no
// mask: lanes past the end read nothing from memory, and in PAD kernels those whose chunk is not below D are sent there too.  Their 16 bytes of LDS keep what they held or become zeros, and nothing
// relies on either: what lies behind the last row is masked by selection and cleared where it is not finite, and chunks not below D were cleared by attn_zero().  A load is two instructions;
// masks and 64-bit addresses took 18, a quarter of all that the forward kernel's loop issued.
template <int DP, bool PAD, int ROWS, int NW>
struct AttnLoad {
    static constexpr int CH = DP / 8, RPL = 64 / CH, LOADS = ROWS / (NW * RPL);
    static_assert(ROWS % (NW * RPL) == 0, "whole wave-loads");
    const uint16_t *base;              // element (0, 0) of the head's rows; uniform
    int64_t ld;
    int wave;
    uint32_t off[LOADS];               // bytes from the tile's first row, at most 64 rows of 2^22 elements
    // A tile on its way
    u32x4 buffer;
    uint32_t to;

    __device__ __forceinline__ AttnLoad(const uint16_t *base, int64_t ld, int wave, int lane, int D)
        : base(reinterpret_cast<const uint16_t *>(attn_uniform(reinterpret_cast<uint64_t>(base)))), ld(ld), wave(wave)
    {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int row = (i * NW + wave) * RPL + lane / CH, chunk = (lane % CH) ^ attn_swizzle<DP>(row);
            off[i] = PAD && chunk * 8 >= D ? 0xfffffff0u : (uint32_t)row * (uint32_t)ld * 2 + chunk * 16;
        }
    }
    // Rows row0 .. ; rows from n on are not read
    __device__ __forceinline__ void begin(int row0, int n, uint32_t tile)
    {
        const uint64_t at = reinterpret_cast<uint64_t>(base) + (uint64_t)((int64_t)row0 * ld * 2);
        const int left = __builtin_amdgcn_readfirstlane(min(n - row0, ROWS));              // keeps the clamp and the product scalar
        const uint32_t bytes = (uint32_t)max(0, left) * (uint32_t)ld * 2;
        buffer = u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)at), (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(at >> 32) & 0xffffu),
                       (uint32_t)__builtin_amdgcn_readfirstlane(bytes), 0x20000u};         // no stride, 32-bit elements
        to = __builtin_amdgcn_readfirstlane(tile + wave * 1024);
    }
    // Load i of them, in order
    __device__ __forceinline__ void next(int i)
    {
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" : : "v"(off[i]), "s"(buffer), "s"(to + i * NW * 1024) : "memory", "m0");
    }
    __device__ __forceinline__ void operator()(int row0, int n, const unsigned char *tile)
    {
        begin(row0, n, attn_lds(tile));
#pragma unroll
        for (int i = 0; i < LOADS; ++i) next(i);
    }
};

// Operands loaded ahead of a loop: the compiler waits for them here.  Otherwise it waits where the loop first uses them, in every round, and with its
// count of its own loads that wait is for the tiles on their way too.
template <int N>
__device__ __forceinline__ void attn_arrived(bf16x8 (&f)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(f[i]));
}

// Clears `bytes` (a multiple of 16) of LDS for PAD kernels, before their first tile
__device__ __forceinline__ void attn_zero(unsigned char *p, int bytes, int threads)
{
    for (int i = threadIdx.x * 16; i < bytes; i += threads * 16) *reinterpret_cast<u32x4 *>(p + i) = u32x4{0, 0, 0, 0};
    __syncthreads();
}

// The two ways in which operands are read from a tile, as byte offsets of a lane.  Steps along the columns change single bits of the chunk's position, which lie
// above the lane's own, so an operand's address is one exclusive or away from that of the first, and rows further on are a constant of the instruction: forming the addresses
// of 64 reads from rows and columns took dK's kernel 150 of its 350 vector instructions a round, and these, not the products, were its time.
template <int DP>
struct AttnLane {
    uint32_t rows, cols;
    __device__ __forceinline__ explicit AttnLane(int lane)
    {
        const int h = lane >> 5, i = lane & 15, r = 4 * h + (i >> 2), c = 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
        rows = (lane & 31) * (DP * 2) + ((h ^ attn_swizzle<DP>(lane & 31)) << 4);
        cols = r * (DP * 2) + ((c ^ attn_swizzle<DP>(r)) << 4) + (i & 1) * 8;
    }
};
// Operand of 32 tile rows x 16 columns: row row_base + lane % 32, columns 16 t + 8 (lane / 32) ..  tile_rows: the tile's LDS address (a multiple of 256) + AttnLane::rows
template <int DP>
__device__ __forceinline__ bf16x8 attn_rows(uint32_t tile_rows, int row_base, int t)
{
    return *(const __attribute__((address_space(3))) bf16x8 *)(uintptr_t)((tile_rows ^ (t << 5)) + row_base * (DP * 2));
}
// Operand of the transposed tile, 32 columns x 16 rows: column 32 db + lane % 32, rows 16 t + 4 (lane / 32) + {0 1 2 3, 8 9 10 11}.  Within 16
// lanes, lane i of a transposing read supplies the address of row i / 4, columns 4 (i % 4) .. and receives column i of the four rows.
template <int DP>
__device__ __forceinline__ bf16x8 attn_cols(uint32_t tile_cols, int t, int db)
{
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const uint32_t p = tile_cols ^ (db << 6);              // eight rows further the swizzle differs in one bit
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)(p + t * 16 * DP * 2));
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)((p ^ 32) + (t * 16 + 8) * DP * 2));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

__device__ __forceinline__ f32x16 attn_mfma(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }

__device__ __forceinline__ uint32_t attn_pack(float a, float b)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}
// Registers 8 half .. 8 half + 7 of an accumulator as an operand, to the nearest bf16
__device__ __forceinline__ bf16x8 attn_operand(const f32x16 &x, int half)
{
    u32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = attn_pack(x[half * 8 + 2 * e], x[half * 8 + 2 * e + 1]);
    return __builtin_bit_cast(bf16x8, v);
}
// The whole accumulator as operands of two products that are added up: its upper bits, cut off, and what they leave, to the nearest bf16: off by 2^-16 at most
__device__ __forceinline__ void attn_two_parts(const f32x16 &x, bf16x8 (&hi)[2], bf16x8 (&lo)[2])
{
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        u32x4 a, b;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float f = x[u * 8 + 2 * e], g = x[u * 8 + 2 * e + 1];                    // a bit cast of an element of the vector takes the first one each time
            const uint32_t p = __builtin_bit_cast(uint32_t, f), q = __builtin_bit_cast(uint32_t, g);
            a[e] = __builtin_amdgcn_perm(q, p, 0x07060302u);
            b[e] = attn_pack(f - __builtin_bit_cast(float, p & 0xffff0000u), g - __builtin_bit_cast(float, q & 0xffff0000u));
        }
        hi[u] = __builtin_bit_cast(bf16x8, a);
        lo[u] = __builtin_bit_cast(bf16x8, b);
    }
}
// Row of the accumulator that register r of a lane of half h holds
__device__ __forceinline__ int attn_acc_row(int r, int h) { return (r & 3) + 8 * (r >> 2) + 4 * h; }

// x of this lane combined with that of lane ^ 32
__device__ __forceinline__ f32x2 attn_halves(float x)
{
    const auto p = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
    const uint32_t a = p[0], b = p[1];                     // a bit cast of an element of the pair takes the first one both times
    return f32x2{__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)};
}

// Four consecutive values of a column of the accumulators, groups g and g + 1 (rows 8 g + 4 h .. and 8 g + 8 + 4 h ..), rounded and exchanged
// between the halves: a lane of half h is left with rows 8 (g + h) .. 8 (g + h) + 7, 16 contiguous bytes of a row-major output.
__device__ __forceinline__ u32x4 attn_store_unit(const float (&lo)[4], const float (&hi)[4])
{
    const auto a = __builtin_amdgcn_permlane32_swap(attn_pack(lo[0], lo[1]), attn_pack(hi[0], hi[1]), false, false);
    const auto b = __builtin_amdgcn_permlane32_swap(attn_pack(lo[2], lo[3]), attn_pack(hi[2], hi[3]), false, false);
    return u32x4{a[0], b[0], a[1], b[1]};
}

// ---------------------------------------------------------------- infinities and NaN behind a mask
// A weight of zero times an infinity or a NaN is NaN, so a row of V that is not finite would reach rows that do not see it.  Tiles that no mask
// touches need nothing.  In the others (one or two for a tile of rows) what is not finite is replaced by zero in LDS before the products, and
// only where there was any, its effect on the rows that do see it is added at the end: a product of the mask (0 or 1) with marks (+inf 1, -inf 2^10,
// NaN 2^20) tells for each output whether it met +inf, -inf, both or a NaN: sums below 2^20 are exact in fp32, above it only that they are counts.  Whatever order a sum takes
// these in, the result is the same, so the end is early enough.

// Not zero if one of eight elements is not finite
__device__ __forceinline__ uint32_t attn_not_finite(u32x4 v)
{
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) top |= ((v[e] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
    return top;
}
// `bytes` of a tile from `tile` on (a multiple of 1024) by one wave; true if something in the first `there` of them (rows behind were not loaded) was not finite
__device__ __forceinline__ bool attn_clean(unsigned char *tile, int bytes, int there, int lane)
{
    bool found = false;
    for (int i = lane * 16; i < bytes; i += 1024) {
        u32x4 v = *reinterpret_cast<const u32x4 *>(tile + i);
        if (attn_not_finite(v)) {
            found |= i < there;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if ((v[e] & 0x7f80u) == 0x7f80u) v[e] &= 0xffff0000u;
                if ((v[e] & 0x7f800000u) == 0x7f800000u) v[e] &= 0xffffu;
            }
            *reinterpret_cast<u32x4 *>(tile + i) = v;
        }
    }
    return __ballot(found) != 0;
}
// The same without touching what was loaded, for a tile that others still read: rows behind it, which nobody's result depends on, are cleared where they are not finite
template <int BYTES>
__device__ __forceinline__ bool attn_check(unsigned char *tile, int there, int lane)
{
    uint32_t top = 0;
    if (there >= BYTES) {
#pragma unroll 4
        for (int i = 0; i < BYTES; i += 1024) top |= attn_not_finite(*reinterpret_cast<const u32x4 *>(tile + i + lane * 16));
    } else
        for (int i = lane * 16; i < BYTES; i += 1024) {
            const uint32_t t = attn_not_finite(*reinterpret_cast<const u32x4 *>(tile + i));
            if (i < there) top |= t;
            else if (t) *reinterpret_cast<u32x4 *>(tile + i) = u32x4{0, 0, 0, 0};
        }
    return __ballot(top != 0) != 0;
}
__device__ __forceinline__ bf16x8 attn_marks(bf16x8 x)
{
    s16x8 v = __builtin_bit_cast(s16x8, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int w = (uint16_t)v[e];
        v[e] = (w & 0x7f80) != 0x7f80 ? 0 : (w & 0x7f) ? 0x4980 : (w & 0x8000) ? 0x4480 : 0x3f80;   // 2^20, 2^10, 1
    }
    return __builtin_bit_cast(bf16x8, v);
}
__device__ __forceinline__ float attn_marked(float o, float marks)
{
    const int n = (int)fminf(marks, 1048576.0f);
    if (n == 0) return o;
    const bool plus = n & 1023, minus = (n >> 10) & 1023;
    if (n >= 1048576 || (plus && minus)) return __builtin_nanf("");
    return o + (plus ? __builtin_inff() : -__builtin_inff());
}
// What the elements of an uncleaned tile of NT x 16 rows that are not finite come to in acc; vis(k): the lane's row sees row k of the tile; met(x, marks): x with what it met
template <int DP, int NT, class Vis, class Met>
__device__ __forceinline__ void attn_add_marks(uint32_t tile_cols, f32x16 (&acc)[DP / 32], int lane, Vis vis, Met met)
{
#pragma unroll
    for (int b = 0; b < DP / 32; ++b) {
        f32x16 marks = {};
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            s16x8 see;
#pragma unroll
            for (int e = 0; e < 8; ++e) see[e] = vis(16 * t + (e & 3) + 8 * (e >> 2) + 4 * (lane >> 5)) ? 0x3f80 : 0;
            marks = attn_mfma(attn_marks(attn_cols<DP>(tile_cols, t, b)), __builtin_bit_cast(bf16x8, see), marks);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[b][r] = met(acc[b][r], marks[r]);
    }
}

// ---------------------------------------------------------------- one tile of keys
// What a wave holds of 32 rows: O^T, and for the lane's row the running maximum of the raw scores and the sum of this half's weights
template <int DP>
struct AttnRows {
    f32x16 o[DP / 32];
    float m, l;
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int b = 0; b < DP / 32; ++b) o[b] = f32x16{};
        m = -__builtin_inff();
        l = 0.0f;
    }
};

// Products 0 .. N - 1 with their LDS operands read a batch of BATCH ahead: left to itself the compiler reads each one where it is used and waits for it there,
// or, where registers seem to be free, all of them at once.  read(i) returns the operand of product i, multiply(i, operand) takes it; the first batch is
// read by the caller, and tail() is called ahead of the last products, to read what comes after them.
template <int BATCH, class Read>
__device__ __forceinline__ void attn_read(bf16x8 (&a)[BATCH], Read read)
{
#pragma unroll
    for (int i = 0; i < BATCH; ++i) a[i] = read(i);
}
template <int N, int BATCH, class Read, class Multiply, class Tail>
__device__ __forceinline__ void attn_products(const bf16x8 (&first)[BATCH], Read read, Multiply multiply, Tail tail)
{
    static_assert(N % BATCH == 0, "whole batches");
    bf16x8 a[2][BATCH];
#pragma unroll
    for (int i = 0; i < BATCH; ++i) a[0][i] = first[i];
#pragma unroll
    for (int n = 0; n < N / BATCH; ++n) {
        if (n + 1 < N / BATCH) {
#pragma unroll
            for (int i = 0; i < BATCH; ++i) a[(n + 1) & 1][i] = read((n + 1) * BATCH + i);
        } else tail();
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < BATCH; ++i) multiply(n * BATCH + i, a[n & 1][i]);
        __builtin_amdgcn_sched_barrier(0);
    }
}
template <int N, int BATCH, class Read, class Multiply>
__device__ __forceinline__ void attn_products(Read read, Multiply multiply)
{
    bf16x8 first[BATCH];
    attn_read<BATCH>(first, read);
    attn_products<N, BATCH>(first, read, multiply, [] {});
}
// S^T of NB x 32 keys and 32 rows; between(i) is called behind product i
template <int DP, int NB, int BATCH, class Between>
__device__ __forceinline__ void attn_scores(uint32_t k_rows, const bf16x8 (&q)[DP / 16], f32x16 (&s)[NB], Between between)
{
#pragma unroll
    for (int b = 0; b < NB; ++b) s[b] = f32x16{};
    attn_products<DP / 16 * NB, BATCH>([&](int i) { return attn_rows<DP>(k_rows, i % NB * 32, i / NB); },
                                       [&](int i, bf16x8 a) {
                                           s[i % NB] = attn_mfma(a, q[i / NB], s[i % NB]);
                                           between(i);
                                       });
}
// The softmax step: scores to weights, rounded, and the rows' maxima and sums.  c = scale * log2(e) > 0.  `masked`: some position is not visible;
// vis(k) says whether key k of the tile is, for the lane's row.  The maximum that the weights are taken relative to is renewed only when some row's
// has grown by more than 2^8 in weight: weights up to 2^8 cost no accuracy in bf16 or fp32, and the multiplications of O^T fall away for nearly
// all tiles.
template <int DP, int NB, class Vis>
__device__ __forceinline__ void attn_weights(f32x16 (&s)[NB], bf16x8 (&p)[2 * NB], AttnRows<DP> &rows, float c, int lane, bool masked, Vis vis)
{
    const int h = lane >> 5;
    if (masked) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[b][r] = vis(b * 32 + attn_acc_row(r, h)) ? s[b][r] : -__builtin_inff();
    }
    float top = s[0][0];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, s[b][r]);
    const f32x2 tops = attn_halves(top);
    top = fmaxf(rows.m, fmaxf(tops[0], tops[1]));
    if (__ballot((top - rows.m) * c > 8.0f)) {             // -inf - -inf is NaN: no row that has seen nothing asks for it
        const float alpha = top == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f((rows.m - top) * c);
        rows.l *= alpha;
        rows.m = top;
#pragma unroll
        for (int b = 0; b < DP / 32; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) rows.o[b][r] *= alpha;
    }
    const float mc = rows.m == -__builtin_inff() ? 0.0f : rows.m * c;
    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            s[b][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][r], c, -mc));
            sum[r & 3] += s[b][r];
        }
    rows.l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
#pragma unroll
    for (int t = 0; t < 2 * NB; ++t) p[t] = attn_operand(s[t >> 1], t & 1);
}
// O^T += V^T P^T
template <int DP, int NB, int BATCH>
__device__ __forceinline__ void attn_values(uint32_t v_cols, const bf16x8 (&p)[2 * NB], f32x16 (&o)[DP / 32])
{
    constexpr int D = DP / 32;
    attn_products<2 * NB * D, BATCH>([&](int i) { return attn_cols<DP>(v_cols, i / D, i % D); }, [&](int i, bf16x8 a) { o[i % D] = attn_mfma(a, p[i / D], o[i % D]); });
}
// Keys of a tile (NB x 32 of them) for 32 rows
template <int DP, int NB, class Vis, class Between>
__device__ __forceinline__ void attn_step(uint32_t k_rows, uint32_t v_cols, const bf16x8 (&q)[DP / 16], AttnRows<DP> &rows, float c, int lane, bool masked, Vis vis,
                                          Between between)
{
    constexpr int D = DP / 32;
    f32x16 s[NB];
    bf16x8 p[2 * NB], first[4];
    attn_scores<DP, NB, 4>(k_rows, q, s, between);
    const auto read = [&](int i) { return attn_cols<DP>(v_cols, i / D, i % D); };
    attn_read<4>(first, read);                             // arrive behind the exponentials
    __builtin_amdgcn_sched_barrier(0);
    attn_weights<DP, NB>(s, p, rows, c, lane, masked, vis);
    attn_products<2 * NB * D, 4>(first, read, [&](int i, bf16x8 a) { rows.o[i % D] = attn_mfma(a, p[i / D], rows.o[i % D]); }, [] {});
}

// ---------------------------------------------------------------- packed sequences
struct AttnSpan {
    int begin, count;
};
// Rows of sequence s of `total`, whatever the offsets hold
__device__ __forceinline__ AttnSpan attn_span(const int32_t *at, int s, int total)
{
    const int a = min(max(at[s], 0), total), b = min(max(at[s + 1], a), total);
    return {a, b - a};
}
// Of one sequence for the whole wave
__device__ __forceinline__ AttnSpan attn_span_of_wave(const int32_t *at, int s, int total)
{
    const AttnSpan x = attn_span(at, s, total);
    return {__builtin_amdgcn_readfirstlane(x.begin), __builtin_amdgcn_readfirstlane(x.count)};
}
// Tiles of `rows` rows are numbered from begin / rows + s in sequence s, so that the number of a tile gives its sequence without anyone having
// counted the tiles: the next sequence's first number is never below this one's last plus one.  Numbers that no sequence uses do nothing.
// Returns the last sequence whose first number is not above t; 64 candidates are looked at at once.
__device__ __forceinline__ int attn_find(const int32_t *at, int n_seqs, int rows, int64_t t, int lane)
{
    int lo = 0, width = n_seqs;
    while (width > 1) {
        const int step = (width + 63) / 64, i = lane * step;
        const bool below = i < width && (int64_t)(max(at[lo + i], 0) / rows) + lo + i <= t;
        const int k = __popcll(__ballot(below));
        if (k > 1) lo += (k - 1) * step;
        width = min(step, n_seqs - lo);
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

}  // namespace coda
