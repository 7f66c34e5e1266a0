// attn_launch.hpp -- host launchers of the attention kernels and of the paged cache.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace coda {

// Rows of packed sequences: Q [Tq x heads * D], K and V [Tk x kv_heads * D], row pitches in elements
struct AttnParams {
    const uint16_t *Q, *K, *V;
    int64_t ldq, ldk, ldv;
    const int32_t *seq_q, *seq_k;      // [n_seqs + 1]
    int n_seqs, heads, kv_heads, D, Tq, Tk, causal;
    float scale;
    uint16_t *out;
    int64_t ldo;
    float *lse;                        // [heads x Tq] or null
};
// About how many tiles of `rows` rows n_seqs sequences of T rows come to, where each but one adds half a tile (their lengths are on the device)
inline int64_t attn_about(int T, int n_seqs, int rows) { return ((int64_t)T - 1) / rows + 1 + (n_seqs - 1) / 2; }
int64_t attn_workgroups(const AttnParams &p);
hipError_t launch_attention(const AttnParams &p, hipStream_t s);

// Backward: f.lse is an input here, f.out is not used
struct BwdParams {
    AttnParams f;
    const uint16_t *O, *dO;
    int64_t ldo, lddo;
    const float *cos, *sin;            // [rope_rows x D / 2], or null
    const int32_t *pos_q, *pos_k;
    int rope_rows;
    uint16_t *dQ, *dK, *dV;
    int64_t lddq, lddk, lddv;
    float *stats;                      // [2][heads][Tq]
};
int64_t bwd_workgroups(const BwdParams &p);
size_t bwd_bytes(int64_t Tq, int heads);
hipError_t launch_attention_bwd(const BwdParams &p, hipStream_t s);

// Who has a part of a tile of rows: the first range and how many ranges; the sequence's first row of Q, the tile's first row and the sequence's number of rows (times the group), its keys
struct CachedSpan {
    int32_t first, parts, q0, row, rows, len;
};
// Rows of Q over a paged cache
struct CachedParams {
    const uint16_t *Q, *K, *V;         // K, V: [pages][kv_heads][page][D]
    int64_t ldq, ld_table;
    const int32_t *table, *lens, *seq_q;
    const uint64_t *tree;              // or null
    int n_seqs, kv_heads, group, D, Tq, page_bits, pages, capacity;   // capacity: keys that a row of the table has room for
    uint32_t page_mask, page_bytes;    // page - 1, bytes of a page of all heads
    int ranges;                        // this and spans: set by the launch
    CachedSpan *spans;                 // of each tile of rows
    float scale;
    uint16_t *out;
    int64_t ldo;
    float *lse;                        // [kv_heads * group x Tq] or null
    float *part;
};
int64_t cached_workgroups(const CachedParams &p);
size_t cached_bytes(int64_t Tq, int n_seqs, int heads, int kv_heads, int D);
hipError_t launch_attention_cached(const CachedParams &p, hipStream_t s);

int64_t cache_store_workgroups(int64_t T, int cols);
hipError_t launch_cache_store(const uint16_t *K, int64_t ldk, const uint16_t *V, int64_t ldv, int64_t T, int cols, int D, const int32_t *slots, uint16_t *k,
                              uint16_t *v, int64_t slots_there, int page_bits, hipStream_t s);

}  // namespace coda
