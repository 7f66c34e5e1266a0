// coda_api.hip -- the C ABI (include/coda.h): argument validation, canonicalisation of
// the epilogue program into one of the pre-instantiated kernel variants, launch.
// Nothing here allocates, synchronises or keeps state beyond the last HIP error.
#include "../../include/coda.h"

#include "attn_launch.hpp"
#include "aux_kernels.hpp"
#include "gemm_launch.hpp"
#include "narrow_launch.hpp"
#include "q8.hpp"
#include "scaled_launch.hpp"
#include "small_launch.hpp"
#include "splitk_plan.hpp"

#include <mutex>

namespace {

static_assert(coda::PLAN_TILE_M == coda::TILE_M && coda::PLAN_TILE_N == coda::TILE_N, "the split-K plan counts the kernels' tiles");

thread_local int g_last_hip_error = 0;

coda_status launch_status(hipError_t e)
{
    if (e == hipSuccess) return CODA_OK;
    g_last_hip_error = (int)e;
    return CODA_ERR_LAUNCH;
}

// The kernels form per-lane byte offsets of up to 256 rows in 32 bits: row pitches are bounded accordingly.
constexpr int64_t MAX_LD = int64_t(1) << 22;

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// Shape / alignment checks of a bf16 operand whose op() shape must be [r x c].
coda_status check_operand(const coda_mat *X, int64_t r, int64_t c)
{
    if (!X) return CODA_ERR_NULL;
    if (X->dtype != CODA_BF16 && X->dtype != CODA_F8E4M3) return CODA_ERR_DTYPE;
    const int64_t sr = X->trans ? c : r, sc = X->trans ? r : c;
    if (X->rows != sr || X->cols != sc || X->ld < sc || X->ld > MAX_LD) return CODA_ERR_SHAPE;
    if (sr > 0 && sc > 0 && !X->ptr) return CODA_ERR_NULL;
    if (!aligned16(X->ptr) || (X->ld & (X->dtype == CODA_F8E4M3 ? 15 : 7))) return CODA_ERR_ALIGN;   // 16-byte rows
    return CODA_OK;
}

coda_status check_tile(const void *p, int64_t ld, int64_t width)
{
    if (!p) return CODA_ERR_NULL;
    if (ld < width || ld > MAX_LD) return CODA_ERR_SHAPE;
    if (!aligned16(p) || (ld & 7)) return CODA_ERR_ALIGN;
    return CODA_OK;
}

coda_status check_vec(const void *p)
{
    if (!p) return CODA_ERR_NULL;
    return aligned4(p) ? CODA_OK : CODA_ERR_ALIGN;
}

// HIP takes fewer than 2^32 work items along a dimension of a launch.
bool launch_fits(int64_t workgroups, int threads) { return workgroups <= (int64_t)UINT32_MAX / threads; }

// An 8-bit tile [M x width]: codes at `p`, scales [ceil(width / 128)][>= M] at `s`.
coda_status check_scales(const void *s, int64_t ld, int64_t rows)
{
    if (!s) return CODA_ERR_NULL;
    if (ld < rows || ld > INT32_MAX) return CODA_ERR_SHAPE;
    return aligned16(s) && (ld & 15) == 0 ? CODA_OK : CODA_ERR_ALIGN;
}
coda_status check_q8_tile(const void *p, int64_t ld, int64_t width, const void *s, int64_t ld_s, int64_t M)
{
    if (!p) return CODA_ERR_NULL;
    if (ld < width || ld > MAX_LD) return CODA_ERR_SHAPE;
    if (!aligned16(p) || (ld & 15)) return CODA_ERR_ALIGN;
    return check_scales(s, ld_s, M);
}

struct Parsed {
    int mode = -1;
    coda::GemmParams p{};
    bool q8 = false;               // the program ends in STORE_Q8: mode is a Q8Mode
    coda::Q8Params q{};
};

// Canonical order: ROW_SCALE < ADD_TILE < ROW_SUMSQ < COL_SCALE_SIDE < final; ROPE only between ROW_SCALE and STORE.
// `scaled`: the programs of coda_gemm_scaled, which has those that end in STORE_Q8 and no ACCUM_F32.
coda_status parse_program(const coda_epi_op *prog, int32_t n_ops, int64_t M, int64_t N, bool scaled, Parsed &out)
{
    if (n_ops < 0 || (n_ops > 0 && !prog)) return CODA_ERR_NULL;
    coda::GemmParams &p = out.p;
    int stage = 0;           // next admissible position in the canonical order
    int pair = 0;            // 0 none, 1 swiglu fwd, 2 swiglu bwd
    bool final_seen = false;
    bool linear_only = false;  // an op that only the linear program supports was used
    int q8_pair = 0;           // 0 none, 1 SWIGLU_FWD_Q8, 2 SWIGLU_BWD_Q8: only STORE_Q8 may follow
    bool rmsbwd = false;       // RMSNORM_BWD seen: only ADD_TILE and a bf16 STORE may follow
    for (int i = 0; i < n_ops; ++i) {
        const coda_epi_op &op = prog[i];
        if (final_seen) return CODA_ERR_PROGRAM;
        if (q8_pair && op.kind != CODA_EPI_STORE_Q8) return CODA_ERR_PROGRAM;
        coda_status st;
        switch (op.kind) {
        case CODA_EPI_ROW_SCALE:
            if (stage > 0 || pair) return CODA_ERR_PROGRAM;
            if ((st = check_vec(op.in)) != CODA_OK) return st;
            p.row_scale = static_cast<const float *>(op.in);
            stage = 1;
            break;
        case CODA_EPI_ROPE:
            if (stage > 1 || pair || rmsbwd) return CODA_ERR_PROGRAM;
            if ((st = check_vec(op.in)) != CODA_OK || (st = check_vec(op.in2)) != CODA_OK || (st = check_vec(op.in3)) != CODA_OK)
                return st;
            if (reinterpret_cast<uintptr_t>(op.in) % coda::ROPE_TABLE_ALIGN || reinterpret_cast<uintptr_t>(op.in2) % coda::ROPE_TABLE_ALIGN) return CODA_ERR_ALIGN;
            if (op.i0 <= 0 || (op.i0 & 7) || op.i0 > INT32_MAX || op.i1 < 0 || (op.i1 & 7) || op.i1 > N || op.ld_in <= 0 ||
                op.ld_in > INT32_MAX / (op.i0 / 2))    // T rows of head_dim / 2 entries, indexed in 31 bits
                return CODA_ERR_SHAPE;
            p.rope_cos = static_cast<const float *>(op.in);
            p.rope_sin = static_cast<const float *>(op.in2);
            p.rope_pos = static_cast<const int *>(op.in3);
            p.rope_half = (int)(op.i0 / 2);
            p.rope_cols = (int)op.i1;
            p.rope_T = (int)op.ld_in;
            stage = 4;          // only STORE may follow
            linear_only = true;
            break;
        case CODA_EPI_LSE_PARTIAL:
            if (stage > 1 || pair || rmsbwd) return CODA_ERR_PROGRAM;
            if ((st = check_vec(op.in3)) != CODA_OK || (st = check_vec(op.out)) != CODA_OK ||
                (st = check_vec(op.out2)) != CODA_OK || (st = check_vec(op.out3)) != CODA_OK)
                return st;
            p.lse_y = static_cast<const int *>(op.in3);
            p.lse_max = static_cast<float *>(op.out);
            p.lse_sum = static_cast<float *>(op.out2);
            p.lse_tgt = static_cast<float *>(op.out3);
            stage = 4;          // only STORE may follow
            linear_only = true;
            break;
        case CODA_EPI_RMSNORM_BWD:
            if (stage > 0 || pair) return CODA_ERR_PROGRAM;
            if ((st = check_tile(op.in, op.ld_in, N)) != CODA_OK) return st;
            if ((st = check_vec(op.in2)) != CODA_OK || (st = check_vec(op.in3)) != CODA_OK || (st = check_vec(op.in4)) != CODA_OK)
                return st;
            if (!aligned16(op.in4)) return CODA_ERR_ALIGN;
            p.rn_c = static_cast<const uint16_t *>(op.in);
            p.ld_rn_c = op.ld_in;
            p.rn_r = static_cast<const float *>(op.in2);
            p.rn_z = static_cast<const float *>(op.in3);
            p.rn_gamma = static_cast<const float *>(op.in4);
            if (op.i0 < 0 || op.i0 > INT32_MAX) return CODA_ERR_SHAPE;
            p.rn_zscale = op.i0 > 0 ? 1.0f / (float)op.i0 : 1.0f;
            if (op.out) {
                if ((st = check_tile(op.out, op.ld_out, N)) != CODA_OK) return st;
                p.out2 = static_cast<uint16_t *>(op.out);
                p.ld_out2 = op.ld_out;
            }
            if (op.out2) {
                if ((st = check_vec(op.out2)) != CODA_OK) return st;
                if ((op.flags & ~1u) != 0) return CODA_ERR_PROGRAM;
                p.colred = static_cast<float *>(op.out2);
                p.colred_mode = (op.flags & CODA_REDUCE_ATOMIC) ? coda::ROWRED_ATOMIC : coda::ROWRED_PARTIALS;
            }
            rmsbwd = true;
            stage = 1;          // only ADD_TILE and STORE may follow
            break;
        case CODA_EPI_ADD_TILE:
            if (stage > 1 || pair) return CODA_ERR_PROGRAM;
            if ((st = check_tile(op.in, op.ld_in, N)) != CODA_OK) return st;
            p.add = static_cast<const uint16_t *>(op.in);
            p.ld_add = op.ld_in;
            stage = 2;
            linear_only = true;
            break;
        case CODA_EPI_ROW_SUMSQ:
            if (stage > 2 || pair || rmsbwd) return CODA_ERR_PROGRAM;
            if ((st = check_vec(op.out)) != CODA_OK) return st;
            if (op.flags != CODA_REDUCE_PARTIALS && op.flags != CODA_REDUCE_ATOMIC) return CODA_ERR_PROGRAM;
            p.rowred = static_cast<float *>(op.out);
            p.rowred_mode = op.flags == CODA_REDUCE_ATOMIC ? coda::ROWRED_ATOMIC : coda::ROWRED_PARTIALS;
            stage = 3;
            linear_only = true;
            break;
        case CODA_EPI_COL_SCALE_SIDE:
            if (stage > 3 || pair || p.rope_cos || rmsbwd) return CODA_ERR_PROGRAM;
            if ((st = check_vec(op.in)) != CODA_OK) return st;
            if (!aligned16(op.in)) return CODA_ERR_ALIGN;
            if ((st = check_tile(op.out, op.ld_out, N)) != CODA_OK) return st;
            p.col_scale = static_cast<const float *>(op.in);
            p.side = static_cast<uint16_t *>(op.out);
            p.ld_side = op.ld_out;
            stage = 4;
            linear_only = true;
            break;
        case CODA_EPI_SWIGLU_FWD:
            if (pair || linear_only || rmsbwd || (N & 1)) return CODA_ERR_PROGRAM;
            if (op.out) {
                if ((st = check_tile(op.out, op.ld_out, N)) != CODA_OK) return st;
                p.out2 = static_cast<uint16_t *>(op.out);
                p.ld_out2 = op.ld_out;
            }
            pair = 1;
            stage = 5;
            break;
        case CODA_EPI_SWIGLU_BWD:
            if (pair || linear_only || stage > 0) return CODA_ERR_PROGRAM;
            if ((st = check_tile(op.in, op.ld_in, 2 * N)) != CODA_OK) return st;
            p.Z = static_cast<const uint16_t *>(op.in);
            p.ldz = op.ld_in;
            if (op.out) {
                if ((st = check_tile(op.out, op.ld_out, N)) != CODA_OK) return st;
                p.out2 = static_cast<uint16_t *>(op.out);
                p.ld_out2 = op.ld_out;
            }
            if (op.out2) {
                if ((st = check_vec(op.out2)) != CODA_OK) return st;
                if ((op.flags & ~1u) != 0) return CODA_ERR_PROGRAM;
                p.rowred = static_cast<float *>(op.out2);
                p.rowred_mode = (op.flags & CODA_REDUCE_ATOMIC) ? coda::ROWRED_ATOMIC : coda::ROWRED_PARTIALS;
            }
            pair = 2;
            stage = 5;
            break;
        case CODA_EPI_STORE: {
            const bool f32 = (op.flags & CODA_STORE_F32) != 0;
            if ((op.flags & ~CODA_STORE_F32) != 0) return CODA_ERR_PROGRAM;
            if ((pair || rmsbwd) && f32) return CODA_ERR_PROGRAM;
            const int64_t width = pair == 1 ? N / 2 : pair == 2 ? 2 * N : N;
            if (!op.out) return CODA_ERR_NULL;
            if (op.ld_out < width || op.ld_out > MAX_LD) return CODA_ERR_SHAPE;
            if (!aligned16(op.out) || (op.ld_out & (f32 ? 3 : 7))) return CODA_ERR_ALIGN;
            p.out = op.out;
            p.ld_out = op.ld_out;
            p.out_f32 = f32 ? 1 : 0;
            out.mode = pair == 1 ? coda::EPI_SWIGLU_FWD : pair == 2 ? coda::EPI_SWIGLU_BWD
                     : rmsbwd  ? coda::EPI_RMSNORM_BWD : coda::EPI_LINEAR;
            final_seen = true;
            break;
        }
        case CODA_EPI_SWIGLU_FWD_Q8:
            if (!scaled || stage > 1 || pair || rmsbwd) return CODA_ERR_PROGRAM;
            if (N & 31) return CODA_ERR_SHAPE;             // rows of the halved width are whole chunks of 16 codes
            if (op.flags != 0) return CODA_ERR_PROGRAM;
            if (op.out) {
                if ((st = check_q8_tile(op.out, op.ld_out, N, op.out2, op.i0, M)) != CODA_OK) return st;
                out.q.z = static_cast<uint8_t *>(op.out);
                out.q.ldz = op.ld_out;
                out.q.z_s = static_cast<uint8_t *>(op.out2);
                out.q.ld_z_s = op.i0;
            }
            q8_pair = 1;
            break;
        case CODA_EPI_SWIGLU_BWD_Q8:
            if (!scaled || stage > 0 || pair || rmsbwd) return CODA_ERR_PROGRAM;
            if ((st = check_q8_tile(op.in, op.ld_in, 2 * N, op.in2, op.i0, M)) != CODA_OK) return st;
            out.q.z = static_cast<uint8_t *>(const_cast<void *>(op.in));
            out.q.ldz = op.ld_in;
            out.q.z_s = static_cast<uint8_t *>(const_cast<void *>(op.in2));
            out.q.ld_z_s = op.i0;
            if ((op.flags & ~1u) != 0) return CODA_ERR_PROGRAM;
            if (op.out2) {
                if ((st = check_vec(op.out2)) != CODA_OK) return st;
                p.rowred = static_cast<float *>(op.out2);
                p.rowred_mode = (op.flags & CODA_REDUCE_ATOMIC) ? coda::ROWRED_ATOMIC : coda::ROWRED_PARTIALS;
            }
            q8_pair = 2;
            break;
        case CODA_EPI_STORE_Q8: {
            if (!scaled || pair || rmsbwd || stage > 1) return CODA_ERR_PROGRAM;
            if (op.flags != 0) return CODA_ERR_PROGRAM;
            const int64_t width = q8_pair == 1 ? N / 2 : q8_pair == 2 ? 2 * N : N;
            if ((st = check_q8_tile(op.out, op.ld_out, width, op.out2, op.i0, M)) != CODA_OK) return st;
            out.q.out = static_cast<uint8_t *>(op.out);
            out.q.ld_out = op.ld_out;
            out.q.out_s = static_cast<uint8_t *>(op.out2);
            out.q.ld_out_s = op.i0;
            out.q8 = true;
            out.mode = q8_pair == 1 ? coda::Q8_SWIGLU_FWD : q8_pair == 2 ? coda::Q8_SWIGLU_BWD : coda::Q8_LINEAR;
            final_seen = true;
            break;
        }
        case CODA_EPI_ACCUM_F32:
            if (scaled || stage > 0 || pair) return CODA_ERR_PROGRAM;
            if (!op.out) return CODA_ERR_NULL;
            if (op.ld_out < N || op.ld_out > MAX_LD) return CODA_ERR_SHAPE;
            if (!aligned16(op.out) || (op.ld_out & 3)) return CODA_ERR_ALIGN;
            p.out = op.out;
            p.ld_out = op.ld_out;
            out.mode = coda::EPI_ACCUM;
            final_seen = true;
            break;
        default:
            return CODA_ERR_PROGRAM;
        }
    }
    return final_seen ? CODA_OK : CODA_ERR_PROGRAM;
}

__global__ void zero_counters_kernel(unsigned *c, int n)
{
    const int i = blockIdx.x * blockDim.x + threadIdx.x;
    if (i < n) c[i] = 0u;
}

template <bool AK, bool BKC, int EPI>
hipError_t dispatch_kind(int kind, const coda::GemmParams &p, hipStream_t s)
{
    using namespace coda;
    switch (kind) {
    case KIND_WHOLE: return launch_gemm<AK, BKC, EPI, KIND_WHOLE>(p, s);
    default: return launch_gemm<AK, BKC, EPI, KIND_RAGGED>(p, s);
    }
}

template <bool AK, bool BKC>
hipError_t dispatch_mode(int mode, int kind, const coda::GemmParams &p, hipStream_t s)
{
    using namespace coda;
    switch (mode) {
    case EPI_LINEAR: return dispatch_kind<AK, BKC, EPI_LINEAR>(kind, p, s);
    case EPI_SWIGLU_FWD: return dispatch_kind<AK, BKC, EPI_SWIGLU_FWD>(kind, p, s);
    case EPI_SWIGLU_BWD: return dispatch_kind<AK, BKC, EPI_SWIGLU_BWD>(kind, p, s);
    case EPI_RMSNORM_BWD: return dispatch_kind<AK, BKC, EPI_RMSNORM_BWD>(kind, p, s);
    default: return dispatch_kind<AK, BKC, EPI_ACCUM>(kind, p, s);
    }
}

template <bool AK, bool BKC, int EPI>
hipError_t dispatch_kind_f8(int kind, const coda::GemmParams &p, hipStream_t s)
{
    using namespace coda;
    return kind == KIND_WHOLE ? launch_gemm_f8<AK, BKC, EPI, KIND_WHOLE>(p, s) : launch_gemm_f8<AK, BKC, EPI, KIND_RAGGED>(p, s);
}

template <bool AK, bool BKC>
hipError_t dispatch_mode_f8(int mode, int kind, const coda::GemmParams &p, hipStream_t s)
{
    using namespace coda;
    switch (mode) {
    case EPI_LINEAR: return dispatch_kind_f8<AK, BKC, EPI_LINEAR>(kind, p, s);
    case EPI_SWIGLU_FWD: return dispatch_kind_f8<AK, BKC, EPI_SWIGLU_FWD>(kind, p, s);
    case EPI_SWIGLU_BWD: return dispatch_kind_f8<AK, BKC, EPI_SWIGLU_BWD>(kind, p, s);
    case EPI_RMSNORM_BWD: return dispatch_kind_f8<AK, BKC, EPI_RMSNORM_BWD>(kind, p, s);
    default: return dispatch_kind_f8<AK, BKC, EPI_ACCUM>(kind, p, s);
    }
}

// Sizes that the kernels index in 32 bits; K is rounded up to whole pairs of K-steps (64 bf16 or 128 8-bit elements) there
bool sizes_fit(int64_t M, int64_t N, int64_t K)
{
    return M >= 0 && N >= 0 && K >= 0 && M <= INT32_MAX - 256 && N <= INT32_MAX / 2 && K <= INT32_MAX - 128;
}

// coda_gemm proper (shared by the entry points that differ only in where the split-K workspace comes from).
coda_status gemm_impl(void *stream, int64_t M, int64_t N, int64_t K, const coda_mat *A, const coda_mat *B,
                      const coda_epi_op *prog, int32_t n_ops, void *workspace, size_t workspace_bytes)
{
    if (!sizes_fit(M, N, K)) return CODA_ERR_SHAPE;
    coda_status st;
    if ((st = check_operand(A, M, K)) != CODA_OK) return st;
    if ((st = check_operand(B, K, N)) != CODA_OK) return st;
    const bool f8 = A->dtype == CODA_F8E4M3 || B->dtype == CODA_F8E4M3;
    if (f8 && A->dtype != B->dtype) return CODA_ERR_DTYPE;                               // both 8-bit
    // 8-bit operands move in 16-byte chunks: 16 elements along whichever index is contiguous in memory
    if (f8 && ((K & 15) || (A->trans && (M & 15)) || (!B->trans && (N & 15)))) return CODA_ERR_SHAPE;
    if ((K & 7) || (N & 7) || (A->trans && (M & 7))) return CODA_ERR_SHAPE;
    Parsed ps;
    if ((st = parse_program(prog, n_ops, M, N, false, ps)) != CODA_OK) return st;
    if (M == 0 || N == 0) return CODA_OK;

    coda::GemmParams &p = ps.p;
    p.A = static_cast<const uint16_t *>(A->ptr);
    p.B = static_cast<const uint16_t *>(B->ptr);
    p.lda = A->ld;
    p.ldb = B->ld;
    p.M = (int)M;
    p.N = (int)N;
    p.K = (int)K;
    if (((M + coda::TILE_M - 1) / coda::TILE_M) * ((N + coda::TILE_N - 1) / coda::TILE_N) * 2 > INT32_MAX) return CODA_ERR_SHAPE;
    const int64_t k_pair = f8 ? 2 * coda::TILE_K : coda::TILE_K;   // elements of a pair of K-steps
    const int kind = ((K % k_pair) || (M % coda::TILE_M) || (N % coda::TILE_N)) ? coda::KIND_RAGGED : coda::KIND_WHOLE;
    const bool ak = !A->trans;   // A stored [M x K]: contraction index contiguous
    const bool bkc = B->trans;   // B stored [N x K]: contraction index contiguous
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e;
    const coda::DirectProgram program = ps.mode == coda::EPI_LINEAR       ? coda::DIRECT_PROG_LINEAR
                                        : ps.mode == coda::EPI_SWIGLU_FWD ? coda::DIRECT_PROG_SWIGLU_FWD
                                        : ps.mode == coda::EPI_SWIGLU_BWD ? coda::DIRECT_PROG_SWIGLU_BWD
                                        : ps.mode == coda::EPI_ACCUM      ? coda::DIRECT_PROG_ACCUM
                                                                          : coda::DIRECT_PROG_RMSNORM_BWD;
    if (ps.mode == coda::EPI_ACCUM) p.out_once = coda::gradient_once(M, N, p.ld_out * 4, reinterpret_cast<uintptr_t>(p.out));
    const bool wide = p.rowred_mode != coda::ROWRED_NONE || p.lse_max;
    const coda::Route route = coda::plan_route(M, N, K, f8, ak, bkc, program, wide, workspace != nullptr);
    if (workspace) {
        if (!aligned16(workspace)) return CODA_ERR_ALIGN;
        if (workspace_bytes < coda::splitk_bytes(route.shared)) return CODA_ERR_WORKSPACE;
    }
    if (route.kind == coda::ROUTE_DIVIDED)
        return launch_status(coda::launch_gemm_small(route.small, ps.mode, f8, ak, bkc, p, route.chain, static_cast<float *>(workspace), s));
    if (route.kind == coda::ROUTE_DIRECT)
        return launch_status(coda::launch_gemm_direct(route.tile, ps.mode, f8, ak, bkc, p, route.chain, route.rot_cols, s));
    if (route.narrow) return launch_status(coda::launch_gemm_narrow(ps.mode, p, s));
    if (route.kind == coda::ROUTE_WHOLE) p.rot_cols = route.rot_cols > 0 ? route.rot_cols : 0;
    if (route.kind == coda::ROUTE_SHARED) {
        const coda::SplitPlan &pl = route.shared;
        p.split_from = pl.first;
        p.tail_tiles = pl.tail;
        p.tail_chunks = pl.chunks;
        p.tail_pieces = pl.pieces;
        p.ws_stride = pl.stride;
        p.ws_cnt = static_cast<unsigned *>(workspace);
        p.ws_part = reinterpret_cast<float *>(static_cast<unsigned char *>(workspace) + coda::SPLITK_CNT_BYTES);
        hipLaunchKernelGGL(zero_counters_kernel, dim3(1), dim3(256), 0, s, p.ws_cnt, pl.tail);
        if ((e = hipGetLastError()) != hipSuccess) return launch_status(e);
    }
    if (f8) {
        if (ak && !bkc)
            e = dispatch_mode_f8<true, false>(ps.mode, kind, p, s);
        else if (ak && bkc)
            e = dispatch_mode_f8<true, true>(ps.mode, kind, p, s);
        else if (!ak && !bkc)
            e = dispatch_mode_f8<false, false>(ps.mode, kind, p, s);
        else
            e = dispatch_mode_f8<false, true>(ps.mode, kind, p, s);
    } else if (ak && !bkc)
        e = dispatch_mode<true, false>(ps.mode, kind, p, s);
    else if (ak && bkc)
        e = dispatch_mode<true, true>(ps.mode, kind, p, s);
    else if (!ak && !bkc)
        e = dispatch_mode<false, false>(ps.mode, kind, p, s);
    else
        e = dispatch_mode<false, true>(ps.mode, kind, p, s);
    return launch_status(e);
}

// ---- static scratch of coda_gemm_static_ws: one array per GPU, in the code object's own data, held until the process ends
constexpr size_t STATIC_WS_BYTES = coda::SPLITK_CNT_BYTES + (size_t)32 * 1024 * 1024;
static __device__ __align__(256) unsigned char scratch[STATIC_WS_BYTES];
constexpr int STATIC_WS_MAX_DEVICES = 64;
std::mutex g_scratch_mutex;
void *g_scratch_ptr[STATIC_WS_MAX_DEVICES] = {};   // device address of `scratch` on each GPU, looked up once per GPU

// Device address of the current GPU's copy of `scratch` (the array's name is only a host-side handle).
hipError_t static_scratch(void **out)
{
    int dev = -1;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    if (dev < 0 || dev >= STATIC_WS_MAX_DEVICES) return hipErrorInvalidDevice;
    std::lock_guard<std::mutex> lock(g_scratch_mutex);
    if (!g_scratch_ptr[dev]) {
        void *ptr = nullptr;
        e = hipGetSymbolAddress(&ptr, HIP_SYMBOL(scratch));
        if (e != hipSuccess) return e;
        if (!ptr) return hipErrorInvalidSymbol;
        g_scratch_ptr[dev] = ptr;
    }
    *out = g_scratch_ptr[dev];
    return hipSuccess;
}

// ---- attention ----------------------------------------------------------------------------------------------------------
constexpr int64_t MAX_ROWS = INT32_MAX - 511;              // rows of the tile behind the last are numbered in 32 bits too

// bf16 [r x c], one row a token
coda_status check_rows(const coda_mat *X, int64_t r, int64_t c)
{
    if (!X) return CODA_ERR_NULL;
    if (X->dtype != CODA_BF16) return CODA_ERR_DTYPE;
    if (X->trans || X->rows < 0 || X->rows > MAX_ROWS) return CODA_ERR_SHAPE;
    return check_operand(X, r, c);
}
bool heads_fit(int32_t heads, int32_t kv_heads, int64_t head_dim)
{
    return kv_heads > 0 && heads > 0 && heads % kv_heads == 0 && head_dim >= 8 && head_dim <= 128 && head_dim % 8 == 0 && heads * head_dim <= MAX_LD;
}
bool scale_fits(float scale) { return scale > 0.0f && scale < 0x1p127f; }        // times log2(e) it is finite

coda_status check_heads(const coda_mat *Q, const coda_mat *K, const coda_mat *V, const int32_t *seq_q, const int32_t *seq_k, int32_t n_seqs, int32_t heads,
                        int32_t kv_heads, float scale, coda::AttnParams &p)
{
    if (!Q || !K || !V) return CODA_ERR_NULL;
    if (heads <= 0 || Q->cols % heads || !heads_fit(heads, kv_heads, Q->cols / heads) || n_seqs < 0 || !scale_fits(scale)) return CODA_ERR_SHAPE;
    const int64_t D = Q->cols / heads;
    coda_status st;
    if ((st = check_rows(Q, Q->rows, heads * D)) != CODA_OK) return st;
    if ((st = check_rows(K, K->rows, kv_heads * D)) != CODA_OK) return st;
    if ((st = check_rows(V, K->rows, kv_heads * D)) != CODA_OK) return st;
    if ((!seq_k && K->rows != Q->rows) || Q->rows * (heads / kv_heads) > MAX_ROWS) return CODA_ERR_SHAPE;
    if (n_seqs > 0 && (Q->rows > 0 || K->rows > 0)) {
        if ((st = check_vec(seq_q)) != CODA_OK) return st;
        if (seq_k && !aligned4(seq_k)) return CODA_ERR_ALIGN;
    }
    p.Q = static_cast<const uint16_t *>(Q->ptr);
    p.K = static_cast<const uint16_t *>(K->ptr);
    p.V = static_cast<const uint16_t *>(V->ptr);
    p.ldq = Q->ld;
    p.ldk = K->ld;
    p.ldv = V->ld;
    p.seq_q = seq_q;
    p.seq_k = seq_k ? seq_k : seq_q;
    p.n_seqs = n_seqs;
    p.heads = heads;
    p.kv_heads = kv_heads;
    p.D = (int)D;
    p.Tq = (int)Q->rows;
    p.Tk = (int)K->rows;
    p.scale = scale;
    return CODA_OK;
}

coda_status check_cache(const coda_cache *c)
{
    if (!c) return CODA_ERR_NULL;
    if (c->pages < 0 || c->page <= 0 || (c->page & (c->page - 1)) || c->pages >= (int64_t(1) << 31) / c->page || !heads_fit(c->kv_heads, c->kv_heads, c->head_dim) ||
        (int64_t)c->page * c->kv_heads * c->head_dim >= int64_t(1) << 31)
        return CODA_ERR_SHAPE;
    return aligned16(c->k) && aligned16(c->v) ? CODA_OK : CODA_ERR_ALIGN;
}

}  // namespace

extern "C" {

coda_status coda_gemm(void *stream, int64_t M, int64_t N, int64_t K, const coda_mat *A, const coda_mat *B,
                      const coda_epi_op *prog, int32_t n_ops, void *workspace, size_t workspace_bytes)
{
    return gemm_impl(stream, M, N, K, A, B, prog, n_ops, workspace, workspace_bytes);
}

coda_status coda_gemm_static_ws(void *stream, int64_t M, int64_t N, int64_t K, const coda_mat *A, const coda_mat *B,
                                const coda_epi_op *prog, int32_t n_ops)
{
    // the size check comes first and needs no GPU: a plan beyond the static array is an error, not a silent unsplit run
    if (M < 0 || N < 0 || K < 0 || M > INT32_MAX - 256 || N > INT32_MAX / 2 || K > INT32_MAX - 128) return CODA_ERR_SHAPE;
    if (!A || !B) return CODA_ERR_NULL;
    const bool f8 = A->dtype == CODA_F8E4M3 || B->dtype == CODA_F8E4M3;
    if (coda::splitk_bytes(coda::plan_splitk(M, N, K, f8)) > STATIC_WS_BYTES) return CODA_ERR_WORKSPACE;
    void *ws = nullptr;
    const hipError_t e = static_scratch(&ws);
    if (e != hipSuccess) return launch_status(e);
    return gemm_impl(stream, M, N, K, A, B, prog, n_ops, ws, STATIC_WS_BYTES);
}

size_t coda_gemm_workspace_bytes(int64_t M, int64_t N, int64_t K, const coda_epi_op *, int32_t)
{
    if (M < 0 || N < 0 || K < 0 || M > INT32_MAX - 256 || N > INT32_MAX / 2 || K > INT32_MAX - 128) return 0;
    // the plan depends on the operand width (an 8-bit K-step covers twice the elements): report what covers both
    const size_t b16 = coda::splitk_bytes(coda::plan_splitk(M, N, K, false)), b8 = coda::splitk_bytes(coda::plan_splitk(M, N, K, true));
    return b16 > b8 ? b16 : b8;
}

int64_t coda_row_partial_blocks(int64_t N, const coda_epi_op *, int32_t)
{
    return N <= 0 ? 0 : (N + coda::TILE_N - 1) / coda::TILE_N;
}

coda_status coda_lse_finalize(void *stream, const float *pmax, const float *psum, int64_t M, int64_t nblk, const float *ztgt,
                              float *lse_out, float *loss_out)
{
    if (M < 0 || nblk <= 0) return CODA_ERR_SHAPE;
    if (!pmax || !psum || (!lse_out && !loss_out) || (loss_out && !ztgt)) return CODA_ERR_NULL;
    if (M == 0) return CODA_OK;
    if (!aligned4(pmax) || !aligned4(psum) || !aligned4(ztgt) || !aligned4(lse_out) || !aligned4(loss_out)) return CODA_ERR_ALIGN;
    return launch_status(coda::launch_lse_finalize(static_cast<hipStream_t>(stream), pmax, psum, M, nblk, ztgt, lse_out, loss_out));
}

int64_t coda_col_partial_blocks(int64_t M)
{
    return M <= 0 ? 0 : (M + coda::TILE_M - 1) / coda::TILE_M;
}

coda_status coda_col_finalize(void *stream, const float *partials, int64_t N, int64_t nblk, float *out)
{
    if (N < 0 || nblk < 0) return CODA_ERR_SHAPE;
    if (!out) return CODA_ERR_NULL;
    if (N == 0) return CODA_OK;
    if (nblk > 0 && !partials) return CODA_ERR_NULL;
    if (!aligned4(partials) || !aligned4(out)) return CODA_ERR_ALIGN;
    return launch_status(coda::launch_col_finalize(static_cast<hipStream_t>(stream), partials, N, nblk, out));
}

coda_status coda_row_finalize(void *stream, const float *partials, int64_t M, int64_t nblk, float *sum_out,
                              float *rstd_out, int64_t d, float eps)
{
    if (M < 0 || nblk < 0 || d <= 0) return CODA_ERR_SHAPE;
    if (!sum_out && !rstd_out) return CODA_ERR_NULL;
    if (M == 0) return CODA_OK;
    if (nblk > 0 && !partials) return CODA_ERR_NULL;
    if (!aligned4(partials) || !aligned4(sum_out) || !aligned4(rstd_out)) return CODA_ERR_ALIGN;
    return launch_status(coda::launch_row_finalize(static_cast<hipStream_t>(stream), partials, M, nblk, sum_out,
                                                   rstd_out, 1.0f / (float)d, eps));
}

coda_status coda_row_sumsq(void *stream, const coda_mat *X, float *sum_out)
{
    if (!X || !sum_out) return CODA_ERR_NULL;
    if (X->dtype != CODA_BF16) return CODA_ERR_DTYPE;
    if (X->trans || X->rows < 0 || X->cols < 0 || X->ld < X->cols || (X->cols & 7)) return CODA_ERR_SHAPE;
    if (X->rows == 0) return CODA_OK;
    if (!X->ptr) return CODA_ERR_NULL;
    if (!aligned16(X->ptr) || (X->ld & 7) || !aligned4(sum_out)) return CODA_ERR_ALIGN;
    return launch_status(coda::launch_row_sumsq(static_cast<hipStream_t>(stream), static_cast<const uint16_t *>(X->ptr),
                                                X->rows, X->cols, X->ld, sum_out));
}

coda_status coda_fold_gamma(void *stream, const coda_mat *W, const float *gamma, void *W_out, int64_t ld_out)
{
    if (!W || !gamma || !W_out) return CODA_ERR_NULL;
    if (W->dtype != CODA_BF16) return CODA_ERR_DTYPE;
    if (W->trans || W->rows < 0 || W->cols < 0 || W->ld < W->cols || ld_out < W->cols || (W->cols & 7))
        return CODA_ERR_SHAPE;
    if (W->rows == 0 || W->cols == 0) return CODA_OK;
    if (!W->ptr) return CODA_ERR_NULL;
    if (!aligned16(W->ptr) || !aligned16(W_out) || (W->ld & 7) || (ld_out & 7) || !aligned4(gamma)) return CODA_ERR_ALIGN;
    return launch_status(coda::launch_fold_gamma(static_cast<hipStream_t>(stream), static_cast<const uint16_t *>(W->ptr),
                                                 W->rows, W->cols, W->ld, gamma, static_cast<uint16_t *>(W_out), ld_out));
}

coda_status coda_interleave_pairs(void *stream, const coda_mat *Wa, const coda_mat *Wb, void *W_out, int64_t ld_out)
{
    if (!Wa || !Wb || !W_out) return CODA_ERR_NULL;
    if (Wa->dtype != CODA_BF16 || Wb->dtype != CODA_BF16) return CODA_ERR_DTYPE;
    if (Wa->trans || Wb->trans || Wa->rows != Wb->rows || Wa->cols != Wb->cols || Wa->rows < 0 || Wa->cols < 0 ||
        Wa->ld < Wa->cols || Wb->ld < Wb->cols || ld_out < 2 * Wa->cols || (Wa->cols & 7))
        return CODA_ERR_SHAPE;
    if (Wa->rows == 0 || Wa->cols == 0) return CODA_OK;
    if (!Wa->ptr || !Wb->ptr) return CODA_ERR_NULL;
    if (!aligned16(Wa->ptr) || !aligned16(Wb->ptr) || !aligned16(W_out) || (Wa->ld & 7) || (Wb->ld & 7) || (ld_out & 7))
        return CODA_ERR_ALIGN;
    return launch_status(coda::launch_interleave_pairs(
        static_cast<hipStream_t>(stream), static_cast<const uint16_t *>(Wa->ptr), Wa->ld,
        static_cast<const uint16_t *>(Wb->ptr), Wb->ld, Wa->rows, Wa->cols, static_cast<uint16_t *>(W_out), ld_out));
}

coda_status coda_quantize(void *stream, const coda_mat *X, int32_t square, void *codes, int64_t ld_codes, void *scales, int64_t ld_scales,
                          void *scales_t, int64_t ld_scales_t)
{
    if (!X) return CODA_ERR_NULL;
    if (X->dtype != CODA_BF16) return CODA_ERR_DTYPE;
    if (X->trans || X->rows < 0 || X->cols < 0 || X->rows > INT32_MAX || X->ld < X->cols || X->ld > MAX_LD || (X->cols & 7)) return CODA_ERR_SHAPE;
    if (!square && scales_t) return CODA_ERR_SHAPE;        // scales along the columns are those of square blocks
    if (X->rows == 0 || X->cols == 0) return CODA_OK;
    if (!X->ptr) return CODA_ERR_NULL;
    if (!aligned16(X->ptr) || (X->ld & 7)) return CODA_ERR_ALIGN;
    coda_status st;
    if ((st = check_q8_tile(codes, ld_codes, X->cols, scales, ld_scales, X->rows)) != CODA_OK) return st;
    if (scales_t && (st = check_scales(scales_t, ld_scales_t, X->cols)) != CODA_OK) return st;
    if (!launch_fits(coda::quantize_workgroups(X->rows, X->cols, square != 0), 256)) return CODA_ERR_SHAPE;
    return launch_status(coda::launch_quantize(static_cast<hipStream_t>(stream), static_cast<const uint16_t *>(X->ptr), X->rows, X->cols, X->ld, square != 0,
                                               static_cast<uint8_t *>(codes), ld_codes, static_cast<uint8_t *>(scales), ld_scales,
                                               static_cast<uint8_t *>(scales_t), ld_scales_t));
}

coda_status coda_dequantize(void *stream, const coda_mat *Q, const void *scales, int64_t ld_scales, void *out, int64_t ld_out)
{
    if (!Q) return CODA_ERR_NULL;
    if (Q->dtype != CODA_F8E4M3) return CODA_ERR_DTYPE;
    if (Q->trans || Q->rows < 0 || Q->cols < 0 || Q->rows > INT32_MAX || (Q->cols & 7)) return CODA_ERR_SHAPE;
    if (Q->rows == 0 || Q->cols == 0) return CODA_OK;
    coda_status st;
    if ((st = check_q8_tile(Q->ptr, Q->ld, Q->cols, scales, ld_scales, Q->rows)) != CODA_OK) return st;
    if ((st = check_tile(out, ld_out, Q->cols)) != CODA_OK) return st;
    if (!launch_fits(coda::dequantize_workgroups(Q->rows, Q->cols), 256)) return CODA_ERR_SHAPE;
    return launch_status(coda::launch_dequantize(static_cast<hipStream_t>(stream), static_cast<const uint8_t *>(Q->ptr), Q->rows, Q->cols, Q->ld,
                                                 static_cast<const uint8_t *>(scales), ld_scales, static_cast<uint16_t *>(out), ld_out));
}

size_t coda_gemm_scaled_workspace_bytes(int64_t M, int64_t N, int64_t K)
{
    if (!sizes_fit(M, N, K) || M == 0 || N == 0) return 0;
    return coda::scaled_bytes(coda::plan_scaled(M, N, K, true, false), M, N);
}

coda_status coda_gemm_scaled(void *stream, int64_t M, int64_t N, int64_t K, const coda_mat *A, const void *scales_a, int64_t ld_scales_a,
                             const coda_mat *B, const void *scales_b, int64_t ld_scales_b, const coda_epi_op *prog, int32_t n_ops, void *workspace,
                             size_t workspace_bytes)
{
    if (!sizes_fit(M, N, K)) return CODA_ERR_SHAPE;
    coda_status st;
    if ((st = check_operand(A, M, K)) != CODA_OK) return st;
    if ((st = check_operand(B, K, N)) != CODA_OK) return st;
    if (A->dtype != CODA_F8E4M3 || B->dtype != CODA_F8E4M3) return CODA_ERR_DTYPE;
    if (A->trans || (K & 15) || (N & 15)) return CODA_ERR_SHAPE;
    if (K > 0) {
        if (M > 0 && (st = check_scales(scales_a, ld_scales_a, M)) != CODA_OK) return st;
        if (N > 0 && (st = check_scales(scales_b, ld_scales_b, N)) != CODA_OK) return st;
    }
    Parsed ps;
    if ((st = parse_program(prog, n_ops, M, N, true, ps)) != CODA_OK) return st;
    if (M == 0 || N == 0) return CODA_OK;
    const bool narrow = !ps.q8 && B->trans && ((ps.mode == coda::EPI_LINEAR && ps.p.rowred_mode == coda::ROWRED_NONE && !ps.p.lse_max) || ps.mode == coda::EPI_SWIGLU_FWD);
    coda::ScaledPlan plan = coda::plan_scaled(M, N, K, workspace != nullptr, narrow);
    if (workspace) {
        if (!aligned16(workspace)) return CODA_ERR_ALIGN;
        if (workspace_bytes < coda_gemm_scaled_workspace_bytes(M, N, K)) return CODA_ERR_WORKSPACE;
    }
    if (!plan.few && plan.nsplit == 0 && !ps.q8 && ps.mode == coda::EPI_RMSNORM_BWD) plan.bm = coda::TILE_M;      // its column partials are per 256 rows
    if (!plan.few && !launch_fits(((M + plan.bm - 1) / plan.bm) * ((N + plan.bn - 1) / plan.bn) * (plan.nsplit ? plan.nsplit : 1), 512)) return CODA_ERR_SHAPE;
    ps.p.M = (int)M;
    ps.p.N = (int)N;
    ps.p.K = (int)K;
    coda::ScaledParams p{};
    p.A = static_cast<const unsigned char *>(A->ptr);
    p.B = static_cast<const unsigned char *>(B->ptr);
    p.sa = static_cast<const unsigned char *>(scales_a);
    p.sb = static_cast<const unsigned char *>(scales_b);
    p.lda = A->ld;
    p.ldb = B->ld;
    p.ld_sa = ld_scales_a;
    p.ld_sb = ld_scales_b;
    p.M = (int)M;
    p.N = (int)N;
    p.K = (int)K;
    p.part = static_cast<float *>(workspace);
    return launch_status(coda::launch_gemm_scaled(plan, ps.mode, ps.q8, B->trans != 0, ps.p, ps.q, p, static_cast<hipStream_t>(stream)));
}

size_t coda_grad_scaled_workspace_bytes(int64_t M, int64_t N, int64_t K)
{
    if (!sizes_fit(M, N, K) || M == 0 || N == 0) return 0;
    return coda::grad_bytes(coda::plan_grad(M, N, K, true), M, N);
}

coda_status coda_grad_scaled(void *stream, int64_t M, int64_t N, int64_t K, const coda_mat *A, const void *scales_a, int64_t ld_scales_a,
                             const coda_mat *B, const void *scales_b, int64_t ld_scales_b, float *G, int64_t ld_g, void *workspace, size_t workspace_bytes)
{
    if (!sizes_fit(M, N, K)) return CODA_ERR_SHAPE;
    coda_status st;
    if ((st = check_operand(A, M, K)) != CODA_OK) return st;
    if ((st = check_operand(B, K, N)) != CODA_OK) return st;
    if (A->dtype != CODA_F8E4M3) return CODA_ERR_DTYPE;
    const bool b8 = B->dtype == CODA_F8E4M3;
    if (!A->trans || B->trans || (M & 15) || (N & (b8 ? 15 : 7))) return CODA_ERR_SHAPE;
    if (!b8 && scales_b) return CODA_ERR_DTYPE;            // a bf16 operand has no scales
    if (K > 0) {
        if (M > 0 && (st = check_scales(scales_a, ld_scales_a, K)) != CODA_OK) return st;
        if (b8 && N > 0 && (st = check_scales(scales_b, ld_scales_b, K)) != CODA_OK) return st;
    }
    if (M == 0 || N == 0) return CODA_OK;
    if (!G) return CODA_ERR_NULL;
    if (ld_g < N || ld_g > MAX_LD) return CODA_ERR_SHAPE;
    if (!aligned16(G) || (ld_g & 3)) return CODA_ERR_ALIGN;
    const coda::GradPlan plan = coda::plan_grad(M, N, K, workspace != nullptr);
    if (workspace) {
        if (!aligned16(workspace)) return CODA_ERR_ALIGN;
        if (workspace_bytes < coda::grad_bytes(plan, M, N)) return CODA_ERR_WORKSPACE;
    }
    if (!launch_fits(((M + plan.tile - 1) / plan.tile) * ((N + plan.tile - 1) / plan.tile) * plan.nsplit, plan.tile * 2)) return CODA_ERR_SHAPE;
    coda::GemmParams g{};
    g.M = (int)M;
    g.N = (int)N;
    g.K = (int)K;
    g.out = G;
    g.ld_out = ld_g;
    g.out_once = coda::gradient_once(M, N, ld_g * 4, reinterpret_cast<uintptr_t>(G));
    coda::GradParams p{};
    p.A = static_cast<const unsigned char *>(A->ptr);
    p.B = static_cast<const unsigned char *>(B->ptr);
    p.sa = static_cast<const unsigned char *>(scales_a);
    p.sb = static_cast<const unsigned char *>(scales_b);
    p.lda = A->ld;
    p.ldb = B->ld * (b8 ? 1 : 2);
    p.ld_sa = ld_scales_a;
    p.ld_sb = ld_scales_b;
    p.M = (int)M;
    p.N = (int)N;
    p.K = (int)K;
    p.part = static_cast<float *>(workspace);
    return launch_status(coda::launch_grad_scaled(plan, b8, g, p, static_cast<hipStream_t>(stream)));
}

coda_status coda_attention(void *stream, const coda_mat *Q, const coda_mat *K, const coda_mat *V, const int32_t *seq_q, const int32_t *seq_k, int32_t n_seqs,
                           int32_t heads, int32_t kv_heads, float scale, int32_t causal, void *out, int64_t ld_out, float *lse)
{
    coda::AttnParams p{};
    coda_status st;
    if ((st = check_heads(Q, K, V, seq_q, seq_k, n_seqs, heads, kv_heads, scale, p)) != CODA_OK) return st;
    p.causal = causal != 0;
    if (p.Tq == 0 || n_seqs == 0) return CODA_OK;
    if ((st = check_tile(out, ld_out, Q->cols)) != CODA_OK) return st;
    if (lse && !aligned4(lse)) return CODA_ERR_ALIGN;
    p.out = static_cast<uint16_t *>(out);
    p.ldo = ld_out;
    p.lse = lse;
    if (!launch_fits(coda::attn_workgroups(p), 256)) return CODA_ERR_SHAPE;
    return launch_status(coda::launch_attention(p, static_cast<hipStream_t>(stream)));
}

size_t coda_attention_bwd_workspace_bytes(int64_t Tq, int64_t Tk, int32_t n_seqs, int32_t heads, int32_t kv_heads, int32_t head_dim)
{
    if (Tq <= 0 || Tq > MAX_ROWS || Tk < 0 || n_seqs <= 0 || !heads_fit(heads, kv_heads, head_dim)) return 0;
    return coda::bwd_bytes(Tq, heads);
}

coda_status coda_attention_bwd(void *stream, const coda_mat *Q, const coda_mat *K, const coda_mat *V, const coda_mat *O, const coda_mat *dO, const float *lse,
                               const int32_t *seq_q, const int32_t *seq_k, int32_t n_seqs, int32_t heads, int32_t kv_heads, float scale, int32_t causal,
                               const coda_rope *rope, void *dQ, int64_t ld_dq, void *dK, int64_t ld_dk, void *dV, int64_t ld_dv, void *workspace,
                               size_t workspace_bytes)
{
    coda::BwdParams p{};
    coda_status st;
    if ((st = check_heads(Q, K, V, seq_q, seq_k, n_seqs, heads, kv_heads, scale, p.f)) != CODA_OK) return st;
    p.f.causal = causal != 0;
    if (!O || !dO) return CODA_ERR_NULL;
    if ((st = check_rows(O, Q->rows, Q->cols)) != CODA_OK) return st;
    if ((st = check_rows(dO, Q->rows, Q->cols)) != CODA_OK) return st;
    if ((p.f.Tq == 0 && p.f.Tk == 0) || n_seqs == 0) return CODA_OK;
    if (p.f.Tq > 0) {
        if ((st = check_vec(lse)) != CODA_OK) return st;
        if ((st = check_tile(dQ, ld_dq, Q->cols)) != CODA_OK) return st;
    }
    if (p.f.Tk > 0 && ((st = check_tile(dK, ld_dk, K->cols)) != CODA_OK || (st = check_tile(dV, ld_dv, K->cols)) != CODA_OK)) return st;
    if (rope) {
        if (!rope->cos || !rope->sin || (p.f.Tq > 0 && !rope->pos_q) || (p.f.Tk > 0 && !rope->pos_k)) return CODA_ERR_NULL;
        if (rope->rows < 1 || rope->rows > INT32_MAX / (p.f.D / 2)) return CODA_ERR_SHAPE;
        if ((reinterpret_cast<uintptr_t>(rope->cos) & 7u) || (reinterpret_cast<uintptr_t>(rope->sin) & 7u) || !aligned4(rope->pos_q) || !aligned4(rope->pos_k))
            return CODA_ERR_ALIGN;
        p.cos = rope->cos;
        p.sin = rope->sin;
        p.pos_q = rope->pos_q;
        p.pos_k = rope->pos_k;
        p.rope_rows = (int)rope->rows;
    }
    if (p.f.Tq > 0) {
        if (!workspace) return CODA_ERR_NULL;
        if (!aligned16(workspace)) return CODA_ERR_ALIGN;
        if (workspace_bytes < coda::bwd_bytes(p.f.Tq, heads)) return CODA_ERR_WORKSPACE;
    }
    p.f.lse = const_cast<float *>(lse);
    p.O = static_cast<const uint16_t *>(O->ptr);
    p.dO = static_cast<const uint16_t *>(dO->ptr);
    p.ldo = O->ld;
    p.lddo = dO->ld;
    p.dQ = static_cast<uint16_t *>(dQ);
    p.dK = static_cast<uint16_t *>(dK);
    p.dV = static_cast<uint16_t *>(dV);
    p.lddq = ld_dq;
    p.lddk = ld_dk;
    p.lddv = ld_dv;
    p.stats = static_cast<float *>(workspace);
    if (!launch_fits(coda::bwd_workgroups(p), 256)) return CODA_ERR_SHAPE;
    return launch_status(coda::launch_attention_bwd(p, static_cast<hipStream_t>(stream)));
}

coda_status coda_cache_store(void *stream, const coda_mat *K, const coda_mat *V, const int32_t *slots, const coda_cache *cache)
{
    coda_status st;
    if ((st = check_cache(cache)) != CODA_OK) return st;
    const int64_t cols = (int64_t)cache->kv_heads * cache->head_dim;
    if (!K || !V) return CODA_ERR_NULL;
    if ((st = check_rows(K, K->rows, cols)) != CODA_OK) return st;
    if ((st = check_rows(V, K->rows, cols)) != CODA_OK) return st;
    if (K->rows == 0) return CODA_OK;
    if ((st = check_vec(slots)) != CODA_OK) return st;
    if (cache->pages == 0) return CODA_OK;                 // no slot is one of the cache's
    if (!cache->k || !cache->v) return CODA_ERR_NULL;
    if (!launch_fits(coda::cache_store_workgroups(K->rows, (int)cols), 256)) return CODA_ERR_SHAPE;
    return launch_status(coda::launch_cache_store(static_cast<const uint16_t *>(K->ptr), K->ld, static_cast<const uint16_t *>(V->ptr), V->ld, K->rows, (int)cols,
                                                  cache->head_dim, slots, static_cast<uint16_t *>(cache->k), static_cast<uint16_t *>(cache->v),
                                                  cache->pages * cache->page, __builtin_ctz((unsigned)cache->page), static_cast<hipStream_t>(stream)));
}

size_t coda_attention_cached_workspace_bytes(int64_t Tq, int32_t n_seqs, int32_t heads, int32_t kv_heads, int32_t head_dim)
{
    if (Tq <= 0 || Tq > MAX_ROWS || n_seqs <= 0 || !heads_fit(heads, kv_heads, head_dim)) return 0;
    return coda::cached_bytes(Tq, n_seqs, heads, kv_heads, head_dim);
}

coda_status coda_attention_cached(void *stream, const coda_mat *Q, const coda_cache *cache, const int32_t *table, int64_t ld_table, int64_t table_pages,
                                  const int32_t *lens, const int32_t *seq_q, int32_t n_seqs, int32_t heads, float scale, const uint64_t *tree, void *out,
                                  int64_t ld_out, float *lse, void *workspace, size_t workspace_bytes)
{
    coda_status st;
    if ((st = check_cache(cache)) != CODA_OK) return st;
    if (!Q) return CODA_ERR_NULL;
    if (!heads_fit(heads, cache->kv_heads, cache->head_dim) || n_seqs < 0 || !scale_fits(scale)) return CODA_ERR_SHAPE;
    if ((st = check_rows(Q, Q->rows, (int64_t)heads * cache->head_dim)) != CODA_OK) return st;
    const int group = heads / cache->kv_heads;
    if (Q->rows * group > MAX_ROWS || table_pages < 0 || ld_table < table_pages || table_pages > (int64_t(1) << 30) / cache->page) return CODA_ERR_SHAPE;
    if (Q->rows == 0 || n_seqs == 0) return CODA_OK;
    if ((st = check_vec(lens)) != CODA_OK || (st = check_vec(seq_q)) != CODA_OK) return st;
    const int64_t capacity = cache->pages ? table_pages * cache->page : 0;
    if (capacity) {
        if (!cache->k || !cache->v) return CODA_ERR_NULL;
        if ((st = check_vec(table)) != CODA_OK) return st;
    }
    if ((st = check_tile(out, ld_out, Q->cols)) != CODA_OK) return st;
    if (lse && !aligned4(lse)) return CODA_ERR_ALIGN;
    if (tree && (reinterpret_cast<uintptr_t>(tree) & 7u)) return CODA_ERR_ALIGN;
    if (!workspace) return CODA_ERR_NULL;
    if (!aligned16(workspace)) return CODA_ERR_ALIGN;
    if (workspace_bytes < coda::cached_bytes(Q->rows, n_seqs, heads, cache->kv_heads, cache->head_dim)) return CODA_ERR_WORKSPACE;
    coda::CachedParams p{};
    p.Q = static_cast<const uint16_t *>(Q->ptr);
    p.K = static_cast<const uint16_t *>(cache->k);
    p.V = static_cast<const uint16_t *>(cache->v);
    p.ldq = Q->ld;
    p.ld_table = ld_table;
    p.table = table;
    p.lens = lens;
    p.seq_q = seq_q;
    p.tree = tree;
    p.n_seqs = n_seqs;
    p.kv_heads = cache->kv_heads;
    p.group = group;
    p.D = cache->head_dim;
    p.Tq = (int)Q->rows;
    p.page_bits = __builtin_ctz((unsigned)cache->page);
    p.pages = (int)cache->pages;
    p.page_mask = (uint32_t)cache->page - 1;
    p.page_bytes = (uint32_t)((int64_t)cache->page * cache->kv_heads * cache->head_dim * 2);
    p.capacity = (int)capacity;
    p.scale = scale;
    p.out = static_cast<uint16_t *>(out);
    p.ldo = ld_out;
    p.lse = lse;
    p.part = static_cast<float *>(workspace);
    if (!launch_fits(coda::cached_workgroups(p), 256)) return CODA_ERR_SHAPE;
    return launch_status(coda::launch_attention_cached(p, static_cast<hipStream_t>(stream)));
}

const char *coda_status_string(coda_status s)
{
    switch (s) {
    case CODA_OK: return "ok";
    case CODA_ERR_NULL: return "required pointer is null";
    case CODA_ERR_SHAPE: return "unsupported or inconsistent shape";
    case CODA_ERR_ALIGN: return "pointer or leading dimension misaligned";
    case CODA_ERR_DTYPE: return "unsupported dtype";
    case CODA_ERR_PROGRAM: return "unsupported epilogue program";
    case CODA_ERR_WORKSPACE: return "workspace too small";
    case CODA_ERR_LAUNCH: return "HIP launch error";
    }
    return "unknown status";
}

int coda_last_hip_error(void) { return g_last_hip_error; }

}  // extern "C"
