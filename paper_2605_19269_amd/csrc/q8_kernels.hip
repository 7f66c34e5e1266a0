// q8_kernels.hip -- bf16 -> codes and scales of blocks of 128, and back.  Both are bound by HBM: three bytes an element.
#include "q8.hpp"

namespace coda {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;

// Largest finite magnitude among bf16 values, two at a time as whole numbers: the bits of magnitudes are in their order, those of infinities
// and NaN from 0x7f80 on.  Where there are any, they are taken out and the maximum found again.
template <int N>
static __device__ __forceinline__ float largest_bf16(const u32x4 (&v)[N])
{
    u16x2 m = {0, 0};
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, v[i][e] & 0x7fff7fffu));
    uint32_t top = m[0] > m[1] ? m[0] : m[1];
    if (__ballot(top >= 0x7f80u)) {                      // a wave's branch: seldom taken
        top = 0;
        for (int i = 0; i < N; ++i)
            for (int e = 0; e < 4; ++e) {
                const uint32_t a = v[i][e] & 0x7fffu, b = (v[i][e] >> 16) & 0x7fffu;
                top = a < 0x7f80u && a > top ? a : top;
                top = b < 0x7f80u && b > top ? b : top;
            }
    }
    return __builtin_bit_cast(float, top << 16);
}
template <int CTRL>
static __device__ __forceinline__ float dpp_max(float m)
{
    return fmaxf(m, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, m), CTRL, 0xf, 0xf, false)));
}
// The maximum over the sixteen lanes of a DPP row, in all of them: pairs, quads, halves, the row
static __device__ __forceinline__ float max16(float m)
{
    m = dpp_max<0xB1>(m);        // quad_perm 1 0 3 2
    m = dpp_max<0x4E>(m);        // quad_perm 2 3 0 1
    m = dpp_max<0x141>(m);       // row_half_mirror
    return dpp_max<0x140>(m);    // row_mirror
}
static __device__ __forceinline__ u32x2 codes8(u32x4 v, float scale)
{
    u32x2 o;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const uint32_t a = v[2 * e], b = v[2 * e + 1];
        q8_pair w = {0, 0};
        w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(bf16x2, a), scale, false);
        o[e] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(bf16x2, b), scale, true));
    }
    return o;
}

// Blocks of 1 x 128: sixteen lanes a row, eight elements a lane, four rows a wave and pass.  The scales of consecutive rows lie
// side by side, so a wave takes 4 PASSES consecutive rows and stores their bytes at once.
template <int PASSES>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const uint16_t *__restrict__ X, int64_t R, int64_t C, int64_t ld, int cblocks,
                                                            uint8_t *__restrict__ q, int64_t ldq, uint8_t *__restrict__ sc, int64_t lds)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, c = lane & 15;
    const int64_t kb = blockIdx.x % (unsigned)cblocks, r0 = ((int64_t)(blockIdx.x / (unsigned)cblocks) * 4 + wave) * (4 * PASSES);
    const int64_t col = kb * Q8_BLOCK + c * 8;
    if (r0 >= R) return;
    u32x4 v[PASSES];
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int64_t r = r0 + p * 4 + g;
        v[p] = u32x4{0u, 0u, 0u, 0u};
        if (r < R && col < C) v[p] = *reinterpret_cast<const u32x4 *>(X + r * ld + col);
    }
    uint32_t word[PASSES];
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int64_t r = r0 + p * 4 + g;
        const u32x4 one[1] = {v[p]};
        const uint32_t byte = q8_scale_byte(max16(largest_bf16(one)));
        if (r < R && col < C) *reinterpret_cast<u32x2 *>(q + r * ldq + col) = codes8(v[p], q8_scale(byte));
        word[p] = (uint32_t)__builtin_amdgcn_readlane((int)byte, 0) | (uint32_t)__builtin_amdgcn_readlane((int)byte, 16) << 8 |
                  (uint32_t)__builtin_amdgcn_readlane((int)byte, 32) << 16 | (uint32_t)__builtin_amdgcn_readlane((int)byte, 48) << 24;
    }
    uint8_t *to = sc + kb * lds + r0;
    if (r0 + 4 * PASSES <= R) {
        if (lane < PASSES) {
            uint32_t w = word[0];
#pragma unroll
            for (int p = 1; p < PASSES; ++p) w = lane == p ? word[p] : w;
            reinterpret_cast<uint32_t *>(to)[lane] = w;
        }
    } else if (lane < 4 * PASSES && r0 + lane < R) {
        uint32_t w = word[0];
#pragma unroll
        for (int p = 1; p < PASSES; ++p) w = lane >> 2 == p ? word[p] : w;
        to[lane] = (uint8_t)(w >> (8 * (lane & 3)));
    }
}

// Blocks of 128 x 128, a workgroup each; the scale goes to every row of the block and, for contractions along the rows, to every column.
__global__ __launch_bounds__(256) void quantize_square_kernel(const uint16_t *__restrict__ X, int64_t R, int64_t C, int64_t ld, int cblocks,
                                                              uint8_t *__restrict__ q, int64_t ldq, uint8_t *__restrict__ sc, int64_t lds,
                                                              uint8_t *__restrict__ sct, int64_t ldst)
{
    __shared__ float largest[4];
    const int tid = threadIdx.x, lane = tid & 63, rl = tid >> 4, c = tid & 15;
    const int64_t kb = blockIdx.x % (unsigned)cblocks, rb = blockIdx.x / (unsigned)cblocks, r0 = rb * Q8_BLOCK, c0 = kb * Q8_BLOCK, col = c0 + c * 8;
    u32x4 v[8];
#pragma unroll
    for (int p = 0; p < 8; ++p) {
        const int64_t r = r0 + p * 16 + rl;
        v[p] = u32x4{0u, 0u, 0u, 0u};
        if (r < R && col < C) v[p] = *reinterpret_cast<const u32x4 *>(X + r * ld + col);
    }
    float m = max16(largest_bf16(v));
    m = fmaxf(m, __shfl_xor(m, 16, 64));
    m = fmaxf(m, __shfl_xor(m, 32, 64));
    if (lane == 0) largest[tid >> 6] = m;
    __syncthreads();
    const uint32_t byte = q8_scale_byte(fmaxf(fmaxf(largest[0], largest[1]), fmaxf(largest[2], largest[3])));
    const float scale = q8_scale(byte);
#pragma unroll
    for (int p = 0; p < 8; ++p) {
        const int64_t r = r0 + p * 16 + rl;
        if (r < R && col < C) *reinterpret_cast<u32x2 *>(q + r * ldq + col) = codes8(v[p], scale);
    }
    if (tid < Q8_BLOCK) {
        if (r0 + tid < R) sc[kb * lds + r0 + tid] = (uint8_t)byte;
    } else if (sct) {
        const int j = tid - Q8_BLOCK;
        if (c0 + j < C) sct[rb * ldst + c0 + j] = (uint8_t)byte;
    }
}

// Codes -> bf16: sixteen lanes a row of a block, eight codes a lane, so that a store covers whole lines (sixteen codes a lane, two stores at a stride: 16384 x 4096
// 47.9 us, 38.0 as here).  Every value is a bf16 value (E4M3 has three bits behind the point) unless it lies below 2^-133.  Plain stores: past the caches the kernel
// alone takes 30.7 us, but with a reader of its output behind it 64.1 instead of 54.0 (and quantising 30.8 instead of 36.0, with a product behind it 254 and 247).
__global__ __launch_bounds__(256) void dequantize_kernel(const uint8_t *__restrict__ q, int64_t R, int64_t C, int64_t ldq, int cblocks,
                                                         const uint8_t *__restrict__ sc, int64_t lds, uint16_t *__restrict__ out, int64_t ld_out)
{
    const int64_t kb = blockIdx.x % (unsigned)cblocks, r0 = (int64_t)(blockIdx.x / (unsigned)cblocks) * (16 * RESTORE_PASSES) + (threadIdx.x >> 4);
    const int64_t col = kb * Q8_BLOCK + (threadIdx.x & 15) * 8;
    if (col >= C) return;                                  // C is a multiple of 8
    u32x2 v[RESTORE_PASSES];
    uint32_t b[RESTORE_PASSES];
#pragma unroll
    for (int p = 0; p < RESTORE_PASSES; ++p) {
        const int64_t r = r0 + p * 16;
        v[p] = u32x2{0u, 0u};
        b[p] = 0;
        if (r >= R) continue;
        v[p] = *reinterpret_cast<const u32x2 *>(q + r * ldq + col);
        b[p] = sc[kb * lds + r];
    }
#pragma unroll
    for (int p = 0; p < RESTORE_PASSES; ++p) {
        const int64_t r = r0 + p * 16;
        if (r >= R) continue;
        const float s = q8_scale(b[p]);
        u32x4 o;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const uint32_t w = v[p][e];
            o[2 * e] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, false));
            o[2 * e + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, true));
        }
        *reinterpret_cast<u32x4 *>(out + r * ld_out + col) = o;
    }
}

hipError_t launch_quantize(hipStream_t s, const uint16_t *X, int64_t R, int64_t C, int64_t ld, bool square, uint8_t *q, int64_t ldq, uint8_t *sc,
                           int64_t lds, uint8_t *sct, int64_t ldst)
{
    const int cb = (int)((C + Q8_BLOCK - 1) / Q8_BLOCK);
    const dim3 grid((unsigned)quantize_workgroups(R, C, square));
    if (square) hipLaunchKernelGGL(quantize_square_kernel, grid, dim3(256), 0, s, X, R, C, ld, cb, q, ldq, sc, lds, sct, ldst);
    else if (R * cb <= 64 * 1024) hipLaunchKernelGGL((quantize_rows_kernel<1>), grid, dim3(256), 0, s, X, R, C, ld, cb, q, ldq, sc, lds);
    else hipLaunchKernelGGL((quantize_rows_kernel<QUANTIZE_PASSES>), grid, dim3(256), 0, s, X, R, C, ld, cb, q, ldq, sc, lds);
    return hipGetLastError();
}

hipError_t launch_dequantize(hipStream_t s, const uint8_t *q, int64_t R, int64_t C, int64_t ldq, const uint8_t *sc, int64_t lds, uint16_t *out,
                             int64_t ld_out)
{
    const int cb = (int)((C + Q8_BLOCK - 1) / Q8_BLOCK);
    hipLaunchKernelGGL(dequantize_kernel, dim3((unsigned)dequantize_workgroups(R, C)), dim3(256), 0, s, q, R, C, ldq, cb, sc, lds, out, ld_out);
    return hipGetLastError();
}

}  // namespace coda
