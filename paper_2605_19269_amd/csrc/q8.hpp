// q8.hpp -- the 8-bit format with a scale for each block of 128, and the host launchers of its kernels.
//
// A code is an OCP E4M3 byte, a scale an E8M0 byte: 2^(byte - 127), 255 NaN.  Powers of two because the matrix instruction of gfx950
// (v_mfma_scale_f32_32x32x64_f8f6f4) takes them with the codes and multiplies by them for nothing: 3.89 PFLOP/s in a register
// loop on random finite codes, 3.59 without scales, and no product is rounded.  fp32 scales would cost an fp32
// multiply-add for every accumulator and block, and a second set of accumulators.
//
// The scale of a block is the least power of two, no less than 2^-126, with |x| <= 448 times it for every finite element: with the
// largest |x| = 1.m 2^(E - 127) the byte is E - 8, one more where 1.m > 1.75 (448 = 1.75 2^8).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace coda {

constexpr int Q8_BLOCK = 128;

__device__ __forceinline__ uint32_t q8_scale_byte(float amax)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, amax);
    const int e = (int)(b >> 23) - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
    return (uint32_t)(e < 1 ? 1 : e);                      // at most 247
}
// 2^(127 - byte) of a byte that q8_scale_byte made
__device__ __forceinline__ float q8_inverse(uint32_t byte) { return __builtin_bit_cast(float, (254u - byte) << 23); }
// 2^(byte - 127) of any byte
__device__ __forceinline__ float q8_scale(uint32_t byte)
{
    return __builtin_bit_cast(float, byte == 0 ? 0x00400000u : (byte == 255 ? 0x7fc00000u : byte << 23));
}
// |v| where it is finite, else 0: a block's scale comes from its finite elements
__device__ __forceinline__ float q8_magnitude(float v)
{
    const float a = __builtin_fabsf(v);
    return a < __builtin_inff() ? a : 0.0f;
}
// Four codes of v * inv, to the nearest, ties to even.  Finite elements are within range; infinities and NaN become NaN.
__device__ __forceinline__ uint32_t q8_codes(float a, float b, float c, float d, float inv)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a * inv, b * inv, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c * inv, d * inv, w, true);
}

hipError_t launch_quantize(hipStream_t s, const uint16_t *X, int64_t R, int64_t C, int64_t ld, bool square, uint8_t *q, int64_t ldq, uint8_t *sc,
                           int64_t lds, uint8_t *sct, int64_t ldst);
hipError_t launch_dequantize(hipStream_t s, const uint8_t *q, int64_t R, int64_t C, int64_t ldq, const uint8_t *sc, int64_t lds, uint16_t *out,
                             int64_t ld_out);

}  // namespace coda
