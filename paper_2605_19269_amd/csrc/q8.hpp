// q8.hpp -- the 8-bit format with a scale for each block of 128, and the host launchers of its kernels.
//
// A code is an OCP E4M3 byte, a scale an E8M0 byte: 2^(byte - 127), 255 NaN.  Powers of two because the matrix instruction of gfx950
// (v_mfma_scale_f32_32x32x64_f8f6f4) takes them with the codes and multiplies by them for nothing, and no product is rounded.  A register loop on random
// finite codes, with scales and without in turn: 3.93 and 3.95 PFLOP/s, on codes of 0.25 to 3 4.24 and 4.21, on zeros 4.97 and 4.97.  fp32 scales would cost an
// fp32 multiply-add for every accumulator and block, and a second set of accumulators.
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
// 2^(byte - 127), as the conversions of gfx950 take it: they use the exponent (all ones: NaN), so 255 needs no case of its own.  Checked over
// all codes and bytes against the product in fp32.
__device__ __forceinline__ float q8_scale(uint32_t byte) { return __builtin_bit_cast(float, byte == 0 ? 0x00400000u : byte << 23); }
typedef __attribute__((ext_vector_type(2))) short q8_pair;
// Four codes of v / scale, to the nearest, ties to even, in two instructions.  Finite elements are within range; infinities and NaN become NaN.
__device__ __forceinline__ uint32_t q8_codes(float a, float b, float c, float d, float scale)
{
    q8_pair w = {0, 0};
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, a, b, scale, false);
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, c, d, scale, true));
}
__device__ __forceinline__ uint16_t q8_codes2(float a, float b, float scale)
{
    return (uint16_t)__builtin_amdgcn_cvt_scalef32_pk_fp8_f32(q8_pair{0, 0}, a, b, scale, false)[0];
}
// |v| where it is finite, else 0: a block's scale comes from its finite elements
__device__ __forceinline__ float q8_magnitude(float v)
{
    const float a = __builtin_fabsf(v);
    return a < __builtin_inff() ? a : 0.0f;
}
// The largest finite magnitude of the values that `each(f)` hands to f two at a time.  The maximum passes over NaN by itself (one instruction
// for two values), so a wave looks at its values again only where an infinity is among them.
template <class F>
__device__ __forceinline__ float q8_largest(F each)
{
    float m = 0.0f;
    each([&](float a, float b) { m = fmaxf(fmaxf(m, __builtin_fabsf(a)), __builtin_fabsf(b)); });
    if (__ballot(m == __builtin_inff())) {
        m = 0.0f;
        each([&](float a, float b) { m = fmaxf(fmaxf(m, q8_magnitude(a)), q8_magnitude(b)); });
    }
    return m;
}

// Workgroups, of 256, that the launches below come to
constexpr int QUANTIZE_PASSES = 4, RESTORE_PASSES = 2;
inline int64_t quantize_workgroups(int64_t R, int64_t C, bool square)
{
    const int64_t cb = (C + Q8_BLOCK - 1) / Q8_BLOCK;
    if (square) return cb * ((R + Q8_BLOCK - 1) / Q8_BLOCK);
    return R * cb <= 64 * 1024 ? cb * ((R + 15) / 16) : cb * ((R + 16 * QUANTIZE_PASSES - 1) / (16 * QUANTIZE_PASSES));
}
inline int64_t dequantize_workgroups(int64_t R, int64_t C) { return (C + Q8_BLOCK - 1) / Q8_BLOCK * ((R + 16 * RESTORE_PASSES - 1) / (16 * RESTORE_PASSES)); }

hipError_t launch_quantize(hipStream_t s, const uint16_t *X, int64_t R, int64_t C, int64_t ld, bool square, uint8_t *q, int64_t ldq, uint8_t *sc,
                           int64_t lds, uint8_t *sct, int64_t ldst);
hipError_t launch_dequantize(hipStream_t s, const uint8_t *q, int64_t R, int64_t C, int64_t ldq, const uint8_t *sc, int64_t lds, uint16_t *out,
                             int64_t ld_out);

}  // namespace coda
