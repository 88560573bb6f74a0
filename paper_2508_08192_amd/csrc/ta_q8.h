// What the kernels of the 8-bit cache share: e8m0 scales and e4m3 codes of gfx950's own conversions.
#pragma once

#include "ta_common.h"

typedef float q8_f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 q8_bf16x2 __attribute__((ext_vector_type(2)));
typedef short q8_s16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short q8_u16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float q8_scale(uint32_t byte)               // 2^(byte - 127); 255: NaN
{
    return __uint_as_float((byte << 23) | (((byte + 1u) & 255u) < 2u ? 0x00400000u : 0u));
}

// The scale byte of a row whose largest finite magnitude has the bits `top`: the smallest 2^e, e >= -126, with top <= 448 * 2^e
// (448 is 1.75 * 2^8).  A power of two costs a floating format nothing of its relative precision, makes every product with it exact,
// and is what the matrix cores take as the scale of an 8-bit operand.
__device__ __forceinline__ uint32_t q8_scale_byte(uint32_t top)
{
    const int e = (int)(top >> 23) - ((top & 0x7fffffu) <= 0x600000u ? 8 : 7);
    return top == 0u ? 127u : (uint32_t)(e < 1 ? 1 : e);
}

__device__ __forceinline__ float q8_power(uint32_t byte)               // 2^(byte - 127) for the bytes that are written, 1 .. 247
{
    return __uint_as_float(byte << 23);
}

__device__ __forceinline__ uint32_t q8_finite_bits(float x)            // |x| as bits, 0 for an infinity or a NaN
{
    const uint32_t u = __float_as_uint(x) & 0x7fffffffu;
    return u < 0x7f800000u ? u : 0u;
}

// Values over a power of two as codes, to nearest, ties to even; what is no number (or above 464 of it) becomes a NaN.  The
// instructions were compared with the definition on all bf16 values and as many fp32 ones at seven powers from 2^-126 to 2^120.
__device__ __forceinline__ uint32_t q8_codes4(float a, float b, float c, float d, float power)
{
    q8_s16x2 r = {0, 0};
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, a, b, power, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, c, d, power, true);
    return __builtin_bit_cast(uint32_t, r);
}

__device__ __forceinline__ uint32_t q8_codes4(uint32_t lo, uint32_t hi, float power)       // of two pairs of bf16 values
{
    q8_s16x2 r = {0, 0};
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(q8_bf16x2, lo), power, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(q8_bf16x2, hi), power, true);
    return __builtin_bit_cast(uint32_t, r);
}

// Two codes times a power of two as bf16 (lower or upper half of the word).
template <bool UPPER>
__device__ __forceinline__ uint32_t q8_bf16_2(uint32_t codes, float power)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)codes, power, UPPER));
}

__device__ __forceinline__ void q8_values4(uint32_t codes, float v[4])
{
    const q8_f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
    v[0] = lo.x; v[1] = lo.y; v[2] = hi.x; v[3] = hi.y;
}

__device__ __forceinline__ float q8_value(uint32_t code)
{
    return __builtin_amdgcn_cvt_f32_fp8((int)code, 0);
}

__device__ __forceinline__ uint32_t q8_pack_bf16(float lo, float hi)
{
    const q8_f32x2 f = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, q8_bf16x2));
}

hipError_t ta_launch_rows(const TARows &r, hipStream_t stream);
hipError_t ta_launch_q8_read(const TAQ8Read &r, hipStream_t stream);
hipError_t ta_launch_q8_compact(const TAQ8Compact &c, hipStream_t stream);
hipError_t ta_launch_q8_generic(const TAQ8Params &p, hipStream_t stream, int dev);
hipError_t ta_launch_q8_mfma(const TAQ8Params &p, hipStream_t stream, int dev);
hipError_t ta_launch_q8_tile(const TAQ8Params &p, hipStream_t stream, int dev);
