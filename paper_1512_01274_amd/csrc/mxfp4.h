// Device side of the 4-bit floating-point format that its files share.
#pragma once
#include "mxc_internal.h"

namespace mxc {

// V values of 16 bytes (or 2 x 16), from memory of the element's own alignment: rows of any length begin anywhere, and the machine
// reads 16 bytes from there at once
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ void load8(const bf16_t *p, float *v)
{
    const u32x4_any u = *reinterpret_cast<const u32x4_any *>(p);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        v[2 * k] = __uint_as_float(u[k] << 16);
        v[2 * k + 1] = __uint_as_float(u[k] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void load8(const float *p, float *v)
{
    const f32x4_any a = *reinterpret_cast<const f32x4_any *>(p), b = *reinterpret_cast<const f32x4_any *>(p + 4);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        v[k] = a[k];
        v[4 + k] = b[k];
    }
}
// eight values of a row of which `left` remain (zeros past the end)
template <typename T>
__device__ __forceinline__ void load8_edge(const T *p, int left, float *v)
{
    if (left >= 8) {
        load8(p, v);
        return;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = k < left ? load_f32(p + k) : 0.f;
}

// the largest magnitude among eight values as bits: a NaN or an infinity shows in the exponent
__device__ __forceinline__ unsigned largest8(const float *v)
{
    unsigned b = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) b = max(b, __float_as_uint(v[k]) & 0x7FFFFFFFu);
    return b;
}

// scale byte of a block whose largest magnitude has these bits: floor(log2) - 2 + 127, at least 0; 255 where one is not finite.
// (Subnormal numbers lie below every scale's reach but the smallest one's.)
__device__ __forceinline__ unsigned mxfp4_scale_byte(unsigned largest)
{
    const unsigned field = largest >> 23;
    return field == 255u ? 255u : field > 2u ? field - 2u : 0u;
}

// codes of eight values, value 0 in the low bits.  The conversion divides by the power of two in its scale operand's exponent
// (0 there means 2^-127), rounds to nearest, ties to the even code, and goes no further than 6.
__device__ __forceinline__ unsigned mxfp4_codes8(const float *v, unsigned byte)
{
    const float scale = __uint_as_float(byte << 23);
    unsigned c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], scale, 3);
    return byte == 255u ? 0u : c;
}

// maximum over the four lanes that share a block
__device__ __forceinline__ unsigned max_quad(unsigned b)
{
    b = max(b, (unsigned)__builtin_amdgcn_update_dpp(0, (int)b, 0xB1, 0xF, 0xF, true));      // lanes 1 0 3 2
    return max(b, (unsigned)__builtin_amdgcn_update_dpp(0, (int)b, 0x4E, 0xF, 0xF, true));   // lanes 2 3 0 1
}

}  // namespace mxc
