// Blocks of 128 entries in 8-bit floating point with a power of two as scale: what the kernels that write or read them share.
#pragma once

#include "cdl_types.h"

namespace cdl {

__device__ __forceinline__ uint32_t row16_max(uint32_t x)      // over the 16 lanes that hold a row
{
#define CDL_ROR(N) x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x120 + N, 0xf, 0xf, false))
    CDL_ROR(8); CDL_ROR(4); CDL_ROR(2); CDL_ROR(1);
#undef CDL_ROR
    return x;
}

// A block's largest magnitude (bits of the float) -> its scale's byte: the exponent rounded up where the fraction is beyond 1.75, the
// largest of both formats, less the format's own exponent `top`.  At least 2^-100: no entry that is not zero then stands for a value below
// 2^-116, and all are normal numbers of bf16 (the matrix cores take smaller ones as zero).
constexpr int kLeast = 27;
__device__ __forceinline__ uint32_t scale_byte(uint32_t largest, int top)
{
    if (largest >= 0x7f800000u) return 255u;
    return (uint32_t)max((int)((largest + 0x1fffffu) >> 23) - top, kLeast);
}
__device__ __forceinline__ float inverse(uint32_t byte)      // 2^(127 - byte)
{
    return __uint_as_float(byte == 255u ? 0x7fc00000u : (254u - byte) << 23);
}

template <bool E5M2>
__device__ __forceinline__ u32x2 eight(const float (&v)[8])
{
    u32x2 q = {0, 0};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        int w = 0;
        if (E5M2) {
            w = __builtin_amdgcn_cvt_pk_bf8_f32(v[4 * h], v[4 * h + 1], w, false);
            w = __builtin_amdgcn_cvt_pk_bf8_f32(v[4 * h + 2], v[4 * h + 3], w, true);
        } else {
            w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h], v[4 * h + 1], w, false);
            w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h + 2], v[4 * h + 3], w, true);
        }
        q[h] = (uint32_t)w;
    }
    return q;
}

// A scale's byte -> the scale, 2^(byte - 127), for bytes 1 .. 254; 255, of a block with an entry that is not finite: NaN
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte == 255u ? 0x7fc00000u : byte << 23); }

// Eight bytes -> their values without the scale
template <bool E5M2>
__device__ __forceinline__ void values8(u32x2 q, float (&v)[8])
{
    typedef float f32x2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const f32x2 lo = E5M2 ? __builtin_amdgcn_cvt_pk_f32_bf8((int)q[h], false) : __builtin_amdgcn_cvt_pk_f32_fp8((int)q[h], false);
        const f32x2 hi = E5M2 ? __builtin_amdgcn_cvt_pk_f32_bf8((int)q[h], true) : __builtin_amdgcn_cvt_pk_f32_fp8((int)q[h], true);
        v[4 * h] = lo.x; v[4 * h + 1] = lo.y; v[4 * h + 2] = hi.x; v[4 * h + 3] = hi.y;
    }
}

}  // namespace cdl
