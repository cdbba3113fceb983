// The e4m3 matrix-core instruction with unit scales.  A lane gives 32 values of
// one row (of the first operand) or column (of the second), lane % 16; which 32
// of the instruction's k is the same for both operands, so any assignment of
// a tile's k to lane groups and bytes that both share computes the same sum.
// Accumulators lie as those of the bf16 instruction of the same shape.
//
// Precision, measured on gfx950 with one large and one small product: among the
// eight products of eight consecutive bytes of a lane, what lies more than 13
// binary places below the largest is cut off; the groups of eight, and the
// accumulator, are added in fp32 (the older 16x16x32 and 32x32x16 instructions
// give the same sums).  For normal operands that is 1.5e-5 of the result, far
// below a bf16 result's rounding (1.7e-3) and above an fp32 one's; where large
// products cancel, up to 2^-10 of the largest of each eight.  Where the
// sums have to be those of fp32, the operands are widened to bf16, which holds
// every e4m3 value, and multiplied by the bf16 instructions, whose sums keep 24
// bits (the same measurement), at half the rate.
#pragma once

#include <hip/hip_runtime.h>

#include "mfma_bf16.h"

namespace xtc {

typedef int i32x8 __attribute__((ext_vector_type(8)));

// Eight e4m3 values (two registers) as bf16, exactly.
__device__ __forceinline__ u16x8 widen_fp8(unsigned lo, unsigned hi) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 v[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true)};
    return __builtin_bit_cast(u16x8, v);
}

// 16x16 products over 128 values of k.
__device__ __forceinline__ f32x4 mma_fp8(const i32x8 &a, const i32x8 &b, const f32x4 &c) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, 0, 0, 0);
}

}  // namespace xtc
