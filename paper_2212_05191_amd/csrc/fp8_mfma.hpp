// The scaled 8-bit matrix instruction, as the product's kernels use it.
#pragma once

#include "fp8_device.hpp"

namespace smile {

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

// Two 16-byte pieces as one operand
__device__ __forceinline__ i32x8 set_low(u32x4 v)
{
    typedef int i32x4 __attribute__((ext_vector_type(4)));
    const i32x4 w = __builtin_bit_cast(i32x4, v);
    return __builtin_shufflevector(w, w, 0, 1, 2, 3, -1, -1, -1, -1);
}
__device__ __forceinline__ i32x8 set_high(i32x8 f, u32x4 v)
{
    return __builtin_shufflevector(f, set_low(v), 0, 1, 2, 3, 8, 9, 10, 11);
}

// D(o, r) += sum over 64 k of W(o, k) X(r, k), e4m3 both (format 0), with the scales' bytes (low byte of sw, sx) of this lane's row of W
// and of X.  A lane holds 32 bytes of its row, in two pieces; which k they are does not matter as long as W and X agree.
__device__ __forceinline__ f32x16 mfma_scaled(i32x8 w, i32x8 x, f32x16 c, uint32_t sw, uint32_t sx)
{
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w, x, c, 0, 0, 0, (int)sw, 0, (int)sx);
}

}  // namespace

}  // namespace smile
