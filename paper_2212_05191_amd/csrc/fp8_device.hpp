// Device-side pieces of the 8-bit operators (HIP, gfx950): the block scale, conversion to and from e4m3 codes, and loads and stores
// of eight neighbouring elements in any storage type.
//
// Scales are powers of two.  The matrix cores multiply them into a product of 32-element blocks by themselves
// (v_mfma_scale_f32_32x32x64_f8f6f4 takes them as exponent bytes), where a scale with a fraction would cost a vector-ALU
// multiply-add for every output and block of 128: 64 of them beside two matrix instructions of 64 cycles each.  They
// cost no accuracy either: a code has three fraction bits wherever the scale puts it, and only values below 2^-14 of the
// block's largest lose some of them to gradual underflow (2^-15 with the best scale).
#pragma once

#include "gemm_device.hpp"

namespace smile {

constexpr int kFp8Block = 128;   // values of a scale
inline int fp8_pitch(int K) { return (K + kFp8Block - 1) / kFp8Block * kFp8Block; }
inline int fp8_blocks(int K) { return (K + kFp8Block - 1) / kFp8Block; }
inline int fp8_scale_pitch(int rows) { return (rows + 15) / 16 * 16; }

namespace {

// What counts for a block's scale, ordered like the magnitudes of finite values: 2 |v| as bits, plus one exponent, so that infinities and NaN wrap
// below 2^24 and every finite value is at or above it (one instruction, and half of another for the maximum of two)
__device__ __forceinline__ uint32_t magnitude_key(float v) { return (__float_as_uint(v) << 1) + 0x01000000u; }
__device__ __forceinline__ uint32_t magnitude_of(uint32_t key) { return (max(key, 0x01000000u) - 0x01000000u) >> 1; }

// max(m, |a|, |b|), NaN passed over, infinities not (half an instruction a value)
__device__ __forceinline__ float max_magnitude(float m, float a, float b)
{
    float r;
    asm("v_max3_f32 %0, %1, |%2|, |%3|" : "=v"(r) : "v"(m), "v"(a), "v"(b));
    return r;
}

// The scale's byte for a block's largest magnitude m 2^p (as bits): 2^(p-8) if m <= 1.75 (448 = 1.75 * 2^8), else 2^(p-7).  At least 1, the
// smallest normal power; at most 247.
__device__ __forceinline__ uint32_t scale_byte(uint32_t largest)
{
    const uint32_t p = (largest + 0x1fffffu) >> 23;   // a fraction beyond .75 carries into the exponent
    return max(p, 9u) - 8u;
}
__device__ __forceinline__ float scale_value(uint32_t byte) { return __uint_as_float(byte << 23); }   // byte >= 1

// Four values over a scale (a power of two) as codes, rounded to nearest even: the instruction divides as it converts
__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d, float scale)
{
    typedef short s16x2 __attribute__((ext_vector_type(2)));
    s16x2 w = {0, 0};
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, a, b, scale, false);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, c, d, scale, true);
    return __builtin_bit_cast(uint32_t, w);
}
__device__ __forceinline__ void unpack4(uint32_t w, float s, float *v)
{
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    v[0] = lo[0] * s, v[1] = lo[1] * s, v[2] = hi[0] * s, v[3] = hi[1] * s;
}

// Eight neighbouring elements of a storage type as they lie in memory, and their conversion
template <int DT>
struct Piece;

template <>
struct Piece<SMILE_DTYPE_F32> {
    typedef float E;
    struct Raw {
        u32x4 a, b;
    };
    __device__ static __forceinline__ Raw load(const void *base, size_t at)
    {
        const u32x4 *p = reinterpret_cast<const u32x4 *>(static_cast<const float *>(base) + at);
        return Raw{p[0], p[1]};
    }
    __device__ static __forceinline__ void store(void *base, size_t at, const Raw &r)
    {
        u32x4 *p = reinterpret_cast<u32x4 *>(static_cast<float *>(base) + at);
        p[0] = r.a, p[1] = r.b;
    }
    __device__ static __forceinline__ void widen(const Raw &r, float *v)
    {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = __uint_as_float(r.a[k]), v[4 + k] = __uint_as_float(r.b[k]);
    }
    __device__ static __forceinline__ Raw narrow(const float *v)
    {
        Raw r;
#pragma unroll
        for (int k = 0; k < 4; ++k) r.a[k] = __float_as_uint(v[k]), r.b[k] = __float_as_uint(v[4 + k]);
        return r;
    }
};

template <typename E16>
struct HalfPiece {
    typedef E16 E;
    struct Raw {
        u32x4 a;
    };
    __device__ static __forceinline__ Raw load(const void *base, size_t at)
    {
        return Raw{*reinterpret_cast<const u32x4 *>(static_cast<const E16 *>(base) + at)};
    }
    __device__ static __forceinline__ void store(void *base, size_t at, const Raw &r)
    {
        *reinterpret_cast<u32x4 *>(static_cast<E16 *>(base) + at) = r.a;
    }
    __device__ static __forceinline__ void widen(const Raw &r, float *v)
    {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[2 * k] = Half<E16>::lo(r.a[k]), v[2 * k + 1] = Half<E16>::hi(r.a[k]);
    }
    __device__ static __forceinline__ Raw narrow(const float *v)
    {
        Raw r;
#pragma unroll
        for (int k = 0; k < 4; ++k) r.a[k] = Half<E16>::pack(v[2 * k], v[2 * k + 1]);
        return r;
    }
};
template <>
struct Piece<SMILE_DTYPE_BF16> : HalfPiece<__bf16> {};
template <>
struct Piece<SMILE_DTYPE_F16> : HalfPiece<_Float16> {};

// Largest value of the 16 lanes of a DPP row, in all of them: a block of 128 is 16 lanes of eight
__device__ __forceinline__ uint32_t max_of_16(uint32_t v)
{
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, false));    // quad_perm 1,0,3,2
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xf, 0xf, false));    // quad_perm 2,3,0,1
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x124, 0xf, 0xf, false));   // row_ror:4
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xf, 0xf, false));   // row_ror:8
    return v;
}

// Eight values of a lane, sixteen lanes a block: the block's scale byte and this lane's codes
__device__ __forceinline__ uint32_t pack_block(const float *v, u32x2 &codes)
{
    uint32_t largest = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) largest = max(largest, magnitude_key(v[k]));
    const uint32_t byte = scale_byte(magnitude_of(max_of_16(largest)));
    const float r = scale_value(byte);
    codes[0] = pack4(v[0], v[1], v[2], v[3], r), codes[1] = pack4(v[4], v[5], v[6], v[7], r);
    return byte;
}

// The activations of the products (ACT: 0 none, 1 ReLU, 3 GELU): activate's, but NaN stays NaN, which is what becomes of a row's or a column's NaN codes (ReLU
// by the maximum that hands NaN on: one instruction), and a sum that overflowed stays infinite: as the largest finite value it would take
// the scale of its block with it, and the other 127 values to zero
template <int ACT>
__device__ __forceinline__ float fp8_activate(float v)
{
    if constexpr (ACT == 1) return __builtin_elementwise_maximum(v, 0.f);
    else return activate<ACT == 3 ? 4 : ACT>(v);
}
// Their derivatives at a kept value; at NaN, which a kept infinity is too: NaN
template <int ACT>
__device__ __forceinline__ float fp8_slope(float g)
{
    if constexpr (ACT == 1) {
        const float v = __builtin_elementwise_maximum(g, 0.f);
        return v > 0.f ? 1.f : v;
    } else {
        return activate_grad<2>(g);
    }
}

__device__ __forceinline__ int rows_of(const int32_t *rows, int e, int C) { return rows ? min(max(rows[e], 0), C) : C; }

}  // namespace

}  // namespace smile
