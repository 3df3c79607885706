// The two 16-bit types of the matrix instructions, and the vectors that kernels hold.
#pragma once

#include <hip/hip_runtime.h>

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
typedef __attribute__((ext_vector_type(4))) _Float16 f16x4;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
typedef __attribute__((ext_vector_type(2))) unsigned u32x2;

// Products of 8 values per lane (16x16x32, 32x32x16), two floats rounded to nearest even and back, and sum_four: every element of acc
// plus the lane's own four values.  In the 4x4x4 products a lane holds one column of its block's B operand, four values of k, and with ones
// for A every row of that column of the result is their sum.
// (v_dot2c_f32_bf16 in their place does not run beside the matrix pipe as the other vector instructions do: synthetic loops,
// two waves per SIMD, 14 ns per 32x32x16 MFMA alone and with four v_fma_f32 beside it, 22 with two dot products; the whole mix of a prefill
// iteration 17.5 -> 17.1 ns per MFMA, against 18.4 with the pairs taken apart and added.  16384 tokens x 32/8 heads x 128 4132 -> 4000 us.)
//
// spare(top): log2 of the factor that softmax weights up to 2^top are packed with; sums carry it too, the division takes it out.  bf16 has the
// exponents of 32 bits and needs none.  fp16 ends at 65504 and rounds what is below 2^-14 to steps of 2^-24: without a factor, 131072 tokens whose
// weights are 2^-26 of the largest would vanish with 2^-9 of the result; with weights up to 2^15 what vanishes is 2^-40 - top of it each.
struct type_bf16 {
    static constexpr float spare(float) { return 0.f; }
    static __device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x4 sum_four(u32x2 v, f32x4 acc)
    {
        const s16x4 ones = {0x3f80, 0x3f80, 0x3f80, 0x3f80};
        return __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(ones, __builtin_bit_cast(s16x4, v), acc, 0, 0, 0);
    }
    static __device__ __forceinline__ unsigned pack(float lo, float hi) { return __builtin_bit_cast(unsigned, bf16x2{(__bf16)lo, (__bf16)hi}); }
    static __device__ __forceinline__ float low(unsigned v) { return __builtin_bit_cast(float, v << 16); }
    static __device__ __forceinline__ float high(unsigned v) { return __builtin_bit_cast(float, v & 0xffff0000u); }
};
struct type_fp16 {
    static constexpr float spare(float top) { return 15.f - top; }
    static __device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x4 sum_four(u32x2 v, f32x4 acc)
    {
        const f16x4 ones = {(_Float16)1, (_Float16)1, (_Float16)1, (_Float16)1};
        return __builtin_amdgcn_mfma_f32_4x4x4f16(ones, __builtin_bit_cast(f16x4, v), acc, 0, 0, 0);
    }
    static __device__ __forceinline__ unsigned pack(float lo, float hi) { return __builtin_bit_cast(unsigned, __builtin_convertvector((f32x2{lo, hi}), f16x2)); }
    static __device__ __forceinline__ float low(unsigned v) { const f16x2 t = __builtin_bit_cast(f16x2, v); return (float)t.x; }
    static __device__ __forceinline__ float high(unsigned v) { const f16x2 t = __builtin_bit_cast(f16x2, v); return (float)t.y; }
};
