// Element types and small pieces that the append and attention kernels share (device code).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace kvl {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));

// Half-precision element types: vectors, conversions and the matrix instructions that take them.
struct Bf16 {
    typedef __bf16 x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 x8 __attribute__((ext_vector_type(8)));
    static constexpr uint32_t kExponent = 0x7f80u;
    static __device__ __forceinline__ f32x2 widen(uint32_t w) { return f32x2{__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)}; }
    static __device__ __forceinline__ f32x16 mma32(x8 a, x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ f32x4 mma16(x8 a, x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
    // two codes of e4m3 times 2 to the exponent of `scale`
    template <bool HI>
    static __device__ __forceinline__ uint32_t from_codes(uint32_t w, float scale) {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HI));
    }
};
struct F16 {
    typedef _Float16 x2 __attribute__((ext_vector_type(2)));
    typedef _Float16 x8 __attribute__((ext_vector_type(8)));
    static constexpr uint32_t kExponent = 0x7c00u;
    static __device__ __forceinline__ f32x2 widen(uint32_t w) {
        const x2 h = __builtin_bit_cast(x2, w);
        return f32x2{(float)h[0], (float)h[1]};
    }
    static __device__ __forceinline__ f32x16 mma32(x8 a, x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ f32x4 mma16(x8 a, x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
    template <bool HI>
    static __device__ __forceinline__ uint32_t from_codes(uint32_t w, float scale) {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, HI));
    }
};

// two floats, each rounded to the nearest element
template <typename T>
__device__ __forceinline__ uint32_t narrow(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), typename T::x2));
}

// The scale of a block and head, as both operators take it (NaN: the least).
__device__ __forceinline__ float in_range(float scale) { return fminf(fmaxf(scale, 0x1p-32f), 0x1p63f); }

// codes of e4m3, as floats
template <int PAIR>
__device__ __forceinline__ f32x2 widen_codes(uint32_t w) {
    return __builtin_bit_cast(f32x2, __builtin_amdgcn_cvt_pk_f32_fp8((int)w, PAIR != 0));
}

}  // namespace kvl
