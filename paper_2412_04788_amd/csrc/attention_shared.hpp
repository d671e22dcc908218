// Matrix instructions and packing shared by the attention kernels.
#pragma once

#include "layer.hpp"

namespace guide {

constexpr float kLog2e = 1.4426950408889634f;

typedef float f32x2 __attribute__((ext_vector_type(2)));

// The greatest of three; a NaN if one is among them (fmaxf would first quiet each operand by an instruction of its own).
__device__ __forceinline__ float max3(float a, float b, float c) {
    return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c);
}

// The 16-bit types as the matrix units take them.  sum2(p, c): p[0] + p[1] + c in 32 bits, for the sums of probabilities that are already
// rounded to the type: a softmax whose numerator has rounded ones and whose denominator has not is no mean of the values any more
// (off by up to half a step of the type; 65504 everywhere gave an infinity).
template <int T> struct Mat;
template <> struct Mat<GUIDE_BF16> {
    using v8 = bf16x8;
    using v2 = bf16x2;
    __device__ static float sum2(v2 p, float c) { return __builtin_amdgcn_fdot2_f32_bf16(p, v2{(__bf16)1.0f, (__bf16)1.0f}, c, false); }
    __device__ static f32x16 mma32(v8 a, v8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
    __device__ static f32x4 mma16(v8 a, v8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Mat<GUIDE_F16> {
    using v8 = f16x8;
    using v2 = f16x2;
    __device__ static float sum2(v2 p, float c) { return __builtin_amdgcn_fdot2(p, v2{(_Float16)1.0f, (_Float16)1.0f}, c, false); }
    __device__ static f32x16 mma32(v8 a, v8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
    __device__ static f32x4 mma16(v8 a, v8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};

// Exponent bits of two packed 16-bit elements: an element with all of them set is an infinity or a NaN.
template <int T> constexpr uint32_t kExpBits = T == GUIDE_BF16 ? 0x7F80u : 0x7C00u;
template <int T>
__device__ inline uint32_t not_finite(uint32_t pair) {
    return (uint32_t)((pair & kExpBits<T>) == kExpBits<T>) | (uint32_t)((pair >> 16 & kExpBits<T>) == kExpBits<T>);
}
template <int T>
__device__ inline uint32_t finite_or_zero(uint32_t pair) {
    if ((pair & kExpBits<T>) == kExpBits<T>) pair &= 0xFFFF0000u;
    if ((pair >> 16 & kExpBits<T>) == kExpBits<T>) pair &= 0xFFFFu;
    return pair;
}

}  // namespace guide
