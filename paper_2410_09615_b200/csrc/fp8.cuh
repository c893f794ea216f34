// 8-bit floating-point operands: how a group of values becomes codes and a scale (include/slim.h, "8-bit operands").
#pragma once
#include "common.cuh"

namespace slim {

constexpr int kF8Group = 128;                    // columns (and rows of a weight) that share a scale

__host__ __device__ constexpr float f8_largest(int format) { return format == SLIM_FP8_E4M3 ? 448.f : 57344.f; }

// Magnitudes are compared as integers: one operation each, subnormals as they are, and a NaN, larger than every number, is found too.
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }
// The larger magnitude of each of two bf16 pairs (bits of the signs cleared).
__device__ __forceinline__ uint32_t magnitude2(uint32_t w) { return w & 0x7FFF7FFFu; }

// The scale of a group from its largest magnitude's bits, and what its values are multiplied with: both correctly rounded, so that a
// scale is reproducible bit for bit.  The division by a constant stays one: a multiplication with 1 / 448 is off by an ulp for some.
struct Scale {
    float scale, inv;
    __device__ __forceinline__ Scale(uint32_t largest, float top) {
        scale = __fdiv_rn(__uint_as_float(largest), top);
        if (scale < 0x1p-126f) scale = 0x1p-126f;             // (a NaN stays)
        inv = __frcp_rn(scale);
    }
};

// Sums and products that keep subnormal numbers (the library is compiled with flush-to-zero).
__device__ __forceinline__ float add_rn(float a, float b) { float v; asm("add.rn.f32 %0, %1, %2;" : "=f"(v) : "f"(a), "f"(b)); return v; }
__device__ __forceinline__ float mul_rn(float a, float b) { float v; asm("mul.rn.f32 %0, %1, %2;" : "=f"(v) : "f"(a), "f"(b)); return v; }
__device__ __forceinline__ float fma_rn(float a, float b, float c) { float v; asm("fma.rn.f32 %0, %1, %2, %3;" : "=f"(v) : "f"(a), "f"(b), "f"(c)); return v; }

// Two codes, v's in the low byte; rounding to nearest even, magnitudes above the largest number become that.
template <int FMT>
__device__ __forceinline__ uint32_t codes2(float v, float w, float inv) {
    const float a = mul_rn(v, inv), b = mul_rn(w, inv);
    uint16_t c;
    if (FMT == SLIM_FP8_E4M3) asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(c) : "f"(b), "f"(a));
    else                      asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(c) : "f"(b), "f"(a));
    return c;
}
template <int FMT>
__device__ __forceinline__ uint32_t codes4(const float* v, float inv) { return codes2<FMT>(v[0], v[1], inv) | codes2<FMT>(v[2], v[3], inv) << 16; }

// bf16 is the upper half of a binary32 number.
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

}  // namespace slim
