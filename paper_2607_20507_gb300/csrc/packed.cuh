// packed.cuh -- the 4-bit cache format (include/cachespec.h): e2m1 codes, an
// e4m3 scale for each group of 16 dims.
#pragma once

#include "cs_device.cuh"

namespace cs {

constexpr int kPackDim = 128;
constexpr int kPackGroup = 16;                          // dims that share a scale
constexpr int kPackGroups = kPackDim / kPackGroup;      // scale bytes of a row
constexpr int kPackCodeBytes = kPackDim / 2;            // code bytes of a row

// The two codes of byte kByte of `w` (the low four bits first) as an fp16 pair.
template <int kByte>
__device__ __forceinline__ uint32_t codes_f16x2(uint32_t w) {
    uint32_t r;
    if constexpr (kByte == 0)
        asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, a;\n\t}" : "=r"(r) : "r"(w));
    else if constexpr (kByte == 1)
        asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, b;\n\t}" : "=r"(r) : "r"(w));
    else if constexpr (kByte == 2)
        asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, c;\n\t}" : "=r"(r) : "r"(w));
    else
        asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, d;\n\t}" : "=r"(r) : "r"(w));
    return r;
}

// The two e4m3 scales in the low half of `w` as an fp16 pair.
__device__ __forceinline__ uint32_t scales_f16x2(uint32_t w) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)w));
    return r;
}

// Products of code and scale are exact in fp16: 2 + 4 significant bits,
// magnitudes from 2^-10 (0.5 times the smallest scale, 2^-9) to 2688.
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

__device__ __forceinline__ float f16_lo(uint32_t w) {
    float f;
    asm("{\n\t.reg .f16 a, b;\n\tmov.b32 {a, b}, %1;\n\tcvt.f32.f16 %0, a;\n\t}" : "=f"(f) : "r"(w));
    return f;
}
__device__ __forceinline__ float f16_hi(uint32_t w) {
    float f;
    asm("{\n\t.reg .f16 a, b;\n\tmov.b32 {a, b}, %1;\n\tcvt.f32.f16 %0, b;\n\t}" : "=f"(f) : "r"(w));
    return f;
}

__device__ __forceinline__ float fmax3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ float fmin3(float a, float b, float c) {
    float d;
    asm("min.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// The e4m3 byte nearest to 0 <= x (ties to even, at most 448).
__device__ __forceinline__ uint32_t to_e4m3(float x) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.f), "f"(x));
    return r & 0xffu;
}

// The byte of the e2m1 codes nearest to lo and hi (ties to even, at most 6).
__device__ __forceinline__ uint32_t to_e2m1x2(float lo, float hi) {
    uint32_t r;
    asm("{\n\t.reg .b8 a;\n\tcvt.rn.satfinite.e2m1x2.f32 a, %1, %2;\n\tcvt.u32.u8 %0, a;\n\t}"
        : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

}  // namespace cs
