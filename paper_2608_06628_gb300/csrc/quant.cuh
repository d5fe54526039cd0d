// quant.cuh -- the 8-bit cache's format: e4m3 codes, and a float32 scale for each kGroup tokens of a
// head, a power of two (hybrid_softmax.h).  Dividing by a power of two is exact, so a value is
// rounded once, and codes move to a larger scale without loss but for e4m3's subnormals.
#pragma once

#include <cuda_fp16.h>

#include "hybrid_common.cuh"
#include "hybrid_softmax.h"

namespace hyb {
namespace quant {

constexpr int kGroup = HYBRID_QUANT_TOKENS;
static_assert(kGroup == 16, "a run's tokens are counted in 16 bits");

// Two values, |x| <= 448 or NaN, to nearest even; `lo` in the low byte.
__device__ __forceinline__ uint32_t encode2(float lo, float hi)
{
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d)
{
    return encode2(a, b) | encode2(c, d) << 16;
}
// Four values, exact in half precision: pairs of the low and of the high 16 bits (which the
// conversion picks by itself).
__device__ __forceinline__ void decode4(uint32_t v, uint32_t &lo, uint32_t &hi)
{
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
        : "=r"(lo), "=r"(hi)
        : "r"(v));
}
__device__ __forceinline__ void decode4(uint32_t v, float (&x)[4])
{
    uint32_t lo, hi;
    decode4(v, lo, hi);
    const float2 a = __half22float2(*reinterpret_cast<const __half2 *>(&lo)), b = __half22float2(*reinterpret_cast<const __half2 *>(&hi));
    x[0] = a.x;
    x[1] = a.y;
    x[2] = b.x;
    x[3] = b.y;
}

// Scales as biased exponents of float32, kLeast ... kMost (of any positive scale: the power of two below).
constexpr int kLeast = 1, kMost = 253;      // 2^-126; the inverse of the largest is a normal number too
__device__ __forceinline__ int scale_of_amax(uint32_t amax)     // of a finite |x|, as bits
{
    const int e = (int)(amax >> 23) - 8 + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0);     // 448 = 1.75 * 2^8
    return e < kLeast ? kLeast : e;
}
__device__ __forceinline__ int scale_of_bits(uint32_t s)
{
    const int e = (int)(s >> 23 & 0xffu);
    return e < kLeast ? kLeast : (e > kMost ? kMost : e);
}
__device__ __forceinline__ float scale_value(int e) { return __uint_as_float((uint32_t)e << 23); }
__device__ __forceinline__ float scale_inverse(int e) { return __uint_as_float((uint32_t)(254 - e) << 23); }
// 2^(from - to), from <= to; 0 below 2^-126 (where every code becomes zero)
__device__ __forceinline__ float scale_ratio(int from, int to)
{
    const int e = 127 + from - to;
    return __uint_as_float(e < 1 ? 0u : (uint32_t)e << 23);
}

}  // namespace quant
}  // namespace hyb
