// e4m3.cuh -- rows of an 8-bit cache: codes c and a scale byte s for the values c 2^(s - 127), written and read.
//
// e is the least integer in [e_min, 7] with max |z| <= 448 2^e.  448 = 0.875 2^9 in the form part 2^x, part in [1/2, 1), so it
// follows from the exponent and the leading bits of max |z| alone.  Reading multiplies each code by a power of two in the
// element type, which is exact: 448 2^7 is below fp16's 65504, and the smallest code, 2^-9, times 2^e_min is no smaller than
// the smallest numbers of the type.
#pragma once

#include <cstdint>

#include "kv_batch.cuh"

namespace wino {

constexpr int kScaleBias = 127, kMaxScaleExp = 7;
constexpr uint32_t kScaleNan = 255;  // the row holds an infinity or NaN
template <bool kBf16>
constexpr int kMinScaleExp = kBf16 ? -110 : -14;

// The scale byte of a row whose largest magnitude has these bits.
template <bool kBf16>
__device__ __forceinline__ uint32_t scale_byte(uint32_t max_bits)
{
    if (max_bits >= 0x7f800000u)
        return kScaleNan;
    const int e = (int)(max_bits >> 23) - 135 + ((max_bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    return (uint32_t)(max(kMinScaleExp<kBf16>, min(kMaxScaleExp, e)) + kScaleBias);
}

// 2^-e, by which a row's values become codes; 0 for a row that is held as NaN.
__device__ __forceinline__ float code_factor(uint32_t scale)
{
    return scale == kScaleNan ? 0.f : __uint_as_float((uint32_t)(2 * 127 - (int)scale) << 23);
}

// Codes of two scaled values, lo in the low byte: nearest, ties to even, kept within +-448.
__device__ __forceinline__ uint32_t codes2(float lo, float hi)
{
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}

// What decode4 multiplies by, twice in a word.  bf16: the codes' bits are read with an exponent too small by 120, so
// 2^(120 + e); scales that are not written (135 to 254) count as 134.
template <bool kBf16>
__device__ __forceinline__ uint32_t read_factor(uint32_t scale)
{
    uint32_t f;
    if (kBf16)
        f = scale == kScaleNan ? 0x7fffu : (min(scale, (uint32_t)(kScaleBias + kMaxScaleExp)) + 120u) << 7;
    else
        f = scale == kScaleNan ? 0x7fffu
                               : (uint32_t)(min(max((int)scale, kScaleBias + kMinScaleExp<kBf16>), kScaleBias + kMaxScaleExp) - kScaleBias + 15) << 10;
    return f | f << 16;
}

// The same, but of rows that are held as NaN something finite.
template <bool kBf16>
__device__ __forceinline__ uint32_t finite_factor(uint32_t scale)
{
    const uint32_t e = min(scale, (uint32_t)(kScaleBias + kMaxScaleExp));
    const uint32_t f = kBf16 ? (e + 120u) << 7 : (uint32_t)(max((int)e, kScaleBias + kMinScaleExp<kBf16>) - kScaleBias + 15) << 10;
    return f | f << 16;
}

// The values of four codes (lowest byte first) as pairs of the element type.
template <bool kBf16>
__device__ __forceinline__ void decode4(uint32_t codes, uint32_t factor, uint32_t &lo, uint32_t &hi)
{
    if (kBf16) {
        // s eeee mmm into the places of a bf16's sign, low exponent bits and high mantissa bits: 16 times the byte, and the sign
        // bit 2^11 moved on to 2^15
        const uint32_t a = __byte_perm(codes, 0u, 0x4140), b = __byte_perm(codes, 0u, 0x4342);
        const uint32_t x = a * 16u + (a & 0x00800080u) * 240u, y = b * 16u + (b & 0x00800080u) * 240u;
        asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(lo) : "r"(x), "r"(factor));
        asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(hi) : "r"(y), "r"(factor));
    } else {
        uint32_t x, y;
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(x) : "h"((uint16_t)codes));
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(y) : "h"((uint16_t)(codes >> 16)));
        asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(lo) : "r"(x), "r"(factor));
        asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(hi) : "r"(y), "r"(factor));
    }
}

// Where the scale of a slot and head lies.
__device__ __forceinline__ int64_t scale_at(const wino_kv_batch &b, int32_t page, int32_t in_page, int32_t head)
{
    return ((int64_t)page * b.n_kv_heads + head) * b.page_size + in_page;
}

}  // namespace wino
