// Values in 8 bits (packed.hip writes them; linear_*.hip reads them).
//
// 32 neighbours of a row share a power of two, 2^(scale - 133): an element is code * 2^(scale - 133) with a code of -127 .. 127, or
// no number (code -128).  133 lets the scales reach from the largest fp32 numbers (254: 127 * 2^121 is the largest value; 64 * 2^122 would be
// none) down to 2^-133, the smallest bf16 number, below which a finer step would be lost in a bf16 tensor.  A code has seven bits, so every value is a bf16 number exactly and
// products of packed tensors are products of bf16 numbers.
#pragma once
#include "typed_device.h"

namespace cg {

constexpr int kPackBlock = 32, kPackBias = 133, kPackTop = 254;

struct Packed {
    const int8_t *codes;
    const uint8_t *scales;
    int64_t codes_ld, scales_ld;
};

namespace {

struct Raw8Packed { uint32_t w[2]; int e; };       // eight codes, the exponent of their step

struct __attribute__((packed, aligned(1))) Loose8 { uint32_t w[2]; };
// n elements (anything below 1: none) from column c (a multiple of 8) of a row on; what is not there is 0
__device__ __forceinline__ Raw8Packed load8(const Packed &p, int64_t row, int c, int n)
{
    Raw8Packed r = {{0, 0}, 0};
    if (n <= 0) return r;
    const int8_t *q = p.codes + row * p.codes_ld + c;
    if (n >= 8) {
        const Loose8 v = *reinterpret_cast<const Loose8 *>(q);
        r.w[0] = v.w[0], r.w[1] = v.w[1];
    } else {
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < n) r.w[i / 4] |= (uint32_t)(uint8_t)q[i] << (8 * (i & 3));
    }
    r.e = (int)p.scales[row * p.scales_ld + c / kPackBlock] - kPackBias;
    return r;
}
__device__ __forceinline__ float elem(const Raw8Packed &r, int i)
{
    const int q = (int)(r.w[i / 4] << (24 - 8 * (i & 3))) >> 24;
    const float f = __builtin_ldexpf((float)q, r.e);
    return q == -128 ? __builtin_nanf("") : f;
}

}  // namespace
}  // namespace cg
