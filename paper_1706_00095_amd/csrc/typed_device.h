// Device code shared by the kernels that take tensors in fp32 or bf16 (rows.hip, attn_*.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <string.h>

namespace cg {
namespace {

typedef uint16_t bf16raw;       // a bf16 tensor's element

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(bf16raw x) { return __uint_as_float((uint32_t)x << 16); }

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
// two values rounded to bf16 (nearest even), the first in the low half
__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_t{a, b}, bf16x2_t));
}
template <class T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ bf16raw from_f32<bf16raw>(float x) { return (bf16raw)(pack_bf16(x, 0.f) & 0xffffu); }

// Eight neighbouring elements as they lie in memory.  Rows start at any element (odd widths, slices of
// wider tensors): the hardware takes 16-byte accesses at any address, so all of a row but its last
// few elements travels in them whatever its alignment.
template <class T> struct Raw8;
template <> struct Raw8<float> { uint32_t w[8]; };
template <> struct Raw8<bf16raw> { uint32_t w[4]; };

template <class T> struct __attribute__((packed, aligned(sizeof(T)))) Loose16 { uint32_t w[4]; };

// n (1 .. 8; anything below 1: none) elements at p; what is not there is 0.  `whole`: n >= 8.
template <class T> __device__ __forceinline__ Raw8<T> load8(const T *p, int n)
{
    Raw8<T> r;
    constexpr int W = sizeof(Raw8<T>) / 16;
    if (n >= 8) {
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const Loose16<T> q = reinterpret_cast<const Loose16<T> *>(p)[i];
#pragma unroll
            for (int j = 0; j < 4; ++j) r.w[4 * i + j] = q.w[j];
        }
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) r.w[i] = i < n ? __float_as_uint(p[i]) : 0u;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            r.w[i] = (2 * i < n ? (uint32_t)p[2 * i] : 0u) | (2 * i + 1 < n ? (uint32_t)p[2 * i + 1] << 16 : 0u);
    }
    return r;
}
template <class T> __device__ __forceinline__ void store8(T *p, const Raw8<T> &r, int n)
{
    constexpr int W = sizeof(Raw8<T>) / 16;
    if (n >= 8) {
#pragma unroll
        for (int i = 0; i < W; ++i) {
            Loose16<T> q;
#pragma unroll
            for (int j = 0; j < 4; ++j) q.w[j] = r.w[4 * i + j];
            reinterpret_cast<Loose16<T> *>(p)[i] = q;
        }
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = __uint_as_float(r.w[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = (bf16raw)(r.w[i / 2] >> (16 * (i & 1)));
    }
}
__device__ __forceinline__ float elem(const Raw8<float> &r, int i) { return __uint_as_float(r.w[i]); }
__device__ __forceinline__ float elem(const Raw8<bf16raw> &r, int i)
{
    return __uint_as_float(i & 1 ? r.w[i / 2] & 0xffff0000u : r.w[i / 2] << 16);
}
template <class T> __device__ __forceinline__ Raw8<T> to_raw(const float (&f)[8])
{
    Raw8<T> r;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) r.w[i] = __float_as_uint(f[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) r.w[i] = pack_bf16(f[2 * i], f[2 * i + 1]);
    }
    return r;
}

}  // namespace
}  // namespace cg
