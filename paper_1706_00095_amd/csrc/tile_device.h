// What the kernels that multiply tiles out of LDS share (attn_*.hip, linear*.hip): operands in one bf16 number or three, accumulators of
// v_mfma_f32_32x32x16_bf16 (attention), loads from memory into LDS.
#pragma once
#include "igemm_device.h"
#include "typed_device.h"

namespace cg {
namespace {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

typedef __attribute__((address_space(3))) char LdsByte;      // LDS by its own addresses: 32 bits, no null checks
#define CG_LDS(type, p) (*reinterpret_cast<__attribute__((address_space(3))) type *>(p))

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;

template <class T> struct Pieces { static constexpr int N = sizeof(T) == 4 ? 3 : 1; };

// ---- operands and accumulators ------------------------------------------------------------------------------------------
template <int NP> struct Frag { u32x4 p[NP]; };      // eight values, NP bf16 pieces each, most significant first

// Two fp32 values in NP bf16 pieces, each the nearest even of what the ones before it left; three hold 24 bits.
template <int NP> __device__ __forceinline__ void cut_pair(float x0, float x1, uint32_t (&pc)[NP])
{
#pragma unroll
    for (int k = 0; k < NP; ++k) {
        pc[k] = pack_bf16(x0, x1);
        if (k + 1 < NP) {
            asm("" : "+v"(pc[k]));         // both values from the pair, not each converted once more on its own
            x0 -= __uint_as_float(pc[k] << 16);
            x1 -= __uint_as_float(pc[k] & 0xffff0000u);
        }
    }
}
template <int NP> __device__ __forceinline__ Frag<NP> cut8(const float *f)
{
    Frag<NP> r;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        uint32_t pc[NP];
        cut_pair<NP>(f[2 * t], f[2 * t + 1], pc);
#pragma unroll
        for (int k = 0; k < NP; ++k) r.p[k][t] = pc[k];
    }
    return r;
}
__device__ __forceinline__ Frag<1> frag_of(const Raw8<bf16raw> &r) { return {{u32x4{r.w[0], r.w[1], r.w[2], r.w[3]}}}; }
__device__ __forceinline__ Frag<3> frag_of(const Raw8<float> &r)
{
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = elem(r, i);
    return cut8<3>(f);
}

__device__ __forceinline__ v16f mfma(u32x4 a, u32x4 b, v16f c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// Three pieces: the products below the first are added up on their own, because an instruction drops what lies below the
// last place of the sum it adds to; the two sums meet in one rounded addition.
template <int NP> struct Acc;
template <> struct Acc<1> {
    v16f big;
    __device__ __forceinline__ void zero() { big = v16f{}; }
    __device__ __forceinline__ void mma(const Frag<1> &a, const Frag<1> &b) { big = mfma(a.p[0], b.p[0], big); }
    __device__ __forceinline__ float get(int i) const { return big[i]; }
};
template <> struct Acc<3> {
    v16f big, small;
    __device__ __forceinline__ void zero() { big = v16f{}, small = v16f{}; }
    __device__ __forceinline__ void mma(const Frag<3> &a, const Frag<3> &b)
    {
        small = mfma(a.p[2], b.p[0], small);
        small = mfma(a.p[0], b.p[2], small);
        small = mfma(a.p[1], b.p[1], small);
        small = mfma(a.p[1], b.p[0], small);
        small = mfma(a.p[0], b.p[1], small);
        big = mfma(a.p[0], b.p[0], big);
    }
    __device__ __forceinline__ float get(int i) const { return big[i] + small[i]; }
};

// A transposing read: lane i of 16 gets column i of the 4 x 16 values that the 16 lanes' addresses name, four lanes a row.
__device__ __forceinline__ s16x4 read_tr(LdsByte *p)
{
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<__attribute__((address_space(3))) s16x4 *>(p));
}

// 64 lanes x 16 bytes from memory to LDS: lane l's land at lds + 16 l.  Assembly, so that the waits stay with this file: the
// compiler would drain every load before each LDS read.  Four wait states, because the descriptor's registers may have been
// written by a vector instruction just before and nothing looks inside.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void dma4(BufferRsrc rsrc, LdsByte *lds, uint32_t voff)
{
    const uint32_t at = __builtin_amdgcn_readfirstlane((uint32_t)(size_t)lds);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(at), "v"(voff), "s"(rsrc) : "memory", "m0");
}
__device__ __forceinline__ void dma16(BufferRsrc rsrc, LdsByte *lds, uint32_t voff)
{
    const uint32_t at = __builtin_amdgcn_readfirstlane((uint32_t)(size_t)lds);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(at), "v"(voff), "s"(rsrc) : "memory", "m0");
}
#pragma clang diagnostic pop

__device__ __forceinline__ BufferRsrc raw_buffer(uint64_t at, uint64_t bytes)
{
    BufferRsrc r;
    r.x = __builtin_amdgcn_readfirstlane((uint32_t)at);
    r.y = __builtin_amdgcn_readfirstlane((uint32_t)(at >> 32) & 0xffffu);
    r.z = __builtin_amdgcn_readfirstlane((uint32_t)(bytes < kMaxBufferBytes ? bytes : kMaxBufferBytes));
    r.w = 0x00020000u;
    return r;
}

// Between tiles: this wave's loads into LDS have landed, and everyone's.
__device__ __forceinline__ void tile_sync()
{
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

}  // namespace
}  // namespace cg
