// Device code shared by the kernels of the linear layers (linear.hip, linear_gemm.hip) and what their host side passes to them.
//
// All three passes are one product, C[r][c] = sum_k A(r, k) B(c, k), of operands that lie with their rows along k (forward: x and w) or
// across it (backward-data: w; backward-weight: dz and x), and one epilogue on rows of fp32 sums.
#pragma once
#include "cg_internal.h"
#include "packed_device.h"
#include "tile_device.h"

namespace cg {

// What becomes of eight neighbouring sums of a row: forward  out = act(sum + bias) + add, z = sum + bias;  backward-data  out = sum *
// slope of act at z_in + add;  backward-weight and sums of a part of k: out = sum.
struct EpiArgs {
    const float *bias;
    const void *add, *z_in;
    Packed z_in8;                     // codes NULL: none
    void *out, *z;
    int64_t add_ld, z_in_ld, out_ld, z_ld;
    int act, slope;                   // CG_ACT_*
};

struct GemmArgs {
    const void *A, *B;
    Packed B8;                        // instead of B
    int64_t a_ld, b_ld;
    int R, C, K;
    int tiles_r, tiles_c, splits, chunk;      // k is cut into `splits` chunks (a multiple of a step each)
    float *part;                      // [splits][R][C] where there are several, then [splits][R] for the bias
    float *dbias;                     // backward-weight, all tiles but those of 256: sums of A over k as well; NULL: not wanted
    EpiArgs epi;
};

// linear_gemm.hip.  Which of its kernels: PASS_*; tiles of 64 x 64, of 128 x 128, or (bf16) of 256 x 256; dma: bf16 operands travel to
// LDS without registers.
struct GemmKind { int type, pass, packed, tile, dma; };
int gemm_launch(const GemmKind &kind, const GemmArgs &a, hipStream_t s);
// Whether either half of a block's waves has half of its values of k: tiles of 64, and bf16 tiles of 128 that are one block a compute unit (2048^3 26 us,
// 28 by four waves a block; 1024 x 4096 x 4096 42 and 46).
inline bool gemm_halves(int type, int tile, int64_t blocks) { return tile == 64 || (type == CG_TYPE_BF16 && tile == 128 && blocks <= 256); }
constexpr int kGemmStep = 64;         // chunks of k are multiples of it

namespace {

// ---- activations ----------------------------------------------------------------------------------------------------------
// gelu(z) = z Phi(z).  Phi(-|z|) = e^(-z^2/2) t P(t), t = 1 / (1 + 0.36 |z|), with a P of degree 8 fitted to the scaled complementary
// error function by iterated least squares on 0 <= |z| <= 40: off by 9e-8 relative at most, and by roundings.  No branch, where the
// library's erff has two sides that both run in a wave: 9 multiply-adds, an exponential, a reciprocal.
__device__ __forceinline__ float tail_of_normal(float z, float &e)
{
    const float a = fabsf(z);
    e = __builtin_amdgcn_exp2f(-0.5f * kLog2e * z * z);
    const float t = __builtin_amdgcn_rcpf(fmaf(0.36f, a, 1.f));
    float p = -0.030240084f;
    p = fmaf(p, t, 0.13951595f);
    p = fmaf(p, t, -0.22361257f);
    p = fmaf(p, t, 0.10738120f);
    p = fmaf(p, t, -0.00039283623f);
    p = fmaf(p, t, 0.096039394f);
    p = fmaf(p, t, 0.12400939f);
    p = fmaf(p, t, 0.14368191f);
    p = fmaf(p, t, 0.14361766f);
    return p * t * e;
}
// For bf16 results, whose own rounding is 2^-9: Phi(-a) = 2^G(a) with a G of degree 7 fitted by iterated least squares on 0 <= a <= 9, off by 1.3e-6 |z| and
// by 2.6e-5 of a result down to z = -5.5, 1.8e-4 to -7, 1e-2 to -9 (where it is 1e-18) and a fourth to -11 (2e-27): from -8.5 on more than its own
// rounding, of numbers below 1e-16.  Half as many instructions, which a tile's epilogue waits for (8192 x 4096
// -> 16384: 876 us, 857 so).  From 15 on Phi(-a) is 0 and a is taken as 15, so that an infinity stays one.
__device__ __forceinline__ float gelu_bf16(float z)
{
    const float a = fabsf(z), b = fminf(a, 15.f);
    float g = -1.58184864e-06f;
    g = fmaf(g, b, 5.64911893e-05f);
    g = fmaf(g, b, -0.000891114699f);
    g = fmaf(g, b, 0.00836254249f);
    g = fmaf(g, b, -0.053697512f);
    g = fmaf(g, b, -0.458680095f);
    g = fmaf(g, b, -1.15118439f);
    g = fmaf(g, b, -1.00000006f);
    return fmaf(-b, __builtin_amdgcn_exp2f(g), fmaf(0.5f, a, 0.5f * z));
}
template <class T> __device__ __forceinline__ float act_of(float z, int act)
{
    if (act == CG_ACT_RELU) return z < 0.f ? 0.f : z;
    if (act == CG_ACT_GELU) {
        if constexpr (sizeof(T) == 2) return gelu_bf16(z);
        float e;
        const float q = tail_of_normal(z, e);
        return z * (z > 0.f ? 1.f - q : q);
    }
    if (act == CG_ACT_SILU) return z * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * z));
    return z;
}
// g times the slope of the activation at z
__device__ __forceinline__ float slope_times(float g, float z, int act)
{
    if (act == CG_ACT_RELU) return z > 0.f ? g : z == z ? 0.f : z;
    if (act == CG_ACT_GELU) {
        float e;
        const float q = tail_of_normal(z, e);
        return g * fmaf(z * 0.3989422804f, e, z > 0.f ? 1.f - q : q);
    }
    if (act == CG_ACT_SILU) {
        const float p = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * z));
        return g * (p * fmaf(z, 1.f - p, 1.f));
    }
    return g;
}

// What the epilogue reads for eight sums of a row, apart from the bias: asked for ahead of its use.  z: the input of the activation, as a
// tensor's values or in 8 bits.
template <class T> struct EpiIn {
    Raw8<T> add, z;
};
enum EpiSide { EPI_EITHER, EPI_FWD, EPI_BWD };       // what a kernel knows of its pass: forward has no slope, backward nothing but it and an addition
template <EpiSide SIDE, class T> __device__ __forceinline__ Raw8<T> epi_load_z(const EpiArgs &e, int64_t row, int c, int n)
{
    Raw8<T> z = {};
    if (SIDE != EPI_FWD && e.slope != CG_ACT_NONE) {
        if (e.z_in8.codes) {
            const Raw8Packed q = load8(e.z_in8, row, c, n);
            z.w[0] = q.w[0], z.w[1] = q.w[1], z.w[2] = (uint32_t)q.e;
        } else z = load8(static_cast<const T *>(e.z_in) + (n > 0 ? row * e.z_in_ld + c : 0), n);
    }
    return z;
}
template <class T> __device__ __forceinline__ Raw8<T> epi_load_add(const EpiArgs &e, int64_t row, int c, int n)
{
    Raw8<T> add = {};
    if (e.add) add = load8(static_cast<const T *>(e.add) + (n > 0 ? row * e.add_ld + c : 0), n);
    return add;
}
template <EpiSide SIDE, class T>
__device__ __forceinline__ void epi_finish(const EpiArgs &e, float (&v)[8], const Raw8<float> &bias, const EpiIn<T> &in, int64_t row, int c, int n)
{
    if constexpr (SIDE != EPI_BWD) {
        if (e.bias) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += elem(bias, i);
        }
        if (e.z) store8(static_cast<T *>(e.z) + row * e.z_ld + c, to_raw<T>(v), n);
        if (e.act != CG_ACT_NONE) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = act_of<T>(v[i], e.act);
        }
    }
    if constexpr (SIDE != EPI_FWD) {
        if (e.slope != CG_ACT_NONE) {
            if (e.z_in8.codes) {
                const Raw8Packed q = {{in.z.w[0], in.z.w[1]}, (int)in.z.w[2]};
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = slope_times(v[i], elem(q, i), e.slope);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = slope_times(v[i], elem(in.z, i), e.slope);
            }
        }
    }
    if (e.add) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += elem(in.add, i);
    }
    store8(static_cast<T *>(e.out) + row * e.out_ld + c, to_raw<T>(v), n);
}
template <class T> __device__ __forceinline__ void finish8(const EpiArgs &e, float (&v)[8], int64_t row, int c, int n)
{
    Raw8<float> bias = {};
    if (e.bias) bias = load8(e.bias + c, n);
    const EpiIn<T> in = {epi_load_add<T>(e, row, c, n), epi_load_z<EPI_EITHER, T>(e, row, c, n)};
    epi_finish<EPI_EITHER, T>(e, v, bias, in, row, c, n);
}

}  // namespace
}  // namespace cg
