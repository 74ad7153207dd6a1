// Tensors into 8 bits and out of them (packed_device.h has the format).
//
// Bound by HBM: each value is read and written once.  A thread takes eight neighbours, four threads a block of 32, whose largest magnitude
// they exchange.
#include "packed_device.h"
#include "row_checks.h"

namespace cg {
namespace {

struct PackArgs {
    const void *x;
    void *y;
    int8_t *codes;
    uint8_t *scales;
    int64_t ld, codes_ld, scales_ld;
    int cols;
    uint32_t count;            // eights, four for each block of 32, the last one of a row filled up
    FastDiv by_chunks;
};

// The exponent (biased) of the step 2^e at which the largest magnitude rounds to 64 .. 127: a number 1.m 2^k has the step 2^(k - 6), and the
// next one where 64 (1.m) would round to 128, which is from 127.5 on.  Subnormal numbers have the step 2^-133, and the next from 127.5 of them on.
// Above the last step's 127.5 the code stays 127.
__device__ __forceinline__ uint32_t scale_of(uint32_t top)
{
    const uint32_t e = top >> 23, m = top & 0x7fffffu;
    return min(e + (m >= (e ? 0x7f0000u : 0x7f8000u)), (uint32_t)kPackTop);
}

template <class T> __global__ __launch_bounds__(256) void pack8_kernel(PackArgs a)
{
    // four lanes at a time, and count is a multiple of 4: a block's lanes are all there
    for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < a.count; i += gridDim.x * 256) {
        const int64_t r = fdiv(i, a.by_chunks);
        const int c = 8 * (int)(i - (uint32_t)r * a.by_chunks.d), n = a.cols - c;
        const Raw8<T> x = load8(static_cast<const T *>(a.x) + (n > 0 ? r * a.ld + c : 0), n);
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t m = __float_as_uint(elem(x, j)) & 0x7fffffffu;
            top = max(top, m < 0x7f800000u ? m : 0u);
        }
        top = max(top, (uint32_t)__shfl_xor((int)top, 1));
        top = max(top, (uint32_t)__shfl_xor((int)top, 2));
        const uint32_t e = scale_of(top);
        uint32_t w[2] = {0, 0};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float f = elem(x, j);
            const bool finite = (__float_as_uint(f) & 0x7fffffffu) < 0x7f800000u;
            const int q = finite ? min(max((int)__builtin_rintf(__builtin_ldexpf(f, kPackBias - (int)e)), -127), 127) : -128;
            w[j / 4] |= ((uint32_t)q & 0xffu) << (8 * (j & 3));
        }
        if (n > 0) {
            int8_t *to = a.codes + r * a.codes_ld + c;
            if (n >= 8) *reinterpret_cast<Loose8 *>(to) = Loose8{{w[0], w[1]}};
            else
#pragma unroll
                for (int j = 0; j < 7; ++j)
                    if (j < n) to[j] = (int8_t)(w[j / 4] >> (8 * (j & 3)));
            if ((threadIdx.x & 3) == 0) a.scales[r * a.scales_ld + c / kPackBlock] = (uint8_t)e;
        }
    }
}

template <class T> __global__ __launch_bounds__(256) void unpack8_kernel(PackArgs a)
{
    const Packed p = {a.codes, a.scales, a.codes_ld, a.scales_ld};
    for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < a.count; i += gridDim.x * 256) {
        const int64_t r = fdiv(i, a.by_chunks);
        const int c = 8 * (int)(i - (uint32_t)r * a.by_chunks.d), n = a.cols - c;
        if (n <= 0) continue;
        const Raw8Packed q = load8(p, r, c, n);
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = elem(q, j);
        store8(static_cast<T *>(a.y) + r * a.ld + c, to_raw<T>(f), n);
    }
}

int args_of(PackArgs &a, int type, int64_t rows, int64_t cols, const void *tensor, int64_t ld, const cg_packed8 *p)
{
    if (!type_ok(type) || rows < 0 || cols < 0) return CG_EINVAL;
    if (rows == 0 || cols == 0) return CG_OK;
    const int64_t blocks = (cols + kPackBlock - 1) / kPackBlock;
    if (!tensor_ok(tensor, ld, cols, type) || !p || !p->codes || !p->scales || p->codes_ld < cols || p->scales_ld < blocks) return CG_EINVAL;
    if (rows > INT32_MAX || cols > INT32_MAX - 65535 || blocks * rows > (INT32_MAX >> 2) - 65535 || !rows_fit(rows, blocks)) return CG_EUNSUPPORTED;
    a.codes = p->codes, a.scales = p->scales, a.codes_ld = p->codes_ld, a.scales_ld = p->scales_ld;
    a.ld = ld, a.cols = (int)cols;
    a.count = (uint32_t)(rows * blocks * 4);
    a.by_chunks = make_fastdiv((uint32_t)(blocks * 4));
    return CG_OK;
}
dim3 grid_of(const PackArgs &a) { const uint32_t b = (a.count + 255) / 256; return dim3(b < 8192 ? b : 8192); }

}  // namespace
}  // namespace cg

using namespace cg;

extern "C" int cg_pack8(int type, int64_t rows, int64_t cols, const void *x, int64_t x_ld, const cg_packed8 *p, void *stream)
{
    PackArgs a{};
    if (int rc = args_of(a, type, rows, cols, x, x_ld, p)) return rc;
    if (a.count == 0) return CG_OK;
    a.x = x;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (type == CG_TYPE_FP32) hipLaunchKernelGGL((pack8_kernel<float>), grid_of(a), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((pack8_kernel<bf16raw>), grid_of(a), dim3(256), 0, s, a);
    CG_HIP_TRY(hipGetLastError());
    return CG_OK;
}

extern "C" int cg_unpack8(int type, int64_t rows, int64_t cols, const cg_packed8 *p, void *y, int64_t y_ld, void *stream)
{
    PackArgs a{};
    if (int rc = args_of(a, type, rows, cols, y, y_ld, p)) return rc;
    if (a.count == 0) return CG_OK;
    a.y = y;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (type == CG_TYPE_FP32) hipLaunchKernelGGL((unpack8_kernel<float>), grid_of(a), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((unpack8_kernel<bf16raw>), grid_of(a), dim3(256), 0, s, a);
    CG_HIP_TRY(hipGetLastError());
    return CG_OK;
}
