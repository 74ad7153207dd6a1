// Attention: joins the partial results of the chunks that a long axis was cut into.
#include "attn_device.h"

namespace cg {
namespace {

// A wave takes an X row, kJoinRows waves' turns a block; DP / 4 lanes hold the row, the other lanes of the wave take other chunks, and the
// groups are added in order.  o: sum_s e^(m_s - M) o_s / sum_s e^(m_s - M) l_s; gradients: sums.  Tiles of one chunk are done already.
constexpr int kJoinRows = 8;

template <class T, int DP, int WHAT> __global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a)
{
    constexpr int L = DP / 4, GROUPS = 64 / L;
    const int lane = threadIdx.x & 63, wave = (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int problems = WHAT == ATTN_JOIN_DKDV ? a.Hkv : a.Hq / a.Gp, pr = blockIdx.x % problems, item = blockIdx.x / problems;
    const int tile = item / (kAttnRows / kJoinRows), part = item % (kAttnRows / kJoinRows);
    int b, t;
    if (WHAT == ATTN_JOIN_DKDV ? !find_tile(a.cu_k, a.Tk, a.B, kAttnRows, 1, tile, b, t) : !find_tile(a.cu_q, a.Tq, a.B, kAttnRows, a.Gp, tile, b, t)) return;
    const Seq s = seq_of(a, b);
    const int row0 = t * kAttnRows, yt = a.yt;
    int n, rows;
    if constexpr (WHAT == ATTN_JOIN_DKDV) {
        rows = s.m;
        n = chunks_of(a, first_seeing(a, s, row0) / yt * yt, s.n * a.Gp);
    } else {
        rows = s.n * a.Gp;
        n = chunks_of(a, 0, keys_seen(a, s, row0 + kAttnRows, rows));
    }
    if (n == 1) return;
    const int64_t at = ((int64_t)pr * a.tiles + tile) * a.splits;
    const int group = lane / L, d = 4 * (lane % L);
    for (int i = wave; i < kJoinRows; i += 4) {
        const int row = row0 + part * kJoinRows + i;
        if (row >= rows) return;
        float M = 0.f, l = 0.f;
        const float *ml = WHAT == ATTN_JOIN_O ? a.part_ml + at * 2 * kAttnRows + (row - row0) : nullptr;
        if constexpr (WHAT == ATTN_JOIN_O) {
            M = -INFINITY;
            for (int k = lane; k < n; k += 64) M = fmaxf(M, ml[(int64_t)k * 2 * kAttnRows]);
#pragma unroll
            for (int x = 32; x; x >>= 1) M = fmaxf(M, __shfl_xor(M, x));
            const float Ms = M == -INFINITY ? 0.f : M;
            for (int k = lane; k < n; k += 64)
                l = fmaf(__builtin_amdgcn_exp2f((ml[(int64_t)k * 2 * kAttnRows] - Ms) * kLog2e), ml[(int64_t)k * 2 * kAttnRows + kAttnRows], l);
#pragma unroll
            for (int x = 32; x; x >>= 1) l += __shfl_xor(l, x);
            M = Ms;
        }
#pragma unroll
        for (int which = 0; which < (WHAT == ATTN_JOIN_DKDV ? 2 : 1); ++which) {
            const float *p = a.part[which] + (at * kAttnRows + (row - row0)) * DP + d;
            float f[4] = {};
            if (group < GROUPS)
#pragma unroll 4
                for (int k = group; k < n; k += GROUPS) {
                    const float4 v = *reinterpret_cast<const float4 *>(p + (int64_t)k * kAttnRows * DP);
                    const float w = WHAT == ATTN_JOIN_O ? __builtin_amdgcn_exp2f((ml[(int64_t)k * 2 * kAttnRows] - M) * kLog2e) : 1.f;
                    f[0] = fmaf(w, v.x, f[0]), f[1] = fmaf(w, v.y, f[1]), f[2] = fmaf(w, v.z, f[2]), f[3] = fmaf(w, v.w, f[3]);
                }
            float r[4] = {f[0], f[1], f[2], f[3]};
#pragma unroll
            for (int g = 1; g < GROUPS; ++g)
#pragma unroll
                for (int e = 0; e < 4; ++e) r[e] += __shfl(f[e], lane % L + g * L);
            if (group != 0) continue;
            if constexpr (WHAT == ATTN_JOIN_DKDV) {
                T *to = which == 0 ? static_cast<T *>(a.dk) + (int64_t)(s.k0 + row) * a.k_tok + (int64_t)pr * a.k_head
                                   : static_cast<T *>(a.dv) + (int64_t)(s.k0 + row) * a.v_tok + (int64_t)pr * a.v_head;
                store4(to + d, r, a.D - d);
            } else {
                const int tok = (int)fdiv((uint32_t)row, a.by_gp), head = pr * a.Gp + row - tok * a.Gp;
                if constexpr (WHAT == ATTN_JOIN_DQ) {
                    store4(static_cast<T *>(a.dq) + (int64_t)(s.q0 + tok) * a.q_tok + (int64_t)head * a.q_head + d, r, a.D - d);
                } else {
                    const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
                    if (lane == 0) a.lse[(int64_t)head * a.Tq + s.q0 + tok] = l == 0.f ? -INFINITY : fmaf(__builtin_amdgcn_logf(l), kLn2, M);
                    const int64_t to = (int64_t)(s.q0 + tok) * a.o_tok + (int64_t)head * a.o_head + d;
#pragma unroll
                    for (int e = 0; e < 4; ++e) r[e] *= inv;
                    store4(static_cast<T *>(a.o) + to, r, a.D - d);
                    if constexpr (sizeof(T) == 2)
                        if (a.o_rest) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) r[e] -= to_f32(from_f32<T>(r[e]));
                            store4(static_cast<T *>(a.o_rest) + to, r, a.D - d);
                        }
                }
            }
        }
    }
}

template <class T, int DP> int join_dp(const AttnArgs &a, int what, hipStream_t s)
{
    const dim3 grid((unsigned)(what == ATTN_JOIN_DKDV ? a.Hkv : a.Hq / a.Gp) * a.tiles * (kAttnRows / kJoinRows));
    if (what == ATTN_JOIN_O) hipLaunchKernelGGL((attn_join_kernel<T, DP, ATTN_JOIN_O>), grid, dim3(256), 0, s, a);
    else if (what == ATTN_JOIN_DQ) hipLaunchKernelGGL((attn_join_kernel<T, DP, ATTN_JOIN_DQ>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((attn_join_kernel<T, DP, ATTN_JOIN_DKDV>), grid, dim3(256), 0, s, a);
    CG_HIP_TRY(hipGetLastError());
    return CG_OK;
}

}  // namespace

int attn_join_launch(const AttnArgs &a, int type, int what, hipStream_t s)
{
#define CG_DP(DP) if (a.D <= DP) return type == CG_TYPE_FP32 ? join_dp<float, DP>(a, what, s) : join_dp<bf16raw, DP>(a, what, s)
    CG_DP(32);
    CG_DP(64);
    CG_DP(96);
    CG_DP(128);
#undef CG_DP
    return CG_EUNSUPPORTED;
}

}  // namespace cg
