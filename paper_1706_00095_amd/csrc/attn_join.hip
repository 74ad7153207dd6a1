// Attention: joins the partial results of the chunks that a long axis was cut into.
#include "attn_device.h"

namespace cg {
namespace {

// Bound by latency, the chunks' results being in the caches: 8 sequences' new tokens, 16 heads of 64, 5.2 us; dq, dk and dv of six packed
// texts, 8 heads of 64, 12.6.
// o: sum_s e^(m_s - M) o_s / sum_s e^(m_s - M) l_s; gradients: sums.  Tiles of one chunk are done already.
// DP / 4 lanes hold a row, so a wave has 2 to 8 such groups.  ROWS: a group takes a row, and its chunks one after the other (many tiles of
// few chunks: 1.8 us a wave, and four times fewer waves); else the groups share a row's chunks and are added in order (few tiles of many).
template <int DP, bool ROWS> struct Join {
    static constexpr int L = DP / 4, GROUPS = 64 / L, PER_BLOCK = ROWS ? 4 * GROUPS : 4;
};

enum { ATTN_JOIN_O = 0, ATTN_JOIN_DQ, ATTN_JOIN_DKDV };

template <class T, int DP, int WHAT, bool ROWS> __device__ __forceinline__ void join_block(const AttnArgs &a, int block)
{
    using J = Join<DP, ROWS>;
    constexpr int L = J::L, GROUPS = J::GROUPS, AT_ONCE = 4, STEP = ROWS ? 1 : GROUPS;
    const int lane = threadIdx.x & 63, wave = (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int problems = WHAT == ATTN_JOIN_DKDV ? a.Hkv : a.Hq / a.Gp, pr = block % problems, item = block / problems;
    const int tile = item / (kAttnRows / J::PER_BLOCK), part = item % (kAttnRows / J::PER_BLOCK);
    constexpr bool X_KEYS = WHAT == ATTN_JOIN_DKDV;
    Place place;
    if (!find_place<X_KEYS, true>(a, tile, place)) return;
    const Seq s = seq_of(a, place.b);
    const int t = place.t;
    const int row0 = t * kAttnRows, yt = a.yt;
    int n, rows;
    if constexpr (WHAT == ATTN_JOIN_DKDV) {
        rows = s.m;
        n = chunks_of(a, first_seeing(a, s, row0) / yt * yt, s.n * a.Gp) * a.gsplit;
    } else {
        rows = s.n * a.Gp;
        n = chunks_of(a, 0, keys_seen(a, s, row0 + kAttnRows, rows));
    }
    if (n == 1) return;
    const int64_t at = (int64_t)pr * a.tiles * a.splits * a.gsplit + place.slot;
    const int group = lane / L, d = 4 * (lane % L);
    {
        const int row = row0 + part * J::PER_BLOCK + (ROWS ? wave * GROUPS + min(group, GROUPS - 1) : wave);
        if (row >= rows) return;
        float M = -INFINITY, l = 0.f;
#pragma unroll
        for (int which = 0; which < (WHAT == ATTN_JOIN_DKDV ? 2 : 1); ++which) {
            // a chunk's statistics and its values are asked for together: one wait for a few chunks
            const float *ml = a.part_ml + at * 2 * kAttnRows + (row - row0), *p = a.part[which] + (at * kAttnRows + (row - row0)) * DP + d;
            float r[4] = {};
            if (group < GROUPS)
                for (int k0 = ROWS ? 0 : group; k0 < n; k0 += AT_ONCE * STEP) {
                    float4 v[AT_ONCE];
                    float mk[AT_ONCE], lk[AT_ONCE];
#pragma unroll
                    for (int u = 0; u < AT_ONCE; ++u) {
                        const int k = k0 + u * STEP;
                        v[u] = k < n ? *reinterpret_cast<const float4 *>(p + (int64_t)k * kAttnRows * DP) : float4{0.f, 0.f, 0.f, 0.f};
                        if constexpr (WHAT == ATTN_JOIN_O) {
                            mk[u] = k < n ? ml[(int64_t)k * 2 * kAttnRows] : -INFINITY;
                            lk[u] = k < n ? ml[(int64_t)k * 2 * kAttnRows + kAttnRows] : 0.f;
                        }
                    }
                    if constexpr (WHAT == ATTN_JOIN_O) {
                        float mn = M;
#pragma unroll
                        for (int u = 0; u < AT_ONCE; ++u) mn = fmaxf(mn, mk[u]);
                        const float ms = mn == -INFINITY ? 0.f : mn, keep = __builtin_amdgcn_exp2f((M - ms) * kLog2e);
                        M = mn, l *= keep;
#pragma unroll
                        for (int e = 0; e < 4; ++e) r[e] *= keep;
#pragma unroll
                        for (int u = 0; u < AT_ONCE; ++u) {
                            const float w = __builtin_amdgcn_exp2f((mk[u] - ms) * kLog2e);
                            l = fmaf(w, lk[u], l);
                            r[0] = fmaf(w, v[u].x, r[0]), r[1] = fmaf(w, v[u].y, r[1]), r[2] = fmaf(w, v[u].z, r[2]), r[3] = fmaf(w, v[u].w, r[3]);
                        }
                    } else
#pragma unroll
                        for (int u = 0; u < AT_ONCE; ++u) r[0] += v[u].x, r[1] += v[u].y, r[2] += v[u].z, r[3] += v[u].w;
                }
            if constexpr (!ROWS) {       // the groups, in order; each knows its own M
                const float mine[4] = {r[0], r[1], r[2], r[3]}, m_mine = M, l_mine = l;
                float w = 1.f;
                if constexpr (WHAT == ATTN_JOIN_O) {
#pragma unroll
                    for (int g = 0; g < GROUPS; ++g) M = fmaxf(M, __shfl(m_mine, lane % L + g * L));
                    w = __builtin_amdgcn_exp2f((m_mine - (M == -INFINITY ? 0.f : M)) * kLog2e);
                    l = 0.f;
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) r[e] = 0.f;
#pragma unroll
                for (int g = 0; g < GROUPS; ++g) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) r[e] += __shfl(mine[e] * w, lane % L + g * L);
                    if constexpr (WHAT == ATTN_JOIN_O) l += __shfl(l_mine * w, lane % L + g * L);
                }
            }
            if (ROWS ? group >= GROUPS : group != 0) continue;
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
                    if (d == 0) a.lse[(int64_t)head * a.Tq + s.q0 + tok] = l == 0.f ? -INFINITY : fmaf(__builtin_amdgcn_logf(l), kLn2, M);
                    const int64_t to = (int64_t)(s.q0 + tok) * a.o_tok + (int64_t)head * a.o_head + d;
#pragma unroll
                    for (int e = 0; e < 4; ++e) r[e] *= inv;
                    store4(static_cast<T *>(a.o) + to, r, a.D - d);
                    if constexpr (sizeof(T) == 2)
                        if (a.o_rest) store_rest4(static_cast<bf16raw *>(a.o_rest) + to, r, a.D - d);
                }
            }
        }
    }
}

template <class T, int DP, bool ROWS> __global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a)
{
    join_block<T, DP, ATTN_JOIN_O, ROWS>(a, blockIdx.x);
}
// blocks 0 .. blocks_q - 1: dq
template <class T, int DP, bool ROWS> __global__ __launch_bounds__(256) void attn_join_bwd_kernel(AttnArgs q, AttnArgs k, int blocks_q)
{
    if ((int)blockIdx.x < blocks_q) join_block<T, DP, ATTN_JOIN_DQ, ROWS>(q, blockIdx.x);
    else join_block<T, DP, ATTN_JOIN_DKDV, ROWS>(k, blockIdx.x - blocks_q);
}

// A row a wave while the chip has room for all the waves at once (8192)
constexpr int64_t kJoinWaves = 8192;

template <class T, int DP, bool ROWS> int join_fwd(const AttnArgs &a, int64_t rows, hipStream_t s)
{
    hipLaunchKernelGGL((attn_join_kernel<T, DP, ROWS>), dim3((unsigned)(rows / Join<DP, ROWS>::PER_BLOCK)), dim3(256), 0, s, a);
    CG_HIP_TRY(hipGetLastError());
    return CG_OK;
}
template <class T, int DP> int fwd_dp(const AttnArgs &a, hipStream_t s)
{
    const int64_t rows = (int64_t)(a.Hq / a.Gp) * a.tiles * kAttnRows;
    return rows > kJoinWaves ? join_fwd<T, DP, true>(a, rows, s) : join_fwd<T, DP, false>(a, rows, s);
}
template <class T, int DP, bool ROWS> int join_bwd(const AttnArgs *q, const AttnArgs *k, int64_t rows_q, int64_t rows_k, hipStream_t s)
{
    const int bq = (int)(rows_q / Join<DP, ROWS>::PER_BLOCK), bk = (int)(rows_k / Join<DP, ROWS>::PER_BLOCK);
    hipLaunchKernelGGL((attn_join_bwd_kernel<T, DP, ROWS>), dim3((unsigned)(bq + bk)), dim3(256), 0, s, q ? *q : *k, k ? *k : *q, bq);
    CG_HIP_TRY(hipGetLastError());
    return CG_OK;
}
template <class T, int DP> int bwd_dp(const AttnArgs *q, const AttnArgs *k, hipStream_t s)
{
    const int64_t rows_q = q ? (int64_t)(q->Hq / q->Gp) * q->tiles * kAttnRows : 0, rows_k = k ? (int64_t)k->Hkv * k->tiles * kAttnRows : 0;
    return rows_q + rows_k > kJoinWaves ? join_bwd<T, DP, true>(q, k, rows_q, rows_k, s) : join_bwd<T, DP, false>(q, k, rows_q, rows_k, s);
}

}  // namespace

int attn_join_launch(const AttnArgs &a, int type, hipStream_t s)
{
#define CG_DP(DP) if (a.D <= DP) return type == CG_TYPE_FP32 ? fwd_dp<float, DP>(a, s) : fwd_dp<bf16raw, DP>(a, s)
    CG_DP(32);
    CG_DP(64);
    CG_DP(96);
    CG_DP(128);
#undef CG_DP
    return CG_EUNSUPPORTED;
}
int attn_join_bwd_launch(const AttnArgs *dq, const AttnArgs *dkdv, int type, hipStream_t s)
{
    if (!dq && !dkdv) return CG_OK;
    const int D = dq ? dq->D : dkdv->D;
#define CG_DP(DP) if (D <= DP) return type == CG_TYPE_FP32 ? bwd_dp<float, DP>(dq, dkdv, s) : bwd_dp<bf16raw, DP>(dq, dkdv, s)
    CG_DP(32);
    CG_DP(64);
    CG_DP(96);
    CG_DP(128);
#undef CG_DP
    return CG_EUNSUPPORTED;
}

}  // namespace cg
