// Attention, forward: one pass over the keys with the running maximum and sum of a softmax.
#include "attn_device.h"

namespace cg {
namespace {

constexpr float kSlack = 8.f;

// A block takes 128 query rows (X) of one problem and walks the keys (Y) they see in tiles of YT.
// Prompts are bound by matrix and vector instructions at a clock that power holds to 1.7 .. 1.8 GHz (the matrix pipeline 56 % busy): 8192
// tokens, 32 heads on 8, 128 wide, causal, bf16 525 .. 600 us, 920 .. 1050 TFLOP/s (a large library product: 1284).  Single tokens are bound by HBM: 64 sequences of 8192
// keys, the same heads, 361 us, 5.9 TB/s; fp32 1790, 2.4, since one of the four waves has rows and six products a term.
// bf16 tensors: probabilities are rounded to 8 bits for the product with V, as they are for P^T do: half a step of the result's type on
// a term (o is 1.2 to 1.4 times as far from 64 bits as with unrounded ones; a second piece would take half as many products again).
// The backward pass subtracts delta, a sum of o times do, from dP.  Where the differences are added up (the bias's gradient) or rows see
// a few keys only, dP is as near to delta as a rounded o is to o: the probabilities that o is made of then keep 24 bits, in three
// pieces.  With a bias that is a kernel of its own (EXACT); without, the two other pieces' products follow the only tile of a sequence
// of kFewKeys keys or fewer, so that what a sequence gets does not depend on the others.
template <class T, int DP> constexpr int kFwdWaves = Pieces<T>::N == 1 || DP <= 64 ? 2 : 1;

template <class T, int DP, bool BIAS, bool DMA, bool EXACT>
__global__ __launch_bounds__(256, (kFwdWaves<T, DP>)) void attn_fwd_kernel(AttnArgs a)
{
    constexpr int NP = Pieces<T>::N, KS = DP / 16, DT = DP / 32, YT = NP == 1 && !(EXACT && DP > 64) ? 64 : 32, SUB = YT / 32, AHEAD = 6;
    using TileY = Tile<DP, YT, NP>;
    __shared__ __align__(16) char lds[2][2][TileY::BYTES];
    LdsByte *const ldsK = (LdsByte *)lds[0][0], *const ldsV = (LdsByte *)lds[1][0];
    __shared__ float window[2][BIAS ? 256 : 1];
    const int lane = threadIdx.x & 63, wave = (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h32 = lane >> 5;
    const int Hr = a.Hq / a.Gp, hr = blockIdx.x % Hr;
    Place place;
    if (!find_place<false>(a, blockIdx.x / Hr, place)) return;
    const int t = place.t, split = place.split;
    const Seq s = seq_of(a, place.b);
    const int row0 = t * kAttnRows, rows = s.n * a.Gp, off = s.m - s.n;
    const int h0 = hr * a.Gp, hkv = h0 / a.G;
    // what this lane's row sees: keys below `limit`
    const int row = row0 + 32 * wave + (lane & 31);
    const bool here = row < rows;
    const int tok = (int)fdiv((uint32_t)min(row, rows - 1), a.by_gp), head = h0 + (here ? row - tok * a.Gp : 0);
    const int limit = a.causal ? min(max(tok + 1 + off, 0), s.m) : s.m;
    const int first_tok = (int)fdiv((uint32_t)min(row0 + 32 * wave, rows - 1), a.by_gp);
    const int wave_limit = a.causal ? min(max(first_tok + 1 + off, 0), s.m) : s.m;       // every row of the wave sees those
    const int wave_kend = row0 + 32 * wave >= rows ? 0 : keys_seen(a, s, row0 + 32 * wave + 32, rows);
    int kend = keys_seen(a, s, row0 + kAttnRows, rows), kbeg = 0;
    const int chunks = chunks_of(a, 0, kend);
    if (split >= chunks) return;
    if (chunks > 1) {
        kbeg = split * a.chunk;
        kend = min(kend, kbeg + a.chunk);
    }

    const FastDiv one = {1, 1, 0};
    const Rows<T> K{static_cast<const T *>(a.k) + (int64_t)s.k0 * a.k_tok + (int64_t)hkv * a.k_head, a.k_tok, 0, s.m, a.D, one};
    const Rows<T> V{static_cast<const T *>(a.v) + (int64_t)s.k0 * a.v_tok + (int64_t)hkv * a.v_head, a.v_tok, 0, s.m, a.D, one};
    const Rows<T> Q{static_cast<const T *>(a.q) + (int64_t)s.q0 * a.q_tok + (int64_t)h0 * a.q_head, a.q_tok, a.q_head, rows, a.D, a.by_gp};
    // Two buffers and one barrier a tile: behind it the tile is there and everyone is done with the one before, whose buffer the
    // next one's loads then fill while this one is multiplied.
    Loader<T, DP, YT, DMA> lk(K), lv(V);
    const int window0 = -(row0 + kAttnRows - 1) - off;
    float bias_next = 0.f;
    if (kbeg < kend) {
        lk.start(kbeg, ldsK);
        lv.start(kbeg, ldsV);
        if constexpr (BIAS) window[0][threadIdx.x] = window_load(a, h0, kbeg + window0);
    }

    Frag<NP> fq[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) fq[ks] = frag_of(Q.load(row, 16 * ks + 8 * h32));

    arrived(fq);

    v16f O[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) O[dt] = v16f{};
    float m = -INFINITY, l = 0.f;
    // without a bias scores stay as the product gives them and the scale enters the exponent: exp2(s c - m c)
    const float c = a.scale * kLog2e;

    if (kbeg < kend) {
        lk.finish(ldsK);
        lv.finish(ldsV);
    }
    int buf = 0;
    for (int k0 = kbeg; k0 < kend; k0 += YT, buf ^= 1) {
        tile_sync();
        const bool more = k0 + YT < kend;
        if (more) {
            lk.start(k0 + YT, ldsK + (buf ^ 1) * TileY::BYTES);
            lv.start(k0 + YT, ldsV + (buf ^ 1) * TileY::BYTES);
            if constexpr (BIAS) bias_next = window_load(a, h0, k0 + YT + window0);
        }
        if (k0 < wave_kend) {       // some row of the wave sees some key of the tile
            float p[SUB][16];
            float mt = -INFINITY;
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                Acc<NP> S;
                S.zero();
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) S.mma(TileY::rows(ldsK + buf * TileY::BYTES, 32 * u, ks, lane), fq[ks]);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int y = 32 * u + 8 * (i / 4) + 4 * h32 + i % 4;
                    p[u][i] = S.get(i);
                    if constexpr (BIAS) p[u][i] = fmaf(p[u][i], a.scale, window[buf][y + kAttnRows - 1 - 32 * wave - (lane & 31)]);
                }
            }
            if constexpr (NP == 1) reads_ahead<SUB * KS, AHEAD, 1>();
            if (k0 + YT > wave_limit)
#pragma unroll
                for (int u = 0; u < SUB; ++u)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (32 * u + 8 * (i / 4) + i % 4 >= limit - k0 - 4 * h32) p[u][i] = -INFINITY;
#pragma unroll
            for (int u = 0; u < SUB; ++u)
#pragma unroll
                for (int i = 0; i < 16; ++i) mt = fmaxf(mt, p[u][i]);
            mt = max_halves(mt);
            // The running maximum follows only where it has grown by a factor of 2^kSlack: p stays below that, at the same relative
            // precision, and the sums are hardly ever scaled again.
            const bool grows = (mt - m) * (BIAS ? kLog2e : c) > kSlack;
            const float mn = grows ? mt : m, ms = mn == -INFINITY ? 0.f : mn;      // a row that has seen no key yet: exp2(-inf) = 0
            const float alpha = grows ? __builtin_amdgcn_exp2f((m - ms) * (BIAS ? kLog2e : c)) : 1.f;
            m = mn;
            float sum = 0.f;
#pragma unroll
            for (int u = 0; u < SUB; ++u)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    p[u][i] = __builtin_amdgcn_exp2f(BIAS ? (p[u][i] - ms) * kLog2e : fmaf(p[u][i], c, -ms * c));
                    sum += p[u][i];
                }
            l = fmaf(l, alpha, sum);
            if constexpr (NP == 1 && !EXACT) {
                if (__any(grows))
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) O[dt] *= alpha;
#pragma unroll
                for (int u = 0; u < SUB; ++u)
#pragma unroll
                    for (int g = 0; g < 2; ++g) {
                        const Frag<1> fp = cut8<1>(&p[u][8 * g]);
#pragma unroll
                        for (int dt = 0; dt < DT; ++dt) O[dt] = mfma(TileY::cols(ldsV + buf * TileY::BYTES, 32 * u + 16 * g, dt, lane).p[0], fp.p[0], O[dt]);
                    }
            } else if constexpr (EXACT) {       // probabilities in three pieces, the least first; a tile's sum from zero as below
                Frag<3> fp[SUB][2];
#pragma unroll
                for (int u = 0; u < SUB; ++u)
#pragma unroll
                    for (int g = 0; g < 2; ++g) fp[u][g] = cut8<3>(&p[u][8 * g]);
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    v16f S = v16f{};
#pragma unroll
                    for (int k = 2; k >= 0; --k)
#pragma unroll
                        for (int u = 0; u < SUB; ++u)
#pragma unroll
                            for (int g = 0; g < 2; ++g) S = mfma(TileY::cols(ldsV + buf * TileY::BYTES, 32 * u + 16 * g, dt, lane).p[0], fp[u][g].p[k], S);
#pragma unroll
                    for (int i = 0; i < 16; ++i) O[dt][i] = fmaf(O[dt][i], alpha, S[i]);
                }
            } else {       // a tile's sum from zero, then one rounding into the running one
                Frag<NP> fp[SUB][2];
#pragma unroll
                for (int u = 0; u < SUB; ++u)
#pragma unroll
                    for (int g = 0; g < 2; ++g) fp[u][g] = cut8<NP>(&p[u][8 * g]);
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    Acc<NP> S;
                    S.zero();
#pragma unroll
                    for (int u = 0; u < SUB; ++u)
#pragma unroll
                        for (int g = 0; g < 2; ++g) S.mma(TileY::cols(ldsV + buf * TileY::BYTES, 32 * u + 16 * g, dt, lane), fp[u][g]);
#pragma unroll
                    for (int i = 0; i < 16; ++i) O[dt][i] = fmaf(O[dt][i], alpha, S.get(i));
                }
            }
        }
        if (more) {
            lk.finish(ldsK + (buf ^ 1) * TileY::BYTES);
            lv.finish(ldsV + (buf ^ 1) * TileY::BYTES);
            if constexpr (BIAS) window[buf ^ 1][threadIdx.x] = bias_next;
        }
    }
    if constexpr (NP == 1 && !BIAS)
        if (__builtin_expect(s.m <= kFewKeys && wave_kend > 0 && a.o_rest, 0)) {       // the tile is in the first buffer still; not expected, so that the end of short kernels stays next to their loop
            static_assert(kFewKeys <= YT, "one tile");
            const float ms = m == -INFINITY ? 0.f : m;
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                if (32 * u >= wave_kend) break;
                Acc<NP> S;
                S.zero();
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) S.mma(TileY::rows(ldsK, 32 * u, ks, lane), fq[ks]);
                float p[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    p[i] = 32 * u + 8 * (i / 4) + 4 * h32 + i % 4 >= limit ? 0.f : __builtin_amdgcn_exp2f(fmaf(S.get(i), c, -ms * c));
                    p[i] -= to_f32(from_f32<bf16raw>(p[i]));       // what the loop above took
                }
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    const Frag<2> fp = cut8<2>(&p[8 * g]);
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) {
                        const u32x4 v = TileY::cols(ldsV, 32 * u + 16 * g, dt, lane).p[0];
                        O[dt] = mfma(v, fp.p[0], O[dt]);
                        O[dt] = mfma(v, fp.p[1], O[dt]);
                    }
                }
            }
        }
    l = sum_halves(l);
    if (chunks > 1) {
        if (!here) return;
        const int64_t at = (int64_t)hr * a.tiles * a.splits + place.slot;
        float *ml = a.part_ml + at * 2 * kAttnRows;
        if (h32 == 0) {
            ml[row - row0] = BIAS ? m : m * a.scale;
            ml[kAttnRows + row - row0] = l;
        }
        store_row(a.part[0] + (at * kAttnRows + (row - row0)) * DP, O, 1.f, DP, h32);
        return;
    }
    if (!here) return;
    const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;      // no key: 0; NaN stays
    if (h32 == 0) a.lse[(int64_t)head * a.Tq + s.q0 + tok] = l == 0.f ? -INFINITY : fmaf(__builtin_amdgcn_logf(l), kLn2, BIAS ? m : m * a.scale);
    const int64_t at = (int64_t)(s.q0 + tok) * a.o_tok + (int64_t)head * a.o_head;
    store_row(static_cast<T *>(a.o) + at, O, inv, a.D, h32);
    if constexpr (NP == 1)
        if (a.o_rest)
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int d = 32 * dt + 8 * j + 4 * h32;
                    const float f[4] = {O[dt][4 * j] * inv, O[dt][4 * j + 1] * inv, O[dt][4 * j + 2] * inv, O[dt][4 * j + 3] * inv};
                    store_rest4(static_cast<bf16raw *>(a.o_rest) + at + d, f, a.D - d);
                }
}

template <class T, int DP, bool DMA> int fwd_run(AttnArgs a, hipStream_t s)
{
    a.levels = levels_of(a, a.Hq / a.Gp, kFwdWaves<T, DP> == 2 && (a.btab || !DMA || DP <= 64));
    a.fold = fold_of(a, a.Hq / a.Gp, kFwdWaves<T, DP>);
    const dim3 grid((unsigned)(a.Hq / a.Gp) * a.tiles * a.splits);
    constexpr bool can = sizeof(T) == 2;
    if (!a.btab) hipLaunchKernelGGL((attn_fwd_kernel<T, DP, false, DMA, false>), grid, dim3(256), 0, s, a);
    else if (can && a.o_rest) hipLaunchKernelGGL((attn_fwd_kernel<T, DP, true, DMA, can>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((attn_fwd_kernel<T, DP, true, DMA, false>), grid, dim3(256), 0, s, a);
    CG_HIP_TRY(hipGetLastError());
    return CG_OK;
}
template <class T, int DP> int fwd_dp(const AttnArgs &a, hipStream_t s)
{
    if (a.dma) return fwd_run<T, DP, true>(a, s);
    return fwd_run<T, DP, false>(a, s);
}

}  // namespace

int attn_fwd_launch(const AttnArgs &a, int type, hipStream_t s)
{
#define CG_DP(DP) if (a.D <= DP) return type == CG_TYPE_FP32 ? fwd_dp<float, DP>(a, s) : fwd_dp<bf16raw, DP>(a, s)
    CG_DP(32);
    CG_DP(64);
    CG_DP(96);
    CG_DP(128);
#undef CG_DP
    return CG_EUNSUPPORTED;
}
}  // namespace cg
