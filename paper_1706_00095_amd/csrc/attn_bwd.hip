// Attention, backward.  The scores are computed again from lse, once with the queries as X (dq, the bias's gradient and delta)
// and once with the keys as X (dk, dv): seven products instead of five, but every sum stays in one block's registers, so no
// gradient is added with atomics and results repeat bit for bit.
//
// bf16 tensors: dS is rounded to 8 bits for dS K and dS^T Q, P for P^T do, half a step of the results' type on a term, which many terms
// average (results are 1.4 times as far from 64 bits as if only they were rounded; second pieces would take three products
// for two).  A few terms do not average: where a sequence has kFewKeys keys or fewer (dq), or kFewRows query rows or fewer (dk, dv), what
// rounding left is multiplied too, behind the loop, from the tile that is in LDS still.  512 texts of 32, 12 heads of 64: dq 96 -> 102 us,
// dk/dv 117 -> 126; calls without such sequences are as fast as without it.  Lanes' numbers are made anew there, lest the loop keep
// addresses for it in registers.
#include "attn_device.h"

namespace cg {
namespace {

// The bias's gradient.  A wave's 32 x 32 part of dS is summed along its 63 diagonals (equal distances): column c of row r goes to row
// r - c + 31 of a square in LDS, at place c; the places of a row that no (r, c) has stay zero, so a lane adds up one whole row
// in eight wide reads.  Rows of kDiag words put eight lanes' reads on different banks.
// Sums over a wave's parts are kept by distance (W <= kNear: a word a distance, which each lane has to itself), else by bucket.
constexpr int kDiag = 36, kLdsBytes = 160 << 10;
// The dq kernel with a bias: LDS of its tiles, windows and squares; the words a wave that are left decide how far distances are kept one
// by one: 1024, which all instances but the widest in fp32 have room for (849 there).
template <class T, int DP> struct DqLds {
    static constexpr int YT = Pieces<T>::N == 1 ? 64 : 32, FIXED = 4 * Tile<DP, YT, Pieces<T>::N>::BYTES + 2 * 256 * 4 + 4 * 63 * kDiag * 4 + 4 * 4;
    static constexpr int LEFT = ((kLdsBytes - FIXED) / 16 - 1) / 2, NEAR = LEFT < 1024 ? LEFT : 1024;
    static __host__ __device__ constexpr int words(int W) { return W <= NEAR ? 2 * W + 1 : kMaxBuckets; }
    static_assert(NEAR > 0 && FIXED + 16 * (2 * NEAR + 1) <= kLdsBytes && FIXED + 16 * kMaxBuckets <= kLdsBytes, "more LDS than a compute unit has");
};

__device__ __forceinline__ float diagonal_sum(const float (&ds)[16], float *sq, int lane)
{
    const int c = lane & 31, h32 = lane >> 5;
#pragma unroll
    for (int i = 0; i < 16; ++i) sq[(8 * (i / 4) + 4 * h32 + i % 4 - c + 31) * kDiag + c] = ds[i];
    // a wave's LDS accesses keep their order; the compiler has to be told to
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    float v[4] = {};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float4 x = *reinterpret_cast<const float4 *>(sq + min(lane, 62) * kDiag + 4 * j);
        v[0] += x.x, v[1] += x.y, v[2] += x.z, v[3] += x.w;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    return (v[0] + v[1]) + (v[2] + v[3]);
}
// Adds a lane's v, whose bucket is `bucket` (-1: none), to acc [buckets].  Neighbouring distances have the same bucket or neighbours, so
// a bucket's lanes are a run: its last lane gets the run's sum.
__device__ __forceinline__ void add_runs(float v, int bucket, float *acc, int lane)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const float u = __shfl_up(v, d);
        const int ub = __shfl_up(bucket, d);
        if (lane >= d && ub == bucket) v += u;
    }
    const int next = __shfl_down(bucket, 1);
    if (bucket >= 0 && (lane == 63 || next != bucket)) acc[bucket] += v;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// With a bias, rows whose lse is far from zero.  lse = m + log l is one number of 24 bits: beside a large m it keeps little of log l (nothing
// where all that a row sees has the type's lowest value as its bias), and e^(s - lse) no longer sums to one.  Such a row gets its m and l
// anew from the scores, and both kernels take e^(s - m - log l).  Below 2^10 a rounded lse costs a probability 2^-14 of itself, no more
// than the score's own rounding does there.  The blocks that have such a row walk the keys once more for it, no others do.  Without a
// bias scores are large only where products are, whose own rounding is as large as lse's.
constexpr float kFar = 1024.f;

// dq, delta and the bias's gradient.  A block takes 128 query rows (X) and walks the keys (Y) they see, as the forward kernel does; the row's
// statistics are known, so a tile is S, dP, dS and dS K: three products.  Bound as the forward kernel: 4 x 4096, 16 heads of 128, causal,
// bf16 450 us, 915 TFLOP/s; 2862 packed tokens, 12 heads of 64, with a bias 45 us, of which the sums along diagonals are 8.
// Waves a SIMD: two where registers and LDS (the squares of the bias's gradient take 36 KB) allow them.
template <class T, int DP, bool BIAS> constexpr int kDqWaves = (Pieces<T>::N == 1 ? !BIAS || DP <= 64 : DP <= (BIAS ? 32 : 64)) ? 2 : 1;

template <class T, int DP, bool BIAS, bool DMA>
__global__ __launch_bounds__(256, (kDqWaves<T, DP, BIAS>)) void attn_dq_kernel(AttnArgs a)
{
    constexpr int NP = Pieces<T>::N, KS = DP / 16, DT = DP / 32, YT = DqLds<T, DP>::YT, SUB = YT / 32;
    using TileY = Tile<DP, YT, NP>;
    __shared__ __align__(16) char lds[2][2][TileY::BYTES];
    LdsByte *const ldsK = (LdsByte *)lds[0][0], *const ldsV = (LdsByte *)lds[1][0];
    __shared__ float window[2][BIAS ? 256 : 1];
    __shared__ __align__(16) float square[BIAS ? 4 : 1][BIAS ? 63 * kDiag : 4];
    __shared__ int far_rows[4];
    extern __shared__ float by_wave[];          // [4][words(W)]
    using Lds = DqLds<T, DP>;
    static_assert(!BIAS || sizeof(lds) + sizeof(window) + sizeof(square) + sizeof(far_rows) == Lds::FIXED, "what the launch's LDS is computed from");
    constexpr int kNear = Lds::NEAR;
    const int lane = threadIdx.x & 63, wave = (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h32 = lane >> 5;
    const int Hr = a.Hq / a.Gp, hr = blockIdx.x % Hr;
    Place place;
    if (!find_place<false>(a, blockIdx.x / Hr, place)) return;
    const int t = place.t, split = place.split;
    const bool want_bias = BIAS && a.dbias_part;
    float *const mine = by_wave + wave * Lds::words(a.W);
    float *const bias_out = want_bias ? a.dbias_part + ((int64_t)hr * a.dbias_parts + place.slot) * a.buckets : nullptr;
    const Seq s = seq_of(a, place.b);
    const int row0 = t * kAttnRows, rows = s.n * a.Gp, off = s.m - s.n;
    const int h0 = hr * a.Gp, hkv = h0 / a.G;
    const int row = row0 + 32 * wave + (lane & 31);
    const bool here = row < rows;
    const int tok = (int)fdiv((uint32_t)min(row, rows - 1), a.by_gp), head = h0 + (here ? row - tok * a.Gp : 0);
    const int limit = a.causal ? min(max(tok + 1 + off, 0), s.m) : s.m;
    const int first_tok = (int)fdiv((uint32_t)min(row0 + 32 * wave, rows - 1), a.by_gp);
    const int wave_limit = a.causal ? min(max(first_tok + 1 + off, 0), s.m) : s.m;
    const int wave_kend = row0 + 32 * wave >= rows ? 0 : keys_seen(a, s, row0 + 32 * wave + 32, rows);
    int kend = keys_seen(a, s, row0 + kAttnRows, rows), kbeg = 0;
    const int chunks = chunks_of(a, 0, kend);
    if (split >= chunks) {
        if (want_bias)
            for (int i = threadIdx.x; i < a.buckets; i += 256) bias_out[i] = 0.f;
        return;
    }
    if (chunks > 1) {
        kbeg = split * a.chunk;
        kend = min(kend, kbeg + a.chunk);
    }
    if (want_bias) {
        for (int i = threadIdx.x; i < 4 * 63 * kDiag; i += 256) square[0][i] = 0.f;
        for (int i = threadIdx.x; i < 4 * Lds::words(a.W); i += 256) by_wave[i] = 0.f;
        __syncthreads();
    }

    const FastDiv one = {1, 1, 0};
    const Rows<T> K{static_cast<const T *>(a.k) + (int64_t)s.k0 * a.k_tok + (int64_t)hkv * a.k_head, a.k_tok, 0, s.m, a.D, one};
    const Rows<T> V{static_cast<const T *>(a.v) + (int64_t)s.k0 * a.v_tok + (int64_t)hkv * a.v_head, a.v_tok, 0, s.m, a.D, one};
    const Rows<T> Q{static_cast<const T *>(a.q) + (int64_t)s.q0 * a.q_tok + (int64_t)h0 * a.q_head, a.q_tok, a.q_head, rows, a.D, a.by_gp};
    const int64_t o_at = (int64_t)s.q0 * a.o_tok + (int64_t)h0 * a.o_head;
    const Rows<T> dO{static_cast<const T *>(a.d_o) + o_at, a.o_tok, a.o_head, rows, a.D, a.by_gp};
    const Rows<T> O{static_cast<const T *>(a.o_in) + o_at, a.o_tok, a.o_head, rows, a.D, a.by_gp};
    const Rows<T> R{static_cast<const T *>(a.o_rest_in) + o_at, a.o_tok, a.o_head, rows, a.D, a.by_gp};
    Loader<T, DP, YT, DMA> lk(K), lv(V);
    const int window0 = -(row0 + kAttnRows - 1) - off;
    float bias_next = 0.f;
    if (kbeg < kend) {
        lk.start(kbeg, ldsK);
        lv.start(kbeg, ldsV);
        if constexpr (BIAS) window[0][threadIdx.x] = window_load(a, h0, kbeg + window0);
    }

    Frag<NP> fq[KS], fdo[KS];
    float delta = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        const int d = 16 * ks + 8 * h32;
        fq[ks] = frag_of(Q.load(row, d));
        const Raw8<T> g = dO.load(row, d), o = O.load(row, d);
        if (NP == 1 && a.o_rest_in) {
            const Raw8<T> r = R.load(row, d);
#pragma unroll
            for (int i = 0; i < 8; ++i) delta = fmaf(elem(g, i), with_rest(elem(o, i), r.w[i / 2 % (sizeof(r.w) / 4)] >> (16 * (i & 1))), delta);
        } else
#pragma unroll
            for (int i = 0; i < 8; ++i) delta = fmaf(elem(g, i), elem(o, i), delta);
        fdo[ks] = frag_of(g);
    }
    delta = sum_halves(delta);
    const int64_t stat = (int64_t)head * a.Tq + s.q0 + tok;
    const float lse = here ? a.lse[stat] : -INFINITY;
    // the exponent takes lse in the scores' own units with a bias, else times log2 e; a row that sees nothing (or is none) has probabilities 0
    const float c = a.scale * kLog2e;
    float lse_b = lse == -INFINITY ? INFINITY : BIAS ? lse : lse * kLog2e, log_l = 0.f;

    arrived(fq);
    arrived(fdo);

    if constexpr (BIAS) {
        const bool is_far = fabsf(lse) >= kFar && fabsf(lse) < INFINITY, any = __any(is_far);
        if (lane == 0) far_rows[wave] = any;
        __syncthreads();
        if (__builtin_amdgcn_readfirstlane(far_rows[0] | far_rows[1] | far_rows[2] | far_rows[3])) {
            tile_sync();       // the tiles asked for above have landed: K's buffer is free
            const int all = keys_seen(a, s, row0 + kAttnRows, rows);       // whatever chunk of them is this block's
            float m = -INFINITY, l = 0.f;
            for (int k0 = 0; k0 < all; k0 += YT) {
                lk.start(k0, ldsK);
                lk.finish(ldsK);
                window[0][threadIdx.x] = window_load(a, h0, k0 + window0);
                tile_sync();
                if (k0 < wave_kend)
#pragma unroll 1
                    for (int u = 0; u < SUB; ++u) {
                        Acc<NP> S;
                        S.zero();
#pragma unroll
                        for (int ks = 0; ks < KS; ++ks) S.mma(TileY::rows(ldsK, 32 * u, ks, lane), fq[ks]);
                        float x[16], top = -INFINITY;
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int y = 32 * u + 8 * (i / 4) + 4 * h32 + i % 4;
                            x[i] = fmaf(S.get(i), a.scale, window[0][y + kAttnRows - 1 - 32 * wave - (lane & 31)]);
                            if (k0 + y >= limit) x[i] = -INFINITY;
                            top = fmaxf(top, x[i]);
                        }
                        const float mn = fmaxf(m, max_halves(top)), ms = mn == -INFINITY ? 0.f : mn;
                        l *= __builtin_amdgcn_exp2f((m - ms) * kLog2e);
                        m = mn;
#pragma unroll
                        for (int i = 0; i < 16; ++i) l += __builtin_amdgcn_exp2f((x[i] - ms) * kLog2e);
                    }
                __syncthreads();       // the tile has been read
            }
            l = sum_halves(l);
            if (is_far) lse_b = m == -INFINITY ? INFINITY : m, log_l = l == 0.f ? 0.f : __builtin_amdgcn_logf(l);
            if (kbeg < kend) {
                lk.start(kbeg, ldsK);
                window[0][threadIdx.x] = window_load(a, h0, kbeg + window0);
            }
        }
    }
    if (here && h32 == 0 && split == 0) {
        a.delta[stat] = delta;
        a.lse_b[stat] = lse_b;
        if constexpr (BIAS) a.log_l[stat] = log_l;
    }

    v16f dQ[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) dQ[dt] = v16f{};
    float far_past = 0.f, far_future = 0.f;

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
        if (k0 < wave_kend) {
            Frag<NP> fds[SUB][2];
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                Acc<NP> S, P;
                S.zero();
                P.zero();
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    S.mma(TileY::rows(ldsK + buf * TileY::BYTES, 32 * u, ks, lane), fq[ks]);
                    P.mma(TileY::rows(ldsV + buf * TileY::BYTES, 32 * u, ks, lane), fdo[ks]);
                }
                float ds[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int y = 32 * u + 8 * (i / 4) + 4 * h32 + i % 4;
                    float p;
                    if constexpr (BIAS) {
                        const float x = fmaf(S.get(i), a.scale, window[buf][y + kAttnRows - 1 - 32 * wave - (lane & 31)]);
                        p = __builtin_amdgcn_exp2f(fmaf(x - lse_b, kLog2e, -log_l));
                    } else p = __builtin_amdgcn_exp2f(fmaf(S.get(i), c, -lse_b));
                    ds[i] = p * (P.get(i) - delta);
                }
                if (k0 + 32 * u + 32 > wave_limit)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (32 * u + 8 * (i / 4) + i % 4 >= limit - k0 - 4 * h32) ds[i] = 0.f;
                if constexpr (BIAS) {
                    if (want_bias) {
                        // distances of this 32 x 32 part: first .. first + 62
                        const int delta0 = k0 + 32 * u - (row0 + 32 * wave) - off;
                        if (delta0 + 31 <= -a.W || delta0 - 31 >= a.W) {
                            float sum = 0.f;
#pragma unroll
                            for (int i = 0; i < 16; ++i) sum += here ? ds[i] : 0.f;
                            (delta0 < 0 ? far_past : far_future) += sum;
                        } else {
                            if (!here)
#pragma unroll
                                for (int i = 0; i < 16; ++i) ds[i] = 0.f;
                            const float v = diagonal_sum(ds, square[wave], lane);
                            const int delta = delta0 + lane - 31;
                            if (a.W > kNear) add_runs(v, lane < 63 ? (int)a.bid[min(max(delta, -a.W), a.W) + a.W] : -1, mine, lane);
                            else if (lane < 63) {
                                if (delta <= -a.W) far_past += v;
                                else if (delta >= a.W) far_future += v;
                                else mine[delta + a.W] += v;
                            }
                        }
                    }
                }
#pragma unroll
                for (int g = 0; g < 2; ++g) fds[u][g] = cut8<NP>(&ds[8 * g]);
            }
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                if constexpr (NP == 1) {
#pragma unroll
                    for (int u = 0; u < SUB; ++u)
#pragma unroll
                        for (int g = 0; g < 2; ++g) dQ[dt] = mfma(TileY::cols(ldsK + buf * TileY::BYTES, 32 * u + 16 * g, dt, lane).p[0], fds[u][g].p[0], dQ[dt]);
                } else {
                    Acc<NP> S;
                    S.zero();
#pragma unroll
                    for (int u = 0; u < SUB; ++u)
#pragma unroll
                        for (int g = 0; g < 2; ++g) S.mma(TileY::cols(ldsK + buf * TileY::BYTES, 32 * u + 16 * g, dt, lane), fds[u][g]);
#pragma unroll
                    for (int i = 0; i < 16; ++i) dQ[dt][i] += S.get(i);
                }
            }
        }
        if (more) {
            lk.finish(ldsK + (buf ^ 1) * TileY::BYTES);
            lv.finish(ldsV + (buf ^ 1) * TileY::BYTES);
            if constexpr (BIAS) window[buf ^ 1][threadIdx.x] = bias_next;
        }
    }
    if constexpr (NP == 1)
        if (__builtin_expect(s.m <= kFewKeys && wave_kend > 0, 0)) {       // the tile is in the first buffers
            int ln = lane;
            asm("" : "+v"(ln));
            const int hf = ln >> 5;
            static_assert(kFewKeys <= YT, "one tile");
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                if (32 * u >= wave_kend) break;
                Acc<NP> S, P;
                S.zero();
                P.zero();
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    S.mma(TileY::rows(ldsK, 32 * u, ks, ln), fq[ks]);
                    P.mma(TileY::rows(ldsV, 32 * u, ks, ln), fdo[ks]);
                }
                float ds[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int y = 32 * u + 8 * (i / 4) + 4 * hf + i % 4;
                    float p;
                    if constexpr (BIAS) {
                        const float x = fmaf(S.get(i), a.scale, window[0][y + kAttnRows - 1 - 32 * wave - (ln & 31)]);
                        p = __builtin_amdgcn_exp2f(fmaf(x - lse_b, kLog2e, -log_l));
                    } else p = __builtin_amdgcn_exp2f(fmaf(S.get(i), c, -lse_b));
                    ds[i] = y >= limit || !here ? 0.f : p * (P.get(i) - delta);
                    ds[i] -= to_f32(from_f32<bf16raw>(ds[i]));
                }
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    const Frag<NP> f = cut8<NP>(&ds[8 * g]);
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) dQ[dt] = mfma(TileY::cols(ldsK, 32 * u + 16 * g, dt, ln).p[0], f.p[0], dQ[dt]);
                }
            }
        }
    if (want_bias) {
#pragma unroll
        for (int m = 32; m; m >>= 1) {
            far_past += __shfl_xor(far_past, m);
            far_future += __shfl_xor(far_future, m);
        }
        float *const sums = a.W <= kNear ? square[wave] : mine;       // [buckets] of this wave
        if (a.W <= kNear) {       // the waves' sums by distance, in order, then by bucket: a quarter of the distances a wave
#pragma unroll
            for (int i = 0; i < 256; i += 64) sums[i + lane] = 0.f;
            __syncthreads();
            const int words = Lds::words(a.W);
            for (int i = 64 * wave; i < words; i += 256) {
                const bool there = i + lane < words;
                const float *w = by_wave + (there ? i + lane : 0);
                add_runs(there ? (w[0] + w[words]) + (w[2 * words] + w[3 * words]) : 0.f, there ? (int)a.bid[i + lane] : -1, sums, lane);
            }
        }
        if (lane == 0) {
            sums[a.bid[0]] += far_past;
            sums[a.bid[2 * a.W]] += far_future;
        }
        __syncthreads();
        const float *const all = a.W <= kNear ? square[0] : by_wave;
        const int apart = a.W <= kNear ? 63 * kDiag : Lds::words(a.W);
        for (int i = threadIdx.x; i < a.buckets; i += 256) bias_out[i] = (all[i] + all[apart + i]) + (all[2 * apart + i] + all[3 * apart + i]);
    }
    if (!here) return;
    if (chunks > 1)
        store_row(a.part[0] + (((int64_t)hr * a.tiles * a.splits + place.slot) * kAttnRows + (row - row0)) * DP, dQ, a.scale, DP, h32);
    else store_row(static_cast<T *>(a.dq) + (int64_t)(s.q0 + tok) * a.q_tok + (int64_t)head * a.q_head, dQ, a.scale, a.D, h32);
}

// dbias[h][bucket]: the dq kernel's items' sums added in a fixed order, in 64 bits.  A block takes a head and 16 buckets, 16 threads a
// bucket.  It rides in the dk/dv launch, behind the blocks of that.
__device__ __forceinline__ void sum_dbias(AttnArgs a, int item, double *lds)
{
    a.splits = a.dbias_splits, a.chunk = a.dbias_chunk, a.gsplit = 1, a.fold = a.levels = 0;
    Place p;
    find_place<false>(a, 0x7fffffff, p);
    const int parts = min(p.slot, a.dbias_parts);       // the dq kernel's items
    const int groups = (a.buckets + 15) / 16, h = item / groups, x = threadIdx.x % 16, j = threadIdx.x / 16, i = item % groups * 16 + x;
    double s = 0;
    if (i < a.buckets)
#pragma unroll 4
        for (int t = j; t < parts; t += 16) s += a.dbias_part[((int64_t)h * a.dbias_parts + t) * a.buckets + i];
    lds[j * 17 + x] = s;
    __syncthreads();
    if (j == 0 && i < a.buckets) {
#pragma unroll
        for (int k = 1; k < 16; ++k) s += lds[k * 17 + x];
        a.dbias[(int64_t)h * a.buckets + i] = (float)s;
    }
}

// X: 128 keys of a key-value head; Y: the query rows that see them, of all Gp heads.  With a bias Gp = 1, and the G heads
// are walked one after the other.  Four products a tile: 4 x 4096, 16 heads of 128, causal, bf16 580 us, 945 TFLOP/s; 2 x 4096, 32 heads on 8,
// 730, 750, because 64 blocks on a die read more rows at a time than its L2 holds.
template <class T, int DP> constexpr int kDkdvWaves = Pieces<T>::N == 1 || DP <= 32 ? 2 : 1;

template <class T, int DP, bool BIAS, bool DMA>
__global__ __launch_bounds__(256, (kDkdvWaves<T, DP>)) void attn_dkdv_kernel(AttnArgs a)
{
    constexpr int NP = Pieces<T>::N, KS = DP / 16, DT = DP / 32, YT = attn_dkdv_yt(NP == 1, DP), SUB = YT / 32;
    using TileY = Tile<DP, YT, NP>;
    // Two waves a SIMD (256 registers each) hide each other's LDS reads and exponentials.  At DP = 128 dK, dV and both operands' fragments
    // leave no room for anything else: V's fragments are read from LDS each time instead.
    constexpr bool V_IN_LDS = NP == 1 && DP >= 96;
    using TileX = Tile<DP, kAttnRows, NP>;
    __shared__ __align__(16) char lds_v[V_IN_LDS ? TileX::BYTES : 16];
    LdsByte *const ldsV = (LdsByte *)lds_v;
    __shared__ __align__(16) char lds[2][2][TileY::BYTES];
    LdsByte *const ldsQ = (LdsByte *)lds[0][0], *const ldsO = (LdsByte *)lds[1][0];
    constexpr int STATS = BIAS ? 3 : 2;
    __shared__ __align__(16) float stats[2][STATS][64];        // lse_b, delta (and log_l) of the tile's rows
    __shared__ float window[2][BIAS ? 256 : 1];
    const int lane = threadIdx.x & 63, wave = (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h32 = lane >> 5;
    if constexpr (BIAS) {
        const int mine = a.Hkv * a.tiles * a.splits * a.gsplit;
        if ((int)blockIdx.x >= mine) {
            __shared__ double sums[16 * 17];
            sum_dbias(a, blockIdx.x - mine, sums);
            return;
        }
    }
    const int hkv = blockIdx.x % a.Hkv;
    Place place;
    if (!find_place<true>(a, blockIdx.x / a.Hkv, place)) return;
    const int t = place.t, split = place.split / a.gsplit;
    const Seq s = seq_of(a, place.b);
    const int key0 = t * kAttnRows, rows = s.n * a.Gp, off = s.m - s.n;
    const int key = key0 + 32 * wave + (lane & 31);
    // Row r of token r / Gp sees the key from first_seeing on.  Keys behind the last one need no mask: what is added up for them is
    // not stored.
    const int first_row = first_seeing(a, s, key), wave_first = first_seeing(a, s, key0 + 32 * wave), wave_all = first_seeing(a, s, key0 + 32 * wave + 31);
    int begin = first_seeing(a, s, key0) / YT * YT, end = rows;
    const int chunks = chunks_of(a, begin, end);
    if (split >= chunks) return;
    if (chunks > 1) {
        begin += split * a.chunk;
        end = min(end, begin + a.chunk);
    }
    const int last = begin < end ? begin + (end - 1 - begin) / YT * YT : begin - YT;

    const FastDiv one = {1, 1, 0};
    const Rows<T> K{static_cast<const T *>(a.k) + (int64_t)s.k0 * a.k_tok + (int64_t)hkv * a.k_head, a.k_tok, 0, s.m, a.D, one};
    const Rows<T> V{static_cast<const T *>(a.v) + (int64_t)s.k0 * a.v_tok + (int64_t)hkv * a.v_head, a.v_tok, 0, s.m, a.D, one};
    Frag<NP> fk[KS], fv[V_IN_LDS ? 1 : KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        fk[ks] = frag_of(K.load(key, 16 * ks + 8 * h32));
        const Frag<NP> f = frag_of(V.load(key, 16 * ks + 8 * h32));
        if constexpr (V_IN_LDS) TileX::put(ldsV, 32 * wave + (lane & 31), 2 * ks + h32, f);      // read by the lane's own wave alone
        else fv[ks] = f;
    }
    arrived(fk);
    if constexpr (!V_IN_LDS) arrived(fv);
    v16f dK[DT], dV[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) dK[dt] = v16f{}, dV[dt] = v16f{};
    const float c = a.scale * kLog2e;
    const int heads = a.G / a.Gp, one_head = place.split % a.gsplit;
    for (int g = a.gsplit > 1 ? one_head : 0; g < (a.gsplit > 1 ? one_head + 1 : heads); ++g) {
        const int h0 = hkv * a.G + g * a.Gp;
        const Rows<T> Q{static_cast<const T *>(a.q) + (int64_t)s.q0 * a.q_tok + (int64_t)h0 * a.q_head, a.q_tok, a.q_head, rows, a.D, a.by_gp};
        const Rows<T> dO{static_cast<const T *>(a.d_o) + (int64_t)s.q0 * a.o_tok + (int64_t)h0 * a.o_head, a.o_tok, a.o_head, rows, a.D, a.by_gp};
        Loader<T, DP, YT, DMA> lq(Q), lo(dO);
        const int window0 = key0 - (YT - 1) - off;
        float bias_next = 0.f, stat_next = 0.f;
        // What the tile's rows have apart from their elements: threads 0 .. 63 lse_b, 64 .. 127 delta, 128 .. 191 log_l, a row each.  Rows
        // that are none get zeros: their elements are zeros as well, so that a probability of 1 adds nothing.
        auto row_start = [&](int y0, int to) {
            if (wave < STATS) {
                const int r = y0 + lane;
                const float *from = (wave == 0 ? a.lse_b : !BIAS || wave == 1 ? a.delta : a.log_l) + (int64_t)h0 * a.Tq + s.q0;
                const bool here = lane < YT && r < rows;
                if constexpr (DMA) {
                    const int tok = (int)fdiv((uint32_t)(here ? r : 0), a.by_gp);
                    const uint32_t at = (uint32_t)(((here ? r : 0) - tok * a.Gp) * a.Tq + tok) * 4u;      // Hq Tq < 2^29
                    dma4(raw_buffer((uint64_t)reinterpret_cast<uintptr_t>(from), kMaxBufferBytes), (LdsByte *)stats[to][wave], here ? at : OOB_ROW);
                } else {
                    const int tok = (int)fdiv((uint32_t)(here ? r : 0), a.by_gp);
                    stat_next = here ? from[(int64_t)(r - tok * a.Gp) * a.Tq + tok] : 0.f;
                }
            }
            if constexpr (BIAS) bias_next = window_load(a, h0, window0 - y0);
        };
        auto row_finish = [&](int to) {
            if constexpr (!DMA)
                if (wave < STATS) stats[to][wave][lane] = stat_next;
            if constexpr (BIAS) window[to][threadIdx.x] = bias_next;
        };
        int buf = 0;
        __syncthreads();      // the head before this one may still be read
        if (begin < end) {
            lq.start(last, ldsQ);
            lo.start(last, ldsO);
            row_start(last, 0);
            lq.finish(ldsQ);
            lo.finish(ldsO);
            row_finish(0);
        }
        // backwards: all blocks of a sequence then ask for the same rows at about the same time
        for (int y0 = last; y0 >= begin; y0 -= YT, buf ^= 1) {
            tile_sync();
            const bool more = y0 > begin;
            if (more) {
                lq.start(y0 - YT, ldsQ + (buf ^ 1) * TileY::BYTES);
                lo.start(y0 - YT, ldsO + (buf ^ 1) * TileY::BYTES);
                row_start(y0 - YT, buf ^ 1);
            }
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                if (y0 + 32 * u + 32 <= wave_first) continue;      // no row of these sees a key of this wave
                Acc<NP> S, P;
                S.zero();
                P.zero();
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    S.mma(TileY::rows(ldsQ + buf * TileY::BYTES, 32 * u, ks, lane), fk[ks]);
                    if constexpr (V_IN_LDS) P.mma(TileY::rows(ldsO + buf * TileY::BYTES, 32 * u, ks, lane), TileX::rows(ldsV, 32 * wave, ks, lane));
                    else P.mma(TileY::rows(ldsO + buf * TileY::BYTES, 32 * u, ks, lane), fv[ks]);
                }
                if constexpr (NP == 1) reads_ahead<2 * KS, 6, V_IN_LDS ? 2 : 1>();
                float p[16], ds[16];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int at = 32 * u + 8 * j + 4 * h32;
                    const float4 l4 = *reinterpret_cast<const float4 *>(stats[buf][0] + at), d4 = *reinterpret_cast<const float4 *>(stats[buf][1] + at);
                    const float4 g4 = BIAS ? *reinterpret_cast<const float4 *>(stats[buf][STATS - 1] + at) : float4{};
                    const float l[4] = {l4.x, l4.y, l4.z, l4.w}, d[4] = {d4.x, d4.y, d4.z, d4.w}, log_l[4] = {g4.x, g4.y, g4.z, g4.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float x;
                        if constexpr (BIAS) {
                            x = fmaf(S.get(4 * j + i), a.scale, window[buf][32 * wave + (lane & 31) - (at + i) + YT - 1]);
                            x = __builtin_amdgcn_exp2f(fmaf(x - l[i], kLog2e, -log_l[i]));
                        } else x = __builtin_amdgcn_exp2f(fmaf(S.get(4 * j + i), c, -l[i]));
                        p[4 * j + i] = x;
                        ds[4 * j + i] = x * (P.get(4 * j + i) - d[i]);
                    }
                }
                const int y = y0 + 32 * u;
                // some row does not see some key; or, with a bias, whose exponential may be an infinity, some row is none
                if (y < wave_all || (BIAS && y + 32 > rows))
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int r = 8 * (i / 4) + i % 4;
                        if (r < first_row - y - 4 * h32 || (BIAS && r >= rows - y - 4 * h32)) p[i] = 0.f, ds[i] = 0.f;
                    }
                Frag<NP> fp[2], fds[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    fp[e] = cut8<NP>(&p[8 * e]);
                    fds[e] = cut8<NP>(&ds[8 * e]);
                }
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    if constexpr (NP == 1) {
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            dV[dt] = mfma(TileY::cols(ldsO + buf * TileY::BYTES, 32 * u + 16 * e, dt, lane).p[0], fp[e].p[0], dV[dt]);
                            dK[dt] = mfma(TileY::cols(ldsQ + buf * TileY::BYTES, 32 * u + 16 * e, dt, lane).p[0], fds[e].p[0], dK[dt]);
                        }
                    } else {
                        Acc<NP> A;
                        A.zero();
#pragma unroll
                        for (int e = 0; e < 2; ++e) A.mma(TileY::cols(ldsO + buf * TileY::BYTES, 32 * u + 16 * e, dt, lane), fp[e]);
#pragma unroll
                        for (int i = 0; i < 16; ++i) dV[dt][i] += A.get(i);
                        A.zero();
#pragma unroll
                        for (int e = 0; e < 2; ++e) A.mma(TileY::cols(ldsQ + buf * TileY::BYTES, 32 * u + 16 * e, dt, lane), fds[e]);
#pragma unroll
                        for (int i = 0; i < 16; ++i) dK[dt][i] += A.get(i);
                    }
                }
            }
            if (more) {
                lq.finish(ldsQ + (buf ^ 1) * TileY::BYTES);
                lo.finish(ldsO + (buf ^ 1) * TileY::BYTES);
                row_finish(buf ^ 1);
            }
        }
        if constexpr (NP == 1)
            if (__builtin_expect(rows <= kFewRows && begin < end && key0 + 32 * wave < s.m, 0)) {       // the rows are in the first buffers
                int ln = lane;
                asm("" : "+v"(ln));
                int y = begin;
                const int hf = ln >> 5;
#pragma unroll 1
                do {
                    Acc<NP> S, P;
                    S.zero();
                    P.zero();
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) {
                        S.mma(TileY::rows(ldsQ, 0, ks, ln), fk[ks]);
                        if constexpr (V_IN_LDS) P.mma(TileY::rows(ldsO, 0, ks, ln), TileX::rows(ldsV, 32 * wave, ks, ln));
                        else P.mma(TileY::rows(ldsO, 0, ks, ln), fv[ks]);
                    }
                    reads_ahead<2 * KS, 6, V_IN_LDS ? 2 : 1>();
                    float p[16], ds[16];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int at = 8 * j + 4 * hf;
                        const float4 l4 = *reinterpret_cast<const float4 *>(stats[0][0] + at), d4 = *reinterpret_cast<const float4 *>(stats[0][1] + at);
                        const float4 g4 = BIAS ? *reinterpret_cast<const float4 *>(stats[0][STATS - 1] + at) : float4{};
                        const float l[4] = {l4.x, l4.y, l4.z, l4.w}, d[4] = {d4.x, d4.y, d4.z, d4.w}, log_l[4] = {g4.x, g4.y, g4.z, g4.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            float x;
                            if constexpr (BIAS) {
                                x = fmaf(S.get(4 * j + i), a.scale, window[0][32 * wave + (ln & 31) - (at + i) + YT - 1]);
                                x = __builtin_amdgcn_exp2f(fmaf(x - l[i], kLog2e, -log_l[i]));
                            } else x = __builtin_amdgcn_exp2f(fmaf(S.get(4 * j + i), c, -l[i]));
                            p[4 * j + i] = x;
                            ds[4 * j + i] = x * (P.get(4 * j + i) - d[i]);
                        }
                    }
                    if (wave_all > 0 || BIAS)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int r = 8 * (i / 4) + i % 4;
                            if (r < first_row - 4 * hf || (BIAS && r >= rows - 4 * hf)) p[i] = 0.f, ds[i] = 0.f;
                        }
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
#pragma unroll
                        for (int i = 8 * e; i < 8 * e + 8; ++i) {
                            p[i] -= to_f32(from_f32<bf16raw>(p[i]));
                            ds[i] -= to_f32(from_f32<bf16raw>(ds[i]));
                        }
                        const Frag<NP> fp = cut8<NP>(&p[8 * e]), fds = cut8<NP>(&ds[8 * e]);
#pragma unroll
                        for (int dt = 0; dt < DT; ++dt) {
                            dV[dt] = mfma(TileY::cols(ldsO, 16 * e, dt, ln).p[0], fp.p[0], dV[dt]);
                            dK[dt] = mfma(TileY::cols(ldsQ, 16 * e, dt, ln).p[0], fds.p[0], dK[dt]);
                        }
                    }
                } while (!BIAS && (y += 32) < rows);       // one turn; told so, the compiler spills in the loop above at 128 wide (600 -> 680 us)
            }
        if constexpr (!BIAS && NP == 1) break;       // all heads that share the keys are one problem
    }
    if (key >= s.m) return;
    if (chunks * a.gsplit > 1) {
        const int64_t at = (((int64_t)hkv * a.tiles * a.splits * a.gsplit + place.slot) * kAttnRows + (key - key0)) * DP;
        store_row(a.part[0] + at, dK, a.scale, DP, h32);
        store_row(a.part[1] + at, dV, 1.f, DP, h32);
    } else {
        store_row(static_cast<T *>(a.dk) + (int64_t)(s.k0 + key) * a.k_tok + (int64_t)hkv * a.k_head, dK, a.scale, a.D, h32);
        store_row(static_cast<T *>(a.dv) + (int64_t)(s.k0 + key) * a.v_tok + (int64_t)hkv * a.v_head, dV, 1.f, a.D, h32);
    }
}

template <class T, int DP, bool DMA> int dq_run(AttnArgs a, hipStream_t s)
{
    const int problems = a.Hq / a.Gp, waves = a.btab ? kDqWaves<T, DP, true> : kDqWaves<T, DP, false>;
    a.levels = levels_of(a, problems, waves == 2 && (a.btab || !DMA));
    a.fold = fold_of(a, problems, waves);
    const dim3 grid((unsigned)(a.Hq / a.Gp) * a.tiles * a.splits);
    const unsigned by_wave = a.dbias_part ? 4 * sizeof(float) * DqLds<T, DP>::words(a.W) : 0;
    if (a.btab) hipLaunchKernelGGL((attn_dq_kernel<T, DP, true, DMA>), grid, dim3(256), by_wave, s, a);
    else hipLaunchKernelGGL((attn_dq_kernel<T, DP, false, DMA>), grid, dim3(256), 0, s, a);
    CG_HIP_TRY(hipGetLastError());
    return CG_OK;
}
template <class T, int DP> int dq_dp(const AttnArgs &a, hipStream_t s)
{
    if (a.dma) return dq_run<T, DP, true>(a, s);
    return dq_run<T, DP, false>(a, s);
}
template <class T, int DP, bool DMA> int dkdv_run(AttnArgs a, hipStream_t s)
{
    a.levels = levels_of(a, a.Hkv, kDkdvWaves<T, DP> == 2 && (a.btab || !DMA));
    a.fold = fold_of(a, a.Hkv, kDkdvWaves<T, DP>);
    const dim3 grid((unsigned)a.Hkv * a.tiles * a.splits * a.gsplit + (a.dbias ? (unsigned)a.Hq * ((a.buckets + 15) / 16) : 0u));
    if (a.btab) hipLaunchKernelGGL((attn_dkdv_kernel<T, DP, true, DMA>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((attn_dkdv_kernel<T, DP, false, DMA>), grid, dim3(256), 0, s, a);
    CG_HIP_TRY(hipGetLastError());
    return CG_OK;
}
template <class T, int DP> int dkdv_dp(const AttnArgs &a, hipStream_t s)
{
    if (a.dma) return dkdv_run<T, DP, true>(a, s);
    return dkdv_run<T, DP, false>(a, s);
}

}  // namespace

int attn_dq_launch(const AttnArgs &a, int type, hipStream_t s)
{
#define CG_DP(DP) if (a.D <= DP) return type == CG_TYPE_FP32 ? dq_dp<float, DP>(a, s) : dq_dp<bf16raw, DP>(a, s)
    CG_DP(32);
    CG_DP(64);
    CG_DP(96);
    CG_DP(128);
#undef CG_DP
    return CG_EUNSUPPORTED;
}
int attn_dkdv_launch(const AttnArgs &a, int type, hipStream_t s)
{
#define CG_DP(DP) if (a.D <= DP) return type == CG_TYPE_FP32 ? dkdv_dp<float, DP>(a, s) : dkdv_dp<bf16raw, DP>(a, s)
    CG_DP(32);
    CG_DP(64);
    CG_DP(96);
    CG_DP(128);
#undef CG_DP
    return CG_EUNSUPPORTED;
}
}  // namespace cg
