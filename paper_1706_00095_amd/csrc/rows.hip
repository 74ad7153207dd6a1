// Operators over rows: dropout from a counter-based generator, layer norm, and the two joined with the residual addition.
//
// All of them are bound by HBM: every kernel reads each input once and writes each output once.  A row's elements stay in
// registers between the passes that its statistics need (mean, then the centred squares: a sum of squares minus a squared
// mean would lose the variance of rows whose mean is large).
#include <cmath>
#include "cg_internal.h"
#include "typed_device.h"

namespace cg {
namespace {

// ---- the generator -----------------------------------------------------------------------------------------------------
// Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3, 2011): ten rounds of two
// 32 x 32 -> 64 bit products.  A block of four words covers eight elements, 16 bits each.  The round keys are uniform and
// live in scalar registers.
struct DropArgs {
    uint32_t key0, key1, off0, off1;
    uint32_t t;               // threshold: 16 bits below it drop the element
    float factor;             // of the kept ones
};

// bit e: element e of block `blk` is kept
__device__ __forceinline__ uint32_t keep8(uint64_t blk, const DropArgs &d)
{
    uint32_t c0 = (uint32_t)blk, c1 = (uint32_t)(blk >> 32), c2 = d.off0, c3 = d.off1, k0 = d.key0, k1 = d.key1;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    const uint32_t w[4] = {c0, c1, c2, c3}, t = d.t << 16;
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m |= (uint32_t)(w[i] << 16 >= t) << (2 * i);
        m |= (uint32_t)(w[i] >= t) << (2 * i + 1);       // the low half cannot reach a multiple of 2^16
    }
    return m;
}
// elements e .. e + 7, which lie in two blocks unless e is a multiple of 8
template <bool ON_BLOCKS> __device__ __forceinline__ uint32_t keep_from(uint64_t e, const DropArgs &d)
{
    if constexpr (ON_BLOCKS) return keep8(e >> 3, d);
    const uint32_t s = (uint32_t)e & 7u;
    return (keep8(e >> 3, d) | keep8((e >> 3) + 1, d) << 8) >> s;
}
__device__ __forceinline__ float dropped(float x, uint32_t keep, int i, const DropArgs &d)
{
    return keep >> i & 1u ? x * d.factor : 0.f;
}

// ---- dropout ----------------------------------------------------------------------------------------------------------
// A thread takes the eight elements of one block of the generator, so each block is computed once whatever the width.
// DENSE: rows follow each other without a gap in all tensors, and a block is eight neighbours.  Otherwise a block's
// elements are neighbours unless a row ends among them.
// Bound by HBM: 16384 x 4096 bf16 with an addend 70 us, 5.8 TB/s (a large copy: 5.1); the generator's 1.7 G multiplications hide behind.
struct DropoutArgs {
    const void *x, *add;
    void *y;
    int64_t x_ld, add_ld, y_ld;
    uint32_t n, cols;         // elements, and of a row
    FastDiv by_cols;
    DropArgs drop;
};

template <class T, bool DENSE, bool ADD> __global__ __launch_bounds__(256) void dropout_rows_kernel(DropoutArgs a)
{
    const uint32_t blocks = (a.n + 7) / 8;
    for (uint32_t b = blockIdx.x * 256 + threadIdx.x; b < blocks; b += gridDim.x * 256) {
        const uint32_t e0 = b * 8;
        uint32_t r = 0, c = e0;
        int n = (int)min(a.n - e0, 8u);
        if constexpr (!DENSE) {
            r = fdiv(e0, a.by_cols);
            c = e0 - r * a.cols;
        }
        const T *x = static_cast<const T *>(a.x) + (int64_t)r * a.x_ld + c;
        const T *add = static_cast<const T *>(a.add) + (int64_t)r * a.add_ld + c;
        T *y = static_cast<T *>(a.y) + (int64_t)r * a.y_ld + c;
        if (DENSE || c + (uint32_t)n <= a.cols) {
            const Raw8<T> xv = load8(x, n);
            Raw8<T> av;
            if constexpr (ADD) av = load8(add, n);
            const uint32_t keep = keep8(b, a.drop);
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                f[i] = dropped(elem(xv, i), keep, i, a.drop);
                if constexpr (ADD) f[i] += elem(av, i);
            }
            store8(y, to_raw<T>(f), n);
        } else {       // rows end among the eight
            const uint32_t keep = keep8(b, a.drop);
            for (int i = 0; i < n; ++i) {
                float f = dropped(to_f32(*x), keep, i, a.drop);
                if constexpr (ADD) f += to_f32(*add);
                *y = from_f32<T>(f);
                ++x, ++add, ++y;
                if (++c == a.cols) {
                    c = 0;
                    x += a.x_ld - a.cols;
                    add += a.add_ld - a.cols;
                    y += a.y_ld - a.cols;
                }
            }
        }
    }
}

// ---- layer norm ---------------------------------------------------------------------------------------------------------
// LANES lanes share a row, each holds CPT chunks of eight columns: chunk k of lane t covers the columns 8 (k LANES + t) ..  A quarter of a
// wave (up to 128 columns), half of one and one need no barrier; wider rows join the waves' sums through LDS.  65536 x 256 bf16, half a
// wave a row: forward 13 us (5.2 TB/s), backward 20 (5.1); with a whole one, half of whose lanes have nothing, 20 and 33.

template <int LANES = 64> __device__ __forceinline__ float wave_sum(float x)
{
#pragma unroll
    for (int m = (LANES < 64 ? LANES : 64) / 2; m; m >>= 1) x += __shfl_xor(x, m);
    return x;
}
// Sums of N numbers over the LANES lanes of a row; every lane gets them.  `lds`: N floats for each of the row's waves, free for
// use (the barrier behind the reads is the next call's or the caller's).
template <int LANES, int N> __device__ __forceinline__ void row_sums(float (&v)[N], float *lds)
{
    constexpr int WPR = LANES / 64;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_sum<LANES>(v[i]);
    if constexpr (WPR > 1) {
        const int wave = (threadIdx.x >> 6) % WPR;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) lds[i * WPR + wave] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = 0.f;
#pragma unroll
            for (int w = 0; w < WPR; ++w) v[i] += lds[i * WPR + w];
        }
    }
}

struct NormArgs {
    const void *x, *branch;           // branch: joined only
    const float *gamma, *beta;
    void *sum, *y;
    float *mean, *rstd;               // NULL: not kept
    int64_t x_ld, branch_ld, sum_ld, y_ld;
    int rows, cols;
    float eps;
    DropArgs drop;
};
struct NormBwdArgs {
    const void *dy, *x, *dsum;        // x: what was normalised; dsum may be NULL
    const float *gamma, *mean, *rstd;
    void *dx, *dbranch;               // dbranch: joined only
    float *part;                      // [gridDim.x][2][cols]: sums over a block's rows
    float *dgamma, *dbeta;            // of a single block: its sums are the result; else NULL
    int64_t dy_ld, x_ld, dsum_ld, dx_ld, dbranch_ld;
    int rows, cols;
    DropArgs drop;
};

// Bound by HBM: 16384 x 2048 bf16 24 us (5.5 TB/s); joined, 8192 x 4096 bf16, 56 (4.8).
// JOIN: 0 = layer norm alone, 1 = joined, rows on the generator's blocks (cols a multiple of 8), 2 = joined, any cols
template <class T, int LANES, int CPT, int JOIN, int BLOCK>
__global__ __launch_bounds__(BLOCK) void norm_fwd_kernel(NormArgs a)
{
    constexpr int ROWS = BLOCK / LANES, WAVES = LANES < 64 ? 1 : LANES / 64;
    __shared__ float lds[ROWS][2][WAVES];
    const int slot = threadIdx.x / LANES, t = threadIdx.x % LANES;
    const float inv = 1.f / (float)a.cols;
    float gam[CPT][8], bet[CPT][8];
#pragma unroll
    for (int k = 0; k < CPT; ++k) {
        const int c = 8 * (k * LANES + t);
        const Raw8<float> g = load8(a.gamma + c, a.cols - c), b = load8(a.beta + c, a.cols - c);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            gam[k][i] = elem(g, i);
            bet[k][i] = elem(b, i);
        }
    }
    // every wave of a block makes the same number of turns: a row's barriers are the block's
    for (int r0 = blockIdx.x * ROWS; r0 < a.rows; r0 += gridDim.x * ROWS) {
        const int r = r0 + slot;
        const bool here = r < a.rows;
        float f[CPT][8];
        float s[1] = {0.f};
#pragma unroll
        for (int k = 0; k < CPT; ++k) {
            const int c = 8 * (k * LANES + t), n = here ? a.cols - c : 0;
            Raw8<T> v = load8(static_cast<const T *>(a.x) + (int64_t)r * a.x_ld + c, n);
            if constexpr (JOIN != 0) {
                const Raw8<T> b = load8(static_cast<const T *>(a.branch) + (int64_t)r * a.branch_ld + c, n);
                const uint32_t keep = keep_from<JOIN == 1>((uint64_t)r * a.cols + c, a.drop);
                float g[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) g[i] = elem(v, i) + dropped(elem(b, i), keep, i, a.drop);
                v = to_raw<T>(g);       // the norm is that of the sum as it is stored
                store8(static_cast<T *>(a.sum) + (int64_t)r * a.sum_ld + c, v, n);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                f[k][i] = elem(v, i);
                s[0] += f[k][i];
            }
        }
        row_sums<LANES, 1>(s, lds[slot][0]);
        const float mean = s[0] * inv;
        float q[1] = {0.f};
#pragma unroll
        for (int k = 0; k < CPT; ++k) {
            const int n = a.cols - 8 * (k * LANES + t);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                f[k][i] = i < n ? f[k][i] - mean : 0.f;
                q[0] = fmaf(f[k][i], f[k][i], q[0]);
            }
        }
        row_sums<LANES, 1>(q, lds[slot][1]);
        const float rstd = 1.f / sqrtf(fmaf(q[0], inv, a.eps));
        if (here && t == 0 && a.mean) {
            a.mean[r] = mean;
            a.rstd[r] = rstd;
        }
#pragma unroll
        for (int k = 0; k < CPT; ++k) {
            const int c = 8 * (k * LANES + t), n = here ? a.cols - c : 0;
            float y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = fmaf(f[k][i] * rstd, gam[k][i], bet[k][i]);
            store8(static_cast<T *>(a.y) + (int64_t)r * a.y_ld + c, to_raw<T>(y), n);
        }
    }
}

// dx of a row needs two sums over it, <g> and <g xh> with g = dy gamma; dgamma and dbeta are sums over the rows, which each
// thread keeps for its columns over all the rows that its block takes.  Blocks write their sums to `part`; sum_parts_kernel adds
// them in order, so results do not depend on scheduling.
// Bound by HBM: 16384 x 2048 bf16 40 us (5.0 TB/s); joined, 8192 x 4096 bf16, 62 (4.3); the sums of the blocks' sums 4 to 7.  With four
// chunks a thread in fp32 (8193 to 16384 columns) 13 to 15 registers are spilled.
template <class T, int LANES, int CPT, int JOIN, int BLOCK>
__global__ __launch_bounds__(BLOCK) void norm_bwd_kernel(NormBwdArgs a)
{
    constexpr int ROWS = BLOCK / LANES, WAVES = LANES < 64 ? 1 : LANES / 64;
    __shared__ float lds[2][ROWS][2][WAVES];
    __shared__ float join[ROWS > 1 ? ROWS - 1 : 1][ROWS > 1 ? LANES * 8 : 1];
    const int slot = threadIdx.x / LANES, t = threadIdx.x % LANES;
    const float inv = 1.f / (float)a.cols;
    // gains, and what else a row needs, in registers from row to row and ahead of the sums, where there is room: four chunks a
    // thread read them again (out of the caches) and later
    constexpr bool ROOM = CPT < 4;
    float dg[CPT][8], db[CPT][8];
    Raw8<float> gam[CPT];
    auto gains = [&](int k) {
        const int c = 8 * (k * LANES + t);
        gam[k] = load8(a.gamma + c, a.cols - c);
    };
#pragma unroll
    for (int k = 0; k < CPT; ++k) {
        if (ROOM) gains(k);
#pragma unroll
        for (int i = 0; i < 8; ++i) dg[k][i] = db[k][i] = 0.f;
    }
    struct Row {
        Raw8<T> x[CPT], d[CPT], s[CPT];
        float mean, rstd;
    };
    auto load = [&](Row &v, int r) {
        const bool here = r < a.rows;
#pragma unroll
        for (int k = 0; k < CPT; ++k) {
            const int c = 8 * (k * LANES + t), n = here ? a.cols - c : 0;
            v.x[k] = load8(static_cast<const T *>(a.x) + (int64_t)r * a.x_ld + c, n);
            v.d[k] = load8(static_cast<const T *>(a.dy) + (int64_t)r * a.dy_ld + c, n);
            if (ROOM && a.dsum) v.s[k] = load8(static_cast<const T *>(a.dsum) + (int64_t)r * a.dsum_ld + c, n);
        }
        v.mean = here ? a.mean[r] : 0.f, v.rstd = here ? a.rstd[r] : 0.f;
    };
    int turn = 0;
    Row row, next;
    if (ROOM) load(row, blockIdx.x * ROWS + slot);
    for (int r0 = blockIdx.x * ROWS; r0 < a.rows; r0 += gridDim.x * ROWS, turn ^= 1) {
        const int r = r0 + slot, r1 = r + gridDim.x * ROWS;
        const bool here = r < a.rows, more = r0 + (int)(gridDim.x * ROWS) < a.rows;
        if (!ROOM) load(row, r);
        else if (more) load(next, r1);       // on its way while this row is worked on
        Raw8<T> (&vx)[CPT] = row.x, (&vd)[CPT] = row.d, (&vs)[CPT] = row.s;
        const float mean = row.mean, rstd = row.rstd;
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int k = 0; k < CPT; ++k) {
            const int n = a.cols - 8 * (k * LANES + t);
            if (!ROOM) gains(k);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float dy = elem(vd[k], i), xh = i < n ? (elem(vx[k], i) - mean) * rstd : 0.f, g = dy * elem(gam[k], i);
                s[0] += g;
                s[1] = fmaf(g, xh, s[1]);
                dg[k][i] = fmaf(dy, xh, dg[k][i]);
                db[k][i] += dy;
            }
        }
        row_sums<LANES, 2>(s, lds[turn][slot][0]);
        const float c1 = s[0] * inv, c2 = s[1] * inv;
#pragma unroll
        for (int k = 0; k < CPT; ++k) {
            const int c = 8 * (k * LANES + t), n = here ? a.cols - c : 0;
            float f[8];
            if (!ROOM) {
                gains(k);
                if (a.dsum) vs[k] = load8(static_cast<const T *>(a.dsum) + (int64_t)r * a.dsum_ld + c, n);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float xh = (elem(vx[k], i) - mean) * rstd, g = elem(vd[k], i) * elem(gam[k], i);
                f[i] = rstd * (g - c1 - xh * c2);
                if (a.dsum) f[i] += elem(vs[k], i);
            }
            const Raw8<T> v = to_raw<T>(f);
            store8(static_cast<T *>(a.dx) + (int64_t)r * a.dx_ld + c, v, n);
            if constexpr (JOIN != 0) {
                const uint32_t keep = keep_from<JOIN == 1>((uint64_t)r * a.cols + c, a.drop);
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] = dropped(elem(v, i), keep, i, a.drop);
                store8(static_cast<T *>(a.dbranch) + (int64_t)r * a.dbranch_ld + c, to_raw<T>(f), n);
            }
        }
        if (ROOM) row = next;
    }
    // the block's rows joined, then one row of sums a block
    float *const out[2] = {a.dgamma ? a.dgamma : a.part + (int64_t)blockIdx.x * 2 * a.cols,
                           a.dbeta ? a.dbeta : a.part + ((int64_t)blockIdx.x * 2 + 1) * a.cols};
#pragma unroll
    for (int k = 0; k < CPT; ++k)
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            float (&v)[8] = which ? db[k] : dg[k];
            if constexpr (ROWS > 1) {
                __syncthreads();
                if (slot > 0)
#pragma unroll
                    for (int i = 0; i < 8; ++i) join[slot - 1][i * LANES + t] = v[i];
                __syncthreads();
                if (slot > 0) continue;
                for (int j = 0; j < ROWS - 1; ++j)
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] += join[j][i * LANES + t];
            }
            const int c = 8 * (k * LANES + t);
            store8(out[which] + c, to_raw<float>(v), a.cols - c);
        }
}

// Rows longer than the registers of a block hold: a block walks the row three times, the second and third time out of L2.
// 1024 x 32768 bf16: 47 us, 2.9 TB/s of what HBM has to move; backward 49, and 24 for the columns' sums.
constexpr int LONG_BLOCK = 1024;
template <class T, int JOIN> __global__ __launch_bounds__(LONG_BLOCK) void norm_fwd_long_kernel(NormArgs a)
{
    constexpr int W = LONG_BLOCK / 64;
    __shared__ float lds[2][2 * W];
    const float inv = 1.f / (float)a.cols;
    for (int r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T *x = static_cast<const T *>(a.x) + (int64_t)r * a.x_ld;
        T *sum = static_cast<T *>(a.sum) + (int64_t)r * a.sum_ld;
        float s[1] = {0.f}, q[1] = {0.f};
        for (int c = 8 * threadIdx.x; c < a.cols; c += 8 * LONG_BLOCK) {
            Raw8<T> v = load8(x + c, a.cols - c);
            if constexpr (JOIN != 0) {
                const Raw8<T> b = load8(static_cast<const T *>(a.branch) + (int64_t)r * a.branch_ld + c, a.cols - c);
                const uint32_t keep = keep_from<JOIN == 1>((uint64_t)r * a.cols + c, a.drop);
                float g[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) g[i] = elem(v, i) + dropped(elem(b, i), keep, i, a.drop);
                v = to_raw<T>(g);
                store8(sum + c, v, a.cols - c);      // read again below by the thread that wrote it
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) s[0] += elem(v, i);
        }
        row_sums<LONG_BLOCK, 1>(s, lds[0]);
        const float mean = s[0] * inv;
        if constexpr (JOIN != 0) x = sum;
        for (int c = 8 * threadIdx.x; c < a.cols; c += 8 * LONG_BLOCK) {
            const Raw8<T> v = load8(x + c, a.cols - c);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = c + i < a.cols ? elem(v, i) - mean : 0.f;
                q[0] = fmaf(d, d, q[0]);
            }
        }
        row_sums<LONG_BLOCK, 1>(q, lds[1]);
        const float rstd = 1.f / sqrtf(fmaf(q[0], inv, a.eps));
        if (threadIdx.x == 0 && a.mean) {
            a.mean[r] = mean;
            a.rstd[r] = rstd;
        }
        for (int c = 8 * threadIdx.x; c < a.cols; c += 8 * LONG_BLOCK) {
            const Raw8<T> v = load8(x + c, a.cols - c);
            const Raw8<float> g = load8(a.gamma + c, a.cols - c), b = load8(a.beta + c, a.cols - c);
            float y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = fmaf((elem(v, i) - mean) * rstd, elem(g, i), elem(b, i));
            store8(static_cast<T *>(a.y) + (int64_t)r * a.y_ld + c, to_raw<T>(y), a.cols - c);
        }
    }
}
template <class T, int JOIN> __global__ __launch_bounds__(LONG_BLOCK) void norm_bwd_long_kernel(NormBwdArgs a)
{
    constexpr int W = LONG_BLOCK / 64;
    __shared__ float lds[2][2 * W];
    const float inv = 1.f / (float)a.cols;
    int turn = 0;
    for (int r = blockIdx.x; r < a.rows; r += gridDim.x, turn ^= 1) {
        const T *x = static_cast<const T *>(a.x) + (int64_t)r * a.x_ld, *dy = static_cast<const T *>(a.dy) + (int64_t)r * a.dy_ld;
        const float mean = a.mean[r], rstd = a.rstd[r];
        float s[2] = {0.f, 0.f};
        for (int c = 8 * threadIdx.x; c < a.cols; c += 8 * LONG_BLOCK) {
            const Raw8<T> vx = load8(x + c, a.cols - c), vd = load8(dy + c, a.cols - c);
            const Raw8<float> gm = load8(a.gamma + c, a.cols - c);
#pragma unroll
            for (int i = 0; i < 8; ++i) {       // behind the row's end g is 0
                const float g = elem(vd, i) * elem(gm, i);
                s[0] += g;
                s[1] = fmaf(g, (elem(vx, i) - mean) * rstd, s[1]);
            }
        }
        row_sums<LONG_BLOCK, 2>(s, lds[turn]);
        const float c1 = s[0] * inv, c2 = s[1] * inv;
        for (int c = 8 * threadIdx.x; c < a.cols; c += 8 * LONG_BLOCK) {
            const Raw8<T> vx = load8(x + c, a.cols - c), vd = load8(dy + c, a.cols - c);
            const Raw8<float> gm = load8(a.gamma + c, a.cols - c);
            Raw8<T> vs;
            if (a.dsum) vs = load8(static_cast<const T *>(a.dsum) + (int64_t)r * a.dsum_ld + c, a.cols - c);
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                f[i] = rstd * (elem(vd, i) * elem(gm, i) - c1 - (elem(vx, i) - mean) * rstd * c2);
                if (a.dsum) f[i] += elem(vs, i);
            }
            const Raw8<T> v = to_raw<T>(f);
            store8(static_cast<T *>(a.dx) + (int64_t)r * a.dx_ld + c, v, a.cols - c);
            if constexpr (JOIN != 0) {
                const uint32_t keep = keep_from<JOIN == 1>((uint64_t)r * a.cols + c, a.drop);
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] = dropped(elem(v, i), keep, i, a.drop);
                store8(static_cast<T *>(a.dbranch) + (int64_t)r * a.dbranch_ld + c, to_raw<T>(f), a.cols - c);
            }
        }
    }
}
// dgamma and dbeta of long rows: a thread keeps the sums of eight columns over the rows of its slice (blockIdx.y of gridDim.y)
template <class T> __global__ __launch_bounds__(64) void norm_columns_kernel(NormBwdArgs a)
{
    const int c = 8 * (blockIdx.x * 64 + threadIdx.x), n = a.cols - c;
    float dg[8] = {}, db[8] = {};
    for (int r = blockIdx.y; r < a.rows; r += gridDim.y) {
        const Raw8<T> vx = load8(static_cast<const T *>(a.x) + (int64_t)r * a.x_ld + c, n);
        const Raw8<T> vd = load8(static_cast<const T *>(a.dy) + (int64_t)r * a.dy_ld + c, n);
        const float mean = a.mean[r], rstd = a.rstd[r];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            dg[i] = fmaf(elem(vd, i), (elem(vx, i) - mean) * rstd, dg[i]);
            db[i] += elem(vd, i);
        }
    }
    float *out = a.part + (int64_t)blockIdx.y * 2 * a.cols;
    store8(out + c, to_raw<float>(dg), n);
    store8(out + a.cols + c, to_raw<float>(db), n);
}

// dgamma, dbeta: the blocks' sums, [parts][2][cols], added.  A block takes 16 of the 2 cols columns, 16 threads each: thread j
// adds the parts j, j + 16, .. and the threads' sums are added in order.  A launch has fewer than 2^32 threads, so blocks of rows
// longer than 2^19 take 16 columns after the other.
constexpr int SUM_BLOCKS = 1 << 16;
__global__ __launch_bounds__(256) void sum_parts_kernel(const float *part, int parts, int cols, float *dgamma, float *dbeta)
{
    __shared__ float lds[16][17];
    const int x = threadIdx.x % 16, j = threadIdx.x / 16;
    const int64_t n = 2 * (int64_t)cols;
    for (int64_t c0 = (int64_t)blockIdx.x * 16; c0 < n; c0 += (int64_t)gridDim.x * 16) {
        const int64_t col = c0 + x;
        float s = 0.f;
        if (col < n)
#pragma unroll 4
            for (int p = j; p < parts; p += 16) s += part[p * n + col];
        lds[j][x] = s;
        __syncthreads();
        if (j == 0 && col < n) {
#pragma unroll
            for (int i = 1; i < 16; ++i) s += lds[i][x];
            (col < cols ? dgamma[col] : dbeta[col - cols]) = s;
        }
        __syncthreads();
    }
}

// ---- host side ----------------------------------------------------------------------------------------------------------

DropArgs drop_args(const cg_drop &d)
{
    DropArgs a;
    const double t = std::floor(65536.0 * d.p + 0.5);
    a.t = t >= 65535.0 ? 65535u : (uint32_t)t;
    a.factor = 65536.f / (float)(65536u - a.t);
    a.key0 = (uint32_t)d.seed;
    a.key1 = (uint32_t)(d.seed >> 32);
    a.off0 = (uint32_t)d.offset;
    a.off1 = (uint32_t)(d.offset >> 32);
    return a;
}
bool drop_ok(const cg_drop *d) { return d && d->p >= 0.0 && d->p < 1.0; }
bool type_ok(int type) { return type == CG_TYPE_FP32 || type == CG_TYPE_BF16; }
size_t type_size(int type) { return type == CG_TYPE_FP32 ? 4 : 2; }
bool rows_fit(int64_t rows, int64_t cols) { return rows <= INT32_MAX && cols <= INT32_MAX && rows * cols <= INT32_MAX; }
// a tensor of `rows` rows: there, on an element's boundary, rows that do not overlap
bool tensor_ok(const void *p, int64_t ld, int64_t cols, int type)
{
    return p && (reinterpret_cast<uintptr_t>(p) & (type_size(type) - 1)) == 0 && ld >= cols;
}
bool optional_ok(const void *p, int64_t ld, int64_t cols, int type) { return !p || tensor_ok(p, ld, cols, type); }
bool floats_ok(const void *p) { return p && (reinterpret_cast<uintptr_t>(p) & 3) == 0; }

template <class T> void dropout_launch_typed(const DropoutArgs &a, bool dense, unsigned grid, hipStream_t s)
{
    if (dense) {
        if (a.add) hipLaunchKernelGGL((dropout_rows_kernel<T, true, true>), dim3(grid), dim3(256), 0, s, a);
        else hipLaunchKernelGGL((dropout_rows_kernel<T, true, false>), dim3(grid), dim3(256), 0, s, a);
    } else {
        if (a.add) hipLaunchKernelGGL((dropout_rows_kernel<T, false, true>), dim3(grid), dim3(256), 0, s, a);
        else hipLaunchKernelGGL((dropout_rows_kernel<T, false, false>), dim3(grid), dim3(256), 0, s, a);
    }
}
int dropout_run(const cg_drop *drop, int type, int64_t rows, int64_t cols, const void *x, int64_t x_ld, const void *add,
                int64_t add_ld, void *y, int64_t y_ld, void *stream)
{
    if (!drop_ok(drop) || !type_ok(type) || rows < 0 || cols < 0) return CG_EINVAL;
    if (rows == 0 || cols == 0) return CG_OK;
    if (!tensor_ok(x, x_ld, cols, type) || !tensor_ok(y, y_ld, cols, type) || !optional_ok(add, add_ld, cols, type)) return CG_EINVAL;
    if (!rows_fit(rows, cols)) return CG_EUNSUPPORTED;
    DropoutArgs a{};
    a.x = x, a.add = add, a.y = y;
    a.x_ld = x_ld, a.add_ld = add_ld, a.y_ld = y_ld;
    a.n = (uint32_t)(rows * cols);
    a.cols = (uint32_t)cols;
    a.by_cols = make_fastdiv(a.cols);
    a.drop = drop_args(*drop);
    const bool dense = rows == 1 || (x_ld == cols && y_ld == cols && (!add || add_ld == cols));
    const uint32_t blocks = (a.n + 7) / 8;
    const unsigned grid = (blocks + 255) / 256;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (type == CG_TYPE_FP32) dropout_launch_typed<float>(a, dense, grid, s);
    else dropout_launch_typed<bf16raw>(a, dense, grid, s);
    CG_HIP_TRY(hipGetLastError());
    return CG_OK;
}

// Which kernel takes rows of `cols` columns.
constexpr int SHORT_COLS = 512, MID_COLS = 4096, WIDE_COLS = 16384;
// Blocks of the backward kernel: each writes a row of column sums, so no more of them than the chip holds at once: two a compute unit of
// the kernels with one chunk a thread, one of the others (8192 x 4096 joined, bf16: 69 us with 512 blocks and no row ahead, 65 so).
// A single block takes ONE_BLOCK turns and writes the sums itself: a turn more costs 2 us at most, a second launch 7.
constexpr int BWD_BLOCKS = 512, LONG_SLICES = 64, ONE_BLOCK = 4;

int bwd_rows_at_once(int64_t cols) { return cols <= SHORT_COLS / 4 ? 32 : cols <= SHORT_COLS / 2 ? 16 : cols <= 2 * SHORT_COLS ? 8 : cols <= MID_COLS ? 2 : 1; }
int bwd_blocks(int64_t cols) { return cols <= SHORT_COLS || (cols > 2 * SHORT_COLS && cols <= MID_COLS / 2) ? BWD_BLOCKS : BWD_BLOCKS / 2; }
int bwd_parts(int64_t rows, int64_t cols)
{
    if (cols > WIDE_COLS) return (int)(rows < LONG_SLICES ? rows : LONG_SLICES);
    const int64_t n = (rows + bwd_rows_at_once(cols) - 1) / bwd_rows_at_once(cols);
    if (n <= ONE_BLOCK) return n > 0;
    const int most = bwd_blocks(cols);
    return (int)(n < most ? n : most);
}

template <class T, int JOIN> int norm_fwd_typed(const NormArgs &a, hipStream_t s)
{
    const int n = a.cols;
    auto grid = [&](int rows_at_once, int most) {
        const int64_t b = ((int64_t)a.rows + rows_at_once - 1) / rows_at_once;
        return dim3((unsigned)(b < most ? b : most));
    };
    if (n <= SHORT_COLS / 4) hipLaunchKernelGGL((norm_fwd_kernel<T, 16, 1, JOIN, 256>), grid(16, 2048), dim3(256), 0, s, a);
    else if (n <= SHORT_COLS / 2) hipLaunchKernelGGL((norm_fwd_kernel<T, 32, 1, JOIN, 256>), grid(8, 2048), dim3(256), 0, s, a);
    else if (n <= SHORT_COLS) hipLaunchKernelGGL((norm_fwd_kernel<T, 64, 1, JOIN, 256>), grid(4, 2048), dim3(256), 0, s, a);
    else if (n <= 2 * SHORT_COLS) hipLaunchKernelGGL((norm_fwd_kernel<T, 64, 2, JOIN, 256>), grid(4, 2048), dim3(256), 0, s, a);
    else if (n <= MID_COLS / 2) hipLaunchKernelGGL((norm_fwd_kernel<T, 256, 1, JOIN, 256>), grid(1, 2048), dim3(256), 0, s, a);
    else if (n <= MID_COLS) hipLaunchKernelGGL((norm_fwd_kernel<T, 256, 2, JOIN, 256>), grid(1, 2048), dim3(256), 0, s, a);
    else if (n <= WIDE_COLS / 2) hipLaunchKernelGGL((norm_fwd_kernel<T, 512, 2, JOIN, 512>), grid(1, 1024), dim3(512), 0, s, a);
    else if (n <= WIDE_COLS) hipLaunchKernelGGL((norm_fwd_kernel<T, 512, 4, JOIN, 512>), grid(1, 1024), dim3(512), 0, s, a);
    else hipLaunchKernelGGL((norm_fwd_long_kernel<T, JOIN>), grid(1, 512), dim3(LONG_BLOCK), 0, s, a);
    CG_HIP_TRY(hipGetLastError());
    return CG_OK;
}
template <class T, int JOIN> int norm_bwd_typed(NormBwdArgs &a, float *dgamma, float *dbeta, hipStream_t s)
{
    const int n = a.cols, parts = bwd_parts(a.rows, n);
    const bool whole = parts == 1 && n <= WIDE_COLS;
    if (whole) a.dgamma = dgamma, a.dbeta = dbeta;
    if (parts > 0) {
        const dim3 grid((unsigned)parts);
        if (n <= SHORT_COLS / 4) hipLaunchKernelGGL((norm_bwd_kernel<T, 16, 1, JOIN, 512>), grid, dim3(512), 0, s, a);
        else if (n <= SHORT_COLS / 2) hipLaunchKernelGGL((norm_bwd_kernel<T, 32, 1, JOIN, 512>), grid, dim3(512), 0, s, a);
        else if (n <= SHORT_COLS) hipLaunchKernelGGL((norm_bwd_kernel<T, 64, 1, JOIN, 512>), grid, dim3(512), 0, s, a);
        else if (n <= 2 * SHORT_COLS) hipLaunchKernelGGL((norm_bwd_kernel<T, 64, 2, JOIN, 512>), grid, dim3(512), 0, s, a);
        else if (n <= MID_COLS / 2) hipLaunchKernelGGL((norm_bwd_kernel<T, 256, 1, JOIN, 512>), grid, dim3(512), 0, s, a);
        else if (n <= MID_COLS) hipLaunchKernelGGL((norm_bwd_kernel<T, 256, 2, JOIN, 512>), grid, dim3(512), 0, s, a);
        else if (n <= WIDE_COLS / 2) hipLaunchKernelGGL((norm_bwd_kernel<T, 512, 2, JOIN, 512>), grid, dim3(512), 0, s, a);
        else if (n <= WIDE_COLS) hipLaunchKernelGGL((norm_bwd_kernel<T, 512, 4, JOIN, 512>), grid, dim3(512), 0, s, a);
        else {
            hipLaunchKernelGGL((norm_bwd_long_kernel<T, JOIN>), dim3((unsigned)(a.rows < 512 ? a.rows : 512)), dim3(LONG_BLOCK), 0, s, a);
            hipLaunchKernelGGL((norm_columns_kernel<T>), dim3((unsigned)((n + 511) / 512), (unsigned)parts), dim3(64), 0, s, a);
        }
        CG_HIP_TRY(hipGetLastError());
        if (whole) return CG_OK;
    }
    const int64_t sums = (2 * (int64_t)n + 15) / 16;
    hipLaunchKernelGGL(sum_parts_kernel, dim3((unsigned)(sums < SUM_BLOCKS ? sums : SUM_BLOCKS)), dim3(256), 0, s, a.part, parts, n, dgamma, dbeta);
    CG_HIP_TRY(hipGetLastError());
    return CG_OK;
}
template <class A, class F> int for_type_and_join(int type, const A &a, bool joined, F &&f)
{
    if (type == CG_TYPE_FP32) {
        if (!joined) return f(float(), std::integral_constant<int, 0>());
        if (a.cols % 8 == 0) return f(float(), std::integral_constant<int, 1>());
        return f(float(), std::integral_constant<int, 2>());
    }
    if (!joined) return f(bf16raw(), std::integral_constant<int, 0>());
    if (a.cols % 8 == 0) return f(bf16raw(), std::integral_constant<int, 1>());
    return f(bf16raw(), std::integral_constant<int, 2>());
}

int desc_check(const cg_layernorm_desc *d)
{
    if (!d || !type_ok(d->type) || d->rows < 0 || d->cols < 1 || !(d->eps >= 0.f)) return CG_EINVAL;
    // a launch's stride behind the last row or column is still a number of 32 bits
    if (!rows_fit(d->rows, d->cols) || d->rows * d->cols > INT32_MAX - 65535) return CG_EUNSUPPORTED;
    return CG_OK;
}

int norm_fwd_run(const cg_layernorm_desc *d, const cg_drop *drop, NormArgs &a, hipStream_t s)
{
    a.rows = (int)d->rows, a.cols = (int)d->cols, a.eps = d->eps;
    if (drop) a.drop = drop_args(*drop);
    return for_type_and_join(d->type, a, drop != nullptr, [&](auto t, auto join) { return norm_fwd_typed<decltype(t), decltype(join)::value>(a, s); });
}
int norm_bwd_run(const cg_layernorm_desc *d, const cg_drop *drop, NormBwdArgs &a, float *dgamma, float *dbeta, void *ws, size_t ws_bytes, hipStream_t s)
{
    const size_t need = cg_layernorm_workspace_bytes(d);
    if (need && (!ws || (reinterpret_cast<uintptr_t>(ws) & 3))) return CG_EINVAL;
    if (ws_bytes < need) return CG_ENOSPC;
    a.rows = (int)d->rows, a.cols = (int)d->cols;
    a.part = static_cast<float *>(ws);
    if (drop) a.drop = drop_args(*drop);
    return for_type_and_join(d->type, a, drop != nullptr,
                             [&](auto t, auto join) { return norm_bwd_typed<decltype(t), decltype(join)::value>(a, dgamma, dbeta, s); });
}

}  // namespace
}  // namespace cg

using namespace cg;

extern "C" int cg_dropout_fwd(const cg_drop *drop, int type, int64_t rows, int64_t cols, const void *x, int64_t x_ld,
                              const void *add, int64_t add_ld, void *y, int64_t y_ld, void *stream)
{
    return dropout_run(drop, type, rows, cols, x, x_ld, add, add_ld, y, y_ld, stream);
}

extern "C" int cg_dropout_bwd(const cg_drop *drop, int type, int64_t rows, int64_t cols, const void *dy, int64_t dy_ld,
                              void *dx, int64_t dx_ld, void *stream)
{
    return dropout_run(drop, type, rows, cols, dy, dy_ld, nullptr, 0, dx, dx_ld, stream);
}

extern "C" int cg_layernorm_fwd(const cg_layernorm_desc *d, const void *x, int64_t x_ld, const float *gamma, const float *beta,
                                void *y, int64_t y_ld, float *mean, float *rstd, void *stream)
{
    if (int rc = desc_check(d)) return rc;
    if (d->rows == 0) return CG_OK;
    if (!tensor_ok(x, x_ld, d->cols, d->type) || !tensor_ok(y, y_ld, d->cols, d->type) || !floats_ok(gamma) || !floats_ok(beta)) return CG_EINVAL;
    if (!mean != !rstd || (mean && (!floats_ok(mean) || !floats_ok(rstd)))) return CG_EINVAL;
    NormArgs a{};
    a.x = x, a.x_ld = x_ld, a.gamma = gamma, a.beta = beta, a.y = y, a.y_ld = y_ld, a.mean = mean, a.rstd = rstd;
    return norm_fwd_run(d, nullptr, a, static_cast<hipStream_t>(stream));
}

extern "C" size_t cg_layernorm_workspace_bytes(const cg_layernorm_desc *d)
{
    if (desc_check(d) != CG_OK) return 0;
    return (size_t)bwd_parts(d->rows, d->cols) * 2 * (size_t)d->cols * sizeof(float);
}

extern "C" int cg_layernorm_bwd(const cg_layernorm_desc *d, const void *dy, int64_t dy_ld, const void *x, int64_t x_ld,
                                const float *gamma, const float *mean, const float *rstd, const void *dsum, int64_t dsum_ld,
                                void *dx, int64_t dx_ld, float *dgamma, float *dbeta, void *ws, size_t ws_bytes, void *stream)
{
    if (int rc = desc_check(d)) return rc;
    if (!floats_ok(dgamma) || !floats_ok(dbeta)) return CG_EINVAL;
    if (d->rows > 0 && (!tensor_ok(dy, dy_ld, d->cols, d->type) || !tensor_ok(x, x_ld, d->cols, d->type) || !tensor_ok(dx, dx_ld, d->cols, d->type) ||
                        !optional_ok(dsum, dsum_ld, d->cols, d->type) || !floats_ok(gamma) || !floats_ok(mean) || !floats_ok(rstd))) return CG_EINVAL;
    NormBwdArgs a{};
    a.dy = dy, a.dy_ld = dy_ld, a.x = x, a.x_ld = x_ld, a.gamma = gamma, a.mean = mean, a.rstd = rstd;
    a.dsum = dsum, a.dsum_ld = dsum_ld, a.dx = dx, a.dx_ld = dx_ld;
    return norm_bwd_run(d, nullptr, a, dgamma, dbeta, ws, ws_bytes, static_cast<hipStream_t>(stream));
}

extern "C" int cg_dropout_add_layernorm_fwd(const cg_layernorm_desc *d, const cg_drop *drop, const void *branch, int64_t branch_ld,
                                            const void *x, int64_t x_ld, const float *gamma, const float *beta, void *sum,
                                            int64_t sum_ld, void *y, int64_t y_ld, float *mean, float *rstd, void *stream)
{
    if (int rc = desc_check(d)) return rc;
    if (!drop_ok(drop)) return CG_EINVAL;
    if (d->rows == 0) return CG_OK;
    if (!tensor_ok(x, x_ld, d->cols, d->type) || !tensor_ok(branch, branch_ld, d->cols, d->type) || !tensor_ok(sum, sum_ld, d->cols, d->type) ||
        !tensor_ok(y, y_ld, d->cols, d->type) || !floats_ok(gamma) || !floats_ok(beta)) return CG_EINVAL;
    if (!mean != !rstd || (mean && (!floats_ok(mean) || !floats_ok(rstd)))) return CG_EINVAL;
    NormArgs a{};
    a.x = x, a.x_ld = x_ld, a.branch = branch, a.branch_ld = branch_ld, a.gamma = gamma, a.beta = beta;
    a.sum = sum, a.sum_ld = sum_ld, a.y = y, a.y_ld = y_ld, a.mean = mean, a.rstd = rstd;
    return norm_fwd_run(d, drop, a, static_cast<hipStream_t>(stream));
}

extern "C" int cg_dropout_add_layernorm_bwd(const cg_layernorm_desc *d, const cg_drop *drop, const void *dy, int64_t dy_ld,
                                            const void *dsum, int64_t dsum_ld, const void *sum, int64_t sum_ld, const float *gamma,
                                            const float *mean, const float *rstd, void *dx, int64_t dx_ld, void *dbranch,
                                            int64_t dbranch_ld, float *dgamma, float *dbeta, void *ws, size_t ws_bytes, void *stream)
{
    if (int rc = desc_check(d)) return rc;
    if (!drop_ok(drop) || !floats_ok(dgamma) || !floats_ok(dbeta)) return CG_EINVAL;
    if (d->rows > 0 && (!tensor_ok(dy, dy_ld, d->cols, d->type) || !tensor_ok(sum, sum_ld, d->cols, d->type) || !tensor_ok(dx, dx_ld, d->cols, d->type) ||
                        !tensor_ok(dbranch, dbranch_ld, d->cols, d->type) || !optional_ok(dsum, dsum_ld, d->cols, d->type) || !floats_ok(gamma) ||
                        !floats_ok(mean) || !floats_ok(rstd))) return CG_EINVAL;
    NormBwdArgs a{};
    a.dy = dy, a.dy_ld = dy_ld, a.x = sum, a.x_ld = sum_ld, a.gamma = gamma, a.mean = mean, a.rstd = rstd;
    a.dsum = dsum, a.dsum_ld = dsum_ld, a.dx = dx, a.dx_ld = dx_ld, a.dbranch = dbranch, a.dbranch_ld = dbranch_ld;
    return norm_bwd_run(d, drop, a, dgamma, dbeta, ws, ws_bytes, static_cast<hipStream_t>(stream));
}
