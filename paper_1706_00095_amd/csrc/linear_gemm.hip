// The linear layers' products on the matrix cores: C[r][c] = sum_k A(r, k) B(c, k), v_mfma_f32_32x32x16_bf16.
//
// A block makes a tile of C, its waves a rectangle of it each.  Per step, STEP values of k of both operands pass through LDS in the
// order they have in memory: a tile of rows along k is read in rows, a tile of rows across k by transposing reads, so no operand is
// ever laid out anew.  bf16 tensors are multiplied as they are; fp32 tensors are cut in three bf16 pieces on their way into LDS, six
// products; 8-bit tensors become bf16 numbers, exactly, on theirs.
//
// The first operand of the instruction is B, so that a lane holds sums of one row r and 4 x 4 neighbouring columns; for the epilogue
// the sums are exchanged through LDS, 32 rows of a wave at a time, and every lane takes eight neighbours of a row.
#include "linear_device.h"

namespace cg {
namespace {

// ---- tiles in LDS -----------------------------------------------------------------------------------------------------------
// ROWS x COLS bf16 as in memory, NP planes.  ACROSS: rows are values of k.  16-byte chunks of a row are exchanged by a function of the row so that
// neither 16 rows' same chunk (reads in rows take 16 lanes at a time) nor four rows' same 64 bytes (transposing reads) fall on the
// same banks (64 of 4 bytes).
template <bool ACROSS, int ROWS, int COLS, int NP> struct LdsTile {
    static constexpr int CH = COLS / 8, PLANE = ROWS * COLS * 2, BYTES = NP * PLANE;
    static_assert(ACROSS ? COLS >= 128 : COLS == 64 || COLS == 32, "the exchange of chunks");
    static __device__ __forceinline__ int swizzle(int row)
    {
        if constexpr (ACROSS) return (row & 3) << 2;
        else if constexpr (COLS == 64) return row >> 1 & 7;
        else return row >> 2 & 3;
    }
    static __device__ __forceinline__ int at(int row, int chunk) { return row * COLS * 2 + ((chunk ^ swizzle(row)) << 4); }
    static __device__ __forceinline__ void put(LdsByte *t, int row, int chunk, const Frag<NP> &f)
    {
#pragma unroll
        for (int k = 0; k < NP; ++k) CG_LDS(u32x4, t + k * PLANE + at(row, chunk)) = f.p[k];
    }
    // operand of 32 rows or columns of C from x0 on, the values 16 ks .. 16 ks + 15 of the step; lane l has those from 8 (l / 32) on
    static __device__ __forceinline__ Frag<NP> read(LdsByte *t, int x0, int ks, int lane)
    {
        Frag<NP> f;
        if constexpr (!ACROSS) {
#pragma unroll
            for (int k = 0; k < NP; ++k) f.p[k] = CG_LDS(u32x4, t + k * PLANE + at(x0 + (lane & 31), 2 * ks + (lane >> 5)));
        } else {
            const int row = 16 * ks + 8 * (lane >> 5) + (lane >> 2 & 3), chunk = (x0 >> 3) + 2 * (lane >> 4 & 1) + (lane >> 1 & 1);
#pragma unroll
            for (int k = 0; k < NP; ++k) {
                LdsByte *base = t + k * PLANE + at(row, chunk) + 8 * (lane & 1);
                const uint2 a = __builtin_bit_cast(uint2, read_tr(base)), b = __builtin_bit_cast(uint2, read_tr(base + 4 * COLS * 2));
                f.p[k] = u32x4{a.x, a.y, b.x, b.y};
            }
        }
        return f;
    }
};

// ---- from memory into LDS -----------------------------------------------------------------------------------------------------
//  start(k, lds): the loads of the step that begins at k leave.  finish(lds): after the multiplications, before the barrier.
// x0: the tile's first row (column) of C, of `count`; kend: where this block's part of k ends.
template <class T, bool ACROSS, int XT, int STEP, int NT, bool DMA> struct TileLoader;

// bf16, rows of whole 16-byte chunks: without registers.  The buffer's base moves with the tile, so that a lane's offsets are the same
// for all steps and 32 bits wide (the host checks the stride); rows behind the last one are out of its range and arrive as zeros, chunks
// behind a row's end are sent out of range.
template <bool ACROSS, int XT, int STEP, int NT> struct TileLoader<bf16raw, ACROSS, XT, STEP, NT, true> {
    static constexpr int NP = 1, ROWS = ACROSS ? STEP : XT, COLS = ACROSS ? XT : STEP, LOADS = ROWS * COLS * 2 / 1024, WAVES = NT / 64, N = LOADS / WAVES;
    static_assert(LOADS % WAVES == 0, "every wave loads as much");
    using Lds = LdsTile<ACROSS, ROWS, COLS, 1>;
    const bf16raw *base;
    int64_t ld;
    int count, kend, x0;
    uint32_t voff[N];
    __device__ __forceinline__ TileLoader(const void *p, const Packed &, int64_t ld_, int x0_, int count_, int kend_)
        : base(static_cast<const bf16raw *>(p)), ld(ld_), count(count_), kend(kend_), x0(x0_)
    {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int row = row_of(j), chunk = chunk_of(j);
            voff[j] = ACROSS && x0 + 8 * chunk >= count ? OOB_ROW : (uint32_t)((int64_t)row * ld * 2 + chunk * 16);
        }
    }
    static __device__ __forceinline__ int at(int j) { return (j * WAVES + (int)(threadIdx.x >> 6)) * 1024 + (int)(threadIdx.x & 63) * 16; }
    static __device__ __forceinline__ int row_of(int j) { return at(j) / (COLS * 2); }
    static __device__ __forceinline__ int chunk_of(int j) { return at(j) % (COLS * 2) / 16 ^ Lds::swizzle(row_of(j)); }
    __device__ __forceinline__ void start(int k, LdsByte *lds) const
    {
        const int row0 = ACROSS ? k : x0, col0 = ACROSS ? x0 : k, rows = (ACROSS ? kend : count) - row0, cols = (ACROSS ? count : kend) - col0;
        const BufferRsrc r = raw_buffer((uint64_t)reinterpret_cast<uintptr_t>(base) + (uint64_t)((row0 * ld + col0) * 2),
                                        (uint64_t)(rows - 1) * (uint64_t)ld * 2 + (uint64_t)cols * 2);
        const int wave = (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        if (!ACROSS && cols < STEP) {        // the last step
#pragma unroll
            for (int j = 0; j < N; ++j) dma16(r, lds + (j * WAVES + wave) * 1024, 8 * chunk_of(j) < cols ? voff[j] : OOB_ROW);
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) dma16(r, lds + (j * WAVES + wave) * 1024, voff[j]);
        }
    }
    __device__ __forceinline__ void finish(LdsByte *) const {}
};

// Otherwise through registers, at any alignment; fp32 is cut on the way.
template <class T, bool ACROSS, int XT, int STEP, int NT> struct TileLoader<T, ACROSS, XT, STEP, NT, false> {
    static constexpr int NP = Pieces<T>::N, ROWS = ACROSS ? STEP : XT, COLS = ACROSS ? XT : STEP, CH = COLS / 8, N = ROWS * CH / NT;
    static_assert(ROWS * CH % NT == 0, "every thread loads as much");
    using Lds = LdsTile<ACROSS, ROWS, COLS, NP>;
    const T *base;
    int64_t ld;
    int count, kend, x0;
    Raw8<T> r[N];
    __device__ __forceinline__ TileLoader(const void *p, const Packed &, int64_t ld_, int x0_, int count_, int kend_)
        : base(static_cast<const T *>(p)), ld(ld_), count(count_), kend(kend_), x0(x0_) {}
    __device__ __forceinline__ void start(int k, LdsByte *)
    {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int i = threadIdx.x + j * NT, row = (ACROSS ? k : x0) + i / CH, c = (ACROSS ? x0 : k) + 8 * (i % CH);
            const int n = row < (ACROSS ? kend : count) ? (ACROSS ? count : kend) - c : 0;
            r[j] = load8(base + (n > 0 ? row * ld + c : 0), n);
        }
    }
    __device__ __forceinline__ void finish(LdsByte *t) const
    {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int i = threadIdx.x + j * NT;
            Lds::put(t, i / CH, i % CH, frag_of(r[j]));
        }
    }
};

// 8-bit tensors
template <bool ACROSS, int XT, int STEP, int NT> struct TileLoader<int8_t, ACROSS, XT, STEP, NT, false> {
    static constexpr int NP = 1, ROWS = ACROSS ? STEP : XT, COLS = ACROSS ? XT : STEP, CH = COLS / 8, N = ROWS * CH / NT;
    static_assert(ROWS * CH % NT == 0, "every thread loads as much");
    using Lds = LdsTile<ACROSS, ROWS, COLS, 1>;
    Packed p;
    int count, kend, x0;
    Raw8Packed r[N];
    __device__ __forceinline__ TileLoader(const void *, const Packed &p_, int64_t, int x0_, int count_, int kend_) : p(p_), count(count_), kend(kend_), x0(x0_) {}
    __device__ __forceinline__ void start(int k, LdsByte *)
    {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int i = threadIdx.x + j * NT, row = (ACROSS ? k : x0) + i / CH, c = (ACROSS ? x0 : k) + 8 * (i % CH);
            r[j] = load8(p, row, c, row < (ACROSS ? kend : count) ? (ACROSS ? count : kend) - c : 0);
        }
    }
    __device__ __forceinline__ void finish(LdsByte *t) const
    {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int i = threadIdx.x + j * NT;
            Frag<1> f;
#pragma unroll
            for (int q = 0; q < 4; ++q) f.p[0][q] = pack_bf16(elem(r[j], 2 * q), elem(r[j], 2 * q + 1));
            Lds::put(t, i / CH, i % CH, f);
        }
    }
};

// ---- sums ------------------------------------------------------------------------------------------------------------------------
// Pieces: the products below the first are added up on their own, because an instruction drops what lies below the last place of the
// sum it adds to; products of pieces i and j with i + j > 2 are below 2^-24 of the whole and left out.
template <int NA, int NB> struct Sums {
    static constexpr bool CUT = NA * NB > 1;
    v16f big, small;
    __device__ __forceinline__ void zero() { big = v16f{}, small = v16f{}; }
    __device__ __forceinline__ void mma(const Frag<NA> &a, const Frag<NB> &b)
    {
#pragma unroll
        for (int d = 2; d > 0; --d)
#pragma unroll
            for (int i = 0; i < NA; ++i)
                if (d - i >= 0 && d - i < NB) small = mfma(b.p[d - i], a.p[i], small);
        big = mfma(b.p[0], a.p[0], big);
    }
    __device__ __forceinline__ float get(int i) const { return CUT ? big[i] + small[i] : big[i]; }
};

// Consecutive blocks run on different XCDs, each with an L2 of its own: every XCD gets a stretch of neighbouring tiles, in groups of
// 8 rows of tiles, so that the 32 blocks it runs at a time read 8 strips of A and 4 of B.
constexpr int kXcds = 8, kGroup = 8;
__device__ __forceinline__ void place_of(const GemmArgs &a, int &tr, int &tc, int &split)
{
    const int n = a.tiles_r * a.tiles_c, all = n * a.splits, id = (int)blockIdx.x;
    const int xcd = id % kXcds, lin = xcd * (all / kXcds) + min(xcd, all % kXcds) + id / kXcds;
    split = lin / n;
    const int t = lin - split * n, group = t / (kGroup * a.tiles_c), within = t - group * kGroup * a.tiles_c;
    const int high = min(kGroup, a.tiles_r - group * kGroup);
    tr = group * kGroup + within % high;
    tc = within / high;
}

template <class T, class TB, bool AX, bool BX, int XT_, bool DMA> struct Config {
    using TA = T;
    static constexpr bool kDmaA = DMA, kDmaB = DMA && sizeof(TB) == 2;
    static constexpr int XT = XT_, NT = XT == 256 ? 512 : 256, WR = 2, WC = NT / 64 / WR;      // waves along the rows and the columns
    static constexpr int NA = Pieces<T>::N, NB = sizeof(TB) == 4 ? 3 : 1;
    // three pieces leave room for one buffer and two blocks a compute unit
    static constexpr int STEP = NA == 3 ? 32 : 64, STAGES = NA == 3 ? 1 : 2;
    using LA = TileLoader<T, AX, XT, STEP, NT, kDmaA>;
    using LB = TileLoader<TB, BX, XT, STEP, NT, kDmaB>;
    static constexpr int MR = XT / WR / 32, MC = XT / WC / 32;       // 32 x 32 tiles of a wave
    static constexpr int STAGE = LA::Lds::BYTES + LB::Lds::BYTES;
    static constexpr int EPI_ROW = (MC * 32 + 4) * 4, EPI = NT / 64 * 32 * EPI_ROW;
    static constexpr int LDS = STAGES * STAGE > EPI ? STAGES * STAGE : EPI;
};

template <class T, class TB, bool AX, bool BX, int XT, bool DMA, class TO>
__global__ __launch_bounds__((XT == 256 ? 512 : 256), 2) void gemm_kernel(GemmArgs a)
{
    using Cfg = Config<T, TB, AX, BX, XT, DMA>;
    using LA = typename Cfg::LA;
    using LB = typename Cfg::LB;
    constexpr int STEP = Cfg::STEP, MR = Cfg::MR, MC = Cfg::MC;
    extern __shared__ __align__(16) char smem[];
    LdsByte *const lds = (LdsByte *)smem;
    const int lane = threadIdx.x & 63, wave = (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wr = wave / Cfg::WC * (MR * 32), wc = wave % Cfg::WC * (MC * 32);
    int tr, tc, split;
    place_of(a, tr, tc, split);
    const int r0 = tr * XT, c0 = tc * XT, kbeg = split * a.chunk, kend = min(a.K, kbeg + a.chunk);

    LA la(a.A, Packed{}, a.a_ld, r0, a.R, kend);
    LB lb(a.B, a.B8, a.b_ld, c0, a.C, kend);
    Sums<Cfg::NA, Cfg::NB> acc[MR][MC];
#pragma unroll
    for (int i = 0; i < MR; ++i)
#pragma unroll
        for (int j = 0; j < MC; ++j) acc[i][j].zero();

    auto multiply = [&](LdsByte *at) {
#pragma unroll
        for (int ks = 0; ks < STEP / 16; ++ks) {
            Frag<Cfg::NA> fa[MR];
            Frag<Cfg::NB> fb[MC];
#pragma unroll
            for (int j = 0; j < MC; ++j) fb[j] = LB::Lds::read(at + LA::Lds::BYTES, wc + 32 * j, ks, lane);
#pragma unroll
            for (int i = 0; i < MR; ++i) fa[i] = LA::Lds::read(at, wr + 32 * i, ks, lane);
#pragma unroll
            for (int i = 0; i < MR; ++i)
#pragma unroll
                for (int j = 0; j < MC; ++j) acc[i][j].mma(fa[i], fb[j]);
        }
    };
    auto start = [&](int k, LdsByte *at) {
        la.start(k, at);
        lb.start(k, at + LA::Lds::BYTES);
    };
    auto finish = [&](LdsByte *at) {
        la.finish(at);
        lb.finish(at + LA::Lds::BYTES);
    };
    if (kbeg < kend) {
        start(kbeg, lds);
        finish(lds);
    }
    if constexpr (Cfg::STAGES == 2) {
        // behind the barrier a step's tiles are there and everyone is done with the ones before, whose buffer is filled while these are multiplied
        int buf = 0;
        for (int k = kbeg; k < kend; k += STEP, buf ^= 1) {
            tile_sync();
            const bool more = k + STEP < kend;
            if (more) start(k + STEP, lds + (buf ^ 1) * Cfg::STAGE);
            multiply(lds + buf * Cfg::STAGE);
            if (more) finish(lds + (buf ^ 1) * Cfg::STAGE);
        }
    } else {
        for (int k = kbeg; k < kend; k += STEP) {
            __syncthreads();
            const bool more = k + STEP < kend;
            if (more) start(k + STEP, lds);
            multiply(lds);
            __syncthreads();
            if (more) finish(lds);
        }
    }
    __syncthreads();

    EpiArgs e = a.epi;
    const bool whole = a.splits == 1;
    LdsByte *const mine = lds + wave * 32 * Cfg::EPI_ROW;
    constexpr int PER = 4 * MC;                     // lanes of a row
#pragma unroll
    for (int i = 0; i < MR; ++i) {
#pragma unroll
        for (int j = 0; j < MC; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                u32x4 v;
#pragma unroll
                for (int u = 0; u < 4; ++u) v[u] = __float_as_uint(acc[i][j].get(4 * q + u));
                CG_LDS(u32x4, mine + (lane & 31) * Cfg::EPI_ROW + (32 * j + 8 * q + 4 * (lane >> 5)) * 4) = v;
            }
        __builtin_amdgcn_wave_barrier();
#pragma unroll 1
        for (int t = 0; t < 32 * PER / 64; ++t) {
            const int row = t * (64 / PER) + lane / PER, c = c0 + wc + 8 * (lane % PER);
            const int r = r0 + wr + 32 * i + row;
            float v[8];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const u32x4 x = CG_LDS(u32x4, mine + row * Cfg::EPI_ROW + (8 * (lane % PER) + 4 * h) * 4);
#pragma unroll
                for (int u = 0; u < 4; ++u) v[4 * h + u] = __uint_as_float(x[u]);
            }
            if (r < a.R && c < a.C) {
                if (whole) finish8<TO>(e, v, r, c, a.C - c);
                else store8(a.part + ((int64_t)split * a.R + r) * a.C + c, to_raw<float>(v), a.C - c);
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

template <class T, class TB, bool AX, bool BX, int XT, bool DMA, class TO> int launch(const GemmArgs &a, hipStream_t s)
{
    using Cfg = Config<T, TB, AX, BX, XT, DMA>;
    auto *const kernel = gemm_kernel<T, TB, AX, BX, XT, DMA, TO>;
    if constexpr (Cfg::LDS > 64 * 1024)       // asked for at every call: it holds for the current device alone
        CG_HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, Cfg::LDS));
    hipLaunchKernelGGL(kernel, dim3((unsigned)(a.tiles_r * a.tiles_c * a.splits)), dim3(Cfg::NT), Cfg::LDS, s, a);
    CG_HIP_TRY(hipGetLastError());
    return CG_OK;
}
template <class T, class TB, bool AX, bool BX, class TO> int launch_bf16(const GemmKind &k, const GemmArgs &a, hipStream_t s)
{
    if (k.large) return launch<T, TB, AX, BX, 256, true, TO>(a, s);
    if (k.dma) return launch<T, TB, AX, BX, 128, true, TO>(a, s);
    return launch<T, TB, AX, BX, 128, false, TO>(a, s);
}

}  // namespace

int gemm_launch(const GemmKind &k, const GemmArgs &a, hipStream_t s)
{
    if (k.type == CG_TYPE_FP32) {
        if (k.pass == CG_PASS_FWD) return launch<float, float, false, false, 128, false, float>(a, s);
        if (k.pass == CG_PASS_BWD_DATA) return launch<float, float, false, true, 128, false, float>(a, s);
        if (k.packed) return launch<float, int8_t, true, true, 128, false, float>(a, s);
        return launch<float, float, true, true, 128, false, float>(a, s);
    }
    if (k.pass == CG_PASS_FWD) return launch_bf16<bf16raw, bf16raw, false, false, bf16raw>(k, a, s);
    if (k.pass == CG_PASS_BWD_DATA) return launch_bf16<bf16raw, bf16raw, false, true, bf16raw>(k, a, s);
    if (k.packed) return launch_bf16<bf16raw, int8_t, true, true, float>(k, a, s);
    return launch_bf16<bf16raw, bf16raw, true, true, float>(k, a, s);
}

}  // namespace cg
