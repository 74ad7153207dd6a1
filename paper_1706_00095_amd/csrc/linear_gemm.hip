// The linear layers' products on the matrix cores: C[r][c] = sum_k A(r, k) B(c, k), on v_mfma_f32_16x16x32_bf16 (v_mfma_f32_32x32x16_bf16 is as
// fast by itself, but power bounds these kernels, and it takes more: 8192^3 1401 TFLOP/s, and 1522 so; on zeros 1914 and 1903).
//
// A block makes a tile of C, its waves a rectangle of it each.  Per step, STEP values of k of both operands pass through LDS in the
// order they have in memory: a tile of rows along k is read in rows, a tile of rows across k by transposing reads, so no operand is
// ever laid out anew.  bf16 tensors are multiplied as they are; fp32 tensors are cut in three bf16 pieces on their way into LDS, six
// products; 8-bit tensors become bf16 numbers, exactly, on theirs.
//
// The first operand of the instruction is B, so that a lane holds sums of one row r and four neighbouring columns; for the epilogue
// the sums are exchanged through LDS, 32 rows of a wave at a time, and every lane takes eight neighbours of a row.
#include "linear_device.h"

namespace cg {
namespace {

typedef float v4f __attribute__((ext_vector_type(4)));

// ---- tiles in LDS -----------------------------------------------------------------------------------------------------------
// ROWS x COLS bf16 as in memory, NP planes.  ACROSS: rows are values of k.  16-byte chunks of a row are exchanged by a function of the row so that
// neither 16 rows' same chunk (reads in rows take 16 lanes at a time) nor four rows' same 64 bytes (transposing reads) fall on the
// same banks (64 of 4 bytes).
template <bool ACROSS, int ROWS, int COLS, int NP> struct LdsTile {
    static constexpr int CH = COLS / 8, PLANE = ROWS * COLS * 2, BYTES = NP * PLANE;
    static_assert(ACROSS ? COLS >= 64 : COLS == 64 || COLS == 32, "the exchange of chunks");
    static __device__ __forceinline__ int swizzle(int row)
    {
        if constexpr (ACROSS && COLS == 64) return (row >> 1 & 1) << 1 | (row >> 3 & 1) << 2;
        else if constexpr (ACROSS) return (row & 3) << 2 | (row >> 3 & 1) << 1;
        else if constexpr (COLS == 64) return row >> 1 & 7;
        else return row >> 2 & 3;
    }
    static __device__ __forceinline__ int at(int row, int chunk) { return row * COLS * 2 + ((chunk ^ swizzle(row)) << 4); }
    static __device__ __forceinline__ void put(LdsByte *t, int row, int chunk, const Frag<NP> &f)
    {
#pragma unroll
        for (int k = 0; k < NP; ++k) CG_LDS(u32x4, t + k * PLANE + at(row, chunk)) = f.p[k];
    }
    // operand of 16 rows or columns of C from x0 on, the values 32 ks .. 32 ks + 31 of the step; lane l has those from 8 (l / 16) on
    static __device__ __forceinline__ u32x4 read(LdsByte *t, int x0, int ks, int lane, int plane = 0)
    {
        if constexpr (!ACROSS) return CG_LDS(u32x4, t + plane * PLANE + at(x0 + (lane & 15), 4 * ks + (lane >> 4)));
        const int row = 32 * ks + 8 * (lane >> 4) + (lane >> 2 & 3), chunk = (x0 >> 3) + (lane >> 1 & 1);
        LdsByte *base = t + plane * PLANE + at(row, chunk) + 8 * (lane & 1);
        const uint2 a = __builtin_bit_cast(uint2, read_tr(base)), b = __builtin_bit_cast(uint2, read_tr(base + 4 * COLS * 2));
        return u32x4{a.x, a.y, b.x, b.y};
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
    __device__ __forceinline__ TileLoader(const void *p, const Packed &, int64_t ld_, int x0_, int count_, int, int kend_, int)
        : base(static_cast<const bf16raw *>(p)), ld(ld_), count(count_), kend(kend_), x0(x0_)
    {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int row = row_of(j), chunk = chunk_of(j);
            voff[j] = ACROSS && x0 + 8 * chunk >= count ? OOB_ROW : (uint32_t)((int64_t)row * ld * 2 + chunk * 16);
        }
    }
    static __device__ __forceinline__ int at(int j) { return (j * WAVES + (int)(threadIdx.x >> 6) % WAVES) * 1024 + (int)(threadIdx.x & 63) * 16; }
    static __device__ __forceinline__ int row_of(int j) { return at(j) / (COLS * 2); }
    static __device__ __forceinline__ int chunk_of(int j) { return at(j) % (COLS * 2) / 16 ^ Lds::swizzle(row_of(j)); }
    __device__ __forceinline__ bool inside(int) const { return true; }
    template <bool> __device__ __forceinline__ void start(int k, LdsByte *lds) const
    {
        const int row0 = ACROSS ? k : x0, col0 = ACROSS ? x0 : k, rows = (ACROSS ? kend : count) - row0, cols = (ACROSS ? count : kend) - col0;
        const BufferRsrc r = raw_buffer((uint64_t)reinterpret_cast<uintptr_t>(base) + (uint64_t)((row0 * ld + col0) * 2),
                                        (uint64_t)(rows - 1) * (uint64_t)ld * 2 + (uint64_t)cols * 2);
        const int wave = (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % WAVES;
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

// The same for one half (128 rows or columns of C) of a large tile, step after step; 512 threads, two loads each.  The buffer is the half's
// rows (of a step, where they lie across k), so that its size is a number of 32 bits.
template <bool ACROSS> struct HalfLoader {
    static constexpr int STEP = 64, ROWS = ACROSS ? STEP : 128, COLS = ACROSS ? 128 : STEP;
    using Lds = LdsTile<ACROSS, ROWS, COLS, 1>;
    uint64_t at, advance;             // address of the next step's tile, bytes from a step to the next
    uint32_t bytes, row;              // from `at` on; from a row to the next (across k)
    int k_left;
    uint32_t voff[2];
    __device__ __forceinline__ HalfLoader(const void *p, int64_t ld, int x0, int count, int kbeg, int kend)
    {
        const int row0 = ACROSS ? kbeg : x0, col0 = ACROSS ? x0 : kbeg, rows = ACROSS ? STEP : min(count - row0, ROWS), cols = (ACROSS ? count : kend) - col0;
        at = (uint64_t)reinterpret_cast<uintptr_t>(p) + (uint64_t)((row0 * ld + col0) * 2);
        row = (uint32_t)ld * 2;
        bytes = rows > 0 && cols > 0 ? (uint32_t)(rows - 1) * row + (uint32_t)min(cols, ACROSS ? 128 : INT32_MAX) * 2 : 0;       // none: zeros
        advance = ACROSS ? (uint64_t)row * STEP : 2 * STEP;
        k_left = kend - kbeg;
#pragma unroll
        for (int j = 0; j < 2; ++j) voff[j] = ACROSS && 8 * chunk_of(j) >= cols ? OOB_ROW : (uint32_t)row_of(j) * row + (uint32_t)chunk_of(j) * 16;
    }
    static __device__ __forceinline__ int place(int j) { return (j * 8 + (int)(threadIdx.x >> 6)) * 1024 + (int)(threadIdx.x & 63) * 16; }
    static __device__ __forceinline__ int row_of(int j) { return place(j) / (COLS * 2); }
    static __device__ __forceinline__ int chunk_of(int j) { return place(j) % (COLS * 2) / 16 ^ Lds::swizzle(row_of(j)); }
    // One of the step's two loads; behind the second the loader stands at the next step.  WHOLE: not the last step.
    template <bool WHOLE, int J> __device__ __forceinline__ void load(LdsByte *lds, int wave)
    {
        BufferRsrc r;
        r.x = __builtin_amdgcn_readfirstlane((uint32_t)at);
        r.y = __builtin_amdgcn_readfirstlane((uint32_t)(at >> 32) & 0xffffu);
        uint32_t size = bytes, off = voff[J];
        if constexpr (!WHOLE) {
            if (ACROSS) size -= k_left < STEP && bytes ? (uint32_t)(STEP - k_left) * row : 0;       // fewer rows
            else off = 8 * chunk_of(J) < k_left ? off : OOB_ROW;
        }
        r.z = __builtin_amdgcn_readfirstlane(size);
        r.w = 0x00020000u;
        dma16(r, lds + (J * 8 + wave) * 1024, off);
        if (J == 1) {
            at += advance;
            if (!ACROSS) bytes -= bytes ? 2 * STEP : 0;
            k_left -= STEP;
        }
    }
    __device__ __forceinline__ void next(LdsByte *lds, int wave)
    {
        load<false, 0>(lds, wave);
        load<false, 1>(lds, wave);
    }
};

// Otherwise through registers, at any alignment; fp32 is cut, and 8-bit numbers become bf16, on the way.  NT threads in a row load a tile; a block
// may have several times as many, with a tile each.
// inside(k): the step that begins at k may be loaded without bounds.  All of its values of k are there, and where rows lie across k another row
// behind them, into which the last chunk of a row may reach; rows and chunks behind the last one are others again: what they give is not stored.
template <class T> struct Source;
template <class T> struct Source {
    const T *base;
    int64_t ld;
    using Raw = Raw8<T>;
    __device__ __forceinline__ Source(const void *p, const Packed &, int64_t ld_) : base(static_cast<const T *>(p)), ld(ld_) {}
    __device__ __forceinline__ Raw load(int64_t row, int c, int n) const { return load8(base + (n > 0 ? row * ld + c : 0), n); }
    struct At {
        const T *p;
        __device__ __forceinline__ Raw take(const Source &s, int rows, int cols)
        {
            const Raw r = load8(p, 8);
            p += rows * s.ld + cols;
            return r;
        }
    };
    __device__ __forceinline__ At at(int64_t row, int c) const { return {base + row * ld + c}; }
};
template <> struct Source<int8_t> {
    Packed p;
    using Raw = Raw8Packed;
    __device__ __forceinline__ Source(const void *, const Packed &p_, int64_t) : p(p_) {}
    __device__ __forceinline__ Raw load(int64_t row, int c, int n) const { return load8(p, row, c, n); }
    struct At {
        const int8_t *q;
        const uint8_t *e;
        __device__ __forceinline__ Raw take(const Source &s, int rows, int)        // rows lie across k: columns stay
        {
            const Loose8 v = *reinterpret_cast<const Loose8 *>(q);
            const Raw r = {{v.w[0], v.w[1]}, (int)*e - kPackBias};
            q += rows * s.p.codes_ld, e += rows * s.p.scales_ld;
            return r;
        }
    };
    __device__ __forceinline__ At at(int64_t row, int c) const { return {p.codes + row * p.codes_ld + c, p.scales + row * p.scales_ld + c / kPackBlock}; }
};
__device__ __forceinline__ Frag<1> frag_of(const Raw8Packed &r)
{
    Frag<1> f;
#pragma unroll
    for (int q = 0; q < 4; ++q) f.p[0][q] = pack_bf16(elem(r, 2 * q), elem(r, 2 * q + 1));
    return f;
}
template <class T, bool ACROSS, int XT, int STEP, int NT> struct TileLoader<T, ACROSS, XT, STEP, NT, false> {
    static constexpr int NP = sizeof(T) == 4 ? 3 : 1, ROWS = ACROSS ? STEP : XT, COLS = ACROSS ? XT : STEP, CH = COLS / 8, N = ROWS * CH / NT;
    static_assert(ROWS * CH % NT == 0, "every thread loads as much");
    using Lds = LdsTile<ACROSS, ROWS, COLS, NP>;
    Source<T> src;
    int count, kend, x0, last;          // last: where the tensor ends along k
    typename Source<T>::At at[N];
    typename Source<T>::Raw r[N];
    __device__ __forceinline__ TileLoader(const void *p, const Packed &p8, int64_t ld, int x0_, int count_, int kbeg, int kend_, int last_)
        : src(p, p8, ld), count(count_), kend(kend_), x0(x0_), last(last_)
    {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int i = threadIdx.x % NT + j * NT, x = x0 + (ACROSS ? 8 * (i % CH) : i / CH), k = kbeg + (ACROSS ? i / CH : 8 * (i % CH));
            const int xc = ACROSS ? min(x, (count - 1) / 8 * 8) : min(x, count - 1);
            at[j] = ACROSS ? src.at(k, xc) : src.at(xc, k);
        }
    }
    __device__ __forceinline__ bool inside(int k) const { return k + STEP <= kend && (!ACROSS || (count >= 8 && (count % 8 == 0 || k + STEP < last))); }
    // steps in order, those inside first
    template <bool INSIDE> __device__ __forceinline__ void start(int k, LdsByte *)
    {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int i = threadIdx.x % NT + j * NT, row = (ACROSS ? k : x0) + i / CH, c = (ACROSS ? x0 : k) + 8 * (i % CH);
            if constexpr (INSIDE) r[j] = at[j].take(src, ACROSS ? STEP : 0, ACROSS ? 0 : STEP);
            else r[j] = src.load(row, c, row < (ACROSS ? kend : count) ? (ACROSS ? count : kend) - c : 0);
        }
    }
    __device__ __forceinline__ void finish_one(LdsByte *t, int j) const
    {
        const int i = threadIdx.x % NT + j * NT;
        Lds::put(t, i / CH, i % CH, frag_of(r[j]));
    }
    __device__ __forceinline__ void finish(LdsByte *t) const
    {
#pragma unroll
        for (int j = 0; j < N; ++j) finish_one(t, j);
    }
};

// ---- sums ------------------------------------------------------------------------------------------------------------------------
// Pieces: the products below the first are added up on their own, because an instruction drops what lies below the last place of the
// sum it adds to; products of pieces i and j with i + j > 2 are below 2^-24 of the whole and left out.
__device__ __forceinline__ v4f mfma16(u32x4 a, u32x4 b, v4f c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// MR x MC tiles of 16 x 16.  A lane has row lane % 16, columns 4 (lane / 16) .. of each.
template <bool CUT, int MR, int MC> struct Sums {
    v4f big[MR][MC], small[CUT ? MR : 1][CUT ? MC : 1];
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < MR; ++i)
#pragma unroll
            for (int j = 0; j < MC; ++j) {
                big[i][j] = v4f{};
                if constexpr (CUT) small[i][j] = v4f{};
            }
    }
    // the product of a piece of A's and one of B's column j; first: of the leading ones
    __device__ __forceinline__ void mma(const u32x4 (&a)[MR], u32x4 b, int j, bool first)
    {
#pragma unroll
        for (int i = 0; i < MR; ++i) {
            if constexpr (CUT)
                if (!first) {
                    small[i][j] = mfma16(b, a[i], small[i][j]);
                    continue;
                }
            big[i][j] = mfma16(b, a[i], big[i][j]);
        }
    }
    __device__ __forceinline__ v4f &of_join(int i, int j) { return CUT ? small[CUT ? i : 0][CUT ? j : 0] : big[i][j]; }      // what sums of another part are added to
    __device__ __forceinline__ u32x4 get(int i, int j) const
    {
        if constexpr (CUT) return __builtin_bit_cast(u32x4, big[i][j] + small[i][j]);
        else return __builtin_bit_cast(u32x4, big[i][j]);
    }
};

// This wave's loads into LDS but the latest LOADS have landed, its reads of LDS but the latest READS are done, and everyone's.  The compiler's
// barrier would wait for all of them.
template <int LOADS, int READS> __device__ __forceinline__ void end_phase()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(%1)\n\ts_barrier" ::"n"(LOADS), "n"(READS) : "memory");
}

// Consecutive blocks run on different XCDs, each with an L2 of its own: every XCD gets a stretch of neighbouring tiles, in groups of
// 4 rows of tiles, so that the 32 blocks it runs at a time read 4 strips of A and 8 of B.
constexpr int kXcds = 8, kGroup = 4;
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

// A wave's tile of sums, 2 MR x 2 MC of 16 x 16 from (r0, c0) on, through `mine` (32 rows of kEpiRow<MC> bytes, the wave's own): rows whose
// lanes have eight neighbours each.  What 32 rows need is asked for at once.
template <int MC> constexpr int kEpiRow = (MC * 32 + 4) * 4;
template <class TO, int MR, int MC, class S> __device__ __forceinline__ void store_wave(const GemmArgs &a, int split, LdsByte *mine, int r0, int c0, int lane, const S &acc)
{
    constexpr int PER = 4 * MC, ROWS = 64 / PER, N = 32 / ROWS;       // lanes of a row, rows at a time
    const EpiArgs e = a.epi;
    const bool whole = a.splits == 1;
    const int c = c0 + 8 * (lane % PER);
    Raw8<float> bias = {};
    if (whole && e.bias && c < a.C) bias = load8(e.bias + c, a.C - c);
#pragma unroll
    for (int i = 0; i < MR; ++i) {
        const int r = r0 + 32 * i + lane / PER;
        auto load = [&](int t) {
            const int n = r + t * ROWS < a.R ? a.C - c : 0;
            return EpiIn<TO>{epi_load_add<TO>(e, r + t * ROWS, c, n), epi_load_z<EPI_EITHER, TO>(e, r + t * ROWS, c, n)};
        };
        constexpr bool AHEAD = sizeof(TO) == 2;        // fp32: registers
        EpiIn<TO> in[N];
        if (AHEAD && whole)
#pragma unroll
            for (int t = 0; t < N; ++t) in[t] = load(t);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < 2 * MC; ++j)
                CG_LDS(u32x4, mine + (16 * h + (lane & 15)) * kEpiRow<MC> + (16 * j + 4 * (lane >> 4)) * 4) = acc.get(2 * i + h, j);
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int t = 0; t < N; ++t) {
            float v[8];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const u32x4 x = CG_LDS(u32x4, mine + (t * ROWS + lane / PER) * kEpiRow<MC> + (8 * (lane % PER) + 4 * h) * 4);
#pragma unroll
                for (int u = 0; u < 4; ++u) v[4 * h + u] = __uint_as_float(x[u]);
            }
            if (r + t * ROWS < a.R && c < a.C) {
                if (whole) epi_finish<EPI_EITHER, TO>(e, v, bias, AHEAD ? in[t] : load(t), r + t * ROWS, c, a.C - c);
                else store8(a.part + ((int64_t)split * a.R + r + t * ROWS) * a.C + c, to_raw<float>(v), a.C - c);
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// The gradient of a bias beside that of the weights: the blocks of the first columns' tiles add up what they read of A.  A lane sees eight values
// of k of its row, in NP pieces, at a time; the lane 16 further the next eight.
template <int NP> __device__ __forceinline__ float sum_of(const u32x4 (&f)[NP])
{
    float s = 0.f;
#pragma unroll
    for (int p = NP - 1; p >= 0; --p) {
        float v[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) v[t] = __uint_as_float(f[p][t] << 16) + __uint_as_float(f[p][t] & 0xffff0000u);
        s += (v[0] + v[1]) + (v[2] + v[3]);
    }
    return s;
}
__device__ __forceinline__ void store_bias(const GemmArgs &a, int split, int row, int lane, float s)
{
    s += __shfl_xor(s, 16);
    s += __shfl_xor(s, 32);
    float *const to = a.splits == 1 ? a.dbias : a.part + (int64_t)a.splits * a.R * a.C + (int64_t)split * a.R;
    if (lane < 16 && row + lane < a.R) to[row + lane] = s;
}

__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }       // lets loads go on
// The sums of the waves that have the same part of a tile in two halves of k meet in the first half's: through `mine`, the part's own.  false: nothing
// is left for this wave to do.
template <int T> constexpr int kJoin = 64 * (T * T * 16 + T * 4);       // bytes of T x T tiles of 16 x 16, and of the bias
template <bool CUT, int T>
__device__ __forceinline__ bool join_halves(const GemmArgs &a, int split, int half, LdsByte *mine, int row, int lane, Sums<CUT, T, T> &acc, const float (&bias)[T], bool with_bias)
{
    if (half == 1) {
#pragma unroll
        for (int t = 0; t < T * T; ++t) CG_LDS(u32x4, mine + (64 * t + lane) * 16) = acc.get(t / T, t % T);
#pragma unroll
        for (int t = 0; t < T; ++t) CG_LDS(float, mine + T * T * 1024 + (64 * t + lane) * 4) = bias[t];
    }
    lds_barrier();
    if (half == 1) return false;
#pragma unroll
    for (int t = 0; t < T * T; ++t) acc.of_join(t / T, t % T) += __builtin_bit_cast(v4f, CG_LDS(u32x4, mine + (64 * t + lane) * 16));
    if (with_bias)
#pragma unroll
        for (int t = 0; t < T; ++t) store_bias(a, split, row + 16 * t, lane, bias[t] + CG_LDS(float, mine + T * T * 1024 + (64 * t + lane) * 4));
    __builtin_amdgcn_wave_barrier();
    return true;
}

// Tiles of 128 x 128 of bf16 (and 8-bit) tensors, four waves, two steps in LDS; two blocks a compute unit.
template <class TB, bool AX, bool BX, bool DMA, class TO> __global__ __launch_bounds__(256, 2) void gemm_kernel(GemmArgs a)
{
    constexpr int STEP = 64, XT = 128;
    using LA = TileLoader<bf16raw, AX, XT, STEP, 256, DMA>;
    using LB = TileLoader<TB, BX, XT, STEP, 256, DMA && sizeof(TB) == 2>;
    constexpr int STAGE = LA::Lds::BYTES + LB::Lds::BYTES;
    __shared__ __align__(16) char smem[2 * STAGE];
    static_assert(4 * 32 * kEpiRow<2> <= 2 * STAGE, "room for the epilogue");
    LdsByte *const lds = (LdsByte *)smem;
    const int lane = threadIdx.x & 63, wave = (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wr = wave / 2 * 64, wc = wave % 2 * 64;
    int tr, tc, split;
    place_of(a, tr, tc, split);
    const int r0 = tr * XT, c0 = tc * XT, kbeg = split * a.chunk, kend = min(a.K, kbeg + a.chunk);

    LA la(a.A, Packed{}, a.a_ld, r0, a.R, kbeg, kend, a.K);
    LB lb(a.B, a.B8, a.b_ld, c0, a.C, kbeg, kend, a.K);
    Sums<false, 4, 4> acc;
    acc.zero();
    const bool with_bias = AX && a.dbias && tc == 0 && wc == 0;
    float bias[4] = {};
    auto start = [&](int k, LdsByte *at, auto inside) {
        la.template start<decltype(inside)::value>(k, at);
        lb.template start<decltype(inside)::value>(k, at + LA::Lds::BYTES);
    };
    auto finish = [&](LdsByte *at) {
        la.finish(at);
        lb.finish(at + LA::Lds::BYTES);
    };
    // behind the barrier a step's tiles are there and everyone is done with the ones before, whose buffer is filled while these are multiplied
    auto step = [&](int k, int buf, auto inside) {
        tile_sync();
        const bool more = decltype(inside)::value || k + STEP < kend;
        if (more) start(k + STEP, lds + (buf ^ 1) * STAGE, inside);
        LdsByte *const at = lds + buf * STAGE;
#pragma unroll
        for (int ks = 0; ks < STEP / 32; ++ks) {
            u32x4 fa[4], fb[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) fb[i] = LB::Lds::read(at + LA::Lds::BYTES, wc + 16 * i, ks, lane);
#pragma unroll
            for (int i = 0; i < 4; ++i) fa[i] = LA::Lds::read(at, wr + 16 * i, ks, lane);
#pragma unroll
            for (int j = 0; j < 4; ++j) acc.mma(fa, fb[j], j, true);
            if (with_bias)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const u32x4 f[1] = {fa[i]};
                    bias[i] += sum_of<1>(f);
                }
        }
        if (more) finish(lds + (buf ^ 1) * STAGE);
    };
    auto is_inside = [&](int k) { return k < kend && la.inside(k) && lb.inside(k); };
    if (kbeg < kend) {
        const bool in = is_inside(kbeg);
        if (in) start(kbeg, lds, std::true_type());
        else start(kbeg, lds, std::false_type());
        finish(lds);
        int buf = 0, k = kbeg;
        if (in)
            for (; is_inside(k + STEP); k += STEP, buf ^= 1) step(k, buf, std::true_type());
        for (; k < kend; k += STEP, buf ^= 1) step(k, buf, std::false_type());
    }
    if (with_bias)
#pragma unroll
        for (int i = 0; i < 4; ++i) store_bias(a, split, r0 + wr + 16 * i, lane, bias[i]);
    __syncthreads();
    store_wave<TO, 2, 2>(a, split, lds + wave * 32 * kEpiRow<2>, r0 + wr, c0 + wc, lane, acc);
}
template <class TB, bool AX, bool BX, bool DMA, class TO> int launch(const GemmArgs &a, hipStream_t s)
{
    hipLaunchKernelGGL((gemm_kernel<TB, AX, BX, DMA, TO>), dim3((unsigned)(a.tiles_r * a.tiles_c * a.splits)), dim3(256), 0, s, a);
    CG_HIP_TRY(hipGetLastError());
    return CG_OK;
}

// The same with four waves and two steps in LDS for either half of a block's values of k, whose sums meet in LDS: small products, which the latency of a
// step's loads bounds, in tiles of 64 x 64 (two steps, one of either half, 0.6 us where a compute unit has one block, 0.38 where it has several; the
// matrix instructions of both take 0.12), and those that have a tile of 128 x 128 for each compute unit at most (1.2 us, of which LDS, written and read,
// takes 0.7 and the matrix instructions 0.46).
template <class TB, bool AX, bool BX, bool DMA, class TO, int XT> __global__ __launch_bounds__(512, XT == 64 ? 4 : 2) void gemm_halves_kernel(GemmArgs a)
{
    constexpr int STEP = 64, T = XT / 32;
    using LA = TileLoader<bf16raw, AX, XT, STEP, 256, DMA>;
    using LB = TileLoader<TB, BX, XT, STEP, 256, DMA && sizeof(TB) == 2>;
    constexpr int STAGE = LA::Lds::BYTES + LB::Lds::BYTES, MINE = kJoin<T> > 32 * kEpiRow<T / 2> ? kJoin<T> : 32 * kEpiRow<T / 2>;
    __shared__ __align__(16) char smem[4 * STAGE];
    static_assert(MINE <= STAGE, "room for the epilogue, and for the sums of a wave");
    const int lane = threadIdx.x & 63, wave = (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = wave >> 2, wr = (wave >> 1 & 1) * XT / 2, wc = (wave & 1) * XT / 2;
    LdsByte *const lds = (LdsByte *)smem + half * 2 * STAGE, *const mine = (LdsByte *)smem + (wave & 3) * MINE;
    int tr, tc, split;
    place_of(a, tr, tc, split);
    const int r0 = tr * XT, c0 = tc * XT, k0 = split * a.chunk, k1 = min(a.K, k0 + a.chunk), each = (k1 - k0 + 2 * STEP - 1) / (2 * STEP);
    const int kbeg = k0 + half * each * STEP, kend = min(k1, kbeg + each * STEP);

    LA la(a.A, Packed{}, a.a_ld, r0, a.R, kbeg, kend, a.K);
    LB lb(a.B, a.B8, a.b_ld, c0, a.C, kbeg, kend, a.K);
    Sums<false, T, T> acc;
    acc.zero();
    const bool with_bias = AX && a.dbias && tc == 0 && wc == 0;
    float bias[T] = {};
    auto start = [&](int k, LdsByte *at) {
        if (la.inside(k) && lb.inside(k)) {
            la.template start<true>(k, at);
            lb.template start<true>(k, at + LA::Lds::BYTES);
        } else {
            la.template start<false>(k, at);
            lb.template start<false>(k, at + LA::Lds::BYTES);
        }
    };
    auto finish = [&](LdsByte *at) {
        la.finish(at);
        lb.finish(at + LA::Lds::BYTES);
    };
    if (kbeg < kend) {
        start(kbeg, lds);
        finish(lds);
    }
    for (int i = 0, k = kbeg; i < each; ++i, k += STEP) {
        tile_sync();
        LdsByte *const at = lds + (i & 1) * STAGE, *const next = lds + (~i & 1) * STAGE;
        const bool more = k + STEP < kend;
        if (more) start(k + STEP, next);
        if (k < kend) {
#pragma unroll
            for (int ks = 0; ks < STEP / 32; ++ks) {
                u32x4 fa[T], fb[T];
#pragma unroll
                for (int t = 0; t < T; ++t) fb[t] = LB::Lds::read(at + LA::Lds::BYTES, wc + 16 * t, ks, lane);
#pragma unroll
                for (int t = 0; t < T; ++t) fa[t] = LA::Lds::read(at, wr + 16 * t, ks, lane);
#pragma unroll
                for (int j = 0; j < T; ++j) acc.mma(fa, fb[j], j, true);
                if (with_bias)
#pragma unroll
                    for (int t = 0; t < T; ++t) {
                        const u32x4 f[1] = {fa[t]};
                        bias[t] += sum_of<1>(f);
                    }
            }
        }
        if (more) finish(next);
    }
    __syncthreads();
    if (join_halves(a, split, half, mine, r0 + wr, lane, acc, bias, with_bias)) store_wave<TO, T / 2, T / 2>(a, split, mine, r0 + wr, c0 + wc, lane, acc);
}
template <class TB, bool AX, bool BX, bool DMA, class TO, int XT> int launch_halves(const GemmArgs &a, hipStream_t s)
{
    hipLaunchKernelGGL((gemm_halves_kernel<TB, AX, BX, DMA, TO, XT>), dim3((unsigned)(a.tiles_r * a.tiles_c * a.splits)), dim3(512), 0, s, a);
    CG_HIP_TRY(hipGetLastError());
    return CG_OK;
}

// fp32 tensors: tiles of 128 x 128, eight waves, one step in LDS; two blocks a compute unit, one of which multiplies while the other cuts.
template <class TB, bool AX, bool BX> __global__ __launch_bounds__(512, 4) void gemm_cut_kernel(GemmArgs a)
{
    constexpr int STEP = 32, XT = 128;
    using LA = TileLoader<float, AX, XT, STEP, 512, false>;
    using LB = TileLoader<TB, BX, XT, STEP, 512, false>;
    constexpr int NB = LB::NP, TILES = LA::Lds::BYTES + LB::Lds::BYTES, EPI = 8 * 32 * kEpiRow<2>;
    __shared__ __align__(16) char smem[TILES > EPI ? TILES : EPI];
    LdsByte *const lds = (LdsByte *)smem;
    const int lane = threadIdx.x & 63, wave = (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wr = wave / 2 * 32, wc = wave % 2 * 64;
    int tr, tc, split;
    place_of(a, tr, tc, split);
    const int r0 = tr * XT, c0 = tc * XT, kbeg = split * a.chunk, kend = min(a.K, kbeg + a.chunk);

    LA la(a.A, Packed{}, a.a_ld, r0, a.R, kbeg, kend, a.K);
    LB lb(a.B, a.B8, a.b_ld, c0, a.C, kbeg, kend, a.K);
    Sums<true, 2, 4> acc;
    acc.zero();
    const bool with_bias = AX && a.dbias && tc == 0 && wc == 0;
    float bias[2] = {};
    auto start = [&](int k, auto inside) {
        la.template start<decltype(inside)::value>(k, lds);
        lb.template start<decltype(inside)::value>(k, lds);
    };
    auto step = [&](int k, auto inside) {
        la.finish(lds);
        lb.finish(lds + LA::Lds::BYTES);
        lds_barrier();
        if (decltype(inside)::value || k + STEP < kend) start(k + STEP, inside);
        u32x4 fa[3][2];
#pragma unroll
        for (int p = 2; p >= 0; --p)
#pragma unroll
            for (int i = 0; i < 2; ++i) fa[p][i] = LA::Lds::read(lds, wr + 16 * i, 0, lane, p);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            u32x4 fb[NB];
#pragma unroll
            for (int p = NB - 1; p >= 0; --p) fb[p] = LB::Lds::read(lds + LA::Lds::BYTES, wc + 16 * j, 0, lane, p);
#pragma unroll
            for (int d = 2; d >= 0; --d)
#pragma unroll
                for (int p = 0; p < 3; ++p)
                    if (d - p >= 0 && d - p < NB) acc.mma(fa[p], fb[d - p < NB && d - p >= 0 ? d - p : 0], j, d == 0);
        }
        if (with_bias)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const u32x4 f[3] = {fa[0][i], fa[1][i], fa[2][i]};
                bias[i] += sum_of<3>(f);
            }
        lds_barrier();
    };
    auto is_inside = [&](int k) { return k < kend && la.inside(k) && lb.inside(k); };
    if (kbeg < kend) {
        const bool in = is_inside(kbeg);
        if (in) start(kbeg, std::true_type());
        else start(kbeg, std::false_type());
        int k = kbeg;
        if (in)
            for (; is_inside(k + STEP); k += STEP) step(k, std::true_type());
        for (; k < kend; k += STEP) step(k, std::false_type());
    }
    if (with_bias)
#pragma unroll
        for (int i = 0; i < 2; ++i) store_bias(a, split, r0 + wr + 16 * i, lane, bias[i]);
    store_wave<float, 1, 2>(a, split, lds + wave * 32 * kEpiRow<2>, r0 + wr, c0 + wc, lane, acc);
}
// Small fp32 products: tiles of 64 x 64, four waves for either half of a block's values of k, whose sums meet in LDS.  Bound by the latency of a
// step's loads, cut and reads in turn (a step of either half 1.06 us where a compute unit has one block, 0.87 each where it has several, of which the
// matrix instructions take 0.35): the halves fill each other's waits without a second launch that joins them.
template <class TB, bool AX, bool BX> __global__ __launch_bounds__(512, 4) void gemm_cut_small_kernel(GemmArgs a)
{
    constexpr int STEP = 32, XT = 64;
    using LA = TileLoader<float, AX, XT, STEP, 256, false>;
    using LB = TileLoader<TB, BX, XT, STEP, 256, false>;
    constexpr int NB = LB::NP, TILES = LA::Lds::BYTES + LB::Lds::BYTES, MINE = 32 * kEpiRow<1>;
    __shared__ __align__(16) char smem[2 * TILES];
    static_assert(4 * MINE <= 2 * TILES && MINE >= kJoin<2>, "room for the epilogue, and for the sums of a wave");
    const int lane = threadIdx.x & 63, wave = (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = wave >> 2, wr = (wave >> 1 & 1) * 32, wc = (wave & 1) * 32;
    LdsByte *const lds = (LdsByte *)smem + half * TILES, *const mine = (LdsByte *)smem + (wave & 3) * MINE;
    int tr, tc, split;
    place_of(a, tr, tc, split);
    const int r0 = tr * XT, c0 = tc * XT, k0 = split * a.chunk, k1 = min(a.K, k0 + a.chunk), each = (k1 - k0 + 2 * STEP - 1) / (2 * STEP);
    const int kbeg = k0 + half * each * STEP, kend = min(k1, kbeg + each * STEP);

    LA la(a.A, Packed{}, a.a_ld, r0, a.R, kbeg, kend, a.K);
    LB lb(a.B, a.B8, a.b_ld, c0, a.C, kbeg, kend, a.K);
    Sums<true, 2, 2> acc;
    acc.zero();
    const bool with_bias = AX && a.dbias && tc == 0 && wc == 0;
    float bias[2] = {};
    auto start = [&](int k) {
        if (la.inside(k) && lb.inside(k)) {
            la.template start<true>(k, lds);
            lb.template start<true>(k, lds);
        } else {
            la.template start<false>(k, lds);
            lb.template start<false>(k, lds);
        }
    };
    if (kbeg < kend) start(kbeg);
    for (int i = 0, k = kbeg; i < each; ++i, k += STEP) {
        if (k < kend) {
            la.finish(lds);
            lb.finish(lds + LA::Lds::BYTES);
        }
        lds_barrier();
        if (k + STEP < kend) start(k + STEP);
        if (k < kend) {
            u32x4 fa[3][2];
#pragma unroll
            for (int p = 2; p >= 0; --p)
#pragma unroll
                for (int t = 0; t < 2; ++t) fa[p][t] = LA::Lds::read(lds, wr + 16 * t, 0, lane, p);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                u32x4 fb[NB];
#pragma unroll
                for (int p = NB - 1; p >= 0; --p) fb[p] = LB::Lds::read(lds + LA::Lds::BYTES, wc + 16 * j, 0, lane, p);
#pragma unroll
                for (int d = 2; d >= 0; --d)
#pragma unroll
                    for (int p = 0; p < 3; ++p)
                        if (d - p >= 0 && d - p < NB) acc.mma(fa[p], fb[d - p < NB && d - p >= 0 ? d - p : 0], j, d == 0);
            }
            if (with_bias)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const u32x4 f[3] = {fa[0][t], fa[1][t], fa[2][t]};
                    bias[t] += sum_of<3>(f);
                }
        }
        lds_barrier();
    }
    if (join_halves(a, split, half, mine, r0 + wr, lane, acc, bias, with_bias)) store_wave<float, 1, 1>(a, split, mine, r0 + wr, c0 + wc, lane, acc);
}
template <class TB, bool AX, bool BX> int launch_cut_small(const GemmArgs &a, hipStream_t s)
{
    hipLaunchKernelGGL((gemm_cut_small_kernel<TB, AX, BX>), dim3((unsigned)(a.tiles_r * a.tiles_c * a.splits)), dim3(512), 0, s, a);
    CG_HIP_TRY(hipGetLastError());
    return CG_OK;
}

template <class TB, bool AX, bool BX> int launch_cut(const GemmKind &k, const GemmArgs &a, hipStream_t s)
{
    if (k.tile == 64) return launch_cut_small<TB, AX, BX>(a, s);
    hipLaunchKernelGGL((gemm_cut_kernel<TB, AX, BX>), dim3((unsigned)(a.tiles_r * a.tiles_c * a.splits)), dim3(512), 0, s, a);
    CG_HIP_TRY(hipGetLastError());
    return CG_OK;
}

// Tiles of 256 x 256 of bf16 tensors, eight waves.  Operands pass through LDS in halves of 128 rows or columns, A0 A1 B0 B1, 64 values of k at
// a time, two steps in LDS.  A wave makes 64 x 32 of each quarter of the tile, a quarter a phase, and reads in each phase the half that it
// needs next, so that its operands are in registers when a phase begins (what a phase uses for the last time is overwritten as it goes):
//     even steps   A0 B0 (reads B1)   A0 B1 (A1)   A1 B1 (B1 of the next step)   A1 B0 (A0 of the next step)
//     odd steps    A0 B1 (reads B0)   A0 B0 (A1)   A1 B0 (B0 of the next step)   A1 B1 (A0 of the next step)
// Two phases after a half was read its place is filled with what is read there eight phases after, so loads have five phases to arrive.  The
// barrier at a phase's end: everyone's reads of the phase before are done, and everyone's part of the next half has landed.
constexpr int kHalf = 128 * 64 * 2, kLargeRow = (32 + 4) * 4;
template <bool AX, bool BX, class TO> __global__ __launch_bounds__(512, 2) void gemm_large_kernel(GemmArgs a)
{
    using LA = HalfLoader<AX>;
    using LB = HalfLoader<BX>;
    extern __shared__ __align__(16) char smem[];
    LdsByte *const lds = (LdsByte *)smem;
    const int lane = threadIdx.x & 63, wave = (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wr = wave >> 2, wc = wave & 3;
    int tr, tc, split;
    place_of(a, tr, tc, split);
    const int r0 = tr * 256, c0 = tc * 256, kbeg = split * a.chunk, kend = min(a.K, kbeg + a.chunk), n = (kend - kbeg + 63) / 64;

    LA la[2] = {LA(a.A, a.a_ld, r0, a.R, kbeg, kend), LA(a.A, a.a_ld, r0 + 128, a.R, kbeg, kend)};
    LB lb[2] = {LB(a.B, a.b_ld, c0, a.C, kbeg, kend), LB(a.B, a.b_ld, c0 + 128, a.C, kbeg, kend)};
    // a lane's places of either operand lie within what an instruction's offset reaches
    auto at_a = [&](int h, int s) { return lds + ((s & 1) * 2 + h) * kHalf; };
    auto at_b = [&](int h, int s) { return lds + (4 + (s & 1) * 2 + h) * kHalf; };
    u32x4 fa[2][4], fb[2][2][2];     // [values of k, 32 at a time][16 rows]; half of B
    v4f acc[2][2][4][2];             // half of A, half of B, 16 rows, 16 columns
#pragma unroll
    for (int i = 0; i < 32; ++i) acc[i >> 4][i >> 3 & 1][i >> 1 & 3][i & 1] = v4f{};

    auto read_a = [&](int h, int s, int ks, int i) { fa[ks][i] = LA::Lds::read(at_a(h, s), 64 * wr + 16 * i, ks, lane); };
    auto read_b = [&](auto h, int s, int ks, int j) { fb[h.value][ks][j] = LB::Lds::read(at_b(h.value, s), 32 * wc + 16 * j, ks, lane); };
    auto multiply = [&](auto ha, auto hb, int ks, int i) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
            acc[ha.value][hb.value][i][j] = mfma16(fb[hb.value][ks][j], fa[ks][i], acc[ha.value][hb.value][i][j]);
    };
    const std::integral_constant<int, 0> _0;
    const std::integral_constant<int, 1> _1;
    // A phase: two products, what they leave to be read, and in the middle the loads (at its beginning all waves would wait for each other's).
    auto phase = [&](auto ha, auto hb, auto full, bool fill, auto &loader, LdsByte *to, auto read) {
        constexpr bool FULL = decltype(full)::value;
#pragma unroll
        for (int t = 0; t < 4; ++t) {         // half a 32 of k: two of four 16 rows
            multiply(ha, hb, t >> 1, 2 * (t & 1));
            multiply(ha, hb, t >> 1, 2 * (t & 1) + 1);
            read(t);
            if (t == 1 && (FULL || fill)) loader.template load<FULL, 0>(to, wave);
            if (t == 3 && (FULL || fill)) loader.template load<FULL, 1>(to, wave);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // first: the half of B that the step begins with.  full: a step behind the one after the next is there too
    auto step = [&](int s, auto first, auto full) {
        constexpr bool FULL = decltype(full)::value;
        const std::integral_constant<int, 1 - decltype(first)::value> second;
        const bool fill = s + 2 < n, more = FULL || s + 1 < n;
        // loads that may still be on their way at a phase's end: five halves' while they go on, one fewer from phase to phase in the last but
        // one step, none in the last
        auto end = [&](auto reads, auto i) {
            if (FULL || fill) end_phase<10, decltype(reads)::value>();
            else if (more) end_phase<8 - 2 * decltype(i)::value, decltype(reads)::value>();
            else end_phase<0, decltype(reads)::value>();
        };
        const std::integral_constant<int, AX ? 15 : 8> reads_a;
        const std::integral_constant<int, BX ? 8 : 4> reads_b;
        phase(_0, first, full, fill, lb[first.value], at_b(first.value, s), [&](int t) { read_b(second, s, t >> 1, t & 1); });
        end(reads_b, _0);
        phase(_0, second, full, fill, la[0], at_a(0, s), [&](int t) { read_a(1, s, t >> 1, 2 * (t & 1)), read_a(1, s, t >> 1, 2 * (t & 1) + 1); });
        end(reads_a, _1);
        phase(_1, second, full, fill, lb[second.value], at_b(second.value, s), [&](int t) {
            // columns' operands serve all rows of their 32 of k: read behind the last of them
            if (more && (t & 1)) read_b(second, s + 1, t >> 1, 0), read_b(second, s + 1, t >> 1, 1);
        });
        end(reads_b, std::integral_constant<int, 2>());
        phase(_1, first, full, fill, la[1], at_a(1, s), [&](int t) { if (more) read_a(0, s + 1, t >> 1, 2 * (t & 1)), read_a(0, s + 1, t >> 1, 2 * (t & 1) + 1); });
        end(reads_a, std::integral_constant<int, 3>());
    };
    if (n > 0) {
        lb[0].next(at_b(0, 0), wave);
        la[0].next(at_a(0, 0), wave);
        lb[1].next(at_b(1, 0), wave);
        la[1].next(at_a(1, 0), wave);
        if (n > 1) {
            lb[1].next(at_b(1, 1), wave);
            la[0].next(at_a(0, 1), wave);
            lb[0].next(at_b(0, 1), wave);
            la[1].next(at_a(1, 1), wave);
        }
        if (n > 1) end_phase<12, 0>();
        else end_phase<0, 0>();
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            if (t < 4) read_b(_0, 0, t >> 1, t & 1);
            read_a(0, 0, t >> 2, t & 3);
        }
        if (n > 1) end_phase<10, 0>();
        else end_phase<0, 0>();
        int s = 0;
        for (; s + 4 < n; s += 2) {
            step(s, _0, std::true_type());
            step(s + 1, _1, std::true_type());
        }
        for (; s < n; s += 2) {
            step(s, _0, std::false_type());
            if (s + 1 < n) step(s + 1, _1, std::false_type());
        }
    }

    // What the epilogue reads is asked for at once, the registers of the operands are free: forward the residual, backward what the slope is
    // taken of.  (A gradient that is added there comes as it is needed.)
    LdsByte *const mine = lds + wave * 32 * kLargeRow;
    const EpiArgs e = a.epi;
    constexpr bool PLAIN = AX;          // backward-weight: sums are the result
    const int c_of = c0 + 32 * wc + 8 * (lane & 3), r_of = r0 + 64 * wr + lane / 4;
    auto row_of = [&](int q) { return r_of + 128 * (q >> 3) + 32 * (q >> 1 & 1) + 16 * (q & 1); };       // q: half of A, half of B, 32 rows, 16 rows
    auto col_of = [&](int q) { return c_of + 128 * (q >> 2 & 1); };
    Raw8<float> bias[2] = {};
    if (!PLAIN && e.bias)
#pragma unroll
        for (int h = 0; h < 2; ++h) bias[h] = load8(e.bias + (c_of + 128 * h < a.C ? c_of + 128 * h : 0), a.C - c_of - 128 * h);
    Raw8<TO> in[16];
    if constexpr (!PLAIN) {
#pragma unroll
        for (int q = 0; q < 16; ++q) {
            const int n = row_of(q) < a.R ? a.C - col_of(q) : 0;
            in[q] = BX ? epi_load_z<EPI_BWD, TO>(e, row_of(q), col_of(q), n) : epi_load_add<TO>(e, row_of(q), col_of(q), n);
        }
    }
#pragma unroll
    for (int p = 0; p < 8; ++p) {
        const int ha = p >> 2, hb = p >> 1 & 1, i = p & 1;
#pragma unroll
        for (int u = 0; u < 4; ++u)       // 16 rows, 16 columns
            CG_LDS(u32x4, mine + (16 * (u >> 1) + (lane & 15)) * kLargeRow + (16 * (u & 1) + 4 * (lane >> 4)) * 4) = __builtin_bit_cast(u32x4, acc[ha][hb][2 * i + (u >> 1)][u & 1]);
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int q = 2 * p + t, r = row_of(q), c = col_of(q);
            float v[8];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const u32x4 x = CG_LDS(u32x4, mine + (16 * t + lane / 4) * kLargeRow + (8 * (lane & 3) + 4 * h) * 4);
#pragma unroll
                for (int y = 0; y < 4; ++y) v[4 * h + y] = __uint_as_float(x[y]);
            }
            if (r < a.R && c < a.C) {
                if constexpr (PLAIN) store8(static_cast<TO *>(e.out) + r * e.out_ld + c, to_raw<TO>(v), a.C - c);
                else {
                    EpiIn<TO> of;
                    of.z = of.add = in[q];
                    if (BX) of.add = epi_load_add<TO>(e, r, c, a.C - c);
                    epi_finish<BX ? EPI_BWD : EPI_FWD, TO>(e, v, bias[hb], of, r, c, a.C - c);
                }
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
}
template <bool AX, bool BX, class TO> int launch_large(const GemmArgs &a, hipStream_t s)
{
    constexpr int LDS = 8 * kHalf;
    auto *const kernel = gemm_large_kernel<AX, BX, TO>;
    CG_HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, LDS));
    hipLaunchKernelGGL(kernel, dim3((unsigned)(a.tiles_r * a.tiles_c)), dim3(512), LDS, s, a);
    CG_HIP_TRY(hipGetLastError());
    return CG_OK;
}

template <class TB, bool AX, bool BX, class TO> int launch_bf16(const GemmKind &k, const GemmArgs &a, hipStream_t s)
{
    if constexpr (sizeof(TB) == 2)
        if (k.tile == 256) return launch_large<AX, BX, TO>(a, s);
    if (gemm_halves(k.type, k.tile, (int64_t)a.tiles_r * a.tiles_c * a.splits)) {
        if (k.tile == 64) return k.dma ? launch_halves<TB, AX, BX, true, TO, 64>(a, s) : launch_halves<TB, AX, BX, false, TO, 64>(a, s);
        return k.dma ? launch_halves<TB, AX, BX, true, TO, 128>(a, s) : launch_halves<TB, AX, BX, false, TO, 128>(a, s);
    }
    return k.dma ? launch<TB, AX, BX, true, TO>(a, s) : launch<TB, AX, BX, false, TO>(a, s);
}

}  // namespace

int gemm_launch(const GemmKind &k, const GemmArgs &a, hipStream_t s)
{
    if (k.type == CG_TYPE_FP32) {
        if (k.pass == CG_PASS_FWD) return launch_cut<float, false, false>(k, a, s);
        if (k.pass == CG_PASS_BWD_DATA) return launch_cut<float, false, true>(k, a, s);
        return k.packed ? launch_cut<int8_t, true, true>(k, a, s) : launch_cut<float, true, true>(k, a, s);
    }
    if (k.pass == CG_PASS_FWD) return launch_bf16<bf16raw, false, false, bf16raw>(k, a, s);
    if (k.pass == CG_PASS_BWD_DATA) return launch_bf16<bf16raw, false, true, bf16raw>(k, a, s);
    return k.packed ? launch_bf16<int8_t, true, true, float>(k, a, s) : launch_bf16<bf16raw, true, true, float>(k, a, s);
}

}  // namespace cg
