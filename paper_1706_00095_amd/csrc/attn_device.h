// Device code shared by the attention kernels (attn_fwd.hip, attn_bwd.hip) and what their host side passes to them.
//
// Common frame.  All products run on v_mfma_f32_32x32x16_bf16: fp32 tensors are cut into three bf16 pieces (NP = 3, six
// products), bf16 tensors are taken as they are (NP = 1).  Of the two sides of the score matrix one, X, lives in registers: a
// wave owns 32 of its rows (queries in the forward and the dq kernel, keys in the dk/dv kernel) and holds them as the
// instruction's second operand.  The other, Y, passes through LDS in tiles all waves share and is the first operand.  A lane
// then holds 16 scores of ONE X row (C layout: column lane % 32, rows 8 (i / 4) + 4 (lane / 32) + i % 4), so softmax statistics are
// sums within a lane and one exchange with lane ^ 32, and the scores are in place as the second operand of the next product,
// whose contraction runs over Y: its slots are filled in the order the C layout has, and the first operand, Y transposed, is read
// from the same LDS tile by transposing reads (ds_read_b64_tr_b16) in that order.  Scores never pass through LDS.
//
// Query rows.  With grouped heads the Gp query heads that share a key-value head are packed into one problem of n Gp rows
// (row r: token r / Gp, head r % Gp), so that K and V are read once for all of them and their dk, dv need no sum afterwards.
// With a bias Gp = 1: the table differs from head to head.
#pragma once
#include "cg_internal.h"
#include "igemm_device.h"
#include "typed_device.h"

namespace cg {

struct AttnArgs {
    const void *q, *k, *v, *d_o, *o_in, *o_rest_in;
    void *o, *o_rest, *dq, *dk, *dv;
    float *lse;                            // [Hq][Tq]
    // [Hq][Tq], written by the dq kernel: sums of do o; lse as the exponent takes it; with a bias, what else it takes (log2, 0 but for rows
    // whose lse is far from zero)
    float *delta, *lse_b, *log_l;
    const int32_t *cu_q, *cu_k;
    int64_t q_tok, q_head, k_tok, k_head, v_tok, v_head, o_tok, o_head;
    int B, Tq, Tk, Hq, Hkv, G, Gp, D;      // G: query heads of a key-value head; Gp of them are packed (1 or G)
    FastDiv by_gp;
    float scale;
    int causal;
    // bias by distance: btab [Hq][2 W + 1], bucket of delta (clamped to -W .. W) bid [2 W + 1]
    const float *btab;
    const uint8_t *bid;
    int W, buckets;
    float *dbias_part, *dbias;             // [Hq][dbias_parts][buckets] of the dq kernel's items; [Hq][buckets]
    int dbias_parts, dbias_splits, dbias_chunk;      // items a head there is room for; how the dq kernel's axis is cut
    int tiles;                             // of X rows over all sequences, an upper bound
    // Y cut into at most `splits` chunks of `chunk` rows, a block each; a tile with several leaves partial results for attn_join_kernel
    int splits, chunk;
    int fold;                              // not 0: from which item of a problem on their order is turned round
    int levels;                            // not 0: items by the length of what they see
    int gsplit;                            // dk/dv kernel with a bias: chunks are of one head each (G), or of all (1)
    int yt;                                // rows of a Y tile in the dk/dv kernel (attn_dkdv_yt)
    int dma;                               // K and V (forward, dq), Q and dO (dk/dv) may travel without registers
    float *part[2], *part_ml;              // [problem][tiles splits gsplit][128][DP] by item (forward: o; dq; dk, dv), [..][2][128]
};

constexpr int kAttnRows = 128;             // X rows of a block: four waves of 32
constexpr int kAttnMaxD = 128;
constexpr int kMaxBuckets = 256;
constexpr int kFewKeys = 64, kFewRows = 32;       // keys, and query rows, of a sequence whose products keep more bits (attn_fwd.hip, attn_bwd.hip)
constexpr int attn_dkdv_yt(bool bf16, int DP) { return bf16 && DP < 128 ? 64 : 32; }

// May the loaders that go by buffers take rows of these strides (elements)?  `per`: heads packed as rows (a tile of 32 begins with
// a token).  Rows behind the last one have to lie behind the buffer's end.  bf16 goes to LDS directly: whole and 16-byte aligned
// chunks of eight; fp32 goes through registers: whole chunks of four.
inline bool attn_dma_ok(int type, const void *p, int64_t tok, int64_t head, int per, int D)
{
    if (!(tok >= (per - 1) * head + D && tok < (1 << 22) && 32 % per == 0)) return false;
    return type == CG_TYPE_FP32 ? D % 4 == 0 : aligned16(p) && D % 8 == 0 && tok % 8 == 0 && head % 8 == 0;
}

// attn_fwd.hip, attn_bwd.hip: DP is D rounded up to a multiple of 32
int attn_fwd_launch(const AttnArgs &a, int type, hipStream_t s);
int attn_dq_launch(const AttnArgs &a, int type, hipStream_t s);
int attn_dkdv_launch(const AttnArgs &a, int type, hipStream_t s);
// The join of the forward pass; of the backward pass, dq and dk, dv in one launch (either NULL: nothing to join).
int attn_join_launch(const AttnArgs &a, int type, hipStream_t s);
int attn_join_bwd_launch(const AttnArgs *dq, const AttnArgs *dkdv, int type, hipStream_t s);

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

// ---- LDS tiles ------------------------------------------------------------------------------------------------------------
// ROWS x DP bf16, NP planes.  16-byte chunks of a row are exchanged by a function of the row so that neither sixteen rows' same chunk
// (a row read takes 16 lanes at a time) nor four rows' same 64 bytes (transposing reads) fall on the same banks (64 of 4 bytes).
template <int DP> __device__ __forceinline__ int swizzle(int row)
{
    if constexpr (DP == 128) return (row & 3) << 2 | (row >> 2 & 3);
    else if constexpr (DP == 64) return (row >> 1 & 1) << 2 | (row >> 2 & 3);
    else return row >> 2 & 3;
}
template <int DP, int ROWS, int NP> struct Tile {
    static constexpr int CH = DP / 8, BYTES = NP * ROWS * DP * 2;
    static __device__ __forceinline__ int at(int row, int chunk) { return row * DP * 2 + ((chunk ^ swizzle<DP>(row)) << 4); }
    static __device__ __forceinline__ void put(LdsByte *t, int row, int chunk, const Frag<NP> &f)
    {
#pragma unroll
        for (int k = 0; k < NP; ++k) CG_LDS(u32x4, t + k * ROWS * DP * 2 + at(row, chunk)) = f.p[k];
    }
    // first operand, rows of the tile: row0 + lane % 32, contraction 16 ks ..
    static __device__ __forceinline__ Frag<NP> rows(LdsByte *t, int row0, int ks, int lane)
    {
        Frag<NP> f;
#pragma unroll
        for (int k = 0; k < NP; ++k)
            f.p[k] = CG_LDS(u32x4, t + k * ROWS * DP * 2 + at(row0 + (lane & 31), 2 * ks + (lane >> 5)));
        return f;
    }
    // first operand, columns of the tile: 32 dt + lane % 32, contraction over the rows row0 .. row0 + 15 in the order of the C layout.
    // A transposing read gives lane i of 16 column i of the 4 x 16 values that the 16 lanes' addresses name, four lanes a row.
    static __device__ __forceinline__ Frag<NP> cols(LdsByte *t, int row0, int dt, int lane)
    {
        const int row = row0 + 4 * (lane >> 5) + (lane >> 2 & 3), chunk = 4 * dt + 2 * (lane >> 4 & 1) + (lane >> 1 & 1);
        Frag<NP> f;
#pragma unroll
        for (int k = 0; k < NP; ++k) {
            LdsByte *base = t + k * ROWS * DP * 2 + 8 * (lane & 1);
            const s16x4 lo = tr(base + at(row, chunk)), hi = tr(base + at(row + 8, chunk));
            const uint2 a = __builtin_bit_cast(uint2, lo), b = __builtin_bit_cast(uint2, hi);
            f.p[k] = u32x4{a.x, a.y, b.x, b.y};
        }
        return f;
    }
    static __device__ __forceinline__ s16x4 tr(LdsByte *p)
    {
        return __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<__attribute__((address_space(3))) s16x4 *>(p));
    }
};

// ---- where rows lie -------------------------------------------------------------------------------------------------------
struct Seq { int b, q0, n, k0, m; };        // query tokens q0 .. q0 + n - 1, key tokens k0 .. k0 + m - 1 (cut to the tensors)

__device__ __forceinline__ void bounds_of(const int32_t *cu, int T, int b, int &first, int &len)
{
    first = min(max(cu[b], 0), T);
    len = min(max(cu[b + 1], first), T) - first;
}
// Work items of a kernel: the X tiles of all sequences, each as often as its sequence has chunks of Y.  X_KEYS: X are keys and Y the
// query rows, else the other way round.
constexpr int kLevels = 4, kUnits = 256, kFoldMost = 640;      // compute units
// Chunks of an axis of n rows, one at least; n + a.chunk may pass 2^31.
__device__ __forceinline__ int chunks_in(const AttnArgs &a, int n) { return max(1, (int)(((uint32_t)max(n, 0) + (uint32_t)a.chunk - 1) / (uint32_t)a.chunk)); }
struct Place { int b, t, split, slot; };        // sequence, its tile, chunk, number of the item
// Only the items that are there have numbers, so that the blocks for which a launch has room beside them end at once and last (32
// sequences of 4096 keys, 4 queries each: 10 240 blocks for 128 items, 82 us; with a number for each tile and possible chunk, 199).  A
// sequence's last row tiles come first: they see most keys under a causal mask.
// Under a causal mask a launch of several rounds would end with the last sequence's longest tiles: its items then come by the length of
// what they see, in kLevels steps of the longest, and by sequence within a step.
__device__ __forceinline__ int wave_sum_upto(int v, int lane)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int u = __shfl_up(v, d);
        if (lane >= d) v += u;
    }
    return v;
}
template <bool X_KEYS> __device__ __forceinline__ bool find_level(const AttnArgs &a, int index, Place &p)
{
    const int lane = threadIdx.x & 63;
    int first, n = 0, m = 0;
    if (lane < a.B) {
        bounds_of(a.cu_q, a.Tq, lane, first, n);
        bounds_of(a.cu_k, a.Tk, lane, first, m);
    }
    const int tiles = ((X_KEYS ? m : n * a.Gp) + kAttnRows - 1) / kAttnRows;
    int top = X_KEYS ? n : m;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) top = max(top, __shfl_xor(top, d));
    p.slot = index, p.split = 0;
    int above = tiles;          // tiles of the sequence that are left: those that see no more than the step's upper end
#pragma unroll 1
    for (int l = kLevels - 1; l >= 0; --l) {
        const int x = (int)((int64_t)top * l / kLevels);
        int below = 0;          // that see no more than x
        if (l > 0) {
            if (X_KEYS) below = x >= n ? tiles : tiles - min(max((m - x + kAttnRows - 1) / kAttnRows, 0), tiles);
            else below = min(min(max(x - (m - n), 0), n) * a.Gp / kAttnRows, tiles);
        }
        below = min(below, above);
        const int mine = above - below, upto = wave_sum_upto(mine, lane);
        const uint64_t beyond = __ballot(upto > index);
        if (beyond) {
            const int at = __builtin_ctzll(beyond), within = index - __shfl(upto - mine, at);
            p.b = at;
            p.t = __builtin_amdgcn_readfirstlane(X_KEYS ? __shfl(tiles - above, at) + within : __shfl(above, at) - 1 - within);
            return true;
        }
        index -= __builtin_amdgcn_readfirstlane(__shfl(upto, 63));
        above = below;
    }
    return false;
}
// Item number `index`, or (BY_TILE) the first item of tile number `index` of all sequences.  64 sequences at a time, one a lane.  false:
// there are fewer.
template <bool X_KEYS, bool BY_TILE = false> __device__ __forceinline__ bool find_place(const AttnArgs &a, int index, Place &p)
{
    if (!BY_TILE && a.levels) return find_level<X_KEYS>(a, index, p);
    const int lane = threadIdx.x & 63;
    int items_before = 0;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
        int first = 0, len = 0, other = 0;
        if (b0 + lane < a.B) {
            if (X_KEYS) bounds_of(a.cu_k, a.Tk, b0 + lane, first, len);
            else bounds_of(a.cu_q, a.Tq, b0 + lane, first, len);
            if (a.splits > 1) {
                if (X_KEYS) bounds_of(a.cu_q, a.Tq, b0 + lane, first, other);
                else bounds_of(a.cu_k, a.Tk, b0 + lane, first, other);
            }
        }
        const int tiles = ((X_KEYS ? len : len * a.Gp) + kAttnRows - 1) / kAttnRows;
        const int chunks = (a.splits > 1 ? chunks_in(a, X_KEYS ? other * a.Gp : other) : 1) * a.gsplit;
        const int items = tiles * chunks, mine = BY_TILE ? tiles : items;
        int upto = mine, items_upto = items;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int u = __shfl_up(upto, d), w = BY_TILE ? __shfl_up(items_upto, d) : 0;
            if (lane >= d) upto += u, items_upto += w;
        }
        if (!BY_TILE) items_upto = upto;
        if (!BY_TILE && a.fold && index >= a.fold) {
            const int all = __builtin_amdgcn_readfirstlane(__shfl(upto, 63));
            if (index >= all) return false;
            index = all - 1 - (index - a.fold);
        }
        const uint64_t beyond = __ballot(upto > index);
        if (beyond) {
            const int at = __builtin_ctzll(beyond);
            const int within = __builtin_amdgcn_readfirstlane(index - __shfl(upto - mine, at)), n = __builtin_amdgcn_readfirstlane(__shfl(chunks, at));
            p.b = b0 + at;
            p.t = BY_TILE ? within : within / n;
            p.split = BY_TILE ? 0 : within - p.t * n;
            p.slot = items_before + __builtin_amdgcn_readfirstlane(__shfl(items_upto - items, at)) + p.t * n + p.split;
            if (!X_KEYS) p.t = __builtin_amdgcn_readfirstlane(__shfl(tiles, at)) - 1 - p.t;
            // sequences that overlap, against the rules, may have more items than there is room for
            return !BY_TILE || p.slot + n <= a.tiles * a.splits * a.gsplit;
        }
        index -= __builtin_amdgcn_readfirstlane(__shfl(upto, 63));
        items_before += __builtin_amdgcn_readfirstlane(__shfl(items_upto, 63));
    }
    p.slot = items_before;       // how many there are
    return false;
}
__device__ __forceinline__ Seq seq_of(const AttnArgs &a, int b)
{
    Seq s;
    s.b = b;
    bounds_of(a.cu_q, a.Tq, b, s.q0, s.n);
    bounds_of(a.cu_k, a.Tk, b, s.k0, s.m);
    return s;
}

// Rows of one operand of one problem: row r of the sequence lies at base + (r / Gp) tok + (r % Gp) head.
template <class T> struct Rows {
    const T *base;
    int64_t tok, head;
    int count, D;               // rows there are
    FastDiv by;                 // d = 1: rows are tokens
    __device__ __forceinline__ const T *at(int r) const
    {
        if (by.d == 1) return base + (int64_t)r * tok;
        const int t = (int)fdiv((uint32_t)r, by);
        return base + (int64_t)t * tok + (int64_t)(r - t * (int)by.d) * head;
    }
    __device__ __forceinline__ Raw8<T> load(int r, int d) const
    {
        const int n = r < count ? D - d : 0;
        return load8(n > 0 ? at(r) + d : base, n);
    }
};

// A tile of Y on its way into one of two LDS buffers while the tile before it is multiplied in the other.
//  start(row0, lds): the loads leave.  finish(lds): after the multiplications, before the barrier.
// DMA: from memory to LDS without registers (bf16, 16-byte aligned rows; attn_dma_ok).  The buffer's base moves with the
// tile, so a lane's offsets stay the same for all tiles and 32 bits wide whatever the length of a sequence; what lies behind the
// last row is out of the buffer's range and arrives as zeros, as do the columns D .. DP - 1.
// Otherwise: through registers, at any alignment, cut in pieces (fp32) on the way.
template <class T, int DP, int ROWS, bool DMA> struct Loader;

template <class T, int DP, int ROWS> struct Loader<T, DP, ROWS, false> {
    static constexpr int NP = Pieces<T>::N, CH = DP / 8, N = (ROWS * CH + 255) / 256;
    Rows<T> src;
    Raw8<T> r[N];
    __device__ __forceinline__ Loader(const Rows<T> &s) : src(s) {}
    __device__ __forceinline__ void start(int row0, LdsByte *)
    {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int i = threadIdx.x + j * 256;
            r[j] = src.load(row0 + i / CH, 8 * (i % CH));
        }
    }
    __device__ __forceinline__ void finish(LdsByte *t) const
    {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int i = threadIdx.x + j * 256;
            if (ROWS * CH % 256 == 0 || i < ROWS * CH) Tile<DP, ROWS, NP>::put(t, i / CH, i % CH, frag_of(r[j]));
        }
    }
};

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

template <int DP, int ROWS> struct Loader<bf16raw, DP, ROWS, true> {
    static constexpr int LOADS = ROWS * DP * 2 / 1024, N = (LOADS + 3) / 4;      // of 64 x 16 bytes; four waves share them
    const bf16raw *base;
    int64_t tok;
    int shift, tokens;      // a token's rows: a power of two
    uint32_t tail;          // bytes of the last token's rows
    uint32_t voff[N];
    __device__ __forceinline__ Loader(const Rows<bf16raw> &s) : base(s.base), tok(s.tok)
    {
        const int gp = (int)s.by.d;
        shift = __builtin_ctz(gp);
        tokens = s.count >> shift;
        const int lane = threadIdx.x & 63, wave = (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        tail = (uint32_t)(((gp - 1) * s.head + s.D) * 2);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int at = (4 * j + wave) * 1024 + lane * 16, row = at / (DP * 2), chunk = at % (DP * 2) / 16 ^ swizzle<DP>(row);
            const int t = row >> shift;
            voff[j] = 8 * chunk < s.D ? (uint32_t)((t * s.tok + (row - (t << shift)) * s.head) * 2 + chunk * 16) : OOB_ROW;
        }
    }
    __device__ __forceinline__ void start(int row0, LdsByte *lds) const
    {
        const int t0 = row0 >> shift, left = tokens - t0;      // a tile begins with a token
        const uint64_t at = (uint64_t)reinterpret_cast<uintptr_t>(base) + (uint64_t)((int64_t)t0 * tok * 2);
        const uint64_t span = left > 0 ? (uint64_t)(left - 1) * (uint64_t)tok * 2 + tail : 0;
        const BufferRsrc r = raw_buffer(at, span);
        const int wave = (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (LOADS % 4 == 0 || 4 * j + wave < LOADS) dma16(r, lds + (4 * j + wave) * 1024, voff[j]);
    }
    __device__ __forceinline__ void finish(LdsByte *) const {}
};

// fp32 with rows of whole 16 bytes: through registers, by loads from such a moving buffer, which need no bounds checks.
template <int DP, int ROWS> struct Loader<float, DP, ROWS, true> {
    static constexpr int CH = DP / 8, N = (ROWS * CH + 255) / 256;
    const float *base;
    int64_t tok;
    int shift, tokens;
    uint32_t tail;
    uint32_t voff[N][2];
    u32x4 r[N][2];
    __device__ __forceinline__ Loader(const Rows<float> &s) : base(s.base), tok(s.tok)
    {
        const int gp = (int)s.by.d;
        shift = __builtin_ctz(gp);
        tokens = s.count >> shift;
        tail = (uint32_t)(((gp - 1) * s.head + s.D) * 4);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int i = threadIdx.x + j * 256, row = i / CH, d = 8 * (i % CH), t = row >> shift;
#pragma unroll
            for (int h = 0; h < 2; ++h)
                voff[j][h] = row < ROWS && d + 4 * h < s.D ? (uint32_t)((t * s.tok + (row - (t << shift)) * s.head + d + 4 * h) * 4) : OOB_ROW;
        }
    }
    __device__ __forceinline__ void start(int row0, LdsByte *)
    {
        const int t0 = row0 >> shift, left = tokens - t0;
        const uint64_t at = (uint64_t)reinterpret_cast<uintptr_t>(base) + (uint64_t)((int64_t)t0 * tok * 4);
        const uint64_t span = left > 0 ? (uint64_t)(left - 1) * (uint64_t)tok * 4 + tail : 0;
        const uint64_t u = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)at) | (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(at >> 32)) << 32;
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void *>((uintptr_t)u), 0,
                                                            (int)__builtin_amdgcn_readfirstlane((uint32_t)(span < kMaxBufferBytes ? span : kMaxBufferBytes)), 0x00020000);
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h) r[j][h] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, voff[j][h], 0, 0));
    }
    __device__ __forceinline__ void finish(LdsByte *t) const
    {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int i = threadIdx.x + j * 256;
            float f[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = __uint_as_float(r[j][e / 4][e % 4]);
            if (ROWS * CH % 256 == 0 || i < ROWS * CH) Tile<DP, ROWS, 3>::put(t, i / CH, i % CH, cut8<3>(f));
        }
    }
};

// Between tiles: this wave's loads into LDS have landed, and everyone's.
__device__ __forceinline__ void tile_sync()
{
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

// Over a lane and lane ^ 32, which hold the two halves of an X row's scores.
__device__ __forceinline__ float max_halves(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_halves(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// The fragments are there from here on.  Without it the compiler waits for them at their first use, inside the loop over tiles, and
// with them, in every turn, for the tile that has just been asked for.
template <int NP, int N> __device__ __forceinline__ void arrived(Frag<NP> (&f)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int k = 0; k < NP; ++k) asm volatile("" : "+v"(f[i].p[k]));
}
__device__ __forceinline__ void arrived(float &x) { asm volatile("" : "+v"(x)); }

// 32 dt + 8 j + 4 (lane / 32) ..: four neighbouring columns of an X row
template <class T> __device__ __forceinline__ void store4(T *p, const float (&f)[4], int n)
{
    if (n >= 4) {
        if constexpr (sizeof(T) == 4) {
            Loose16<T> q;
#pragma unroll
            for (int i = 0; i < 4; ++i) q.w[i] = __float_as_uint(f[i]);
            *reinterpret_cast<Loose16<T> *>(p) = q;
        } else {
            struct __attribute__((packed, aligned(2))) Loose8 { uint32_t w[2]; } q = {{pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3])}};
            *reinterpret_cast<Loose8 *>(p) = q;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) p[i] = from_f32<T>(f[i]);
    }
}

// The order of a stretch of code without branches: `ahead` LDS reads first, then one more (two for transposing reads) behind each
// of N matrix instructions.  Left to itself the compiler reads one or two operands ahead, and an LDS read takes as long as
// four matrix instructions and more.
template <int N, int AHEAD, int EACH> __device__ __forceinline__ void reads_ahead()
{
    __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
    static_for<0, N>([](auto) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, EACH, 0);
    });
}

// What o loses when it is rounded to bf16, in the 16 bits an element of o_rest has: a whole number of 2^-16 of o's last place, which
// makes 24 bits of o together (a second bf16 number would make 17, and delta, a sum of o times do, is taken from others nearly
// as large in the gradient of the bias).
__device__ __forceinline__ uint32_t rest_exponent(float o) { return min(max(__float_as_uint(o) & 0x7f800000u, 0x20000000u), 0x7e800000u); }
__device__ __forceinline__ float with_rest(float o, uint32_t rest) { return fmaf((float)(int16_t)rest * 0x1p-23f, __uint_as_float(rest_exponent(o)), o); }
// of four neighbouring elements of an X row, stored like o's
__device__ __forceinline__ void store_rest4(bf16raw *p, const float (&f)[4], int n)
{
    uint32_t r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float o = to_f32(from_f32<bf16raw>(f[i]));
        r[i] = (uint32_t)(int)fminf(rintf((f[i] - o) * __uint_as_float(0x7f000000u - rest_exponent(o)) * 0x1p23f), 32767.f) & 0xffffu;
    }
    if (n >= 4) {
        struct __attribute__((packed, aligned(2))) Loose8 { uint32_t w[2]; } q = {{r[0] | r[1] << 16, r[2] | r[3] << 16}};
        *reinterpret_cast<Loose8 *>(p) = q;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) p[i] = (bf16raw)r[i];
    }
}

// An X row's accumulators, times `factor`, to a row of T: four neighbouring columns at a time.
template <class T, int DT> __device__ __forceinline__ void store_row(T *to, const v16f (&acc)[DT], float factor, int D, int h32)
{
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int d = 32 * dt + 8 * j + 4 * h32;
            const float f[4] = {acc[dt][4 * j] * factor, acc[dt][4 * j + 1] * factor, acc[dt][4 * j + 2] * factor, acc[dt][4 * j + 3] * factor};
            store4(to + d, f, D - d);
        }
}

// Chunks that Y rows [begin, end) of a tile are cut into (at least one, which may be empty).
__device__ __forceinline__ int chunks_of(const AttnArgs &a, int begin, int end)
{
    return a.splits == 1 ? 1 : chunks_in(a, end - begin);
}
// What the rows of a tile see, row0 .. of `rows`: keys 0 .. the return value - 1.
__device__ __forceinline__ int keys_seen(const AttnArgs &a, const Seq &s, int row_end, int rows)
{
    const int last = (int)fdiv((uint32_t)(min(max(row_end, 1), rows) - 1), a.by_gp);
    return a.causal ? min(max(last + 1 + s.m - s.n, 0), s.m) : s.m;
}
// The first row, of Gp to a token, that sees key k.
__device__ __forceinline__ int first_seeing(const AttnArgs &a, const Seq &s, int k)
{
    return a.causal ? (int)min(max((int64_t)(k - (s.m - s.n)) * a.Gp, (int64_t)0), (int64_t)s.n * a.Gp) : 0;
}

// The bias of a tile: entry e is that of delta = first + e, clamped to the table.  At most 256 entries, one a thread.
__device__ __forceinline__ float window_load(const AttnArgs &a, int h, int first)
{
    return a.btab[(int64_t)h * (2 * a.W + 1) + a.W + min(max(first + (int)threadIdx.x, -a.W), a.W)];
}

// Where the items come by length (`gains`).  What the rounds' end saves, the sequences lose that no longer follow one another in L2:
// with two waves a SIMD it pays for kernels with a bias (4 x 2048, 16 heads of 64, both causal: forward 130 -> 109 us, dk/dv 124 -> 109) and
// for those without loads into LDS (the same of 100: forward 305 -> 250), and for the forward kernel of narrow heads (4 x 4096, 16 of 64: 211
// -> 193); the others, which the chip's power holds back, lose up to 4 %.
inline int levels_of(const AttnArgs &a, int problems, bool gains)
{
    return gains && a.causal && a.splits == 1 && a.gsplit == 1 && a.B > 1 && a.B <= 64 && (int64_t)problems * a.tiles > kFoldMost;
}
// Where the order of a launch's items is turned round: if all blocks are resident at once, two a compute unit (block i and block i + 256,
// as measured), the second ones would else meet first ones with as much work, a causal mask's long tiles twice in one place: dk/dv of
// 4 x 2048, 32 heads on 8, 128 wide, 502 -> 446 us.
inline int fold_of(const AttnArgs &a, int problems, int waves)
{
    const int64_t blocks = (int64_t)problems * a.tiles * a.gsplit;
    return waves == 2 && a.splits == 1 && a.B <= 64 && blocks > kUnits && blocks <= kFoldMost ? (kUnits + problems - 1) / problems : 0;
}

}  // namespace
}  // namespace cg
