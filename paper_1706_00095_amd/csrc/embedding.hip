// Embedding: rows of a table by token, scaled, and the gradient of the table by sorted tokens.
//
// The gradient is dense (the update takes whole buckets): row v is the sum of dy over the places that hold v, zero where there are none.
// Places are sorted by token, stably, so that each row's sum is taken in the order of the places and results are the same bits run to
// run.  A token that is frequent has thousands of places: the sorted places are cut into chunks, chunks of one token alone are summed by
// blocks of their own, and the row adds what they leave.  Every row of the gradient is then written once.
#include <algorithm>
#include "cg_internal.h"
#include "row_checks.h"
#include "typed_device.h"

namespace cg {
namespace {

// ---- lookup ---------------------------------------------------------------------------------------------------------------------
struct LookupArgs {
    const int32_t *tokens;
    const void *table;
    void *y;
    int64_t table_ld, y_ld;
    int vocab, cols;
    uint32_t count;
    FastDiv by_chunks;
    float scale;
};
// A thread takes eight neighbours of a row.  Bound by HBM.
template <class TT, class T> __global__ __launch_bounds__(256) void lookup_kernel(LookupArgs a)
{
    for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < a.count; i += gridDim.x * 256) {
        const int64_t t = fdiv(i, a.by_chunks);
        const int c = 8 * (int)(i - (uint32_t)t * a.by_chunks.d), n = a.cols - c;
        const int v = a.tokens[t];
        float f[8] = {};
        if ((uint32_t)v < (uint32_t)a.vocab) {
            const Raw8<TT> x = load8(static_cast<const TT *>(a.table) + v * a.table_ld + c, n);
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = elem(x, j) * a.scale;
        }
        store8(static_cast<T *>(a.y) + t * a.y_ld + c, to_raw<T>(f), n);
    }
}

// ---- places sorted by token --------------------------------------------------------------------------------------------------------
// Least significant digit first, stably.  A wave numbers 64 places at a time: those with its digit among the lanes before it, and
// those the wave has had before (counted in LDS).  Places without a token have the key `vocab` and come last.
constexpr int kItems = 16;                  // of a lane
constexpr int kDigits = 256;
constexpr int kOneBlock = 1024, kTileBlock = 256, kTile = kTileBlock * kItems;       // threads; places of a block where there are several
constexpr int kMostOne = kOneBlock * kItems;

__device__ __forceinline__ uint32_t key_of(const int32_t *tokens, int i, int n, int vocab)
{
    if (i >= n) return 0xffffffffu;         // behind everything
    const uint32_t v = (uint32_t)tokens[i];
    return v < (uint32_t)vocab ? v : (uint32_t)vocab;
}
// Numbers this wave's items by digit: rank[j] among the wave's of the same digit; counts[] (of the wave, zeroed) ends with their numbers.
__device__ __forceinline__ void number_items(const uint32_t (&key)[kItems], int items, int shift, int bits, uint32_t *counts, uint32_t (&rank)[kItems])
{
    const int lane = threadIdx.x & 63;
    const uint64_t below = ((uint64_t)1 << lane) - 1;
#pragma unroll
    for (int j = 0; j < kItems; ++j) {
        if (j < items) {
            const uint32_t d = key[j] >> shift & ((1u << bits) - 1);
            uint64_t same = ~(uint64_t)0;
            for (int b = 0; b < bits; ++b) {
                const uint64_t m = __ballot(d >> b & 1);
                same &= d >> b & 1 ? m : ~m;
            }
            const uint32_t before = counts[d];
            __builtin_amdgcn_wave_barrier();
            if ((same & below) == 0) counts[d] = before + (uint32_t)__popcll(same);
            __builtin_amdgcn_wave_barrier();
            rank[j] = before + (uint32_t)__popcll(same & below);
        }
    }
}
// Exclusive sums over a block's threads; `lds`: one word a wave, free for use.
template <int THREADS> __device__ __forceinline__ uint32_t block_before(uint32_t x, uint32_t *lds)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t upto = x;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t u = (uint32_t)__shfl_up((int)upto, d);
        if (lane >= d) upto += u;
    }
    if (lane == 63) lds[wave] = upto;
    __syncthreads();
    uint32_t before = 0;
    for (int w = 0; w < wave; ++w) before += lds[w];
    __syncthreads();
    return before + upto - x;
}

struct SortArgs {
    const int32_t *tokens;                   // NULL: keys and places as they lie in key_in, place_in
    const uint32_t *key_in, *place_in;
    uint32_t *key, *place;
    uint32_t *counts;                        // [kDigits][tiles]
    int n, vocab, shift, bits, tiles;
};

// All of up to kMostOne places by one block, the items going through LDS between passes.
__global__ __launch_bounds__(kOneBlock) void sort_one_kernel(const int32_t *tokens, int n, int vocab, int passes, int bits, uint32_t *keys, uint32_t *places)
{
    constexpr int W = kOneBlock / 64;
    extern __shared__ __align__(16) uint32_t smem[];
    uint32_t *const counts = smem, *const sums = counts + W * kDigits, *const ex_key = sums + W;      // counts [W][kDigits]
    uint16_t *const ex_place = reinterpret_cast<uint16_t *>(ex_key + kMostOne);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, items = (n + kOneBlock - 1) / kOneBlock, at = wave * items * 64 + lane;
    uint32_t key[kItems], place[kItems], rank[kItems];
#pragma unroll
    for (int j = 0; j < kItems; ++j) {
        if (j < items) {
            place[j] = (uint32_t)(at + 64 * j);
            key[j] = key_of(tokens, at + 64 * j, n, vocab);
        }
    }
    for (int p = 0; p < passes; ++p) {
        for (int i = threadIdx.x; i < W * kDigits; i += kOneBlock) counts[i] = 0;
        __syncthreads();
        number_items(key, items, p * bits, bits, counts + wave * kDigits, rank);
        __syncthreads();
        // in the order of digits, then waves: thread t has digit t / 4 of four waves
        const int d = threadIdx.x >> 2, w0 = 4 * (threadIdx.x & 3);
        uint32_t c[4], sum = 0;
#pragma unroll
        for (int u = 0; u < 4; ++u) c[u] = counts[(w0 + u) * kDigits + d], sum += c[u];
        uint32_t before = block_before<kOneBlock>(sum, sums);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            counts[(w0 + u) * kDigits + d] = before;
            before += c[u];
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kItems; ++j) {
            if (j < items) {
                const uint32_t to = counts[wave * kDigits + (key[j] >> (p * bits) & ((1u << bits) - 1))] + rank[j];
                ex_key[to] = key[j];
                ex_place[to] = (uint16_t)place[j];
            }
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kItems; ++j) {
            if (j < items) {
                key[j] = ex_key[at + 64 * j];
                place[j] = ex_place[at + 64 * j];
            }
        }
    }
#pragma unroll
    for (int j = 0; j < kItems; ++j) {
        if (j < items && at + 64 * j < n) keys[at + 64 * j] = key[j], places[at + 64 * j] = place[j];
    }
}
constexpr int kOneLds = (kOneBlock / 64 * kDigits + kOneBlock / 64 + kMostOne) * 4 + kMostOne * 2;

// Several blocks, a pass in three launches: how often each digit occurs in each tile, sums before in the order of digits, then tiles, and
// the items to their places.
__device__ __forceinline__ void load_items(const SortArgs &a, uint32_t (&key)[kItems], uint32_t (&place)[kItems])
{
    const int at = blockIdx.x * kTile + (threadIdx.x >> 6) * kItems * 64 + (threadIdx.x & 63);
#pragma unroll
    for (int j = 0; j < kItems; ++j) {
        const int i = at + 64 * j;
        place[j] = a.tokens || i >= a.n ? (uint32_t)i : a.place_in[i];
        key[j] = a.tokens ? key_of(a.tokens, i, a.n, a.vocab) : i < a.n ? a.key_in[i] : 0xffffffffu;
    }
}
__global__ __launch_bounds__(kTileBlock) void sort_count_kernel(SortArgs a)
{
    __shared__ uint32_t counts[kDigits];
    counts[threadIdx.x] = 0;
    __syncthreads();
    uint32_t key[kItems], place[kItems];
    load_items(a, key, place);
#pragma unroll
    for (int j = 0; j < kItems; ++j) atomicAdd(&counts[key[j] >> a.shift & ((1u << a.bits) - 1)], 1u);       // whole numbers: in any order
    __syncthreads();
    a.counts[threadIdx.x * a.tiles + blockIdx.x] = counts[threadIdx.x];
}
__global__ __launch_bounds__(1024) void sort_sums_kernel(uint32_t *counts, int n)
{
    __shared__ uint32_t sums[16], total;
    uint32_t carry = 0;
    for (int i0 = 0; i0 < n; i0 += 4096) {
        uint32_t c[4], sum = 0;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int i = i0 + 4 * threadIdx.x + u;
            c[u] = i < n ? counts[i] : 0, sum += c[u];
        }
        uint32_t before = carry + block_before<1024>(sum, sums);
        if (threadIdx.x == 1023) total = before + sum;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int i = i0 + 4 * threadIdx.x + u;
            if (i < n) counts[i] = before;
            before += c[u];
        }
        __syncthreads();
        carry = total;
        __syncthreads();
    }
}
__global__ __launch_bounds__(kTileBlock) void sort_move_kernel(SortArgs a)
{
    constexpr int W = kTileBlock / 64;
    __shared__ uint32_t counts[W][kDigits];
    const int wave = threadIdx.x >> 6;
#pragma unroll
    for (int w = 0; w < W; ++w) counts[w][threadIdx.x] = 0;
    uint32_t key[kItems], place[kItems], rank[kItems];
    load_items(a, key, place);
    __syncthreads();
    number_items(key, kItems, a.shift, a.bits, counts[wave], rank);
    __syncthreads();
    uint32_t before = a.counts[threadIdx.x * a.tiles + blockIdx.x];
#pragma unroll
    for (int w = 0; w < W; ++w) {
        const uint32_t c = counts[w][threadIdx.x];
        counts[w][threadIdx.x] = before;
        before += c;
    }
    __syncthreads();
    // what lies behind the last place has the largest key in every digit and comes last in the last tile
#pragma unroll
    for (int j = 0; j < kItems; ++j) {
        const uint32_t to = counts[wave][key[j] >> a.shift & ((1u << a.bits) - 1)] + rank[j];
        if (to < (uint32_t)a.n && key[j] != 0xffffffffu) a.key[to] = key[j], a.place[to] = place[j];
    }
}

// ---- sums --------------------------------------------------------------------------------------------------------------------------
struct GradArgs {
    const uint32_t *key, *place;
    const void *dy;
    float *part;                             // [chunks][cols]
    uint32_t *first;                         // [vocab + 1]: where each token's places begin
    float *dtable;
    int64_t dy_ld;
    int n, vocab, cols, chunk, chunk_shift;
    float scale;
};
constexpr int kGradThreads = 64;

template <class T> __device__ __forceinline__ void add_places(const GradArgs &a, int from, int to, int c, float (&v)[8])
{
    constexpr int AHEAD = 8;
    const int n = a.cols - c;
    for (int i = from; i < to; i += AHEAD) {
        Raw8<T> x[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
            x[u] = load8(static_cast<const T *>(a.dy) + (int64_t)a.place[min(i + u, to - 1)] * a.dy_ld + c, i + u < to ? n : 0);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += elem(x[u], j);
    }
}
// Blocks 0 .. bounds - 1: where each token's places begin, by halving, a thread a token.  The others: chunks of one token alone.
template <class T> __global__ __launch_bounds__(kGradThreads) void chunk_sums_kernel(GradArgs a, int bounds, int per_chunk)
{
    if ((int)blockIdx.x < bounds) {
        for (int v = blockIdx.x * kGradThreads + threadIdx.x; v <= a.vocab; v += bounds * kGradThreads) {
            int lo = 0, hi = a.n;
            while (lo < hi) {
                const int m = lo + (hi - lo) / 2;
                if (a.key[m] < (uint32_t)v) lo = m + 1;
                else hi = m;
            }
            a.first[v] = (uint32_t)lo;
        }
        return;
    }
    const int b = (int)blockIdx.x - bounds, chunk = b / per_chunk, c = (b - chunk * per_chunk) * kGradThreads * 8 + 8 * threadIdx.x;
    const int from = chunk << a.chunk_shift, to = from + a.chunk;       // whole chunks only
    if (c >= a.cols || a.key[from] != a.key[to - 1] || a.key[from] >= (uint32_t)a.vocab) return;
    float v[8] = {};
    add_places<T>(a, from, to, c, v);
    store8(a.part + (int64_t)chunk * a.cols + c, to_raw<float>(v), a.cols - c);
}
// LANES lanes a row, eight columns each at a time.  Bound by writing the table's gradient.
template <class T, int LANES> __global__ __launch_bounds__(256) void rows_kernel(GradArgs a)
{
    constexpr int ROWS = 256 / LANES;
    const int lane = threadIdx.x % LANES;
    for (int64_t r = (int64_t)blockIdx.x * ROWS + threadIdx.x / LANES; r < a.vocab; r += (int64_t)gridDim.x * ROWS) {
        const int from = (int)a.first[r], to = (int)a.first[r + 1];
        // whole chunks among the row's places
        const int c0 = (int)(((uint32_t)from + a.chunk - 1) >> a.chunk_shift), c1 = to >> a.chunk_shift;
        for (int c = 8 * lane; c < a.cols; c += 8 * LANES) {
            float v[8] = {};
            if (c0 >= c1) add_places<T>(a, from, to, c, v);
            else {
                add_places<T>(a, from, c0 << a.chunk_shift, c, v);
                const float *p = a.part + (int64_t)c0 * a.cols + c;
                for (int k = c0; k < c1; k += 4, p += 4 * (int64_t)a.cols) {
                    Raw8<float> x[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) x[u] = load8(k + u < c1 ? p + u * (int64_t)a.cols : p, k + u < c1 ? a.cols - c : 0);
#pragma unroll
                    for (int u = 0; u < 4; ++u)
#pragma unroll
                        for (int j = 0; j < 8; ++j) v[j] += elem(x[u], j);
                }
                add_places<T>(a, c1 << a.chunk_shift, to, c, v);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= a.scale;
            store8(a.dtable + r * a.cols + c, to_raw<float>(v), a.cols - c);
        }
    }
}

// ---- host side ------------------------------------------------------------------------------------------------------------------------
int desc_check(const cg_embedding_desc *d)
{
    if (!d || !type_ok(d->table_type) || !type_ok(d->type) || d->vocab < 1 || d->cols < 1 || d->tokens < 0) return CG_EINVAL;
    const int64_t most = INT32_MAX - 65535, chunks = (d->cols + 7) / 8;
    if (d->vocab > most || d->cols > most || d->tokens > (1 << 28) || d->tokens * chunks > INT32_MAX / 2) return CG_EUNSUPPORTED;
    return CG_OK;
}
int chunk_shift_of(int64_t tokens) { return tokens <= 1 << 16 ? 5 : tokens <= 1 << 20 ? 7 : 9; }
size_t round16(size_t n) { return (n + 15) & ~(size_t)15; }
struct Layout {
    size_t key[2], place[2], counts, first, part, total;
    int tiles;                // 0: one block
};
Layout layout_of(const cg_embedding_desc *d)
{
    Layout l{};
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t p = at; at += round16(bytes); return p; };
    const size_t n = (size_t)d->tokens;
    l.tiles = n <= (size_t)kMostOne ? 0 : (int)((n + kTile - 1) / kTile);
    for (int i = 0; i < (l.tiles ? 2 : 1); ++i) l.key[i] = take(4 * n), l.place[i] = take(4 * n);
    l.counts = take(l.tiles ? sizeof(uint32_t) * kDigits * (size_t)l.tiles : 0);
    l.first = take(4 * ((size_t)d->vocab + 1));
    l.part = take(4 * (n >> chunk_shift_of(d->tokens)) * (size_t)d->cols);
    l.total = at;
    return l;
}

template <class TT> int lookup_typed(const LookupArgs &a, int type, dim3 grid, hipStream_t s)
{
    if (type == CG_TYPE_FP32) hipLaunchKernelGGL((lookup_kernel<TT, float>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((lookup_kernel<TT, bf16raw>), grid, dim3(256), 0, s, a);
    CG_HIP_TRY(hipGetLastError());
    return CG_OK;
}
template <class T, int LANES> void rows_launch(const GradArgs &a, hipStream_t s)
{
    const int64_t b = ((int64_t)a.vocab + 256 / LANES - 1) / (256 / LANES);
    hipLaunchKernelGGL((rows_kernel<T, LANES>), dim3((unsigned)(b < 65536 ? b : 65536)), dim3(256), 0, s, a);
}
template <class T> int grad_typed(const GradArgs &a, hipStream_t s)
{
    const int per = (a.cols + kGradThreads * 8 - 1) / (kGradThreads * 8), bounds = (int)std::min<int64_t>(((int64_t)a.vocab + kGradThreads) / kGradThreads, 4096);
    hipLaunchKernelGGL((chunk_sums_kernel<T>), dim3((unsigned)(bounds + (a.n >> a.chunk_shift) * per)), dim3(kGradThreads), 0, s, a, bounds, per);
    CG_HIP_TRY(hipGetLastError());
    if (a.cols <= 32) rows_launch<T, 4>(a, s);
    else if (a.cols <= 128) rows_launch<T, 16>(a, s);
    else if (a.cols <= 512) rows_launch<T, 64>(a, s);
    else rows_launch<T, 128>(a, s);
    CG_HIP_TRY(hipGetLastError());
    return CG_OK;
}

}  // namespace
}  // namespace cg

using namespace cg;

extern "C" int cg_embedding_fwd(const cg_embedding_desc *d, const int32_t *tokens, const void *table, int64_t table_ld, void *y, int64_t y_ld, void *stream)
{
    if (int rc = desc_check(d)) return rc;
    if (d->tokens == 0) return CG_OK;
    if (!floats_ok(tokens) || !tensor_ok(table, table_ld, d->cols, d->table_type) || !tensor_ok(y, y_ld, d->cols, d->type)) return CG_EINVAL;
    LookupArgs a{};
    a.tokens = tokens, a.table = table, a.y = y, a.table_ld = table_ld, a.y_ld = y_ld;
    a.vocab = (int)d->vocab, a.cols = (int)d->cols, a.scale = d->scale;
    const uint32_t chunks = (uint32_t)((d->cols + 7) / 8);
    a.count = (uint32_t)d->tokens * chunks;
    a.by_chunks = make_fastdiv(chunks);
    const uint32_t b = (a.count + 255) / 256;
    const dim3 grid(b < 8192 ? b : 8192);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    return d->table_type == CG_TYPE_FP32 ? lookup_typed<float>(a, d->type, grid, s) : lookup_typed<bf16raw>(a, d->type, grid, s);
}

extern "C" size_t cg_embedding_workspace_bytes(const cg_embedding_desc *d) { return desc_check(d) == CG_OK ? layout_of(d).total : 0; }

extern "C" int cg_embedding_bwd(const cg_embedding_desc *d, const int32_t *tokens, const void *dy, int64_t dy_ld, float *dtable, void *ws, size_t ws_bytes, void *stream)
{
    if (int rc = desc_check(d)) return rc;
    if (!floats_ok(dtable) || (d->tokens > 0 && (!floats_ok(tokens) || !tensor_ok(dy, dy_ld, d->cols, d->type)))) return CG_EINVAL;
    const Layout l = layout_of(d);
    if (!ws || !aligned16(ws)) return CG_EINVAL;
    if (ws_bytes < l.total) return CG_ENOSPC;
    char *const base = static_cast<char *>(ws);
    auto words = [&](size_t at) { return reinterpret_cast<uint32_t *>(base + at); };
    const hipStream_t s = static_cast<hipStream_t>(stream);
    int bits = 1;
    while (d->vocab >> bits) ++bits;           // keys are at most vocab
    const int passes = (bits + 7) / 8, per = (bits + passes - 1) / passes, n = (int)d->tokens;
    int last = 0;
    if (n > 0 && l.tiles == 0) {
        CG_HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void *>(&sort_one_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kOneLds));
        hipLaunchKernelGGL(sort_one_kernel, dim3(1), dim3(kOneBlock), kOneLds, s, tokens, n, (int)d->vocab, passes, per, words(l.key[0]), words(l.place[0]));
        CG_HIP_TRY(hipGetLastError());
    } else if (n > 0) {
        for (int p = 0; p < passes; ++p) {
            last = p & 1;
            SortArgs a{};
            a.tokens = p == 0 ? tokens : nullptr;
            a.key_in = words(l.key[1 - last]), a.place_in = words(l.place[1 - last]), a.key = words(l.key[last]), a.place = words(l.place[last]);
            a.counts = words(l.counts), a.n = n, a.vocab = (int)d->vocab, a.shift = p * per, a.bits = per, a.tiles = l.tiles;
            hipLaunchKernelGGL(sort_count_kernel, dim3((unsigned)l.tiles), dim3(kTileBlock), 0, s, a);
            hipLaunchKernelGGL(sort_sums_kernel, dim3(1), dim3(1024), 0, s, a.counts, kDigits * l.tiles);
            hipLaunchKernelGGL(sort_move_kernel, dim3((unsigned)l.tiles), dim3(kTileBlock), 0, s, a);
            CG_HIP_TRY(hipGetLastError());
        }
    }
    GradArgs g{};
    g.key = words(l.key[last]), g.place = words(l.place[last]), g.dy = dy, g.dy_ld = dy_ld, g.part = reinterpret_cast<float *>(base + l.part);
    g.first = words(l.first), g.dtable = dtable, g.n = n, g.vocab = (int)d->vocab, g.cols = (int)d->cols, g.scale = d->scale;
    g.chunk_shift = chunk_shift_of(d->tokens), g.chunk = 1 << g.chunk_shift;
    return d->type == CG_TYPE_FP32 ? grad_typed<float>(g, s) : grad_typed<bf16raw>(g, s);
}
