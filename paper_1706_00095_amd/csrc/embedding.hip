// Embedding: rows of a table by token, scaled, and the gradient of the table by sorted tokens.
//
// The gradient is dense (the update takes whole buckets): row v is the sum of dy over the places that hold v, zero where there are none.
// Places are sorted by token, stably, so that each row's sum is taken in the order of the places and results are the same bits run to
// run.  A token that is frequent has thousands of places: the sorted places are cut into chunks, a wave each, and what runs that cross a
// border leave in their chunks is added by a second kernel, stretches of chunks first and then these, all of them in order.  The table's gradient is filled with zeros by blocks beside those that sort,
// and the rows of tokens that occur are written over.
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
// A thread takes eight neighbours of a row, AHEAD of them at a time: their tokens are asked for together, then their rows.
template <class TT, class T, int AHEAD> __global__ __launch_bounds__(256) void lookup_kernel(LookupArgs a)
{
    const uint32_t step = gridDim.x * 256;
    for (uint32_t i0 = blockIdx.x * 256 + threadIdx.x; i0 < a.count; i0 += AHEAD * step) {
        int t[AHEAD], c[AHEAD], v[AHEAD];
        Raw8<TT> x[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const uint32_t i = min(i0 + u * step, a.count - 1);       // the last one several times, the same
            t[u] = (int)fdiv(i, a.by_chunks);
            c[u] = 8 * (int)(i - (uint32_t)t[u] * a.by_chunks.d);
            v[u] = a.tokens[t[u]];
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const bool some = (uint32_t)v[u] < (uint32_t)a.vocab;
            x[u] = load8(static_cast<const TT *>(a.table) + (some ? v[u] : 0) * a.table_ld + c[u], a.cols - c[u]);
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const float scale = a.scale;
            const bool some = (uint32_t)v[u] < (uint32_t)a.vocab;
            float f[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = some ? elem(x[u], j) * scale : 0.f;
            store8(static_cast<T *>(a.y) + (int64_t)t[u] * a.y_ld + c[u], to_raw<T>(f), a.cols - c[u]);
        }
    }
}

// ---- places sorted by token --------------------------------------------------------------------------------------------------------
// Least significant digit first, stably.  A wave numbers 64 places at a time: those with its digit among the lanes before it, and
// those the wave has had before (counted in LDS).  Places without a token have the key `vocab` and come last.
// A digit has up to 10 bits where a pass is one launch (a table of a million rows takes two passes), up to 8 beyond.  Six at least, so that a block's
// threads share out the waves' counts of all digits in whole lines.
constexpr int kDigits = 256, kMostDigits = 1 << 10, kLeastBits = 6;
constexpr int kOneBlock = 1024, kOneItems = 4, kMostOne = kOneBlock * kOneItems;      // threads, places of a lane, of the block
constexpr int kMostPass = 1 << 16;          // places up to which a pass is one launch
constexpr int kTileBlock = 256, kItems = 16, kTile = kTileBlock * kItems;             // beyond: threads, places of a lane, of a block

__device__ __forceinline__ uint32_t key_of(const int32_t *tokens, int i, int n, int vocab)
{
    if (i >= n) return 0xffffffffu;         // behind everything
    const uint32_t v = (uint32_t)tokens[i];
    return v < (uint32_t)vocab ? v : (uint32_t)vocab;
}
// Numbers this wave's items by digit: rank[j] among the wave's of the same digit; counts[] (of the wave, zeroed) ends with their numbers.
template <int ITEMS> __device__ __forceinline__ void number_items(const uint32_t (&key)[ITEMS], int items, int shift, int bits, uint32_t *counts, uint32_t (&rank)[ITEMS])
{
    const int lane = threadIdx.x & 63;
    const uint64_t below = ((uint64_t)1 << lane) - 1;
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
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
// Counts of digits with an LDS atomic a place (whole numbers: in any order): in kMostDigits >> bits copies by lane, because places that share a digit wait
// for each other, and few tokens or a frequent one make many of them (60000 places of 2 tokens, 16 columns: 36 us the gradient, 60 in one copy).
__device__ __forceinline__ void count_digit(uint32_t *counts, uint32_t digit, int bits)
{
    const int copies = kMostDigits >> bits;
    atomicAdd(&counts[(digit << (10 - bits)) + (threadIdx.x & (copies - 1))], 1u);
}
__device__ __forceinline__ uint32_t counted(const uint32_t *counts, int digit, int bits)
{
    uint32_t n = 0;
    if (digit < 1 << bits)
        for (int i = 0; i < kMostDigits >> bits; ++i) n += counts[(digit << (10 - bits)) + i];
    return n;
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

// Zeros for `count` floats, by the blocks from `first` on: beside those of a launch that leaves the chip empty, so that sorting costs little.
struct Fill {
    float *to;
    int64_t count;
    int first;
};
__device__ __forceinline__ bool fills(const Fill &f)
{
    if ((int)blockIdx.x < f.first) return false;
    const int64_t step = (int64_t)(gridDim.x - f.first) * blockDim.x * 4;
    for (int64_t i = ((int64_t)(blockIdx.x - f.first) * blockDim.x + threadIdx.x) * 4; i < f.count; i += step) {
        if (i + 4 <= f.count) *reinterpret_cast<Loose16<float> *>(f.to + i) = Loose16<float>{{0, 0, 0, 0}};
        else
            for (int64_t j = i; j < f.count; ++j) f.to[j] = 0.f;
    }
    return true;
}
__global__ __launch_bounds__(1024) void fill_kernel(Fill f) { fills(f); }

struct SortArgs {
    const int32_t *tokens;                   // NULL: keys and places as they lie in key_in, place_in
    const uint32_t *key_in, *place_in;
    uint32_t *key, *place;
    uint32_t *counts;                        // [kDigits][tiles]
    int n, vocab, shift, bits, tiles;
    Fill fill;
};

// What a block of kOneBlock threads counts: counts[wave][digit].  They become where each wave's places of a digit begin: in the order of digits, then
// waves, from `base`[digit] (NULL: from 0 on, all digits one after the other).  Thread t has digit t / E of some waves, E threads a digit.
constexpr int kOneWaves = kOneBlock / 64;
__device__ __forceinline__ void places_of_waves(uint32_t *counts, int bits, const uint32_t *base, uint32_t *sums)
{
    const int digits = 1 << bits, shift = bits < 10 ? 10 - bits : 0, each = kOneWaves >> shift;
    const int d = threadIdx.x >> shift, w0 = (threadIdx.x & ((1 << shift) - 1)) * each;
    uint32_t c[kOneWaves], sum = 0;
#pragma unroll
    for (int u = 0; u < kOneWaves; ++u) {
        c[u] = u < each ? counts[(w0 + u) * digits + d] : 0;
        sum += c[u];
    }
    uint32_t at = block_before<kOneBlock>(sum, sums);
    if (base) {          // what the threads of the same digit before this one have
        const uint32_t first = (uint32_t)__shfl((int)at, (int)((threadIdx.x & 63) >> shift << shift));
        at = at - first + base[d];
    }
#pragma unroll
    for (int u = 0; u < kOneWaves; ++u) {
        if (u < each) counts[(w0 + u) * digits + d] = at;
        at += c[u];
    }
}

// All of up to kMostOne places by one block, the items going through LDS between passes.  16384 places in one block (16 a lane) took 35 us.
__global__ __launch_bounds__(kOneBlock) void sort_one_kernel(SortArgs a, int passes)
{
    if (fills(a.fill)) return;
    __shared__ uint32_t counts[kOneWaves * kMostDigits], sums[kOneWaves], ex_key[kMostOne];
    __shared__ uint16_t ex_place[kMostOne];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, items = (a.n + kOneBlock - 1) / kOneBlock, at = wave * items * 64 + lane, digits = 1 << a.bits;
    const uint32_t mask = (uint32_t)digits - 1;
    uint32_t *const mine = counts + wave * digits;
    uint32_t key[kOneItems], place[kOneItems], rank[kOneItems];
#pragma unroll
    for (int j = 0; j < kOneItems; ++j)
        if (j < items) {
            place[j] = (uint32_t)(at + 64 * j);
            key[j] = key_of(a.tokens, at + 64 * j, a.n, a.vocab);
        }
    for (int p = 0; p < passes; ++p) {
        const int shift = p * a.bits;
        for (int i = threadIdx.x; i < kOneWaves * digits; i += kOneBlock) counts[i] = 0;
        __syncthreads();
        number_items(key, items, shift, a.bits, mine, rank);
        __syncthreads();
        places_of_waves(counts, a.bits, nullptr, sums);
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kOneItems; ++j)
            if (j < items) {
                const uint32_t to = mine[key[j] >> shift & mask] + rank[j];
                ex_key[to] = key[j];
                ex_place[to] = (uint16_t)place[j];
            }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kOneItems; ++j)
            if (j < items) {
                key[j] = ex_key[at + 64 * j];
                place[j] = ex_place[at + 64 * j];
            }
    }
#pragma unroll
    for (int j = 0; j < kOneItems; ++j)
        if (j < items && at + 64 * j < a.n) a.key[at + 64 * j] = key[j], a.place[at + 64 * j] = place[j];
}

// A pass over up to kMostPass places in one launch, a place a thread: every block counts the digits of all places, before its own and from
// there on, so that no other launch has to.
__global__ __launch_bounds__(kOneBlock) void sort_pass_kernel(SortArgs a)
{
    if (fills(a.fill)) return;
    __shared__ uint32_t counts[kOneWaves * kMostDigits], ahead[kMostDigits], rest[kMostDigits], sums[kOneWaves];
    const int wave = threadIdx.x >> 6, own = blockIdx.x * kOneBlock, i = own + threadIdx.x, digits = 1 << a.bits, all = a.tiles * kOneBlock;
    const uint32_t mask = (uint32_t)digits - 1;
    uint32_t *const mine = counts + wave * digits;
    auto key_at = [&](int j) { return a.tokens ? key_of(a.tokens, j, a.n, a.vocab) : j < a.n ? a.key_in[j] : 0xffffffffu; };
    for (int j = threadIdx.x; j < kOneWaves * digits; j += kOneBlock) counts[j] = 0;
    ahead[threadIdx.x] = rest[threadIdx.x] = 0;
    uint32_t key[1] = {key_at(i)}, rank[1];
    const uint32_t place = a.tokens || i >= a.n ? (uint32_t)i : a.place_in[i];
    __syncthreads();
    for (int j0 = threadIdx.x; j0 < all; j0 += 16 * kOneBlock) {
        uint32_t k[16];
#pragma unroll
        for (int u = 0; u < 16; ++u) k[u] = key_at(j0 + u * kOneBlock);
#pragma unroll
        for (int u = 0; u < 16; ++u) {
            const int j = j0 + u * kOneBlock;
            if (j < all) count_digit(j < own ? ahead : rest, k[u] >> a.shift & mask, a.bits);
        }
    }
    number_items(key, 1, a.shift, a.bits, mine, rank);
    __syncthreads();
    const uint32_t earlier = counted(ahead, threadIdx.x, a.bits), before = block_before<kOneBlock>(earlier + counted(rest, threadIdx.x, a.bits), sums);
    rest[threadIdx.x] = before + earlier;
    __syncthreads();
    places_of_waves(counts, a.bits, rest, sums);
    __syncthreads();
    const uint32_t to = mine[key[0] >> a.shift & mask] + rank[0];
    if (i < a.n) a.key[to] = key[0], a.place[to] = place;       // what lies behind the last place comes last
}

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
    if (fills(a.fill)) return;
    __shared__ uint32_t counts[kMostDigits];
#pragma unroll
    for (int j = 0; j < kMostDigits / kTileBlock; ++j) counts[threadIdx.x + j * kTileBlock] = 0;
    __syncthreads();
    uint32_t key[kItems], place[kItems];
    load_items(a, key, place);
#pragma unroll
    for (int j = 0; j < kItems; ++j) count_digit(counts, key[j] >> a.shift & ((1u << a.bits) - 1), a.bits);
    __syncthreads();
    a.counts[threadIdx.x * a.tiles + blockIdx.x] = counted(counts, threadIdx.x, a.bits);
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
    // [chunks][cols]: sums of the run that a chunk begins with, where it began earlier, and of the one that it ends with, where it goes on and
    // began here
    float *head, *tail;
    float *dtable;
    int64_t dy_ld;
    int n, vocab, cols, chunk_shift;
    float scale;
};

// The columns of a lane: eight, the last ones of a row where it would reach past them (two lanes then make the same numbers), so that loads
// need no bounds and many are on their way at a time; fewer only where a row has fewer.
struct Columns {
    int c, n;
    __device__ __forceinline__ Columns(int at, int cols) : c(cols >= 8 ? min(at, cols - 8) : 0), n(cols >= 8 ? 8 : cols) {}
};
// WIDE: rows of eight columns and more
template <bool WIDE, class T> __device__ __forceinline__ Raw8<T> load_row(const GradArgs &a, uint32_t place, Columns at)
{
    return load8(static_cast<const T *>(a.dy) + (int64_t)place * a.dy_ld + at.c, WIDE ? 8 : at.n);
}
// What the lanes of a group, LANES of them with eight columns each, have to do: a chunk, and as many groups as its columns take.
template <int LANES> struct Group {
    int chunk, lane, c, from, to;
    bool some;
    __device__ __forceinline__ Group(const GradArgs &a, int per_chunk, int64_t groups)
    {
        const int64_t g = (int64_t)blockIdx.x * (256 / LANES) + (LANES == 64 ? (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : (int)threadIdx.x / LANES);
        some = g < groups;
        chunk = (int)(g / per_chunk), lane = threadIdx.x % LANES;
        c = (int)(g - (int64_t)chunk * per_chunk) * 8 * LANES + 8 * lane;
        from = chunk << a.chunk_shift, to = min(from + (1 << a.chunk_shift), a.n);
    }
};
// Sums of the runs of equal tokens in a chunk.  Bound by latency: a chunk's places, then their rows, a few at a time.
template <class T, int LANES, bool WIDE> __global__ __launch_bounds__(256) void runs_kernel(GradArgs a, int per_chunk, int64_t groups)
{
    constexpr int MOST = 32 / (int)sizeof(T), STEP = LANES < MOST ? LANES : MOST;
    const Group<LANES> g(a, per_chunk, groups);
    if (!g.some) return;
    const Columns at(g.c, a.cols);
    const bool here = g.c < a.cols;            // lanes behind the last column go along
    const int from = g.from, to = g.to;
    const uint32_t none = (uint32_t)a.vocab, before = from > 0 ? a.key[from - 1] : none, behind = to < a.n ? a.key[to] : none;
    // of lane i of the group; the same number in all lanes of a wave may live in a scalar register
    auto lanes = [](uint32_t x, int i) { return LANES == 64 ? (uint32_t)__builtin_amdgcn_readlane((int)x, i) : (uint32_t)__shfl((int)x, i, LANES); };
    float v[8] = {};
    uint32_t now = none;                       // the run that is being summed
    auto store = [&](bool goes_on) {
        const bool whole = now != before && !goes_on;
        float *const p = (whole ? a.dtable + (int64_t)now * a.cols : (now == before ? a.head : a.tail) + (int64_t)g.chunk * a.cols) + at.c;
        const float scale = whole ? a.scale : 1.f;
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = v[j] * scale, v[j] = 0.f;
        if (here) store8(p, to_raw<float>(f), at.n);
    };
    // The next places' rows are asked for before these are added: a row that is stored in between would have to be there first.
    uint32_t key = 0, place = 0, k[2][STEP];
    Raw8<T> x[2][STEP];
    auto ask = [&](int i, auto half) {
        const int b = (i - from) % LANES;
        if (b == 0) {        // a lane has a place of its own at hand, all of them take it from there
            const int own = min(i + g.lane, to - 1);
            key = a.key[own], place = a.place[own];
        }
#pragma unroll
        for (int u = 0; u < STEP; ++u) {
            k[half.value][u] = lanes(key, b + u);
            x[half.value][u] = load_row<WIDE, T>(a, lanes(place, b + u), at);
        }
    };
    auto take = [&](int i, auto half) {
#pragma unroll
        for (int u = 0; u < STEP; ++u) {
            const uint32_t q = k[half.value][u];
            if (i + u >= to) continue;
            if (q != now) {
                if (now != none) store(false);
                now = q;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += now != none ? elem(x[half.value][u], j) : 0.f;
        }
    };
    const std::integral_constant<int, 0> _0;
    const std::integral_constant<int, 1> _1;
    ask(from, _0);
    for (int i = from; i < to; i += 2 * STEP) {
        if (i + STEP < to) ask(i + STEP, _1);
        take(i, _0);
        if (i + 2 * STEP < to) ask(i + 2 * STEP, _0);
        if (i + STEP < to) take(i + STEP, _1);
    }
    if (now != none) store(behind == now);
}
// The runs that end in another chunk than they began in: what they left, added in order.  A block looks at a chunk's last run.  Its groups of lanes take
// 16 of the chunks behind it each, whose sums meet neighbour by neighbour, in a wave and then in LDS, and so on with the next block's worth: places stay
// in order, and a sum of n chunks takes the roundings of n / (16 GROUPS) additions and some 25 more.  Bound by latency, which a frequent token's hundreds
// of chunks would take one after the other (9663 places of 9 tokens, 8 columns: 70 us the gradient with one group a run, 18 so).
template <int LANES, bool WIDE> __global__ __launch_bounds__(256) void join_runs_kernel(GradArgs a, int per_chunk)
{
    constexpr int AHEAD = 16, GROUPS = 256 / LANES, WAVES = 4;
    __shared__ __align__(16) float lds[2][WAVES][8 * LANES];
    const int chunk = (int)blockIdx.x / per_chunk, from = chunk << a.chunk_shift, to = from + (1 << a.chunk_shift);
    if (to >= a.n) return;
    const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
    const int chunks = (int)(((int64_t)a.n + (1 << a.chunk_shift) - 1) >> a.chunk_shift);
    auto key_at = [&](int q) { return q < chunks ? a.key[q << a.chunk_shift] : (uint32_t)a.vocab; };
    // keys are asked for ahead of their use: of the next chunk, of this group's chunks, of the next round's
    const uint32_t now = a.key[to - 1], behind = a.key[to], before = from > 0 ? a.key[from - 1] : (uint32_t)a.vocab;
    uint32_t own = key_at(chunk + 1 + group * AHEAD), next = key_at(chunk + 1 + GROUPS * AHEAD);
    if (behind != now || now >= (uint32_t)a.vocab || before == now) return;
    const int c = ((int)blockIdx.x - chunk * per_chunk) * 8 * LANES + 8 * lane;
    const Columns at(c < a.cols ? c : 0, a.cols);
    float v[8] = {}, sum[8] = {};              // of this group's chunks; of the rounds before (group 0)
    if (group == 0) {
        const Raw8<float> first = load8(a.tail + (int64_t)chunk * a.cols + at.c, WIDE ? 8 : at.n);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = elem(first, j);
    }
    bool more = true;
    for (int q0 = chunk + 1, buf = 0; more; q0 += GROUPS * AHEAD, buf ^= 1) {
        const int q = q0 + group * AHEAD;
        const bool some = own == now;          // keys ascend: it is the run that chunk q begins with
        more = next == now;
        own = key_at(q + GROUPS * AHEAD), next = key_at(q0 + 2 * GROUPS * AHEAD);
        if (some) {
            bool mine[AHEAD];
            Raw8<float> x[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int r = min(q + u, chunks - 1);
                mine[u] = key_at(q + u) == now;
                x[u] = load8(a.head + (int64_t)r * a.cols + at.c, WIDE ? 8 : at.n);      // of other chunks: anything
            }
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] += mine[u] ? elem(x[u], j) : 0.f;
        }
        // a wave's groups, then the waves: group 0 adds these while the others read the next round, whose sums go to the other half, which is free,
        // because a round's barrier is behind group 0's additions of the round before
#pragma unroll
        for (int d = LANES; d < 64; d *= 2)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += __shfl_down(v[j], d);
        if ((threadIdx.x & 63) < LANES)
#pragma unroll
            for (int j = 0; j < 8; ++j) lds[buf][threadIdx.x >> 6][8 * lane + j] = v[j];
        __syncthreads();
        if (group == 0) {
#pragma unroll
            for (int w = 1; w < WAVES; ++w)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] += lds[buf][w][8 * lane + j];
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] += v[j];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = 0.f;
    }
    if (group > 0 || c >= a.cols) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] *= a.scale;
    store8(a.dtable + (int64_t)now * a.cols + at.c, to_raw<float>(sum), at.n);
}

// ---- host side ------------------------------------------------------------------------------------------------------------------------
int desc_check(const cg_embedding_desc *d)
{
    if (!d || !type_ok(d->table_type) || !type_ok(d->type) || d->vocab < 1 || d->cols < 1 || d->tokens < 0) return CG_EINVAL;
    const int64_t most = INT32_MAX - 65535, chunks = (d->cols + 7) / 8;
    if (d->vocab > most || d->cols > most || d->tokens > (1 << 28) || d->tokens * chunks > INT32_MAX / 2) return CG_EUNSUPPORTED;
    return CG_OK;
}
// More chunks, more waves; fewer, fewer parts of a frequent token to add: 3001 places of 769 columns 23 us with chunks of 8, 25 with 16, 29 with 32; 8000
// of 256 32, 32 and 35; 16384 of 1024 62, 60 and 57 (64: 60); 300000 of 64 143 with 64, 149 with 32, 153 with 128.
int chunk_shift_of(int64_t tokens, int64_t cols) { return tokens <= 4096 ? 3 : tokens <= kMostPass ? cols <= 256 ? 4 : 5 : tokens <= 1 << 20 ? 6 : 7; }
size_t round16(size_t n) { return (n + 15) & ~(size_t)15; }
struct Layout {
    size_t key[2], place[2], counts, head, tail, total;
    int tiles;                // of the sort; 1: one block
    bool passes;              // a pass is one launch
};
Layout layout_of(const cg_embedding_desc *d)
{
    Layout l{};
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t p = at; at += round16(bytes); return p; };
    const size_t n = (size_t)d->tokens;
    l.passes = n <= (size_t)kMostPass;
    l.tiles = n <= (size_t)kMostOne ? 1 : (int)(l.passes ? (n + kOneBlock - 1) / kOneBlock : (n + kTile - 1) / kTile);
    for (int i = 0; i < (l.tiles > 1 ? 2 : 1); ++i) l.key[i] = take(4 * n), l.place[i] = take(4 * n);
    l.counts = take(l.passes ? 0 : sizeof(uint32_t) * kDigits * (size_t)l.tiles);
    const size_t chunks = (n + ((size_t)1 << chunk_shift_of(d->tokens, d->cols)) - 1) >> chunk_shift_of(d->tokens, d->cols);
    if (chunks > 1) l.head = take(4 * chunks * (size_t)d->cols), l.tail = take(4 * chunks * (size_t)d->cols);
    l.total = at;
    return l;
}

// One at a time where that does not fill the chip.
template <class TT, class T> void lookup_launch(const LookupArgs &a, hipStream_t s)
{
    const uint32_t b = (a.count + 255) / 256;
    if (b <= 2048) hipLaunchKernelGGL((lookup_kernel<TT, T, 1>), dim3(b), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((lookup_kernel<TT, T, 4>), dim3(b < 4 * 8192 ? (b + 3) / 4 : 8192), dim3(256), 0, s, a);
}
template <class TT> int lookup_typed(const LookupArgs &a, int type, hipStream_t s)
{
    if (type == CG_TYPE_FP32) lookup_launch<TT, float>(a, s);
    else lookup_launch<TT, bf16raw>(a, s);
    CG_HIP_TRY(hipGetLastError());
    return CG_OK;
}
template <class T, int LANES, bool WIDE> void runs_launch(const GradArgs &a, hipStream_t s)
{
    const int per = (a.cols + 8 * LANES - 1) / (8 * LANES);
    const int64_t chunks = ((int64_t)a.n + (1 << a.chunk_shift) - 1) >> a.chunk_shift, groups = chunks * per;
    const dim3 grid((unsigned)((groups + 256 / LANES - 1) / (256 / LANES)));
    hipLaunchKernelGGL((runs_kernel<T, LANES, WIDE>), grid, dim3(256), 0, s, a, per, groups);
    if (chunks > 1) hipLaunchKernelGGL((join_runs_kernel<LANES, WIDE>), dim3((unsigned)groups), dim3(256), 0, s, a, per);
}
template <class T> int grad_typed(const GradArgs &a, hipStream_t s)
{
    if (a.cols < 8) runs_launch<T, 4, false>(a, s);
    else if (a.cols <= 32) runs_launch<T, 4, true>(a, s);
    else if (a.cols <= 128) runs_launch<T, 16, true>(a, s);
    else runs_launch<T, 64, true>(a, s);
    CG_HIP_TRY(hipGetLastError());
    return CG_OK;
}
// Blocks of 1024 threads that fill `count` floats, 16 a thread at least.
unsigned fillers(int64_t count) { return (unsigned)std::min<int64_t>((count + 16383) / 16384, 1024); }

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
    const hipStream_t s = static_cast<hipStream_t>(stream);
    return d->table_type == CG_TYPE_FP32 ? lookup_typed<float>(a, d->type, s) : lookup_typed<bf16raw>(a, d->type, s);
}

extern "C" size_t cg_embedding_workspace_bytes(const cg_embedding_desc *d) { return desc_check(d) == CG_OK ? layout_of(d).total : 0; }

extern "C" int cg_embedding_bwd(const cg_embedding_desc *d, const int32_t *tokens, const void *dy, int64_t dy_ld, float *dtable, void *ws, size_t ws_bytes, void *stream)
{
    if (int rc = desc_check(d)) return rc;
    if (!floats_ok(dtable) || (d->tokens > 0 && (!floats_ok(tokens) || !tensor_ok(dy, dy_ld, d->cols, d->type)))) return CG_EINVAL;
    const Layout l = layout_of(d);
    if (l.total && (!ws || !aligned16(ws))) return CG_EINVAL;
    if (ws_bytes < l.total) return CG_ENOSPC;
    char *const base = static_cast<char *>(ws);
    auto words = [&](size_t at) { return reinterpret_cast<uint32_t *>(base + at); };
    const hipStream_t s = static_cast<hipStream_t>(stream);
    int bits = 1;
    while (d->vocab >> bits) ++bits;           // keys are at most vocab
    const int most = l.passes ? 10 : 8, passes = (bits + most - 1) / most, n = (int)d->tokens;
    const int per = std::max((bits + passes - 1) / passes, kLeastBits);
    const int64_t count = d->vocab * d->cols;
    if (n == 0) {
        hipLaunchKernelGGL(fill_kernel, dim3(fillers(count)), dim3(1024), 0, s, Fill{dtable, count, 0});
        CG_HIP_TRY(hipGetLastError());
        return CG_OK;
    }
    int last = 0;
    SortArgs a{};
    a.tokens = tokens, a.counts = words(l.counts), a.n = n, a.vocab = (int)d->vocab, a.bits = per, a.tiles = l.tiles;
    // a part beside each launch of the sort that goes over the places once
    const int shares = l.tiles > 1 && l.passes ? passes : 1;
    const int64_t share = (count + shares - 1) / shares;
    int64_t filled = 0;
    auto fill = [&](int first) {
        const Fill f{dtable + filled, std::min(share, count - filled), first};
        filled += f.count;
        return f;
    };
    if (l.tiles == 1) {
        a.key = words(l.key[0]), a.place = words(l.place[0]);
        a.fill = fill(1);
        hipLaunchKernelGGL(sort_one_kernel, dim3(1 + fillers(a.fill.count)), dim3(kOneBlock), 0, s, a, passes);
        CG_HIP_TRY(hipGetLastError());
    } else {
        for (int p = 0; p < passes; ++p) {
            last = p & 1;
            a.key_in = words(l.key[1 - last]), a.place_in = words(l.place[1 - last]), a.key = words(l.key[last]), a.place = words(l.place[last]);
            a.shift = p * per;
            a.fill = fill(l.tiles);
            const unsigned beside = fillers(a.fill.count);
            if (l.passes) hipLaunchKernelGGL(sort_pass_kernel, dim3((unsigned)l.tiles + beside), dim3(kOneBlock), 0, s, a);
            else {
                hipLaunchKernelGGL(sort_count_kernel, dim3((unsigned)l.tiles + 4 * beside), dim3(kTileBlock), 0, s, a);
                hipLaunchKernelGGL(sort_sums_kernel, dim3(1), dim3(1024), 0, s, a.counts, kDigits * l.tiles);
                hipLaunchKernelGGL(sort_move_kernel, dim3((unsigned)l.tiles), dim3(kTileBlock), 0, s, a);
            }
            CG_HIP_TRY(hipGetLastError());
            a.tokens = nullptr;
        }
    }
    GradArgs g{};
    g.key = words(l.key[last]), g.place = words(l.place[last]), g.dy = dy, g.dy_ld = dy_ld;
    g.head = reinterpret_cast<float *>(base + l.head), g.tail = reinterpret_cast<float *>(base + l.tail);
    g.dtable = dtable, g.n = n, g.vocab = (int)d->vocab, g.cols = (int)d->cols, g.scale = d->scale;
    g.chunk_shift = chunk_shift_of(d->tokens, d->cols);
    return d->type == CG_TYPE_FP32 ? grad_typed<float>(g, s) : grad_typed<bf16raw>(g, s);
}
