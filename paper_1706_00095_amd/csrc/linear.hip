// Linear layers: what the entry points check and plan, and the kernels beside the tiles of linear_gemm.hip: few tokens, the join of a
// cut k, sums of columns, the gradient through an activation alone.
#include "linear_device.h"
#include "row_checks.h"

namespace cg {
namespace {

// ---- few tokens -------------------------------------------------------------------------------------------------------------
// Forward for up to 16 MT tokens: the weights are read once and that is all there is to do.  A block takes 16 rows of w, its eight waves every
// eighth step along k; a step is a lane's 16 bytes of one row (4 lanes a row), AHEAD to 2 AHEAD of
// them in flight (one token, 4096 -> 16384, weights out of HBM: 24.5 us, 5.5 TB/s; 26 with twice as many that all land before the next are asked
// for, 28 with twice as many so).  w is the matrix instruction's first operand, the
// tokens are the second; bf16: 16x16x32, fp32: 16x16x4 on the values as they are.  The waves' sums meet in LDS.
constexpr int kFewWaves = 8, kFewRows = 16;
typedef float v4f __attribute__((ext_vector_type(4)));
struct FewArgs {
    const void *x, *w;
    int64_t x_ld, w_ld;
    int M, N, K;
    EpiArgs epi;
};

template <class T> struct FewStep;
template <> struct FewStep<bf16raw> {
    static constexpr int PER = 8;         // values of a lane
    static __device__ __forceinline__ u32x4 load(const bf16raw *p, int n)
    {
        const Raw8<bf16raw> r = load8(p, n);
        return u32x4{r.w[0], r.w[1], r.w[2], r.w[3]};
    }
    static __device__ __forceinline__ v4f mma(u32x4 w, u32x4 x, v4f c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, x), c, 0, 0, 0);
    }
};
template <> struct FewStep<float> {
    static constexpr int PER = 4;
    static __device__ __forceinline__ u32x4 load(const float *p, int n)
    {
        if (n >= 4) {
            const Loose16<float> q = *reinterpret_cast<const Loose16<float> *>(p);
            return u32x4{q.w[0], q.w[1], q.w[2], q.w[3]};
        }
        u32x4 r = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < n) r[i] = __float_as_uint(p[i]);
        return r;
    }
    static __device__ __forceinline__ v4f mma(u32x4 w, u32x4 x, v4f c)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[i]), __uint_as_float(x[i]), c, 0, 0, 0);
        return c;
    }
};

template <class T, int MT> __global__ __launch_bounds__(64 * kFewWaves) void few_tokens_kernel(FewArgs a)
{
    using S = FewStep<T>;
    constexpr int STEP = 4 * S::PER, AHEAD = MT == 1 ? 4 : 2;
    __shared__ __align__(16) float sums[kFewWaves][MT * 16][kFewRows + 4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, at = lane & 15, k0 = (lane >> 4) * S::PER;
    const int n0 = blockIdx.x * kFewRows, row = n0 + at;
    const T *w = static_cast<const T *>(a.w) + (row < a.N ? row * a.w_ld : 0);
    const T *x[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) x[t] = static_cast<const T *>(a.x) + (16 * t + at < a.M ? (16 * t + at) * a.x_ld : 0);
    v4f acc[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[t] = v4f{};
    // rows and tokens that are none read the first one's values, and their sums go nowhere; the next AHEAD steps are asked for before these are multiplied
    u32x4 vw[2][AHEAD], vx[2][MT][AHEAD];
    auto ask = [&](int s0, auto half) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int k = s0 + u * STEP + k0;
            vw[half.value][u] = S::load(w + k, a.K - k);
#pragma unroll
            for (int t = 0; t < MT; ++t) vx[half.value][t][u] = S::load(x[t] + k, a.K - k);
        }
    };
    auto multiply = [&](auto half) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
#pragma unroll
            for (int t = 0; t < MT; ++t) acc[t] = S::mma(vw[half.value][u], vx[half.value][t][u], acc[t]);
    };
    constexpr int ALL = kFewWaves * AHEAD * STEP;
    const std::integral_constant<int, 0> _0;
    const std::integral_constant<int, 1> _1;
    const int first = wave * AHEAD * STEP;
    if (first < a.K) ask(first, _0);
    for (int s0 = first; s0 < a.K; s0 += 2 * ALL) {
        if (s0 + ALL < a.K) ask(s0 + ALL, _1);
        multiply(_0);
        if (s0 + 2 * ALL < a.K) ask(s0 + 2 * ALL, _0);
        if (s0 + ALL < a.K) multiply(_1);
    }
#pragma unroll
    for (int t = 0; t < MT; ++t) *reinterpret_cast<v4f *>(&sums[wave][16 * t + at][4 * (lane >> 4)]) = acc[t];
    __syncthreads();
    if (threadIdx.x < MT * 32) {
        const int m = threadIdx.x / 2, c = 8 * (threadIdx.x & 1);
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i] = 0.f;
#pragma unroll
            for (int u = 0; u < kFewWaves; ++u) v[i] += sums[u][m][c + i];
        }
        if (m < a.M && n0 + c < a.N) finish8<T>(a.epi, v, m, n0 + c, a.N - n0 - c);
    }
}

// ---- the join of a cut k --------------------------------------------------------------------------------------------------
template <class T> __global__ __launch_bounds__(256) void gemm_join_kernel(const float *part, int splits, int R, int C, FastDiv by_chunks, uint32_t count, EpiArgs e, float *dbias)
{
    const int64_t plane = (int64_t)R * C;
    if (dbias)
        for (uint32_t r = blockIdx.x * 256 + threadIdx.x; r < (uint32_t)R; r += gridDim.x * 256) {
            float s = 0.f;
            for (int i = 0; i < splits; ++i) s += part[splits * plane + (int64_t)i * R + r];
            dbias[r] = s;
        }
    for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < count; i += gridDim.x * 256) {
        const int r = (int)fdiv(i, by_chunks), c = 8 * (int)(i - r * by_chunks.d), n = C - c;
        const float *p = part + (int64_t)r * C + c;
        Raw8<float> bias = {};
        if (e.bias) bias = load8(e.bias + c, n);
        const EpiIn<T> in = {epi_load_add<T>(e, r, c, n), epi_load_z<EPI_EITHER, T>(e, r, c, n)};
        float v[8] = {};
        for (int s = 0; s < splits; s += 4) {        // four parts on their way at a time
            Raw8<float> x[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) x[u] = load8(p + min(s + u, splits - 1) * plane, n);
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] += s + u < splits ? elem(x[u], j) : 0.f;
        }
        epi_finish<EPI_EITHER, T>(e, v, bias, in, r, c, n);
    }
}

// ---- sums of columns: the gradient of a bias ----------------------------------------------------------------------------------
// A block sums a slice of the rows for 256 columns, eight neighbours a thread, eight threads a column; slices are added in order.
constexpr int kColumns = 256;
template <class T> __global__ __launch_bounds__(256) void column_sums_kernel(const T *x, int64_t ld, int rows, int cols, int slice, float *out)
{
    __shared__ __align__(16) float lds[8][kColumns];
    const int c = blockIdx.x * kColumns + 8 * (threadIdx.x & 31), ty = threadIdx.x >> 5, n = cols - c;
    const int64_t r0 = (int64_t)blockIdx.y * slice;
    const int r1 = (int)min((int64_t)rows, r0 + slice);
    float v[8] = {};
    for (int64_t r = r0 + ty; r < r1; r += 32) {
        Raw8<T> q[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) q[u] = load8(x + (r + 8 * u < r1 && n > 0 ? (r + 8 * u) * ld + c : 0), r + 8 * u < r1 ? n : 0);
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += elem(q[u], i);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) lds[ty][8 * (threadIdx.x & 31) + i] = v[i];
    __syncthreads();
    const int mine = blockIdx.x * kColumns + threadIdx.x;
    if (mine < cols) {
        float s = 0.f;
#pragma unroll
        for (int u = 0; u < 8; ++u) s += lds[u][threadIdx.x];
        out[(int64_t)blockIdx.y * cols + mine] = s;
    }
}
// The slices of 32 columns a block: eight threads a column take every eighth, four of them asked for at a time.
__global__ __launch_bounds__(256) void column_join_kernel(const float *part, int slices, int cols, float *out)
{
    __shared__ float lds[8][32];
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5, c = blockIdx.x * 32 + tx;
    float s = 0.f;
    if (c < cols)
        for (int i = ty; i < slices; i += 32) {
            float v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = i + 8 * u < slices ? part[(int64_t)(i + 8 * u) * cols + c] : 0.f;
#pragma unroll
            for (int u = 0; u < 4; ++u) s += v[u];
        }
    lds[ty][tx] = s;
    __syncthreads();
    if (ty == 0 && c < cols) {
#pragma unroll
        for (int u = 1; u < 8; ++u) s += lds[u][tx];
        out[c] = s;
    }
}

// ---- the gradient through an activation alone -----------------------------------------------------------------------------------
template <class T> __global__ __launch_bounds__(256) void act_bwd_kernel(const T *dy, int64_t dy_ld, int cols, FastDiv by_chunks, uint32_t count, EpiArgs e)
{
    for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < count; i += gridDim.x * 256) {
        const int64_t r = fdiv(i, by_chunks);
        const int c = 8 * (int)(i - (uint32_t)r * by_chunks.d), n = cols - c;
        const Raw8<T> g = load8(dy + r * dy_ld + c, n);
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = elem(g, j);
        finish8<T>(e, v, r, c, n);
    }
}

// ---- plans ------------------------------------------------------------------------------------------------------------------------
constexpr int64_t kMostBlocks = 1 << 22;       // of 512 threads a launch has room for less than 2^32
// Up to 32 tokens by few_tokens_kernel.  Measured at 17 and 32 tokens with weights out of HBM, and the same in tiles: bf16 1000 -> 2000 4.3 and 4.7 us, 9.1 and
// 9.0 in tiles (whose k is cut: a launch more); 4096 -> 4096 12.9 and 15.9, 13.1 and 14.8.  With more inputs tiles are the faster (10240 -> 4096 32 and
// 39, 23 and 23; 4096 -> 16384 43 and 55, 31 and 42), with more tokens everywhere but in short rows (64 tokens, 4096 -> 4096: 24, 16 in tiles).
constexpr int kFewTokens = 32;
constexpr int kMostSplits = 32;

bool act_ok(int act) { return act >= CG_ACT_NONE && act <= CG_ACT_SILU; }
int desc_check(const cg_linear_desc *d)
{
    if (!d || !type_ok(d->type) || d->M < 0 || d->N < 1 || d->K < 1 || !act_ok(d->act) || !act_ok(d->act_in)) return CG_EINVAL;
    const int64_t most = 1 << 26;
    if (d->M > most || d->N > most || d->K > most) return CG_EUNSUPPORTED;
    auto tiles = [](int64_t n) { return (n + 127) / 128; };
    if (tiles(d->M) * tiles(d->N) > kMostBlocks || tiles(d->M) * tiles(d->K) > kMostBlocks || tiles(d->N) * tiles(d->K) > kMostBlocks) return CG_EUNSUPPORTED;
    return CG_OK;
}
// Microseconds that `blocks` tiles of 128 x 128 take for `steps` steps of 64 values of k each, and that the join of a cut k takes: what was measured
// on products of 64 to 9216 rows, columns and values of k.  A compute unit's second block costs less than its first, others as much
// again.  bf16, 1024^3: 14 us uncut, 17 in two parts, 20 in four; 64 x 4096 x 4096: 15 in eight parts, 19 in sixteen, 17 in four.  fp32, 256 x
// 9216 x 4096: 120 us in three parts, 186 uncut.
double cost(int type, int64_t blocks, int64_t steps)
{
    const int64_t each = (blocks + 255) / 256;
    const double of = type == CG_TYPE_FP32 ? each == 1 ? 2.8 : 2.4 * (double)each : each == 1 ? 0.55 : 0.4 * (double)each;
    return 4.0 + of * (double)steps;
}
// The same of tiles of 64 x 64: a quarter of the work a tile in more than a quarter of the time, but four times the tiles, so that k need not be cut.
// fp32: 1500 x 515 x 771 18 us (26 in four parts of tiles of 128), 1024^3 22 (30), 2048^3 118 (104), 256 x 4096 x 9216 136 (115).  bf16: 1024^3 8
// (15), 1000 x 2048 x 2048 17 (25), 64 x 4096 x 4096 13 in four parts (15 in eight of tiles of 128), 2048^3 32 (27).
double small_cost(int type, int64_t blocks, int64_t steps)
{
    const int64_t each = (blocks + 255) / 256;
    const double of = type == CG_TYPE_FP32 ? each == 1 ? 1.06 : 0.87 * (double)each : each == 1 ? 0.3 : 0.19 * (double)each;
    return 4.0 + of * (double)steps + 1.2 * (double)(each - 1);
}
double join_cost(int64_t splits, int64_t R, int64_t C) { return 4.5 + (double)splits * (double)R * (double)C * 2e-6; }
struct Plan {
    int R, C, K;              // of the product
    bool few;
    bool small;               // tiles of 64 x 64, else 128 x 128
    bool large;               // tiles of 256 x 256, k uncut, where rows allow it (bf16)
    int splits, chunk;        // of k, for tiles of 64 and 128
};
Plan plan_of(const cg_linear_desc *d, int pass)
{
    Plan p{};
    const int M = (int)d->M, N = (int)d->N, K = (int)d->K;
    p.R = pass == CG_PASS_BWD_WEIGHT ? N : M;
    p.C = pass == CG_PASS_FWD ? N : K;
    p.K = pass == CG_PASS_FWD ? K : pass == CG_PASS_BWD_DATA ? N : M;
    p.few = pass == CG_PASS_FWD && M <= kFewTokens;
    p.splits = 1, p.chunk = p.K;
    if (p.few || p.K == 0) return p;
    auto tiles = [&](int64_t t) { return ((p.R + t - 1) / t) * ((p.C + t - 1) / t); };
    const int64_t pieces = (p.K + kGemmStep - 1) / kGemmStep;
    double best = 1e30;
    const int64_t splits = (int64_t)p.R * p.C <= 1 << 28 ? kMostSplits : 1;       // of large outputs there are tiles enough
    for (int tile = 128; tile >= 64; tile /= 2) {
        const int64_t n = tiles(tile);
        for (int64_t s = 1; s <= splits && s <= pieces; ++s) {
            const int64_t per = (pieces + s - 1) / s, have = (pieces + per - 1) / per;
            if (have != s || n * s > kMostBlocks) continue;
            const double t = (tile == 64 ? small_cost(d->type, n * s, per) : cost(d->type, n * s, per)) + (s > 1 ? join_cost(s, p.R, p.C) : 0);
            if (t < best) best = t, p.small = tile == 64, p.splits = (int)s, p.chunk = (int)(s > 1 ? per * kGemmStep : p.K);
        }
    }
    // a block a compute unit: microseconds a step, and before and after the steps
    p.large = d->type == CG_TYPE_BF16 && (double)((tiles(256) + 255) / 256) * (9.0 + 1.0 * (double)pieces) < best + 4.0;
    return p;
}
size_t part_bytes(const Plan &p) { return p.splits > 1 ? (size_t)p.splits * (size_t)p.R * ((size_t)p.C + 1) * sizeof(float) : 0; }
int column_slices(int64_t M, int64_t N)
{
    const int64_t blocks = (N + kColumns - 1) / kColumns, most = 1024 / blocks, want = (M + 63) / 64;
    int64_t s = want < most ? want : most;
    return (int)(s < 1 ? 1 : s > 256 ? 256 : s);
}
// As far as rows may lie apart where a lane's offsets have 32 bits: what is sent out of range (2^31) stays out of it for 128 rows of 2 bytes an element.
constexpr int64_t kMostDmaLd = 1 << 21;
// Backward-weight in large tiles multiplies bf16 numbers: x in 8 bits is unpacked first.  Eight rows of tiles would each turn it into bf16 on
// its way into LDS otherwise (8192 tokens, 8192 x 2048 weights: 521 us in tiles of 256 through registers, 812 in tiles of 128; 36 and 208 so).
bool unpacks(const cg_linear_desc *d, const Plan &p)
{
    return p.large && d->K % 8 == 0 && d->K <= kMostDmaLd && d->M * ((d->K + kPackBlock - 1) / kPackBlock) <= (INT32_MAX >> 2) - 65535;
}
size_t unpacked_bytes(const cg_linear_desc *d) { return (size_t)d->M * (size_t)d->K * 2; }
size_t slice_bytes(const cg_linear_desc *d)
{
    const int s = column_slices(d->M, d->N);
    return s > 1 ? (size_t)s * (size_t)d->N * sizeof(float) : 0;
}

bool dma_ok(const void *p, int64_t ld, int64_t cols) { return aligned16(p) && ld % 8 == 0 && cols % 8 == 0 && ld <= kMostDmaLd; }
int ws_check(void *ws, size_t ws_bytes, size_t need)
{
    if (need && (!ws || !aligned16(ws))) return CG_EINVAL;
    return ws_bytes < need ? CG_ENOSPC : CG_OK;
}
unsigned blocks_for(uint64_t n, unsigned most) { const uint64_t b = (n + 255) / 256; return (unsigned)(b < most ? b : most); }

// What a product takes of its plan, with operands as they are: its tile; a: its tiles and the parts of k.
int tile_of(const Plan &p, bool packed, bool dma, GemmArgs &a)
{
    const bool large = p.large && dma && !packed;
    const int tile = large ? 256 : p.small ? 64 : 128;
    a.R = p.R, a.C = p.C, a.K = p.K;
    a.tiles_r = (p.R + tile - 1) / tile, a.tiles_c = (p.C + tile - 1) / tile;
    a.splits = large ? 1 : p.splits, a.chunk = large ? p.K : p.chunk;
    return tile;
}
int product(const cg_linear_desc *d, int pass, const Plan &p, GemmArgs &a, bool packed, bool dma, void *ws, hipStream_t s)
{
    const int tile = tile_of(p, packed, dma, a);
    a.part = static_cast<float *>(ws);
    if (int rc = gemm_launch({d->type, pass, packed, tile, dma}, a, s)) return rc;
    if (a.splits == 1) return CG_OK;
    const uint32_t chunks = (uint32_t)((p.C + 7) / 8), count = chunks * (uint32_t)p.R;
    const dim3 grid(blocks_for(count, 4096));
    const FastDiv by = make_fastdiv(chunks);
    if (pass == CG_PASS_BWD_WEIGHT || d->type == CG_TYPE_FP32)
        hipLaunchKernelGGL((gemm_join_kernel<float>), grid, dim3(256), 0, s, a.part, a.splits, p.R, p.C, by, count, a.epi, a.dbias);
    else hipLaunchKernelGGL((gemm_join_kernel<bf16raw>), grid, dim3(256), 0, s, a.part, a.splits, p.R, p.C, by, count, a.epi, a.dbias);
    CG_HIP_TRY(hipGetLastError());
    return CG_OK;
}

// dbias by a pass of its own; its slices' sums lie in the workspace until it is done.
int bias_pass(const cg_linear_desc *d, const void *dz, int64_t dz_ld, float *dbias, void *ws, hipStream_t s)
{
    const int M = (int)d->M, N = (int)d->N, slices = column_slices(M, N), slice = (M + slices - 1) / slices;
    float *const to = slices > 1 ? static_cast<float *>(ws) : dbias;
    const dim3 grid((unsigned)((N + kColumns - 1) / kColumns), (unsigned)slices);
    hipLaunchKernelGGL((column_sums_kernel<bf16raw>), grid, dim3(256), 0, s, static_cast<const bf16raw *>(dz), dz_ld, M, N, slice, to);
    CG_HIP_TRY(hipGetLastError());
    if (slices > 1) {
        hipLaunchKernelGGL(column_join_kernel, dim3((unsigned)((N + 31) / 32)), dim3(256), 0, s, to, slices, N, dbias);
        CG_HIP_TRY(hipGetLastError());
    }
    return CG_OK;
}

template <class T> int few_tokens(const FewArgs &a, hipStream_t s)
{
    const dim3 grid((unsigned)((a.N + kFewRows - 1) / kFewRows)), block(64 * kFewWaves);
    if (a.M <= 16) hipLaunchKernelGGL((few_tokens_kernel<T, 1>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((few_tokens_kernel<T, 2>), grid, block, 0, s, a);
    CG_HIP_TRY(hipGetLastError());
    return CG_OK;
}

bool packed_ok(const cg_packed8 *p, int64_t cols)
{
    return p->codes && p->scales && p->codes_ld >= cols && p->scales_ld >= (cols + kPackBlock - 1) / kPackBlock;
}
// where an activation's slope is wanted: its inputs in one form or the other
bool slope_ok(int act, const void *z, int64_t z_ld, const cg_packed8 *z8, int64_t cols, int type)
{
    if (act == CG_ACT_NONE) return true;
    if (z8) return !z && packed_ok(z8, cols);
    return tensor_ok(z, z_ld, cols, type);
}
void slope_args(EpiArgs &e, int act, const void *z, int64_t z_ld, const cg_packed8 *z8)
{
    e.slope = act;
    if (act == CG_ACT_NONE) return;
    if (z8) e.z_in8 = {z8->codes, z8->scales, z8->codes_ld, z8->scales_ld};
    else e.z_in = z, e.z_in_ld = z_ld;
}

}  // namespace
}  // namespace cg

using namespace cg;

extern "C" size_t cg_linear_workspace_bytes(const cg_linear_desc *d, int pass)
{
    if (desc_check(d) != CG_OK || d->M == 0 || (pass != CG_PASS_FWD && pass != CG_PASS_BWD_DATA && pass != CG_PASS_BWD_WEIGHT)) return 0;
    const Plan p = plan_of(d, pass);
    size_t need = part_bytes(p);
    if (pass != CG_PASS_BWD_WEIGHT) return need;
    if (p.large && slice_bytes(d) > need) need = slice_bytes(d);
    if (unpacks(d, p) && unpacked_bytes(d) > need) need = unpacked_bytes(d);
    return need;
}

extern "C" int cg_debug_linear_plan(const cg_linear_desc *d, int pass, int whole, int packed, int *tile, int *parts, int *halves)
{
    if (int rc = desc_check(d)) return rc;
    if ((pass != CG_PASS_FWD && pass != CG_PASS_BWD_DATA && pass != CG_PASS_BWD_WEIGHT) || !tile || !parts || !halves) return CG_EINVAL;
    const Plan p = plan_of(d, pass);
    const bool dma = whole && d->type == CG_TYPE_BF16;
    GemmArgs a{};
    *tile = p.few ? 16 : tile_of(p, packed && !(dma && unpacks(d, p)), dma, a);
    *parts = p.few ? 1 : a.splits;
    *halves = !p.few && gemm_halves(d->type, *tile, (int64_t)a.tiles_r * a.tiles_c * a.splits);
    return CG_OK;
}

extern "C" int cg_linear_fwd(const cg_linear_desc *d, const void *x, int64_t x_ld, const void *w, int64_t w_ld, const float *bias,
                             const void *residual, int64_t residual_ld, void *y, int64_t y_ld, void *z, int64_t z_ld, void *ws,
                             size_t ws_bytes, void *stream)
{
    if (int rc = desc_check(d)) return rc;
    if (d->M == 0) return CG_OK;
    if (!tensor_ok(x, x_ld, d->K, d->type) || !tensor_ok(w, w_ld, d->K, d->type) || (bias && !floats_ok(bias)) ||
        !optional_ok(residual, residual_ld, d->N, d->type) || !tensor_ok(y, y_ld, d->N, d->type) || !optional_ok(z, z_ld, d->N, d->type)) return CG_EINVAL;
    const Plan p = plan_of(d, CG_PASS_FWD);
    if (int rc = ws_check(ws, ws_bytes, part_bytes(p))) return rc;
    EpiArgs e{};
    e.bias = bias, e.add = residual, e.add_ld = residual_ld, e.out = y, e.out_ld = y_ld, e.z = z, e.z_ld = z_ld, e.act = d->act;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (p.few) {
        const FewArgs a = {x, w, x_ld, w_ld, (int)d->M, (int)d->N, (int)d->K, e};
        return d->type == CG_TYPE_FP32 ? few_tokens<float>(a, s) : few_tokens<bf16raw>(a, s);
    }
    GemmArgs a{};
    a.A = x, a.a_ld = x_ld, a.B = w, a.b_ld = w_ld, a.epi = e;
    return product(d, CG_PASS_FWD, p, a, false, d->type == CG_TYPE_BF16 && dma_ok(x, x_ld, d->K) && dma_ok(w, w_ld, d->K), ws, s);
}

extern "C" int cg_linear_bwd_data(const cg_linear_desc *d, const void *dz, int64_t dz_ld, const void *w, int64_t w_ld, const void *z_in,
                                  int64_t z_in_ld, const cg_packed8 *z_in8, const void *add, int64_t add_ld, void *dx, int64_t dx_ld,
                                  void *ws, size_t ws_bytes, void *stream)
{
    if (int rc = desc_check(d)) return rc;
    if (d->M == 0) return CG_OK;
    if (!tensor_ok(dz, dz_ld, d->N, d->type) || !tensor_ok(w, w_ld, d->K, d->type) || !tensor_ok(dx, dx_ld, d->K, d->type) ||
        !optional_ok(add, add_ld, d->K, d->type) || !slope_ok(d->act_in, z_in, z_in_ld, z_in8, d->K, d->type)) return CG_EINVAL;
    const Plan p = plan_of(d, CG_PASS_BWD_DATA);
    if (int rc = ws_check(ws, ws_bytes, part_bytes(p))) return rc;
    GemmArgs a{};
    a.A = dz, a.a_ld = dz_ld, a.B = w, a.b_ld = w_ld;
    a.epi.add = add, a.epi.add_ld = add_ld, a.epi.out = dx, a.epi.out_ld = dx_ld;
    slope_args(a.epi, d->act_in, z_in, z_in_ld, z_in8);
    return product(d, CG_PASS_BWD_DATA, p, a, false, d->type == CG_TYPE_BF16 && dma_ok(dz, dz_ld, d->N) && dma_ok(w, w_ld, d->K), ws,
                   static_cast<hipStream_t>(stream));
}

extern "C" int cg_linear_bwd_weight(const cg_linear_desc *d, const void *dz, int64_t dz_ld, const void *x, int64_t x_ld, const cg_packed8 *x8,
                                    float *dw, float *dbias, void *ws, size_t ws_bytes, void *stream)
{
    if (int rc = desc_check(d)) return rc;
    if (!floats_ok(dw) || (dbias && !floats_ok(dbias)) || (x && x8)) return CG_EINVAL;
    if (d->M > 0 && (!tensor_ok(dz, dz_ld, d->N, d->type) || (x8 ? !packed_ok(x8, d->K) : !tensor_ok(x, x_ld, d->K, d->type)))) return CG_EINVAL;
    if (int rc = ws_check(ws, ws_bytes, cg_linear_workspace_bytes(d, CG_PASS_BWD_WEIGHT))) return rc;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const Plan p = plan_of(d, CG_PASS_BWD_WEIGHT);
    const bool dz_dma = d->type == CG_TYPE_BF16 && dma_ok(dz, dz_ld, d->N), unpack = x8 && dz_dma && unpacks(d, p);
    GemmArgs a{};
    a.A = dz, a.a_ld = dz_ld, a.epi.out = dw, a.epi.out_ld = d->K;
    const bool dma = dz_dma && (x8 || dma_ok(x, x_ld, d->K));
    // large tiles leave no room for the bias's sums: they come first, and the workspace is the product's afterwards
    if (p.large && dma && (!x8 || unpack)) {
        if (dbias)
            if (int rc = bias_pass(d, dz, dz_ld, dbias, ws, s)) return rc;
    } else a.dbias = dbias;
    if (unpack) {
        if (int rc = cg_unpack8(d->type, d->M, d->K, x8, ws, d->K, stream)) return rc;
        x = ws, x_ld = d->K, x8 = nullptr;
    }
    if (x8) a.B8 = {x8->codes, x8->scales, x8->codes_ld, x8->scales_ld};
    else a.B = x, a.b_ld = x_ld;
    return product(d, CG_PASS_BWD_WEIGHT, p, a, x8 != nullptr, dma, ws, s);
}

extern "C" int cg_act_bwd(int act, int type, int64_t rows, int64_t cols, const void *dy, int64_t dy_ld, const void *z, int64_t z_ld,
                          const cg_packed8 *z8, void *dz, int64_t dz_ld, void *stream)
{
    if (!act_ok(act) || act == CG_ACT_NONE || !type_ok(type) || rows < 0 || cols < 0) return CG_EINVAL;
    if (rows == 0 || cols == 0) return CG_OK;
    if (!tensor_ok(dy, dy_ld, cols, type) || !tensor_ok(dz, dz_ld, cols, type) || !slope_ok(act, z, z_ld, z8, cols, type)) return CG_EINVAL;
    const int64_t chunks = (cols + 7) / 8;
    if (rows > INT32_MAX || cols > INT32_MAX - 65535 || rows * chunks > INT32_MAX / 2) return CG_EUNSUPPORTED;
    EpiArgs e{};
    e.out = dz, e.out_ld = dz_ld;
    slope_args(e, act, z, z_ld, z8);
    const uint32_t count = (uint32_t)(rows * chunks);
    const dim3 grid(blocks_for(count, 16384));
    const FastDiv by = make_fastdiv((uint32_t)chunks);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (type == CG_TYPE_FP32) hipLaunchKernelGGL((act_bwd_kernel<float>), grid, dim3(256), 0, s, static_cast<const float *>(dy), dy_ld, (int)cols, by, count, e);
    else hipLaunchKernelGGL((act_bwd_kernel<bf16raw>), grid, dim3(256), 0, s, static_cast<const bf16raw *>(dy), dy_ld, (int)cols, by, count, e);
    CG_HIP_TRY(hipGetLastError());
    return CG_OK;
}
