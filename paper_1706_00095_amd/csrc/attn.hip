// Attention: descriptors, workspaces, the table of the bias by distance, and the order of the launches.
#include <cmath>
#include <utility>
#include "attn_device.h"

namespace cg {
namespace {

constexpr int64_t kMaxRows = INT32_MAX - 65535;      // a tile's end behind the last row is still a number of 32 bits
constexpr int kMaxDistance = 65536;
constexpr int64_t kMaxBlocks = (1 << 24) - 1;        // of 256 threads: a launch has fewer than 2^32

// From which distance on the buckets E + 1 .. n - 1 apply: bucket(dist) = dist below E, else E + (how many are <= dist).
struct Thresholds {
    int n, E, both;
    int from[kMaxBuckets / 2 + 1];
};

// Bias and bucket by distance, for the heads' tables [2 W + 1] in the workspace: a kernel of 4 to 9 microseconds, so that the
// attention kernels look a distance up instead of taking its logarithm for every pair.
__global__ __launch_bounds__(256) void bias_table_kernel(Thresholds th, const float *bias, int buckets, int W, float *tab, uint8_t *bid)
{
    __shared__ int from[kMaxBuckets / 2 + 1];
    const int i = blockIdx.x * 256 + threadIdx.x, h = blockIdx.y;
    if (threadIdx.x < sizeof(from) / sizeof(int)) from[threadIdx.x] = th.from[threadIdx.x];
    __syncthreads();
    if (i > 2 * W) return;
    const int delta = i - W, dist = th.both ? abs(delta) : max(-delta, 0);
    int b = dist;
    if (dist >= th.E) {
        int lo = 0, hi = th.n - 1 - th.E;       // thresholds there are
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (from[mid] <= dist) lo = mid + 1;
            else hi = mid;
        }
        b = th.E + lo;
    }
    if (th.both && delta > 0) b += th.n;
    tab[(int64_t)h * (2 * W + 1) + i] = bias[(int64_t)h * buckets + b];
    if (h == 0) bid[i] = (uint8_t)b;
}

// dist >= E reaches bucket E + t where log(dist / E) / log(max / E) * (n - E) + 1e-9 >= t, that is
// dist >= E (max / E)^((t - 1e-9) / (n - E)); the 1e-9 keeps distances that reach it exactly from falling short in their last place.
Thresholds thresholds(const cg_attn_desc &d)
{
    Thresholds th{};
    th.both = d.both != 0;
    th.n = d.both ? d.buckets / 2 : d.buckets;
    th.E = th.n / 2;
    const double ratio = (double)d.max_distance / th.E;
    for (int t = 1; t < th.n - th.E; ++t)
        th.from[t - 1] = (int)std::ceil(th.E * std::pow(ratio, (t - 1e-9) / (th.n - th.E)));
    return th;
}

int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

int check(const cg_attn_desc *d, int pass)
{
    if (!d || (d->type != CG_TYPE_FP32 && d->type != CG_TYPE_BF16)) return CG_EINVAL;
    if (d->B < 0 || d->Hq < 1 || d->Hkv < 1 || d->D < 1 || d->Hq % d->Hkv || d->Tq < 0 || d->Tk < 0) return CG_EINVAL;
    if (!(d->scale > 0.f) || !std::isfinite(d->scale) || d->buckets < 0) return CG_EINVAL;
    if (d->q_tok < 0 || d->q_head < 0 || d->k_tok < 0 || d->k_head < 0 || d->v_tok < 0 || d->v_head < 0 || d->o_tok < 0 || d->o_head < 0) return CG_EINVAL;
    if (d->buckets > 0) {
        const int n = d->both ? d->buckets / 2 : d->buckets;
        if (n < 2 || (d->both && d->buckets % 2) || d->max_distance <= n / 2) return CG_EINVAL;
        if (d->buckets > kMaxBuckets || d->max_distance > kMaxDistance) return CG_EUNSUPPORTED;
    }
    if (d->D > kAttnMaxD || d->Tq > kMaxRows || d->Tk > kMaxRows || d->Tq * d->Hq > kMaxRows || d->Tk * d->Hkv > kMaxRows) return CG_EUNSUPPORTED;
    // the blocks of the kernels whose X are queries, and keys (with the blocks that add up dbias); axes are cut only where these are few
    const int64_t Gp = d->buckets ? 1 : d->Hq / d->Hkv;
    if (d->Hq / Gp * (d->Tq * Gp / kAttnRows + d->B) > kMaxBlocks) return CG_EUNSUPPORTED;
    if (pass != CG_PASS_FWD && d->Hkv * (d->Tk / kAttnRows + d->B) + (int64_t)d->Hq * ((d->buckets + 15) / 16) > kMaxBlocks) return CG_EUNSUPPORTED;
    return CG_OK;
}

// Few X tiles leave most of the chip idle while each walks a long Y axis: the axis is then cut into chunks, a block each, and a
// second kernel joins what they found.
struct Split { int splits, chunk; };

// How a kernel over problems x tiles of X (an upper bound) is cut along Y: not at all where there are blocks for the chip (kFull), nor
// where Y is short (on average over the B sequences, and in all).  Otherwise into as many chunks as bring about kTarget blocks
// where the sequences are alike, of kMinChunk rows at least: a chunk's set-up and its partial result cost about what 64 rows do.  At most
// kMaxChunks, because the grid has room for them in every tile, whichever sequence is the long one: y being all sequences' rows, unlike
// sequences come out coarser (8 of 90 to 8000 keys, 19 513 in all: chunks of 320).
constexpr int kFull = 256, kTarget = 512, kMinChunk = 128, kMaxChunks = 64;
constexpr int64_t kPartBytes = 256ll << 20;

Split split_of(int64_t problems, int64_t tiles, int64_t y, int64_t B, int64_t row_bytes, int type)
{
    const int64_t blocks = problems * tiles;
    int64_t chunk = type == CG_TYPE_FP32 ? kMinChunk / 2 : kMinChunk;
    if (blocks == 0 || blocks >= kFull || (y < 4 * chunk && y < 2 * chunk * B)) return {1, 0};
    for (const int64_t least : {up(y / B * blocks / kTarget, 64), up((y + kMaxChunks - 1) / kMaxChunks, 64)})
        if (chunk < least) chunk = least;
    while (blocks * ((y + chunk - 1) / chunk) * kAttnRows * row_bytes > kPartBytes) chunk *= 2;
    const int64_t n = (y + chunk - 1) / chunk;
    return n > 1 ? Split{(int)n, (int)chunk} : Split{1, 0};
}

// How the pass is laid out and what it keeps in the workspace (offsets; bytes in all).
struct Plan {
    int Gp, tiles_q, tiles_k, W, DP;
    int gsplit;
    Split q, k;                 // of the kernels whose X are queries (forward, dq) and keys (dk, dv)
    size_t tab, bid, part_q, part_ml, part_k[2], delta, lse_b, log_l, dbias, bytes;
};

Plan plan_of(const cg_attn_desc &d, int pass)
{
    Plan p{};
    p.Gp = d.buckets ? 1 : d.Hq / d.Hkv;
    p.tiles_q = (int)(d.Tq * p.Gp / kAttnRows + d.B);
    p.tiles_k = (int)(d.Tk / kAttnRows + d.B);
    p.W = d.buckets ? d.max_distance : 0;
    p.DP = (int)up(d.D, 32);
    const int64_t Hr = d.Hq / p.Gp;
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const size_t here = (size_t)at;
        at += up(bytes, 256);
        return here;
    };
    if (d.buckets) {
        p.tab = take(d.Hq * (2ll * p.W + 1) * 4);
        p.bid = take(2ll * p.W + 1);
    }
    p.q = split_of(Hr, p.tiles_q, d.Tk, d.B, (p.DP + 2) * 4, d.type);
    const int64_t q_rows = p.q.splits > 1 ? Hr * p.tiles_q * p.q.splits * kAttnRows : 0;
    if (pass == CG_PASS_FWD) {
        p.part_q = take(q_rows * p.DP * 4);
        p.part_ml = take(q_rows * 2 * 4);
    } else {
        // with a bias a block walks the heads of its keys one after the other; where blocks are few each gets blocks of its own
        const int64_t G = d.Hq / d.Hkv, blocks_k = (int64_t)d.Hkv * p.tiles_k;
        p.gsplit = d.buckets && G > 1 && blocks_k < kFull && blocks_k * G * kAttnRows * 2 * p.DP * 4 <= kPartBytes ? (int)G : 1;
        p.k = split_of((int64_t)d.Hkv * p.gsplit, p.tiles_k, d.Tq * p.Gp, d.B, 2 * p.DP * 4, d.type);
        const int64_t k_rows = p.k.splits * p.gsplit > 1 ? blocks_k * p.gsplit * p.k.splits * kAttnRows : 0;
        p.part_q = take(q_rows * p.DP * 4);
        p.part_k[0] = take(k_rows * p.DP * 4);
        p.part_k[1] = take(k_rows * p.DP * 4);
        p.delta = take(d.Tq * d.Hq * 4);
        p.lse_b = take(d.Tq * d.Hq * 4);
        p.log_l = take(d.buckets ? d.Tq * d.Hq * 4 : 0);
        p.dbias = take((int64_t)d.Hq * p.tiles_q * p.q.splits * d.buckets * 4);
    }
    p.bytes = (size_t)at;
    return p;
}

bool tensor_ok(const void *p, int type, int64_t n)
{
    return n == 0 || (p && (reinterpret_cast<uintptr_t>(p) & (type == CG_TYPE_FP32 ? 3 : 1)) == 0);
}
// May a tensor [T][H][D] of these strides be written: no two of its elements in one place?
bool strides_ok(int64_t T, int64_t H, int64_t tok, int64_t head, int64_t D)
{
    if (T > H) std::swap(T, H), std::swap(tok, head);
    if (T < 1) return true;
    if ((T > 1 && tok < D) || (H > 1 && head < D)) return false;
    if (T == 1 || (tok - D) / head >= H - 1 || (head - D) / tok >= T - 1) return true;      // one inside the other
    for (int64_t i = 1; i < T; ++i) {       // T <= 2^15.5: i steps of tok, and the steps of head next to them
        const __int128 at = (__int128)i * tok, n = at / head;
        for (__int128 j = n; j <= n + 1 && j < H; ++j)
            if (const __int128 gap = at - j * head; gap < D && -gap < D) return false;
    }
    return true;
}
bool words_ok(const void *p, int64_t n) { return n == 0 || (p && (reinterpret_cast<uintptr_t>(p) & 3) == 0); }

AttnArgs args_of(const cg_attn_desc &d, const Plan &p, const void *q, const void *k, const void *v, const int32_t *cu_q, const int32_t *cu_k, char *ws)
{
    AttnArgs a{};
    a.q = q, a.k = k, a.v = v, a.cu_q = cu_q, a.cu_k = cu_k;
    a.q_tok = d.q_tok, a.q_head = d.q_head, a.k_tok = d.k_tok, a.k_head = d.k_head;
    a.v_tok = d.v_tok, a.v_head = d.v_head, a.o_tok = d.o_tok, a.o_head = d.o_head;
    a.B = d.B, a.Tq = (int)d.Tq, a.Tk = (int)d.Tk, a.Hq = d.Hq, a.Hkv = d.Hkv, a.G = d.Hq / d.Hkv, a.Gp = p.Gp, a.D = d.D;
    a.by_gp = make_fastdiv((uint32_t)p.Gp);
    a.scale = d.scale;
    a.causal = d.causal != 0;
    a.buckets = d.buckets;
    a.W = p.W;
    a.tiles = p.tiles_q;
    a.splits = p.q.splits, a.chunk = p.q.chunk, a.gsplit = 1;
    a.part[0] = reinterpret_cast<float *>(ws + p.part_q);
    a.part_ml = reinterpret_cast<float *>(ws + p.part_ml);
    a.yt = attn_dkdv_yt(d.type == CG_TYPE_BF16, p.DP);
    a.dma = attn_dma_ok(d.type, k, d.k_tok, 0, 1, d.D) && attn_dma_ok(d.type, v, d.v_tok, 0, 1, d.D) &&
            (d.type == CG_TYPE_FP32 || (d.k_head % 8 == 0 && d.v_head % 8 == 0));
    if (d.buckets) {
        a.btab = reinterpret_cast<const float *>(ws + p.tab);
        a.bid = reinterpret_cast<const uint8_t *>(ws + p.bid);
    }
    return a;
}
int table_launch(const cg_attn_desc &d, const Plan &p, const float *bias, char *ws, hipStream_t s)
{
    if (!d.buckets) return CG_OK;
    hipLaunchKernelGGL(bias_table_kernel, dim3((unsigned)(2 * p.W + 1 + 255) / 256, (unsigned)d.Hq), dim3(256), 0, s, thresholds(d), bias, d.buckets, p.W,
                       reinterpret_cast<float *>(ws + p.tab), reinterpret_cast<uint8_t *>(ws + p.bid));
    CG_HIP_TRY(hipGetLastError());
    return CG_OK;
}
int ws_check(const Plan &p, const void *ws, size_t ws_bytes)
{
    if (p.bytes && (!ws || !aligned16(ws))) return CG_EINVAL;
    return ws_bytes < p.bytes ? CG_ENOSPC : CG_OK;
}

}  // namespace
}  // namespace cg

using namespace cg;

extern "C" size_t cg_attn_workspace_bytes(const cg_attn_desc *d, int pass)
{
    if ((pass != CG_PASS_FWD && pass != CG_PASS_BWD_DATA) || check(d, pass) != CG_OK) return 0;
    return plan_of(*d, pass).bytes;
}

extern "C" int cg_attn_fwd(const cg_attn_desc *d, const void *q, const void *k, const void *v, const int32_t *cu_q, const int32_t *cu_k,
                           const float *bias, void *o, float *lse, void *o_rest, void *ws, size_t ws_bytes, void *stream)
{
    if (int rc = check(d, CG_PASS_FWD)) return rc;
    if (d->B == 0 || d->Tq == 0) return CG_OK;
    if (!tensor_ok(q, d->type, 1) || !tensor_ok(k, d->type, d->Tk) || !tensor_ok(v, d->type, d->Tk) || !tensor_ok(o, d->type, 1) || !words_ok(lse, 1) ||
        !words_ok(cu_q, 1) || !words_ok(cu_k, 1) || !words_ok(bias, d->buckets)) return CG_EINVAL;
    if (o_rest && (d->type != CG_TYPE_BF16 || !tensor_ok(o_rest, d->type, 1))) return CG_EINVAL;
    if (!strides_ok(d->Tq, d->Hq, d->o_tok, d->o_head, d->D)) return CG_EINVAL;
    const Plan p = plan_of(*d, CG_PASS_FWD);
    if (int rc = ws_check(p, ws, ws_bytes)) return rc;
    char *w = static_cast<char *>(ws);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (int rc = table_launch(*d, p, bias, w, s)) return rc;
    AttnArgs a = args_of(*d, p, q, k, v, cu_q, cu_k, w);
    a.o = o, a.o_rest = o_rest, a.lse = lse;
    if (int rc = attn_fwd_launch(a, d->type, s)) return rc;
    return a.splits > 1 ? attn_join_launch(a, d->type, s) : CG_OK;
}

extern "C" int cg_attn_bwd(const cg_attn_desc *d, const void *d_o, const void *q, const void *k, const void *v, const int32_t *cu_q,
                           const int32_t *cu_k, const float *bias, const void *o, const void *o_rest, const float *lse, void *dq,
                           void *dk, void *dv, float *dbias, void *ws, size_t ws_bytes, void *stream)
{
    if (int rc = check(d, CG_PASS_BWD_DATA)) return rc;
    if (!tensor_ok(q, d->type, d->Tq) || !tensor_ok(k, d->type, d->Tk) || !tensor_ok(v, d->type, d->Tk) || !tensor_ok(o, d->type, d->Tq) ||
        !tensor_ok(d_o, d->type, d->Tq) || !tensor_ok(dq, d->type, d->Tq) || !tensor_ok(dk, d->type, d->Tk) || !tensor_ok(dv, d->type, d->Tk) ||
        !words_ok(lse, d->Tq) || !words_ok(cu_q, d->B) || !words_ok(cu_k, d->B) || !words_ok(bias, d->buckets)) return CG_EINVAL;
    if (!strides_ok(d->Tq, d->Hq, d->q_tok, d->q_head, d->D) || !strides_ok(d->Tk, d->Hkv, d->k_tok, d->k_head, d->D) ||
        !strides_ok(d->Tk, d->Hkv, d->v_tok, d->v_head, d->D)) return CG_EINVAL;
    if ((o_rest && (d->type != CG_TYPE_BF16 || !tensor_ok(o_rest, d->type, 1))) || (dbias && (!d->buckets || !words_ok(dbias, 1)))) return CG_EINVAL;
    const Plan p = plan_of(*d, CG_PASS_BWD_DATA);
    if (int rc = ws_check(p, ws, ws_bytes)) return rc;
    char *w = static_cast<char *>(ws);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (int rc = table_launch(*d, p, bias, w, s)) return rc;
    AttnArgs a = args_of(*d, p, q, k, v, cu_q, cu_k, w);
    a.d_o = d_o, a.o_in = o, a.o_rest_in = o_rest, a.lse = const_cast<float *>(lse);
    a.dq = dq, a.dk = dk, a.dv = dv;
    a.delta = reinterpret_cast<float *>(w + p.delta);
    a.lse_b = reinterpret_cast<float *>(w + p.lse_b);
    a.log_l = reinterpret_cast<float *>(w + p.log_l);
    const bool any_q = d->B > 0 && d->Tq > 0, any_k = d->B > 0 && d->Tk > 0;
    if (dbias) {
        a.dbias = dbias;
        a.dbias_part = reinterpret_cast<float *>(w + p.dbias);
        a.dbias_parts = any_q ? p.tiles_q * p.q.splits : 0;
        a.dbias_splits = p.q.splits, a.dbias_chunk = p.q.chunk;
    }
    AttnArgs k_side = a;       // the dk/dv kernel's, which also adds up dbias
    if (any_q)
        if (int rc = attn_dq_launch(a, d->type, s)) return rc;
    k_side.tiles = any_k ? p.tiles_k : 0;
    k_side.dma = attn_dma_ok(d->type, q, d->q_tok, d->q_head, p.Gp, d->D) && attn_dma_ok(d->type, d_o, d->o_tok, d->o_head, p.Gp, d->D) &&
                 d->Tq * d->Hq < (1 << 29);
    k_side.splits = p.k.splits, k_side.chunk = p.k.chunk, k_side.gsplit = p.gsplit;
    k_side.part[0] = reinterpret_cast<float *>(w + p.part_k[0]), k_side.part[1] = reinterpret_cast<float *>(w + p.part_k[1]);
    if (any_k || dbias)
        if (int rc = attn_dkdv_launch(k_side, d->type, s)) return rc;
    return attn_join_bwd_launch(any_q && a.splits > 1 ? &a : nullptr, any_k && p.k.splits * p.gsplit > 1 ? &k_side : nullptr, d->type, s);
}
