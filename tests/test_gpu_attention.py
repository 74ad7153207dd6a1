"""Attention over packed sequences, with and without a bias by distance, forward and backward on the GPU, against its plain form
in 64 bits.  How far a result may be off is derived in sublayer_util.Attention."""
import pytest
import torch

import paper_1706_00095_amd as cg
from sublayer_util import DTYPES, Attention, half_step

pytestmark = pytest.mark.gpu


def inputs(dtype, lens_q, lens_k, Hq, Hkv, D, fused=False, shift=0, seed=1, lead=0, trail=0):
    """q, k, v, do as device tensors (`shift` elements off an allocation's start; fused: slices of one tensor; `lead`, `trail`
    tokens of NaN around the sequences) and in float64 on the host."""
    dt = DTYPES[dtype]
    g = torch.Generator().manual_seed(seed)
    Tq, Tk = sum(lens_q), sum(lens_k)

    def put(values, around):
        T, H, _ = values.shape
        flat = torch.full(((T + 2 * around) * H * D + shift,), float("nan"), dtype=dt, device="cuda")
        t = flat[shift:].view(T + 2 * around, H, D)
        t[around:around + T] = values.cuda()
        return t[around - lead:around + T + trail] if around else t

    def make(T, H, std=1.0):
        return torch.empty(T, H, D, dtype=torch.float64).normal_(0, std, generator=g).to(dt)

    vals = [make(Tq, Hq), make(Tk, Hkv), make(Tk, Hkv), make(Tq, Hq, 0.02)]
    around = max(lead, trail)
    if fused:
        both = put(torch.cat(vals[:3], 1), around)
        q, k, v = both[:, :Hq], both[:, Hq:Hq + Hkv], both[:, Hq + Hkv:]
    else:
        q, k, v = (put(t, around) for t in vals[:3])
    return (q, k, v, put(vals[3], around)), [t.double() for t in vals]


def lengths(lens, lead=0):
    return torch.tensor([0] + lens, device="cuda").cumsum(0).add(lead).int()


def like(t):
    """An output of t's shape and strides, filled with NaN."""
    n = 1 + sum((s - 1) * st for s, st in zip(t.shape, t.stride())) if t.numel() else 0
    return torch.full((n,), float("nan"), dtype=t.dtype, device="cuda").as_strided(t.shape, t.stride())


def call(x, B, cu_q, cu_k, scale, causal, bias, far, both, rest, train=True):
    q, k, v, do = x
    n = bias.shape[1] if bias is not None else 0
    o = torch.full(do.shape, float("nan"), dtype=q.dtype, device="cuda").as_strided(do.shape, do.stride())
    d = cg.attn_desc(q, k, v, o, B, scale, causal, n, far, both)
    lse = torch.full((q.shape[1], q.shape[0]), float("nan"), device="cuda")
    ws = torch.full((cg.cg_attn_workspace_bytes(d, cg.CG_PASS_FWD) + 16,), 255, dtype=torch.uint8, device="cuda")
    r = {"o": o, "lse": lse}
    rest = like(o) if rest else None
    cg.cg_attn_fwd(d, q, k, v, cu_q, cu_k, bias, o, lse, rest, ws)
    if train:
        r["dq"], r["dk"], r["dv"] = like(q), like(k), like(v)
        db = torch.full_like(bias, float("nan")) if bias is not None else None
        ws = torch.full((cg.cg_attn_workspace_bytes(d, cg.CG_PASS_BWD_DATA) + 16,), 255, dtype=torch.uint8, device="cuda")
        cg.cg_attn_bwd(d, do, q, k, v, cu_q, cu_k, bias, o, rest, lse, r["dq"], r["dk"], r["dv"], db, ws)
        if db is not None:
            r["dbias"] = db
    torch.cuda.synchronize()
    return r


def near(name, got, ref, tol, dtype):
    got = got.double().cpu()
    same = (got == ref) | (torch.isnan(got) & torch.isnan(ref))      # infinities
    d = (got - ref).abs()
    ok = same | (d <= half_step(dtype) * (ref.abs() + tol) + tol + 1e-30)
    assert ok.all(), (name, int((~ok).sum()), float(torch.nan_to_num(d[~ok], nan=float("inf")).max()), float(ref.abs().max()))


def check(r, a, dtype, trains=True):
    f32 = torch.float32
    near("o", r["o"], a.o, a.tol_o, dtype)
    near("lse", r["lse"], a.lse, a.tol_lse, f32)
    if trains:
        near("dq", r["dq"], a.dq, a.tol_dq, dtype)
        near("dk", r["dk"], a.dk, a.tol_dk, dtype)
        near("dv", r["dv"], a.dv, a.tol_dv, dtype)
        if "dbias" in r:
            near("dbias", r["dbias"], a.dbias, a.tol_dbias, f32)


def run(dtype, lens_q, lens_k, Hq, Hkv, D, causal, fused=False, shift=0, bias=0, far=0, both=False, rest=None, seed=1):
    x, vals = inputs(dtype, lens_q, lens_k, Hq, Hkv, D, fused, shift, seed)
    dt = DTYPES[dtype]
    rest = dt == torch.bfloat16 if rest is None else rest
    table = torch.empty(Hq, bias).normal_(0, 0.5, generator=torch.Generator().manual_seed(seed + 9)).cuda() if bias else None
    scale = D ** -0.5
    r = call(x, len(lens_q), lengths(lens_q), lengths(lens_k), scale, causal, table, far, both, rest)
    a = Attention(*vals, lens_q, lens_k, float(torch.tensor(scale, dtype=torch.float32)), causal, table.double().cpu() if bias else None, bias, far, both, dt, rest)
    check(r, a, dt)


ODD = [1, 0, 63, 64, 65, 127, 128, 129, 5, 0, 200]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("D", [1, 8, 17, 32, 33, 40, 48, 64, 72, 77, 96, 100, 128])
def test_head_sizes(dtype, causal, D):
    run(dtype, [70, 1, 129], [70, 1, 129], 2, 2, D, causal)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("fused", [False, True])
def test_lengths_at_the_borders_of_tiles(dtype, causal, fused):
    run(dtype, ODD, ODD, 2, 1, 64, causal, fused)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 1), (6, 2), (8, 1), (3, 3), (15, 3)])
def test_grouped_heads(dtype, causal, Hq, Hkv):
    run(dtype, [37, 300, 2], [37, 300, 2], Hq, Hkv, 40, causal)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("causal", [False, True])
def test_other_queries_than_keys(dtype, causal):
    """Fewer and more queries than keys: with a causal mask the first queries of the latter see nothing.  Either side empty."""
    run(dtype, [5, 100, 40, 0, 7, 200, 1], [300, 60, 0, 9, 7, 130, 1000], 4, 2, 64, causal)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shift", [1, 3, 4])
def test_tensors_off_the_alignment_of_wide_loads(dtype, shift):
    run(dtype, [70, 33], [70, 33], 2, 2, 64, True, True, shift)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("lens_q,lens_k,Hq,Hkv,D", [
    ([1], [5000], 4, 1, 64), ([1, 5, 16, 1], [4096, 1500, 777, 1], 16, 4, 64), ([3, 1], [1024, 2049], 2, 2, 128),
    ([130, 2], [1500, 64], 3, 1, 40), ([1, 0, 1], [0, 3000, 1200], 8, 8, 33)])
@pytest.mark.parametrize("causal", [False, True])
def test_few_queries_of_long_sequences(dtype, lens_q, lens_k, Hq, Hkv, D, causal):
    """The keys are cut into chunks and joined."""
    run(dtype, lens_q, lens_k, Hq, Hkv, D, causal)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_without_the_rest_of_o(dtype):
    run(dtype, [200, 31], [200, 31], 2, 2, 64, True, rest=False)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("causal,both,n,far", [(False, True, 32, 128), (True, False, 32, 128), (False, False, 8, 11), (True, True, 64, 200),
                                               (False, True, 4, 500), (True, False, 2, 2), (False, True, 256, 65)])
def test_bias_by_distance(dtype, causal, both, n, far):
    run(dtype, [300, 1, 65, 0], [300, 1, 65, 4], 4, 2, 48, causal, bias=n, far=far, both=both)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("D", [32, 64, 96, 128])
def test_bias_with_other_queries_than_keys(dtype, causal, D):
    run(dtype, [40, 100, 3], [300, 60, 1300], 2, 1, D, causal, bias=32, far=100, both=not causal)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_bias_of_minus_infinity_masks(dtype):
    """Distances whose bias is -inf are not seen; the type's lowest value alike where another distance is seen, and equally
    where nothing else is."""
    lens = [150, 33]
    x, vals = inputs(dtype, lens, lens, 2, 2, 64)
    for low in (float("-inf"), torch.finfo(torch.float32).min):
        table = torch.zeros(2, 8)
        table[0, 3:] = low           # head 0 sees three distances
        table[1, 0] = low            # head 1 does not see itself (nor, one-sided, what is behind it)
        r = call(x, 2, lengths(lens), lengths(lens), 0.125, True, table.cuda(), 20, False, dtype == "bf16")
        a = Attention(*vals, lens, lens, 0.125, True, table.double(), 8, 20, False, DTYPES[dtype], dtype == "bf16")
        near("o", r["o"], a.o, a.tol_o, DTYPES[dtype])
        if low == float("-inf"):
            a.tol_lse[:] = a.tol_lse.nan_to_num(posinf=0.0)
            check(r, a, DTYPES[dtype])
            assert bool((r["o"][0, 1] == 0).all() and r["lse"][1, 0] == float("-inf"))      # the first query of head 1 sees nothing


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("causal", [False, True])
def test_tokens_of_no_sequence_are_neither_read_nor_written(dtype, causal):
    """NaN before the first and behind the last sequence; outputs keep what they held there."""
    lens = [33, 100]
    x, vals = inputs(dtype, lens, lens, 4, 2, 40, lead=3, trail=5)
    r = call(x, 2, lengths(lens, 3), lengths(lens, 3), 0.2, causal, None, 0, False, False)
    T = sum(lens)
    for name in ("o", "dq", "dk", "dv"):
        assert torch.isnan(r[name][:3].float()).all() and torch.isnan(r[name][3 + T:].float()).all(), name
        r[name] = r[name][3:3 + T]
    assert torch.isnan(r["lse"][:, :3]).all() and torch.isnan(r["lse"][:, 3 + T:]).all()
    r["lse"] = r["lse"][:, 3:3 + T]
    a = Attention(*vals, lens, lens, float(torch.tensor(0.2)), causal, None, 0, 0, False, DTYPES[dtype], False)
    check(r, a, DTYPES[dtype])


def test_bad_lengths_stay_within_the_tensors():
    """Lengths that run past the tensors, backwards or overlap are cut: the call returns, and writes nothing outside."""
    x, _ = inputs("bf16", [100], [100], 2, 2, 64)
    for cu in ([0, 200], [-50, 60], [90, 10], [1000, 2000]):
        c = torch.tensor(cu, device="cuda").int()
        call(x, 1, c, c, 0.125, True, None, 0, False, True)
    c = torch.tensor([0, 70, 30, 1 << 30], device="cuda").int()
    call(x, 3, c, c, 0.125, False, None, 0, False, True)


def test_results_repeat_and_replay():
    """The same bits on every call, on another stream and from a captured graph, with a bias and without."""
    lens = [300, 17, 200]
    x, _ = inputs("bf16", lens, lens, 4, 2, 64)
    for n in (0, 32):
        table = torch.randn(4, n, generator=torch.Generator().manual_seed(3)).cuda() if n else None
        q, k, v, do = x
        cu = lengths(lens)
        o, rest, lse = torch.empty_like(q), torch.empty_like(q), torch.empty(4, q.shape[0], device="cuda")
        d = cg.attn_desc(q, k, v, o, 3, 0.125, n == 0, n, 128 if n else 0, n > 0)
        ws = [torch.empty(cg.cg_attn_workspace_bytes(d, p) + 16, dtype=torch.uint8, device="cuda") for p in (cg.CG_PASS_FWD, cg.CG_PASS_BWD_DATA)]
        dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
        db = torch.empty_like(table) if n else None
        outs = [t for t in (o, lse, dq, dk, dv, db) if t is not None]

        def step(stream=None):
            cg.cg_attn_fwd(d, q, k, v, cu, cu, table, o, lse, rest, ws[0], stream)
            cg.cg_attn_bwd(d, do, q, k, v, cu, cu, table, o, rest, lse, dq, dk, dv, db, ws[1], stream)

        def results():
            torch.cuda.synchronize()
            got = [t.clone() for t in outs]
            for t in outs:
                t.fill_(float("nan"))
            torch.cuda.synchronize()
            return got

        step()
        first = results()
        side = torch.cuda.Stream()
        step(side)
        assert all(torch.equal(a, b) for a, b in zip(first, results()))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
        for _ in range(3):
            graph.replay()
            assert all(torch.equal(a, b) for a, b in zip(first, results()))
            step()
            assert all(torch.equal(a, b) for a, b in zip(first, results()))


def test_gradients_against_differences():
    """Along a random direction the gradients give the change of <o, do>, by central differences in 64 bits of the plain form;
    the library's fp32 gradients are off by less than 2^-12, the differences by h^2."""
    lens, H, D, h = [60, 35], 2, 32, 1e-4
    x, vals = inputs("fp32", lens, lens, H, H, D)
    table = torch.randn(H, 16, generator=torch.Generator().manual_seed(3))
    r = call(x, 2, lengths(lens), lengths(lens), 0.25, True, table.cuda(), 40, False, False)
    g = torch.Generator().manual_seed(4)
    dirs = [torch.empty_like(t).normal_(0, 1, generator=g) for t in vals[:3]] + [torch.empty(H, 16, dtype=torch.float64).normal_(0, 1, generator=g)]
    along = sum(float((r[n].double().cpu() * t).sum()) for n, t in zip(("dq", "dk", "dv", "dbias"), dirs))
    size = sum(float((r[n].double().cpu() * t).norm()) for n, t in zip(("dq", "dk", "dv", "dbias"), dirs))

    def value(e):
        q, k, v = (t + e * s for t, s in zip(vals[:3], dirs))
        a = Attention(q, k, v, vals[3], lens, lens, 0.25, True, table.double() + e * dirs[3], 16, 40, False, torch.float32, False)
        return float((a.o * vals[3]).sum())
    assert abs(along - (value(h) - value(-h)) / (2 * h)) < 1e-3 * size


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_cache_longer_than_32_bits_of_bytes(dtype):
    """Keys and values as slices of one tensor of over 4 GiB, the last tokens beyond 2^32 bytes."""
    dt, D, Tk, tok, Tq = DTYPES[dtype], 64, 36000, 1 << (16 if dtype == "bf16" else 15), 3
    wide = torch.empty(Tk, tok, dtype=dt, device="cuda")
    assert wide.numel() * wide.element_size() > 1 << 32
    g = torch.Generator().manual_seed(1)
    vals = [torch.empty(T, 1, D, dtype=torch.float64).normal_(0, s, generator=g).to(dt) for T, s in ((Tq, 1), (Tk, 1), (Tk, 1), (Tq, 0.02))]
    q, do = vals[0].cuda(), vals[3].cuda()
    k, v = wide[:, None, :D], wide[:, None, 4096:4096 + D]
    k.copy_(vals[1].cuda())
    v.copy_(vals[2].cuda())
    dwide = torch.full_like(wide, float("nan"))
    dk, dv = dwide[:, None, :D], dwide[:, None, 4096:4096 + D]
    o, dq, rest = torch.empty_like(q), torch.empty_like(q), torch.empty_like(q) if dtype == "bf16" else None
    d = cg.attn_desc(q, k, v, o, 1, 0.125, True)
    lse = torch.empty(1, Tq, device="cuda")
    ws = [torch.empty(cg.cg_attn_workspace_bytes(d, p) + 16, dtype=torch.uint8, device="cuda") for p in (cg.CG_PASS_FWD, cg.CG_PASS_BWD_DATA)]
    cq, ck = lengths([Tq]), lengths([Tk])
    cg.cg_attn_fwd(d, q, k, v, cq, ck, None, o, lse, rest, ws[0])
    cg.cg_attn_bwd(d, do, q, k, v, cq, ck, None, o, rest, lse, dq, dk, dv, None, ws[1])
    a = Attention(*[t.double() for t in vals], [Tq], [Tk], 0.125, True, None, 0, 0, False, dt, dtype == "bf16")
    check({"o": o, "lse": lse, "dq": dq, "dk": dk, "dv": dv}, a, dt)
    assert torch.isnan(dwide[:, D:4096].float()).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_strides_wider_than_a_buffer_of_a_tile(dtype):
    """Tokens more than 2^22 elements apart, and heads outside tokens (all tokens of a head together)."""
    dt, T, H, D = DTYPES[dtype], 20, 2, 32
    x, vals = inputs(dtype, [T], [T], H, H, D)
    far = torch.zeros(T * ((1 << 22) + 8), dtype=dt, device="cuda")
    q, k, v, do = x
    k2 = far.as_strided((T, H, D), ((1 << 22) + 8, D, 1))
    k2.copy_(k)
    by_head = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in (q, v, do)]
    a = Attention(*vals, [T], [T], 0.25, False, None, 0, 0, False, dt, False)
    check(call((by_head[0], k2, by_head[1], by_head[2]), 1, lengths([T]), lengths([T]), 0.25, False, None, 0, False, False), a, dt)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("bias", [0, 32])
def test_heads_packed_in_memory_orders_of_their_own(dtype, bias):
    """Grouped heads whose query heads lie outside the tokens: packed rows are then not in the order of their addresses."""
    dt, lens, Hq, Hkv, D = DTYPES[dtype], [70, 9], 4, 2, 64
    x, vals = inputs(dtype, lens, lens, Hq, Hkv, D)
    q, k, v, do = (t.transpose(0, 1).contiguous().transpose(0, 1) for t in x)
    table = torch.randn(Hq, bias, generator=torch.Generator().manual_seed(2)).cuda() if bias else None
    a = Attention(*vals, lens, lens, 0.125, True, table.double().cpu() if bias else None, bias, 100, False, dt, dtype == "bf16")
    check(call((q, k, v, do), 2, lengths(lens), lengths(lens), 0.125, True, table, 100 if bias else 0, False, dtype == "bf16"), a, dt)


@pytest.mark.parametrize("far", [1024, 1025, 3000])
def test_bias_of_far_distances(far):
    """On both sides of the number of distances whose sums a wave keeps one by one."""
    run("bf16", [900, 130], [1400, 130], 2, 1, 64, False, bias=32, far=far, both=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_bias_whose_exponential_overflows(dtype):
    """Softmax does not change with a constant: tables about 300 (and -300), with rows and keys behind the ends of tiles."""
    lens = [33, 70]
    x, vals = inputs(dtype, lens, lens, 2, 1, 32)
    for shift in (300.0, -300.0):
        table = torch.randn(2, 16, generator=torch.Generator().manual_seed(2)) + shift
        a = Attention(*vals, lens, lens, 0.125, False, table.double(), 16, 50, True, DTYPES[dtype], dtype == "bf16")
        check(call(x, 2, lengths(lens), lengths(lens), 0.125, False, table.cuda(), 50, True, dtype == "bf16"), a, DTYPES[dtype])


def test_many_sequences():
    """More sequences than a wave looks through at once, some of them empty."""
    lens = [(7 * i) % 13 for i in range(150)]
    run("bf16", lens, lens, 2, 1, 32, True)
    run("fp32", lens, [n + 3 for n in lens], 1, 1, 32, False, bias=8, far=9)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("bias", [0, 16])
def test_long_axes_of_many_unequal_sequences(dtype, causal, bias):
    """Sequences cut into different numbers of chunks, one or more tiles each, more of them than a wave looks through at once."""
    lens_q, lens_k = [1, 0, 300, 2, 140], [700, 64, 1500, 0, 129]
    run(dtype, lens_q, lens_k, 2, 1, 40, causal, bias=bias, far=64)
    many = [(i % 3) for i in range(70)] + [260]
    run(dtype, many, [n + 5 * (i % 2) for i, n in enumerate(many[:-1])] + [2000], 2, 1, 32, causal, bias=bias, far=64)


def test_overlapping_lengths_of_cut_axes():
    """More items than there is room for: the call returns, and writes nothing outside."""
    x, _ = inputs("bf16", [300], [3000], 2, 1, 64)
    cu_q, cu_k = (torch.tensor([0, n] * 40 + [0], device="cuda").int() for n in (300, 3000))
    table = torch.zeros(2, 8, device="cuda")
    for bias in (None, table):
        call(x, 80, cu_q, cu_k, 0.125, False, bias, 9 if bias is not None else 0, True, True)


@pytest.mark.parametrize("dtype,D,bias", [("bf16", 33, 0), ("bf16", 64, 0), ("bf16", 64, 8), ("fp32", 32, 0), ("fp32", 32, 8)])
@pytest.mark.parametrize("lens_k", [None, 40, -40])
def test_many_tiles_under_a_causal_mask(dtype, D, bias, lens_k):
    """More blocks than the chip holds at once, with sequences of unlike lengths, and as many as it holds."""
    lens = [400, 1, 0, 130, 257, 700, 65]
    for H in (48, 16):
        run(dtype, lens, [max(n + (lens_k or 0), 0) for n in lens], H, H, D, True, bias=bias, far=30)
