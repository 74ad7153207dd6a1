"""Linear layers against their 64-bit form: every kernel, odd sizes, strides, epilogues, sums that are whole numbers bit for bit."""
import pytest
import torch

import block_util as bu

pytestmark = pytest.mark.gpu


def _cg():
    import paper_1706_00095_amd as cg
    return cg


def _ws(n):
    return torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") if n else None


class Layer:
    """A layer's tensors on the host in 64 bits and on the device."""

    def __init__(self, dtype, M, K, N, act="none", act_in="none", bias=True, residual=False, pad=0, values=None, seed=1):
        self.dt, self.M, self.K, self.N, self.pad = bu.DTYPES[dtype], M, K, N, pad
        make = values or (lambda shape, i: bu.normal(shape, self.dt, seed + i, [1.0, K ** -0.5, 0.5, 1.0, 0.1, 1.0, 0.1][i]))
        h = dict(x=make((M, K), 0), w=make((N, K), 1), bias=make((N,), 2).float().double() if bias else None, residual=make((M, N), 3) if residual else None,
                 dz=make((M, N), 4), z_in=make((M, K), 5) if act_in != "none" else None, add=make((M, K), 6) if residual else None)
        self.h = h
        self.d = {k: v.float().cuda() if k == "bias" else bu.wide(v, pad, self.dt)[0] for k, v in h.items() if v is not None}
        self.act, self.act_in = act, act_in
        self.desc = _cg().linear_desc(self.d["x"], self.d["w"], act, act_in)

    def out(self, rows, cols):
        return bu.wide(torch.full((rows, cols), 7.0), self.pad, self.dt, fill=5.0)

    def fwd(self, keep=True):
        cg, d = _cg(), self.d
        (y, all_y), (z, all_z) = self.out(self.M, self.N), self.out(self.M, self.N)
        cg.cg_linear_fwd(self.desc, d["x"], d["w"], d.get("bias"), d.get("residual"), y, z if keep else None, _ws(cg.cg_linear_workspace_bytes(self.desc, cg.CG_PASS_FWD)))
        for t in (all_y, all_z):
            assert bool((t[:, self.N:] == 5.0).all()), "wrote between rows"
        return y, z

    def dx(self, z_in=None):
        cg, d = _cg(), self.d
        dx, all_dx = self.out(self.M, self.K)
        cg.cg_linear_bwd_data(self.desc, d["dz"], d["w"], z_in if z_in is not None else d.get("z_in"), d.get("add"), dx,
                              _ws(cg.cg_linear_workspace_bytes(self.desc, cg.CG_PASS_BWD_DATA)))
        assert bool((all_dx[:, self.K:] == 5.0).all()), "wrote between rows"
        return dx

    def dw(self, x=None, bias=True):
        cg = _cg()
        dw, db = torch.full((self.N, self.K), 7.0, device="cuda"), torch.full((self.N,), 7.0, device="cuda")
        cg.cg_linear_bwd_weight(self.desc, self.d["dz"], x if x is not None else self.d["x"], dw, db if bias else None,
                                _ws(cg.cg_linear_workspace_bytes(self.desc, cg.CG_PASS_BWD_WEIGHT)))
        return dw, db

    def packed(self, name):
        cg, t = _cg(), self.d[name]
        p = cg.packed8_like(t)
        cg.cg_pack8(t, p)
        return p


def check(L, pack=False):
    h = L.h
    y, z = L.fwd()
    want_y, tol_y, want_z, tol_z = bu.linear(h["x"], h["w"], h["bias"], h["residual"], L.act, L.dt)
    bu.near(z, want_z, tol_z, "z")
    bu.near(y, want_y, tol_y, "y")
    z_in, x = h["z_in"], h["x"]
    if pack:
        x = bu.packed(x)[2]
        z_in = None if z_in is None else bu.packed(z_in)[2]
    got = L.dx(L.packed("z_in") if pack and z_in is not None else None)
    bu.near(got, *bu.linear_dx(h["dz"], h["w"], z_in, L.act_in, h["add"], L.dt), "dx")
    dw, db = L.dw(L.packed("x") if pack else None)
    bu.near(dw, *bu.linear_dw(h["dz"], x), "dw")
    bu.near(db, h["dz"].sum(0), (L.M / 8 + 300) * bu.U * h["dz"].abs().sum(0), "dbias")


SIZES = [  # M, K, N, pad
    (1, 1, 1, 0), (1, 8, 16, 0), (2, 33, 17, 3), (7, 130, 8, 0), (16, 256, 40, 8), (17, 100, 33, 1), (32, 515, 129, 0), (33, 64, 128, 0), (64, 72, 200, 8),
    (127, 31, 257, 5), (128, 128, 128, 0), (129, 264, 136, 0), (300, 1000, 72, 8), (300, 7, 130, 0), (5, 3000, 9, 0), (40, 2056, 24, 0),
]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("M,K,N,pad", SIZES)
def test_sizes(dtype, M, K, N, pad):
    check(Layer(dtype, M, K, N, pad=pad, seed=M + K + N))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("M,K,N,pad", [(3, 40, 50, 0), (200, 48, 136, 0), (130, 45, 77, 3), (140, 1500, 40, 0)])
def test_epilogues(dtype, act, M, K, N, pad):
    """Every activation, forward and through the one that made the inputs, with a residual and an added gradient."""
    check(Layer(dtype, M, K, N, act, act, True, True, pad, seed=9))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("M,K,N,pad,act_in", [(1, 5, 3, 0, "none"), (70, 96, 40, 0, "gelu"), (129, 200, 130, 5, "silu"), (513, 264, 136, 0, "relu"), (1000, 31, 8, 2, "gelu")])
def test_packed(dtype, M, K, N, pad, act_in):
    """The backward pass from what 8 bits keep of the inputs."""
    check(Layer(dtype, M, K, N, "none", act_in, True, False, pad, seed=4), pack=True)


@pytest.mark.parametrize("dtype,M,K,N,pad,pack", [
    ("fp32", 2040, 250, 2044, 1, False), ("fp32", 2040, 2044, 250, 0, False), ("fp32", 250, 2044, 2040, 0, True), ("fp32", 256, 9216, 4096, 0, False),
    ("bf16", 2048, 2048, 2048, 0, False), ("bf16", 2048, 2048, 2048, 0, True), ("bf16", 2045, 2047, 2041, 3, False), ("bf16", 2045, 2047, 2041, 3, True),
    ("bf16", 128, 8192, 6144, 0, False), ("bf16", 2100, 2111, 2077, 3, False), ("bf16", 2100, 2111, 2077, 0, True), ("bf16", 2104, 2112, 2080, 0, True)])
def test_tiles_of_128(dtype, M, K, N, pad, pack):
    """Products for which tiles of 128 are taken, whole or with a k that is cut."""
    check(Layer(dtype, M, K, N, "gelu", "silu", True, True, pad, seed=11), pack)


@pytest.mark.parametrize("M,K,N", [(2048, 2104, 2056), (2050, 2048, 4096)])
@pytest.mark.parametrize("pack", [False, True])
def test_large_tiles_whole_numbers(M, K, N, pack):
    """Tiles of 256, where every sum is a whole number below 2^24: bit for bit."""
    L = Layer("bf16", M, K, N, bias=True, residual=True, values=lambda s, i: bu.whole(s, 3, 20 + i))
    h = {k: None if v is None else v.float() for k, v in L.h.items()}       # exact in fp32 in any order
    y, z = L.fwd()
    want = h["x"] @ h["w"].T + h["bias"]
    assert torch.equal(z.cpu(), want.bfloat16()) and torch.equal(y.cpu(), (want + h["residual"]).bfloat16())
    assert torch.equal(L.dx().cpu(), (h["dz"] @ h["w"] + h["add"]).bfloat16())
    dw, db = L.dw(L.packed("x") if pack else None)
    assert torch.equal(dw.cpu(), h["dz"].T @ h["x"]) and torch.equal(db.cpu(), h["dz"].sum(0))


@pytest.mark.parametrize("M,K,N", [(4096, 136, 4096), (4104, 200, 4088), (4096, 72, 4096), (4096, 4096, 136), (136, 4096, 4096), (72, 4096, 4096), (8, 4096, 4096)])
def test_large_tiles_of_few_steps(M, K, N):
    """Tiles of 256 whose k ends within their first steps."""
    L = Layer("bf16", M, K, N, bias=True, residual=False, values=lambda s, i: bu.whole(s, 3, 60 + i))
    h = {k: None if v is None else v.float() for k, v in L.h.items()}
    y, _ = L.fwd()
    assert torch.equal(y.cpu(), (h["x"] @ h["w"].T + h["bias"]).bfloat16())
    assert torch.equal(L.dx().cpu(), (h["dz"] @ h["w"]).bfloat16())
    dw, db = L.dw()
    assert torch.equal(dw.cpu(), h["dz"].T @ h["x"]) and torch.equal(db.cpu(), h["dz"].sum(0))


@pytest.mark.parametrize("act,act_in,packed", [("gelu", "silu", False), ("silu", "gelu", True), ("relu", "relu", False)])
def test_large_tiles_with_epilogues(act, act_in, packed):
    """Tiles of 256 with all that an epilogue has, rows of wider tensors and tiles that reach past the last row and column."""
    L = Layer("bf16", 2056, 1064, 4104, act, act_in, True, True, 8, seed=12)
    check(L, pack=packed)


def test_large_tiles_in_a_graph():
    """Captured, and replayed between eager calls: the same bits."""
    L = Layer("bf16", 2048, 2048, 4096, "gelu", "none", seed=2)
    cg, d = _cg(), L.d
    y, dw, db = torch.empty(L.M, L.N, dtype=L.dt, device="cuda"), torch.empty(L.N, L.K, device="cuda"), torch.empty(L.N, device="cuda")
    x8, ws = L.packed("x"), _ws(cg.cg_linear_workspace_bytes(L.desc, cg.CG_PASS_BWD_WEIGHT))

    def into():
        cg.cg_linear_fwd(L.desc, d["x"], d["w"], d["bias"], None, y)
        cg.cg_linear_bwd_weight(L.desc, d["dz"], x8, dw, db, ws)

    into()
    first = [t.clone() for t in (y, dw, db)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        into()
    for _ in range(3):
        for t in (y, dw, db):
            t.fill_(3.0)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, (y, dw, db)))
        into()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("M,K,N,pad", [(1, 4096, 48, 0), (16, 1000, 100, 8), (31, 77, 130, 1), (200, 520, 136, 0), (333, 129, 65, 2), (128, 4096, 128, 0)])
def test_whole_numbers(dtype, M, K, N, pad):
    L = Layer(dtype, M, K, N, bias=True, residual=True, pad=pad, values=lambda s, i: bu.whole(s, 3, 40 + i))
    h = {k: None if v is None else v.float() for k, v in L.h.items()}
    y, z = L.fwd()
    want = h["x"] @ h["w"].T + h["bias"]
    assert torch.equal(z.cpu(), want.to(L.dt)) and torch.equal(y.cpu(), (want + h["residual"]).to(L.dt))
    assert torch.equal(L.dx().cpu(), (h["dz"] @ h["w"] + h["add"]).to(L.dt))
    for x in (None, L.packed("x")):
        dw, db = L.dw(x)
        assert torch.equal(dw.cpu(), h["dz"].T @ h["x"]) and torch.equal(db.cpu(), h["dz"].sum(0))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_no_tokens(dtype):
    cg, dt = _cg(), bu.DTYPES[dtype]
    x, w, dz = torch.empty(0, 24, dtype=dt, device="cuda"), torch.ones(40, 24, dtype=dt, device="cuda"), torch.empty(0, 40, dtype=dt, device="cuda")
    d = cg.linear_desc(x, w, "gelu")
    y = torch.empty(0, 40, dtype=dt, device="cuda")
    cg.cg_linear_fwd(d, x, w, None, None, y)
    cg.cg_linear_bwd_data(d, dz, w, None, None, x)
    dw, db = torch.full((40, 24), 7.0, device="cuda"), torch.full((40,), 7.0, device="cuda")
    cg.cg_linear_bwd_weight(d, dz, x, dw, db)
    assert not dw.any() and not db.any()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("M", [5, 150])
def test_not_finite(dtype, M):
    """What is not finite stays in the rows and columns that meet it."""
    L = Layer(dtype, M, 40, 50, "gelu", "gelu", seed=3)
    L.d["x"][2, 5], L.d["w"][7, 3], L.d["dz"][3, 4] = float("nan"), float("inf"), float("nan")
    y, _ = L.fwd()
    bad = ~torch.isfinite(y).cpu()
    assert bad[2].all() and not bad[[i for i in range(M) if i != 2]][:, [j for j in range(50) if j != 7]].any()
    dw, db = L.dw()
    assert torch.isnan(db).nonzero().flatten().tolist() == [4]
    bad = ~torch.isfinite(dw).cpu()
    assert bad[4].all() and bad[:, 5].all() and int(bad.sum()) == 40 + 50 - 1


def test_slopes_far_out():
    """Activations and slopes where an exponential leaves its range."""
    cg = _cg()
    z = torch.tensor([[-3e38, -1e4, -90.0, -40.0, -15.0, -6.0, -1.0, -1e-30, 0.0, 1e-30, 1.0, 6.0, 15.0, 40.0, 90.0, 1e4]], device="cuda")
    one, eye = torch.ones_like(z), torch.eye(16, device="cuda")
    for act in ("relu", "gelu", "silu"):
        dz = torch.empty_like(z)
        cg.cg_act_bwd(act, one, z, dz)
        bu.near(dz, bu.slope(z.double().cpu(), act), bu.ACT, f"slope of {act}")
        v = z.clamp(min=-1e4)
        y = torch.empty_like(z)
        cg.cg_linear_fwd(cg.linear_desc(v, eye, act), v, eye, None, None, y)
        bu.near(y, bu.act(v.double().cpu(), act), bu.ACT * v.abs().double().cpu().clamp(max=64) + 2 * bu.U * bu.act(v.double().cpu(), act).abs(), act)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (5, 33, 3), (130, 264, 0)])
def test_act_bwd(dtype, act, rows, cols, pad):
    cg, dt = _cg(), bu.DTYPES[dtype]
    dy, z = bu.normal((rows, cols), dt, 1), bu.normal((rows, cols), dt, 2)
    (out, whole_out), dz_in, z_d = bu.wide(dy, pad, dt, fill=5.0), bu.wide(dy, pad, dt)[0], bu.wide(z, pad, dt)[0]
    p = cg.packed8_like(z_d)
    cg.cg_pack8(z_d, p)
    for kept, value in ((z_d, z), (p, bu.packed(z)[2])):
        out.fill_(7.0)
        cg.cg_act_bwd(act, dz_in, kept, out)
        want = dy * bu.slope(value, act)
        bu.near(out, want, bu.ACT * dy.abs() + (bu.half_step(dt) + bu.U) * want.abs(), "dz")
        assert bool((whole_out[:, cols:] == 5.0).all())


def test_act_bwd_of_many():
    """More than 2^31 elements, in place."""
    cg, rows, cols = _cg(), (1 << 16) + 3, (1 << 15) + 40
    dy, z = bu.normal((40, cols), torch.bfloat16, 1), bu.normal((40, cols), torch.bfloat16, 2)
    g, zd = (torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for t, values in ((g, dy), (zd, z)):
        t[:20], t[-20:] = values[:20].bfloat16().cuda(), values[20:].bfloat16().cuda()
    p = cg.packed8_like(zd)
    cg.cg_pack8(zd, p)
    del zd
    cg.cg_act_bwd("silu", g, p, g)
    want = dy * bu.slope(bu.packed(z)[2], "silu")
    bu.near(torch.cat([g[:20], g[-20:]]), want, bu.ACT * dy.abs() + (bu.half_step(torch.bfloat16) + bu.U) * want.abs(), "dz")
    assert not g[20:-20].any()


def test_two_streams_at_once():
    """Calls on two streams, a workspace each, that run beside each other: the bits of calls one after the other."""
    layers = [Layer(t, 300, 520, 264, "gelu", "silu", True, True, seed=i) for i, t in enumerate(("bf16", "fp32"))]
    want = [[*L.fwd(), L.dx(), *L.dw()] for L in layers]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in layers], [[], []]
    for _ in range(5):
        for i, L in enumerate(layers):
            with torch.cuda.stream(streams[i]):
                got[i] = [*L.fwd(), L.dx(), *L.dw()]
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_gradients_by_differences():
    """dx and dw against central differences of a sum over y, in fp32 through the kernels themselves."""
    cg = _cg()
    L = Layer("fp32", 40, 24, 36, "none", "none", seed=6)
    dx, (dw, db) = L.dx().double().cpu(), L.dw()
    x, w = L.d["x"], L.d["w"]
    coef = L.h["dz"]

    def total():
        y, _ = L.fwd(keep=False)
        return float((y.double().cpu() * coef).sum())

    for t, g, at in ((x, dx, (3, 7)), (x, dx, (39, 23)), (w, dw.double().cpu(), (0, 0)), (w, dw.double().cpu(), (35, 11))):
        h = 0.25          # the layer is linear: the difference is exact but for roundings
        old = float(t[at])
        t[at] = old + h
        up = total()
        t[at] = old - h
        down = total()
        t[at] = old
        # both sums are off by sum_error and a rounding of every y; divided by 2 h
        size = float((bu.sum_error(L.h["x"], L.h["w"].T) * coef.abs()).sum()) + 4 * bu.U * float((L.h["x"].abs() @ L.h["w"].abs().T * coef.abs()).sum())
        assert abs((up - down) / (2 * h) - float(g[at])) <= 2 * size / (2 * h) + 1e-6, at


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("M,K,N", [(9, 300, 50), (150, 1064, 136)])
def test_same_bits_and_graphs(dtype, M, K, N):
    """Run to run, on another stream and in a captured graph that is replayed between eager calls: the same bits."""
    L = Layer(dtype, M, K, N, "gelu", "silu", True, True, seed=8)

    def all_of():
        y, z = L.fwd()
        return [y, z, L.dx(), *L.dw()]

    first = [t.clone() for t in all_of()]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        again = all_of()
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(a, b) for a, b in zip(first, again))

    cg, d = _cg(), L.d
    y, z, dx = (torch.empty(a, b, dtype=L.dt, device="cuda") for a, b in ((M, N), (M, N), (M, K)))
    dw, db = torch.empty(N, K, device="cuda"), torch.empty(N, device="cuda")
    ws = _ws(max(16, *(cg.cg_linear_workspace_bytes(L.desc, p) for p in (0, 1, 2))))

    def into():
        cg.cg_linear_fwd(L.desc, d["x"], d["w"], d["bias"], d["residual"], y, z, ws)
        cg.cg_linear_bwd_data(L.desc, d["dz"], d["w"], d["z_in"], d["add"], dx, ws)
        cg.cg_linear_bwd_weight(L.desc, d["dz"], d["x"], dw, db, ws)

    with torch.cuda.stream(s):
        into()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        into()
    for _ in range(3):
        for t in (y, z, dx, dw, db):
            t.fill_(3.0)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, (y, z, dx, dw, db)))
        all_of()


@pytest.mark.parametrize("M", [9, 1030])
def test_far_rows(M):
    """Rows that lie more than 2^31 elements from the first."""
    cg, K, N = _cg(), 40, 48
    ld = (1 << 31) // (M - 2) // 8 * 8
    big = torch.empty(M * ld, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(big, (M, K), (ld, 1))
    values = bu.whole((M, K), 3, 1)
    x.copy_(values.bfloat16().cuda())
    w, dz = bu.whole((N, K), 3, 2), bu.whole((M, N), 3, 3)
    wd, dzd = w.bfloat16().cuda(), dz.bfloat16().cuda()
    d = cg.linear_desc(x, wd)
    y = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    cg.cg_linear_fwd(d, x, wd, None, None, y, None, _ws(cg.cg_linear_workspace_bytes(d, 0)))
    assert torch.equal(y.cpu(), (values @ w.T).bfloat16())
    dw = torch.empty(N, K, device="cuda")
    cg.cg_linear_bwd_weight(d, dzd, x, dw, None, _ws(cg.cg_linear_workspace_bytes(d, 2)))
    assert torch.equal(dw.cpu(), (dz.T @ values).float())
    cg.cg_linear_bwd_data(d, dzd, wd, None, None, x, _ws(cg.cg_linear_workspace_bytes(d, 1)))
    assert torch.equal(x.cpu(), (dz @ w).bfloat16())


@pytest.mark.parametrize("M,K,N", [(100, 70, 72), (300, 1500, 330), (20, 70, 72)])
def test_ends_of_the_range(M, K, N):
    """fp32 operands near the smallest numbers, off by half of 2^-133 where their third piece ends there, and up to where they count as infinite."""
    L, most = Layer("fp32", M, K, N, bias=False), float.fromhex("0x1.fefffep127")

    def near(size_x, size_w, off):
        h = dict(L.h)
        for k, size in (("x", size_x), ("dz", size_x), ("w", size_w)):
            h[k] = (h[k] * size).clamp(-most, most).float().double()
            L.d[k].copy_(h[k])
        y, _ = L.fwd()
        bu.near(y, h["x"] @ h["w"].T, bu.sum_error(h["x"], h["w"].T) + off * h["w"].abs().sum(1) + bu.U * (h["x"] @ h["w"].T).abs(), "y")
        bu.near(L.dx(), h["dz"] @ h["w"], bu.sum_error(h["dz"], h["w"]) + off * h["w"].abs().sum(0) + bu.U * (h["dz"] @ h["w"]).abs(), "dx")

    near(2.0 ** -122, 2.0 ** 30, 2.0 ** -134)
    near(2.0 ** 127, 2.0 ** -30, 0.0)          # many are clamped to the largest that has three pieces


def test_gelu_far_down_in_bf16():
    """gelu of a bf16 result relative to itself where it is small: its rounding and what its power of two is off by there."""
    cg = _cg()
    z = torch.linspace(-9, 9, 16 * 128).view(128, 16).bfloat16().cuda()
    y = torch.empty_like(z)
    eye = torch.eye(16, device="cuda").bfloat16()
    cg.cg_linear_fwd(cg.linear_desc(z, eye, "gelu"), z, eye, None, None, y, None, _ws(cg.cg_linear_workspace_bytes(cg.linear_desc(z, eye, "gelu"), 0)))
    v = z.double().cpu()
    want = v * torch.erfc(-v / 2 ** 0.5) / 2          # as far down as 64 bits go
    off = torch.where(v > -5.5, 2.6e-5, torch.where(v > -7, 1.8e-4, 1e-2)) + 4 * bu.U
    bu.near(y, want, (off * (1 + bu.half_step(torch.bfloat16)) + bu.half_step(torch.bfloat16)) * want.abs(), "gelu")
