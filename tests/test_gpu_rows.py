"""Dropout from the counter-based generator, layer norm and the two joined with the residual addition, on the GPU, against
their plain forms in 64 bits.

Tolerances.  Every result is one rounding of its type (half a step) of a sum held in fp32.  A row's sums are added in at
most 8 * 4 (a lane's elements) + 6 (lanes) + 8 (waves) = 46 additions in a row, or cols / 1024 + 6 + 16 in the kernel for
long rows, and a value passes through fewer than 16 further roundings; what follows uses 64 + cols / 1024 roundings of
2^-24 of the largest terms that enter the value.  Column sums are added over the rows of a block in order (at most
rows / blocks + 8, below 64 here), then over at most 512 / 16 + 16 blocks: 128 roundings of the sum of magnitudes."""
import numpy as np
import pytest
import torch

import paper_1706_00095_amd as cg
from sublayer_util import DTYPES, half_step, keep_factors, norm, norm_bwd, rows_of

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
SEED, OFFSET = 0x9E3779B97F4A7C15, 0x1_2345_6789

# widths at the borders of the kernels (512, 1024, 2048, 4096, 8192, 16384), odd ones, one column; few rows and many
SHAPES = [(1, 1), (3, 1), (2, 7), (5, 8), (33, 9), (1, 256), (9, 511), (4, 512), (7, 513), (130, 769), (3, 1024), (3, 1025), (2, 2048),
          (5, 2049), (700, 64), (2, 4096), (3, 4100), (2, 8192), (2, 8200), (2, 16384), (3, 16390), (2, 40001)]


def out_like(x, pad):
    wide = torch.full((x.shape[0], x.shape[1] + pad), float("nan"), dtype=x.dtype, device="cuda")
    return wide, wide[:, :x.shape[1]]


def near(got, ref, dtype, scale):
    """got (device) within one rounding of its type and `scale` (float64, absolute) of ref."""
    d = (got.double().cpu() - ref).abs()
    bad = d > half_step(dtype) * (ref.abs() + scale) + scale
    assert not bad.any(), (float(d[bad].max()), float(ref.abs().max()), int(bad.sum()))


@pytest.mark.parametrize("shape", SHAPES + [(4099, 1000), (70000, 3)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("pad,add,p", [(0, True, 0.1), (0, False, 0.5), (13, True, 0.2), (8, False, 0.0)])
def test_dropout(shape, dtype, pad, add, p):
    dt = DTYPES[dtype]
    x, xr = rows_of(shape, pad, dt, 1)
    b, br = rows_of(shape, pad, dt, 2)
    f = keep_factors(*shape, p, SEED, OFFSET)
    drop = cg.drop(p, SEED, OFFSET)
    wide, y = out_like(x, pad)
    cg.cg_dropout_fwd(drop, x, b if add else None, y)
    ref = xr * f + (br if add else 0)
    near(y, ref, dt, 2 * U * (xr.abs() * f + br.abs()))      # the product's and the sum's rounding
    assert torch.isnan(wide[:, shape[1]:]).all()
    if p and not add:
        assert torch.equal(y.cpu() != 0, (f != 0) & (xr != 0))       # exactly the definition's elements
    wide, dx = out_like(x, pad)
    cg.cg_dropout_bwd(drop, x, dx)
    near(dx, xr * f, dt, U * xr.abs() * f)
    assert torch.isnan(wide[:, shape[1]:]).all()


def test_dropout_drops_nan_and_infinity():
    x = torch.full((3, 64), float("nan"), device="cuda")
    x[1] = float("inf")
    y = torch.empty_like(x)
    cg.cg_dropout_fwd(cg.drop(0.5, SEED, OFFSET), x, None, y)
    kept = keep_factors(3, 64, 0.5, SEED, OFFSET) != 0
    assert torch.equal(y.cpu() == 0, ~kept)


def test_dropout_of_nothing():
    y = torch.full((4,), 7.0, device="cuda")
    cg.cg_dropout_fwd(cg.drop(0.5, 1), y[:0].view(0, 4), None, y[:0].view(0, 4))
    cg.cg_dropout_fwd(cg.drop(0.5, 1), y.view(4, 1)[:, :0], None, y.view(4, 1)[:, :0])
    torch.cuda.synchronize()
    assert bool((y == 7).all())


def run_norm(x, xr, gamma, beta, dy, dyr, ds, dsr, joined, pad, eps=1e-5, p=0.2):
    """One forward and backward pass through the library, compared with the plain form."""
    dt, (R, N) = x.dtype, x.shape
    g64, b64 = gamma.double().cpu(), beta.double().cpu()
    c = (64 + N / 1024) * U
    d = cg.layernorm_desc(x, eps)
    mean, rstd = (torch.full((R,), float("nan"), device="cuda") for _ in range(2))
    wy, y = out_like(x, pad)
    wx, dx = out_like(x, pad)
    dgamma, dbeta = (torch.full((N,), float("nan"), device="cuda") for _ in range(2))
    ws = torch.empty(cg.cg_layernorm_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    if joined is not None:
        br, brr = joined
        f = keep_factors(R, N, p, SEED, OFFSET)
        drop = cg.drop(p, SEED, OFFSET)
        wt, total = out_like(x, pad)
        wb, db = out_like(x, pad)
        cg.cg_dropout_add_layernorm_fwd(d, drop, br, x, gamma, beta, total, y, mean, rstd)
        near(total, xr + f * brr, dt, 2 * U * (xr.abs() + f * brr.abs()))
        xr = total.double().cpu()      # the norm is that of the stored sum
        cg.cg_dropout_add_layernorm_bwd(d, drop, dy, ds, total, gamma, mean, rstd, dx, db, dgamma, dbeta, ws)
        near(db, dx.double().cpu() * f, dt, U * dx.double().cpu().abs() * f)
        assert torch.isnan(wt[:, N:]).all() and torch.isnan(wb[:, N:]).all()
    else:
        cg.cg_layernorm_fwd(d, x, gamma, beta, y, mean, rstd)
        y2 = torch.empty_like(y)
        cg.cg_layernorm_fwd(d, x, gamma, beta, y2)
        assert torch.equal(y, y2)      # the same with the statistics not kept
        cg.cg_layernorm_bwd(d, dy, x, gamma, mean, rstd, ds, dx, dgamma, dbeta, ws)
    yr, xh, mr, rr = norm(xr, g64, b64, eps)
    # the mean is off by c of the largest element, which the division by the deviation enlarges; a row of equal elements
    # has nothing else in its deviation
    big = xr.abs().max(1, keepdim=True).values
    off = c * (1 + xh.abs()) * (1 + big * rr[:, None])
    assert bool(((mean.double().cpu() - mr).abs() <= c * big[:, 0] + 1e-300).all())
    near(y, yr, dt, off * g64.abs() + 2 * U * b64.abs())
    dxr, dgr, dbr = norm_bwd(dyr, xh, rr, g64)
    g = (dyr * g64).abs()
    gm = g.max(1, keepdim=True).values
    xm = xh.abs().max(1, keepdim=True).values
    # three terms of up to gm, the last with xh twice, xh and rstd off as above
    tol = 4 * c * rr[:, None] * gm * (1 + xm * xm) * (1 + big * rr[:, None])
    near(dx, dxr + (0 if dsr is None else dsr), dt, tol + (0 if dsr is None else 2 * U * dsr.abs()))
    near(dgamma, dgr, torch.float32, (128 * U * (dyr.abs() * (1 + xh.abs())) + dyr.abs() * off).sum(0))
    near(dbeta, dbr, torch.float32, 128 * U * dyr.abs().sum(0))
    assert torch.isnan(wy[:, N:]).all() and torch.isnan(wx[:, N:]).all()


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("pad,dsum,joined", [(0, False, False), (13, True, False), (0, True, True), (8, False, True)])
def test_layernorm(shape, dtype, pad, dsum, joined):
    dt = DTYPES[dtype]
    x, xr = rows_of(shape, pad, dt, 1, 1.0, 0.25)
    dy, dyr = rows_of(shape, pad, dt, 2, 0.01)
    ds, dsr = rows_of(shape, pad, dt, 3, 0.01) if dsum else (None, None)
    br = rows_of(shape, pad, dt, 4, 0.5) if joined else None
    g = torch.Generator().manual_seed(5)
    gamma, beta = (torch.empty(shape[1]).normal_(m, 0.2, generator=g).cuda() for m in (1.0, 0.0))
    run_norm(x, xr, gamma, beta, dy, dyr, ds, dsr, br, pad)


def test_layernorm_of_many_rows():
    """More rows than a launch has room for at once: every block takes several."""
    shape = (20011, 72)
    x, xr = rows_of(shape, 0, torch.float32, 1, 1.0, 0.25)
    dy, dyr = rows_of(shape, 0, torch.float32, 2, 0.01)
    run_norm(x, xr, torch.ones(72, device="cuda"), torch.zeros(72, device="cuda"), dy, dyr, None, None, None, 0)


def test_layernorm_of_rows_with_a_large_mean_and_of_equal_elements():
    """A deviation of 1 about a mean of 1000 loses no more than the elements' own last places; equal elements give beta."""
    x, xr = rows_of((6, 1000), 0, torch.float32, 1, 1.0, 1000.0)
    dy, dyr = rows_of((6, 1000), 0, torch.float32, 2, 0.01)
    run_norm(x, xr, torch.ones(1000, device="cuda"), torch.zeros(1000, device="cuda"), dy, dyr, None, None, None, 0)
    x = torch.full((3, 256), 0.5, device="cuda")
    beta = torch.arange(256.0, device="cuda")
    y = torch.empty_like(x)
    cg.cg_layernorm_fwd(cg.layernorm_desc(x), x, torch.ones(256, device="cuda"), beta, y)
    assert torch.equal(y, beta.expand(3, 256))


def test_layernorm_of_no_rows():
    x = torch.empty(0, 40, device="cuda")
    d = cg.layernorm_desc(x)
    dg, db = (torch.full((40,), float("nan"), device="cuda") for _ in range(2))
    w, e = torch.ones(40, device="cuda"), torch.empty(0, device="cuda")
    cg.cg_layernorm_fwd(d, x, w, w, x, e, e)
    cg.cg_layernorm_bwd(d, x, x, w, e, e, None, x, dg, db, None)
    assert bool((dg == 0).all() and (db == 0).all())


def test_layernorm_gradients_against_differences():
    """<dx, r> + <dgamma, s> + <dbeta, t> is the derivative of <y, dy> along (r, s, t), by central differences in 64 bits of the
    plain forward pass; the library's gradients are off by 2^-13 at most (tolerances above), the differences by h^2."""
    shape, eps, h = (12, 200), 1e-5, 1e-4
    x, xr = rows_of(shape, 0, torch.float32, 1)
    dy, dyr = rows_of(shape, 0, torch.float32, 2)
    g = torch.Generator().manual_seed(5)
    gamma, beta, s, t = (torch.empty(200, dtype=torch.float64).normal_(0, 1, generator=g).float().double() for _ in range(4))
    r = torch.empty(shape, dtype=torch.float64).normal_(0, 1, generator=g)
    d = cg.layernorm_desc(x, eps)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = torch.empty(12, device="cuda"), torch.empty(12, device="cuda")
    dg, db = torch.empty(200, device="cuda"), torch.empty(200, device="cuda")
    ws = torch.empty(cg.cg_layernorm_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    cg.cg_layernorm_fwd(d, x, gamma.float().cuda(), beta.float().cuda(), y, mean, rstd)
    cg.cg_layernorm_bwd(d, dy, x, gamma.float().cuda(), mean, rstd, None, dx, dg, db, ws)
    along = float((dx.double().cpu() * r).sum() + (dg.double().cpu() * s).sum() + (db.double().cpu() * t).sum())
    up, down = ((norm(xr + e * r, gamma + e * s, beta + e * t, eps)[0] * dyr).sum() for e in (h, -h))
    size = float((dx.double().cpu() * r).norm() + (dg.double().cpu() * s).norm() + (db.double().cpu() * t).norm())
    assert abs(along - float(up - down) / (2 * h)) < 1e-3 * size


def test_layernorm_results_repeat_and_follow_the_stream():
    """The same bits on every call, also on a stream of its own and replayed from a captured graph."""
    x, _ = rows_of((3001, 769), 31, torch.float32, 1)
    dy, _ = rows_of((3001, 769), 31, torch.float32, 2)
    w = torch.ones(769, device="cuda")
    d = cg.layernorm_desc(x)
    y, dx = torch.empty(3001, 769, device="cuda"), torch.empty(3001, 769, device="cuda")
    mean, rstd = torch.empty(3001, device="cuda"), torch.empty(3001, device="cuda")
    dg, db = torch.empty(769, device="cuda"), torch.empty(769, device="cuda")
    ws = torch.empty(cg.cg_layernorm_workspace_bytes(d), dtype=torch.uint8, device="cuda")

    def step(stream=None):
        cg.cg_layernorm_fwd(d, x, w, w, y, mean, rstd, stream)
        cg.cg_layernorm_bwd(d, dy, x, w, mean, rstd, None, dx, dg, db, ws, stream)

    def results():
        torch.cuda.synchronize()
        got = [t.clone() for t in (y, dx, dg, db)]
        for t in (y, dx, dg, db, mean, rstd):
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


@pytest.mark.parametrize("cols", [120, 128, 129, 250, 256, 257])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("joined", [False, True])
def test_layernorm_of_rows_that_share_a_wave(cols, dtype, joined):
    """Widths around a quarter and half of a wave's; one row, a block's rows and one more, more than a single block's, many."""
    dt = DTYPES[dtype]
    g = torch.Generator().manual_seed(5)
    gamma, beta = (torch.empty(cols).normal_(m, 0.2, generator=g).cuda() for m in (1.0, 0.0))
    for rows in (1, 17, 32, 65, 129, 6001):
        x, xr = rows_of((rows, cols), 3, dt, 1, 1.0, 0.25)
        dy, dyr = rows_of((rows, cols), 3, dt, 2, 0.01)
        br = rows_of((rows, cols), 3, dt, 4, 0.5) if joined else None
        run_norm(x, xr, gamma, beta, dy, dyr, None, None, br, 3)
