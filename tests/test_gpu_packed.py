"""Tensors in 8 bits: codes and scales bit for bit against their definition, and what is not finite."""
import pytest
import torch

import block_util as bu

pytestmark = pytest.mark.gpu


def _cg():
    import paper_1706_00095_amd as cg
    return cg


def _pack(x, pad=0):
    cg = _cg()
    rows, cols = x.shape
    blocks = (cols + 31) // 32
    codes = torch.full((rows, cols + pad), 99, dtype=torch.int8, device="cuda")
    scales = torch.full((rows, blocks + pad), 99, dtype=torch.uint8, device="cuda")
    p = cg.Packed8(codes[:, :cols], scales[:, :blocks])
    cg.cg_pack8(x, p)
    assert bool((codes[:, cols:] == 99).all()) and bool((scales[:, blocks:] == 99).all()), "wrote between rows"
    return p


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (3, 7, 1), (2, 32, 0), (5, 33, 3), (17, 100, 0), (64, 256, 8), (130, 1001, 5), (1000, 8, 0), (9, 40, 13)])
@pytest.mark.parametrize("std", [1.0, 1e-37, 1e36])
def test_definition(dtype, rows, cols, pad, std):
    cg, dt = _cg(), bu.DTYPES[dtype]
    x = bu.normal((rows, cols), dt, rows + cols, std)
    x[:, :: max(1, cols // 3)] *= 8.0
    x = x.to(dt).double()
    x[0] = 0.0
    d, _ = bu.wide(x, pad, dt)
    p = _pack(d, pad)
    codes, scales, values = bu.packed(x)
    assert torch.equal(p.scales.cpu(), scales) and torch.equal(p.codes.cpu(), codes)
    y, whole = bu.wide(torch.full((rows, cols), 7.0), pad, dt, fill=5.0)
    cg.cg_unpack8(p, y)
    assert torch.equal(y.double().cpu(), values) and bool((whole[:, cols:] == 5.0).all())
    for other in bu.DTYPES.values():      # every value is a number of both types
        z = torch.empty(rows, cols, dtype=other, device="cuda")
        cg.cg_unpack8(p, z)
        assert torch.equal(z.double().cpu(), values)


def test_borders():
    """The largest magnitudes on both sides of where a block's step doubles, for every exponent, and the ends of the type."""
    tops = [t * 2.0 ** e for e in range(-140, 128) for t in (1.0, 127 / 128 * 2 - 2.0 ** -22, 127 / 64, 1.9999, 127.5 / 64, 127.5 / 64 - 2.0 ** -23)]
    tops += [3.4028234663852886e38, 2.0 ** -149, 2.0 ** -133, 127 * 2.0 ** -133, 127.5 * 2.0 ** -133, 127.5 * 2.0 ** -133 - 2.0 ** -149, 0.0]
    x = torch.tensor(tops, dtype=torch.float64).float().double()
    x = x[torch.isfinite(x)]
    rows = torch.zeros(len(x), 32, dtype=torch.float64)
    rows[:, 5] = -x
    rows[:, 9] = (x * 0.37).float().double()
    p = _pack(rows.float().cuda())
    codes, scales, _ = bu.packed(rows.float().double())
    assert torch.equal(p.scales.cpu(), scales) and torch.equal(p.codes.cpu(), codes)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_largest(dtype):
    """The largest numbers of a type come back finite: off by 1/127 of the block's largest at most."""
    cg, dt = _cg(), bu.DTYPES[dtype]
    top = float(torch.finfo(dt).max)
    x = torch.zeros(4, 33, dtype=torch.float64)
    x[0, 3], x[1, 32], x[2, 0], x[3, :] = top, -top, 127.5 * 2.0 ** 121, 127 * 2.0 ** 121
    x[0, 4], x[2, 1] = 0.3 * top, -63.4 * 2.0 ** 121
    x = x.to(dt).double()
    p = _pack(x.to(dt).cuda())
    codes, scales, values = bu.packed(x)
    assert torch.equal(p.scales.cpu(), scales) and torch.equal(p.codes.cpu(), codes)
    for other in bu.DTYPES.values():
        y = torch.empty(4, 33, dtype=other, device="cuda")
        cg.cg_unpack8(p, y)
        assert torch.equal(y.double().cpu(), values)
    assert bool(((values - x).abs() <= x.abs().amax(1, keepdim=True) / 127).all())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_not_finite(dtype):
    cg, dt = _cg(), bu.DTYPES[dtype]
    x = bu.normal((3, 70), dt, 5)
    want = x.clone()
    for i, v in ((0, float("nan")), (40, float("inf")), (69, -float("inf"))):
        x[1, i], want[1, i] = v, 0.0
    x[2, 32:64], want[2, 32:64] = float("inf"), 0.0
    p = _pack(x.to(dt).cuda())
    codes, scales, values = bu.packed(want)
    bad = ~torch.isfinite(x)
    assert torch.equal(p.scales.cpu(), scales) and torch.equal(p.codes.cpu()[~bad], codes[~bad]) and bool((p.codes.cpu()[bad] == -128).all())
    y = torch.empty(3, 70, dtype=dt, device="cuda")
    cg.cg_unpack8(p, y)
    y = y.double().cpu()
    assert torch.equal(torch.isnan(y), bad) and torch.equal(y[~bad], values[~bad])


def test_far_rows():
    cg, cols, M = _cg(), 40, 9
    ld = (1 << 31) // (M - 2) // 8 * 8
    big = torch.empty(M * ld, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(big, (M, cols), (ld, 1))
    values = bu.normal((M, cols), torch.bfloat16, 1)
    x.copy_(values.bfloat16().cuda())
    far = torch.as_strided(big.view(torch.int8), (M, cols), (ld + 64, 1), ld // 2)       # codes between the rows of x, as far apart
    p = cg.Packed8(far, torch.empty(M, 2, dtype=torch.uint8, device="cuda"))
    cg.cg_pack8(x, p)
    codes, _, kept = bu.packed(values)
    assert torch.equal(p.codes.cpu(), codes)
    cg.cg_unpack8(p, x)
    assert torch.equal(x.double().cpu(), kept)


def test_room():
    """packed8_like: codes and scales are the rows that are written, whatever the sizes."""
    cg = _cg()
    for rows, cols in ((1, 1), (3, 33), (17, 100)):
        x = bu.normal((rows, cols), torch.float32, rows)
        p = cg.packed8_like(x.float().cuda())
        cg.cg_pack8(x.float().cuda(), p)
        codes, scales, _ = bu.packed(x)
        assert torch.equal(p.codes.cpu(), codes) and torch.equal(p.scales.cpu(), scales)
        again = cg.Packed8(p.codes, p.scales)
        y = torch.empty(rows, cols, device="cuda")
        cg.cg_unpack8(again, y)
        assert torch.equal(y.double().cpu(), bu.packed(x)[2])


def test_nothing():
    cg = _cg()
    for shape in ((0, 40), (3, 0)):
        x = torch.empty(shape, device="cuda")
        p = cg.packed8_like(x)
        cg.cg_pack8(x, p)
        cg.cg_unpack8(p, x)
