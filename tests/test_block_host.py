"""CPU-only checks of the operators of a block over tokens: what the entry points refuse before anything is launched, how much workspace
they ask for, and the plain forms that the GPU tests compare with."""
import ctypes as C

import pytest
import torch

import block_util as bu
import paper_1706_00095_amd as cg

PACKED = cg.cg_packed8(64, 64, 65, 2)


def embedding(table_type=0, type=1, vocab=100, cols=24, tokens=10, scale=1.0):
    return cg.cg_embedding_desc(table_type, type, vocab, cols, tokens, scale)


def embed_fwd(d, tokens=64, table=64, table_ld=24, y=64, y_ld=24):
    return cg.lib().cg_embedding_fwd(d, tokens, table, table_ld, y, y_ld, None)


def embed_bwd(d, tokens=64, dy=64, dy_ld=24, dtable=64, ws=64, n=1 << 40):
    return cg.lib().cg_embedding_bwd(d, tokens, dy, dy_ld, dtable, ws, n, None)


def test_embedding_refusals():
    for d in (None, embedding(table_type=2), embedding(type=-1), embedding(vocab=0), embedding(cols=0), embedding(tokens=-1)):
        assert embed_fwd(d) == cg.CG_EINVAL and embed_bwd(d) == cg.CG_EINVAL
        assert cg.lib().cg_embedding_workspace_bytes(d) == 0
    for d in (embedding(tokens=(1 << 28) + 1), embedding(vocab=(1 << 31) - 1), embedding(tokens=1 << 28, cols=40)):
        assert embed_fwd(d, table_ld=40, y_ld=40) == cg.CG_EUNSUPPORTED and embed_bwd(d, dy_ld=40) == cg.CG_EUNSUPPORTED
    for bad in (dict(tokens=None), dict(tokens=66), dict(table=None), dict(table=66), dict(table_ld=23), dict(y=None), dict(y=65), dict(y_ld=23)):
        assert embed_fwd(embedding(), **bad) == cg.CG_EINVAL, bad
    for bad in (dict(tokens=None), dict(dy=None), dict(dy=65), dict(dy_ld=23), dict(dtable=None), dict(dtable=66), dict(ws=None), dict(ws=72)):
        assert embed_bwd(embedding(), **bad) == cg.CG_EINVAL, bad
    assert embed_fwd(embedding(tokens=0), tokens=None, table=None, y=None) == cg.CG_OK
    for tokens in (1, 1000, 4097, 16384, 65537, 1 << 20):
        d = embedding(tokens=tokens)
        n = cg.cg_embedding_workspace_bytes(d)
        assert 8 * tokens <= n <= 16 * tokens + 16 * tokens * 24 + 4096 + 256 * (tokens // 4096 + 1) * 4
        assert embed_bwd(d, n=n - 1) == cg.CG_ENOSPC


def test_pack_refusals():
    L = cg.lib()

    def pack(type=0, rows=2, cols=64, x=64, ld=64, p=PACKED):
        a, b = L.cg_pack8(type, rows, cols, x, ld, p, None), L.cg_unpack8(type, rows, cols, p, x, ld, None)
        assert a == b
        return a
    for bad in (dict(type=2), dict(rows=-1), dict(cols=-1), dict(x=None), dict(x=66), dict(ld=63), dict(p=None), dict(p=cg.cg_packed8(None, 64, 64, 2)),
                dict(p=cg.cg_packed8(64, 64, None, 2)), dict(p=cg.cg_packed8(64, 63, 64, 2)), dict(p=cg.cg_packed8(64, 64, 64, 1)), dict(type=1, x=65)):
        assert pack(**bad) == cg.CG_EINVAL, bad
    big = cg.cg_packed8(64, 1 << 40, 64, 1 << 40)
    assert pack(rows=1 << 29, cols=1, ld=1, p=big) == cg.CG_EUNSUPPORTED and pack(rows=1, cols=1 << 31, ld=1 << 31, p=big) == cg.CG_EUNSUPPORTED
    assert pack(rows=0, x=None, p=None) == cg.CG_OK and pack(cols=0, x=None, p=None) == cg.CG_OK


def linear(type=1, M=100, N=40, K=24, act=0, act_in=0):
    return cg.cg_linear_desc(type, M, N, K, act, act_in)


def fwd(d, x=64, x_ld=24, w=64, w_ld=24, bias=None, res=None, res_ld=40, y=64, y_ld=40, z=None, z_ld=40, ws=64, n=1 << 40):
    return cg.lib().cg_linear_fwd(d, x, x_ld, w, w_ld, bias, res, res_ld, y, y_ld, z, z_ld, ws, n, None)


def bwd_data(d, dz=64, dz_ld=40, w=64, w_ld=24, z=None, z_ld=24, z8=None, add=None, add_ld=24, dx=64, dx_ld=24, ws=64, n=1 << 40):
    return cg.lib().cg_linear_bwd_data(d, dz, dz_ld, w, w_ld, z, z_ld, z8, add, add_ld, dx, dx_ld, ws, n, None)


def bwd_weight(d, dz=64, dz_ld=40, x=64, x_ld=24, x8=None, dw=64, db=None, ws=64, n=1 << 40):
    return cg.lib().cg_linear_bwd_weight(d, dz, dz_ld, x, x_ld, x8, dw, db, ws, n, None)


def test_linear_refusals():
    for d in (None, linear(type=2), linear(M=-1), linear(N=0), linear(K=0), linear(act=4), linear(act=-1), linear(act_in=4)):
        assert fwd(d) == cg.CG_EINVAL and bwd_data(d) == cg.CG_EINVAL and bwd_weight(d) == cg.CG_EINVAL
        assert all(cg.lib().cg_linear_workspace_bytes(d, p) == 0 for p in range(3))
    most = 1 << 26
    for d in (linear(M=most + 1), linear(N=most + 1), linear(K=most + 1), linear(M=most, N=most), linear(N=1 << 20, K=1 << 20)):
        n = dict(x_ld=most, w_ld=most)
        assert fwd(d, **n, y_ld=most) == cg.CG_EUNSUPPORTED and bwd_data(d, dz_ld=most, w_ld=most, dx_ld=most) == cg.CG_EUNSUPPORTED
        assert bwd_weight(d, dz_ld=most, x_ld=most) == cg.CG_EUNSUPPORTED
    for bad in (dict(x=None), dict(x=65), dict(x_ld=23), dict(w=None), dict(w_ld=23), dict(bias=66), dict(res=64, res_ld=39), dict(res=65), dict(y=None), dict(y_ld=39),
                dict(z=64, z_ld=39), dict(z=65)):
        assert fwd(linear(), **bad) == cg.CG_EINVAL, bad
    for bad in (dict(dz=None), dict(dz_ld=39), dict(w=None), dict(w=65), dict(dx=None), dict(dx_ld=23), dict(add=64, add_ld=23)):
        assert bwd_data(linear(), **bad) == cg.CG_EINVAL, bad
    for bad in (dict(), dict(z=64, z_ld=23), dict(z=65), dict(z=64, z8=PACKED), dict(z8=cg.cg_packed8(64, 23, 64, 1)), dict(z8=cg.cg_packed8(None, 24, 64, 1))):
        assert bwd_data(linear(act_in=2), **bad) == cg.CG_EINVAL, bad
    for bad in (dict(dz=None), dict(x=None), dict(x=65), dict(x_ld=23), dict(x8=PACKED), dict(x=None, x8=cg.cg_packed8(64, 23, 64, 1)), dict(dw=None), dict(dw=66), dict(db=66)):
        assert bwd_weight(linear(), **bad) == cg.CG_EINVAL, bad
    assert fwd(linear(M=0), x=None, y=None) == cg.CG_OK and bwd_data(linear(M=0), dz=None, dx=None) == cg.CG_OK
    assert cg.cg_linear_workspace_bytes(linear(), 3) == 0


@pytest.mark.parametrize("type", [0, 1])
@pytest.mark.parametrize("M,N,K", [(1, 4096, 4096), (40, 512, 8192), (100, 4096, 9216), (256, 4096, 9216), (1500, 515, 771), (16384, 4096, 4096), (7, 3, 100000)])
def test_linear_workspaces(type, M, N, K):
    """Sums of parts of k: at most 32 of the output, and x unpacked; what is too small is refused, what is misplaced too."""
    d = linear(type, M, N, K)
    for which, out, call in ((0, M * N, lambda **a: fwd(d, x_ld=K, w_ld=K, y_ld=N, **a)), (1, M * K, lambda **a: bwd_data(d, dz_ld=N, w_ld=K, dx_ld=K, **a)),
                             (2, N * K, lambda **a: bwd_weight(d, dz_ld=N, x_ld=K, **a))):
        n = cg.cg_linear_workspace_bytes(d, which)
        assert n <= 32 * 4 * (out + max(M, N, K)) + 2 * M * K + 4 * 256 * N
        if n:
            assert call(n=n - 1) == cg.CG_ENOSPC and call(ws=None) == cg.CG_EINVAL and call(ws=72) == cg.CG_EINVAL


def test_act_bwd_refusals():
    def call(act=2, type=0, rows=2, cols=64, dy=64, dy_ld=64, z=64, z_ld=64, z8=None, dz=64, dz_ld=64):
        return cg.lib().cg_act_bwd(act, type, rows, cols, dy, dy_ld, z, z_ld, z8, dz, dz_ld, None)
    for bad in (dict(act=0), dict(act=4), dict(type=2), dict(rows=-1), dict(dy=None), dict(dy_ld=63), dict(z=None), dict(z8=PACKED), dict(z_ld=63), dict(dz=None), dict(dz=66), dict(dz_ld=63)):
        assert call(**bad) == cg.CG_EINVAL, bad
    assert call(rows=0, dy=None, z=None, dz=None) == cg.CG_OK
    assert call(rows=1 << 20, cols=1 << 14, dy_ld=1 << 14, z_ld=1 << 14, dz_ld=1 << 14) == cg.CG_EUNSUPPORTED


def test_the_binding_refuses_what_does_not_fit():
    x, w = torch.zeros(4, 8), torch.zeros(5, 8)
    for f in (lambda: cg.linear_desc(x, w[:, :7]), lambda: cg.embedding_desc(w, torch.zeros(3, 7)), lambda: cg.linear_desc(x[0], w)):
        with pytest.raises(ValueError):
            f()
    with pytest.raises(TypeError):
        cg.linear_desc(x, w.bfloat16())
    with pytest.raises(KeyError):
        cg.linear_desc(x, w, "tanh")
    d = cg.linear_desc(x, w)
    with pytest.raises(TypeError):
        cg.cg_linear_fwd(d, x, w, None, None, torch.zeros(4, 5))         # not on a device
    with pytest.raises(TypeError):
        cg.cg_embedding_fwd(cg.embedding_desc(w, x), torch.zeros(4, dtype=torch.int32), w, x)
    with pytest.raises(TypeError):
        cg.packed8_like(x)


def test_the_plain_forms():
    """Slopes are the activations' derivatives; 8 bits are what their definition says."""
    z = torch.linspace(-6, 6, 41, dtype=torch.float64).requires_grad_()
    for name in ("relu", "gelu", "silu", "none"):
        (g,) = torch.autograd.grad(bu.act(z, name).sum(), z)
        keep = z.detach() != 0
        assert torch.allclose(g[keep], bu.slope(z.detach(), name)[keep])
    x = bu.normal((3, 70), torch.float32, 1, 5.0)
    codes, scales, values = bu.packed(x)
    step = torch.exp2(scales.double() - 133).repeat_interleave(32, 1)[:, :70]
    assert torch.equal(values, codes.double() * step) and bool(((values - x).abs() <= step / 2).all())
    top = codes.abs().max(1).values
    assert bool((top >= 64).all()) and bool((top <= 127).all())
    t = torch.tensor([1, -1, 1, 3, 0], dtype=torch.int32)
    dy = bu.normal((5, 4), torch.float32, 2)
    g, _ = bu.embedding_grad(t, dy, 3, 2.0)
    assert torch.equal(g, torch.stack([2 * dy[4], 2 * (dy[0] + dy[2]), torch.zeros(4, dtype=torch.float64)]))
