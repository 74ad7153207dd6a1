"""CPU-only checks of the operators of an attention sublayer: what the entry points refuse before anything is launched, how
much workspace they ask for, and the plain forms that the GPU tests compare with."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import paper_1706_00095_amd as cg
from sublayer_util import Attention, bucket_of, keep_factors, norm, norm_bwd, philox

NAN = float("nan")


def test_the_generator_gives_the_published_answers():
    """Known answers of Philox4x32-10 (Salmon et al. 2011, the test vectors published with the paper)."""
    full = 0xFFFFFFFF
    for ctr, key, want in (
            ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
            ((full,) * 4, (full, full), (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
            ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))):
        got = philox(np.array([ctr], np.uint32), key)[0]
        assert tuple(int(x) for x in got) == want


def test_the_share_of_dropped_elements():
    f = keep_factors(1000, 999, 0.2, 7, 1)
    assert abs(float((f == 0).double().mean()) - 0.2) < 4 * math.sqrt(0.16 / f.numel())
    assert float(f.max()) == 65536.0 / (65536 - 13107)
    assert bool((keep_factors(10, 10, 0.0, 7, 1) == 1).all())


def test_the_plain_gradients_are_those_of_the_plain_forms():
    g = torch.Generator().manual_seed(1)
    r = lambda *s: torch.empty(s, dtype=torch.float64).normal_(0, 1, generator=g).requires_grad_()  # noqa: E731
    x, ga, be, dy = r(5, 9), r(9), r(9), r(5, 9).detach()
    y, xh, _, rstd = norm(x, ga, be, 1e-3)
    (y * dy).sum().backward()
    dx, dg, db = norm_bwd(dy, xh.detach(), rstd.detach(), ga.detach())
    assert torch.allclose(dx, x.grad) and torch.allclose(dg, ga.grad) and torch.allclose(db, be.grad)
    q, k, v, do = r(6, 4, 3), r(7, 2, 3), r(7, 2, 3), r(6, 4, 3).detach()
    bias = r(4, 6)
    a = Attention(q.detach(), k.detach(), v.detach(), do, [4, 0, 2], [5, 0, 2], 0.5, True, bias.detach(), 6, 5, True, torch.float32, False)
    out = []
    for q0, n, k0, m in ((0, 4, 0, 5), (4, 2, 5, 2)):
        delta = torch.arange(m)[None, :] - torch.arange(n)[:, None] - (m - n)
        b = torch.tensor([[bucket_of(min(abs(int(t)), 5), 3, 5) + (3 if t > 0 else 0) for t in row] for row in delta])
        for h in range(4):
            S = q[q0:q0 + n, h] @ k[k0:k0 + m, h // 2].T * 0.5 + bias[h][b]
            out.append(((torch.softmax(torch.where(delta <= 0, S, -math.inf), 1) @ v[k0:k0 + m, h // 2]) * do[q0:q0 + n, h]).sum())
    sum(out).backward()
    for got, want in ((a.dq, q.grad), (a.dk, k.grad), (a.dv, v.grad), (a.dbias, bias.grad)):
        assert torch.allclose(got, want)


def test_dropout_refusals():
    L = cg.lib()
    drop = cg.drop(0.5, 1)

    def call(d=drop, type=0, rows=2, cols=8, x=64, x_ld=8, add=None, add_ld=0, y=128, y_ld=8):
        return L.cg_dropout_fwd(d, type, rows, cols, x, x_ld, add, add_ld, y, y_ld, None)
    assert call(d=None) == cg.CG_EINVAL
    for p in (-0.1, 1.0, NAN):
        assert call(d=cg.drop(p, 1)) == cg.CG_EINVAL
    for bad in (dict(type=2), dict(type=-1), dict(rows=-1), dict(cols=-1), dict(x=None), dict(y=None), dict(x=66), dict(y=129),
                dict(x_ld=7), dict(y_ld=7), dict(add=64, add_ld=7), dict(add=65, add_ld=8), dict(type=1, x=65)):
        assert call(**bad) == cg.CG_EINVAL, bad
    assert call(rows=1 << 20, cols=1 << 12, x_ld=1 << 12, y_ld=1 << 12) == cg.CG_EUNSUPPORTED
    assert call(rows=0, x=None, y=None) == cg.CG_OK and call(cols=0, x=None, y=None) == cg.CG_OK
    assert L.cg_dropout_bwd(drop, 0, 2, 8, None, 8, 64, 8, None) == cg.CG_EINVAL


def test_layernorm_refusals_and_workspace():
    L = cg.lib()

    def desc(type=0, rows=4, cols=8, eps=1e-5):
        return cg.cg_layernorm_desc(type, rows, cols, eps)

    def fwd(d, x=64, x_ld=8, gamma=64, beta=64, y=64, y_ld=8, mean=None, rstd=None):
        return L.cg_layernorm_fwd(d, x, x_ld, gamma, beta, y, y_ld, mean, rstd, None)

    def bwd(d, dy=64, dy_ld=8, x=64, x_ld=8, gamma=64, mean=64, rstd=64, dsum=None, dsum_ld=0, dx=64, dx_ld=8, dgamma=64, dbeta=64, ws=64, n=1 << 30):
        return L.cg_layernorm_bwd(d, dy, dy_ld, x, x_ld, gamma, mean, rstd, dsum, dsum_ld, dx, dx_ld, dgamma, dbeta, ws, n, None)
    for d in (None, desc(type=3), desc(rows=-1), desc(cols=0), desc(eps=-1.0), desc(eps=NAN)):
        assert fwd(d) == cg.CG_EINVAL and bwd(d) == cg.CG_EINVAL
    assert fwd(desc(rows=1 << 20, cols=1 << 12)) == cg.CG_EUNSUPPORTED
    for bad in (dict(x=None), dict(y=None), dict(gamma=None), dict(beta=66), dict(x_ld=7), dict(y_ld=4), dict(mean=64), dict(rstd=64), dict(mean=64, rstd=65)):
        assert fwd(desc(), **bad) == cg.CG_EINVAL, bad
    for bad in (dict(dy=None), dict(dx=None), dict(x=None), dict(mean=None), dict(rstd=None), dict(dgamma=None), dict(dbeta=None), dict(ws=None), dict(ws=66),
                dict(dsum=64, dsum_ld=7), dict(dx_ld=7)):
        assert bwd(desc(), **bad) == cg.CG_EINVAL, bad
    for rows, cols in ((1, 8), (40, 769), (100000, 16), (3, 20000), (5000, 12288)):
        d = desc(rows=rows, cols=cols)
        n = cg.cg_layernorm_workspace_bytes(d)
        assert n >= 8 * cols and n % (8 * cols) == 0 and n <= 512 * 8 * cols
        assert bwd(d, dy_ld=cols, x_ld=cols, dx_ld=cols, n=n - 1) == cg.CG_ENOSPC
    assert cg.cg_layernorm_workspace_bytes(desc(rows=0)) == 0 and cg.cg_layernorm_workspace_bytes(desc(cols=0)) == 0
    drop = cg.drop(0.5, 1)
    args = (64, 8, 64, 8, 64, 64, 64, 8, 64, 8, None, None, None)
    assert L.cg_dropout_add_layernorm_fwd(desc(), cg.drop(1.5, 1), *args) == cg.CG_EINVAL
    assert L.cg_dropout_add_layernorm_fwd(desc(), drop, None, *args[1:]) == cg.CG_EINVAL
    assert L.cg_dropout_add_layernorm_fwd(desc(), drop, *args[:6], None, *args[7:]) == cg.CG_EINVAL
    back = (64, 8, None, 0, 64, 8, 64, 64, 64, 64, 8, 64, 8, 64, 64, 64, 0, None)
    assert L.cg_dropout_add_layernorm_bwd(desc(), drop, *back) == cg.CG_ENOSPC
    assert L.cg_dropout_add_layernorm_bwd(desc(), None, *back) == cg.CG_EINVAL
    assert L.cg_dropout_add_layernorm_bwd(desc(), drop, *back[:11], None, *back[12:]) == cg.CG_EINVAL


def attn(type=1, B=2, Hq=8, Hkv=2, D=64, Tq=100, Tk=100, scale=0.125, causal=1, buckets=0, far=0, both=0, **strides):
    s = dict(q_tok=Hq * D, q_head=D, k_tok=Hkv * D, k_head=D, v_tok=Hkv * D, v_head=D, o_tok=Hq * D, o_head=D)
    s.update(strides)
    return cg.cg_attn_desc(type, B, Hq, Hkv, D, Tq, Tk, *(s[n] for n in ("q_tok", "q_head", "k_tok", "k_head", "v_tok", "v_head", "o_tok", "o_head")),
                           scale, causal, buckets, far, both)


def fwd(d, q=64, k=64, v=64, cu_q=64, cu_k=64, bias=None, o=64, lse=64, rest=None, ws=64, n=1 << 40):
    return cg.lib().cg_attn_fwd(C.byref(d) if d is not None else None, q, k, v, cu_q, cu_k, bias, o, lse, rest, ws, n, None)


def bwd(d, do=64, q=64, k=64, v=64, cu_q=64, cu_k=64, bias=None, o=64, rest=None, lse=64, dq=64, dk=64, dv=64, dbias=None, ws=64, n=1 << 40):
    return cg.lib().cg_attn_bwd(C.byref(d) if d is not None else None, do, q, k, v, cu_q, cu_k, bias, o, rest, lse, dq, dk, dv, dbias, ws, n, None)


def test_attention_refusals():
    bad = [None, attn(type=2), attn(B=-1), attn(Hq=0), attn(Hkv=0), attn(Hq=7), attn(D=0), attn(Tq=-1), attn(Tk=-1), attn(scale=0.0), attn(scale=-1.0),
           attn(scale=NAN), attn(scale=math.inf), attn(buckets=-1), attn(q_tok=-1), attn(o_head=-8), attn(buckets=1, far=8), attn(buckets=3, far=8, both=1),
           attn(buckets=2, far=8, both=1), attn(buckets=32, far=16), attn(buckets=32, far=8, both=1)]
    for d in bad:
        assert fwd(d, bias=64) == cg.CG_EINVAL and bwd(d, bias=64) == cg.CG_EINVAL
        assert d is None or (cg.cg_attn_workspace_bytes(d, cg.CG_PASS_FWD) == 0 and cg.cg_attn_workspace_bytes(d, cg.CG_PASS_BWD_DATA) == 0)
    for d in (attn(D=129), attn(buckets=257, far=1000), attn(buckets=32, far=65537), attn(Tq=1 << 30), attn(Tk=1 << 31, Hkv=1, Hq=4)):
        assert fwd(d, bias=64) == cg.CG_EUNSUPPORTED and bwd(d, bias=64) == cg.CG_EUNSUPPORTED
    for name in ("q", "k", "v", "o", "lse", "cu_q", "cu_k"):
        for value in (None, 65):
            assert fwd(attn(), **{name: value}) == cg.CG_EINVAL, name
    for name in ("do", "q", "k", "v", "o", "lse", "cu_q", "cu_k", "dq", "dk", "dv"):
        for value in (None, 65):
            assert bwd(attn(), **{name: value}) == cg.CG_EINVAL, name
    b = attn(buckets=32, far=128)
    assert fwd(b) == cg.CG_EINVAL and bwd(b) == cg.CG_EINVAL                    # the table is missing
    assert bwd(attn(), dbias=64) == cg.CG_EINVAL                                # a gradient of no table
    assert fwd(attn(type=0), rest=64) == cg.CG_EINVAL and bwd(attn(type=0), rest=64) == cg.CG_EINVAL
    assert fwd(b, bias=64, ws=None) == cg.CG_EINVAL and bwd(attn(), ws=None) == cg.CG_EINVAL and bwd(attn(), ws=72) == cg.CG_EINVAL
    for d, f, which, more in ((b, fwd, cg.CG_PASS_FWD, dict(bias=64)), (attn(), bwd, cg.CG_PASS_BWD_DATA, {})):
        assert f(d, n=cg.cg_attn_workspace_bytes(d, which) - 1, **more) == cg.CG_ENOSPC
    assert cg.cg_attn_workspace_bytes(attn(), cg.CG_PASS_BWD_WEIGHT) == 0


def test_attention_calls_without_work():
    assert fwd(attn(B=0), q=None, o=None, lse=None, cu_q=None, cu_k=None) == cg.CG_OK
    assert fwd(attn(Tq=0), q=None, o=None, lse=None) == cg.CG_OK
    assert bwd(attn(Tq=0, Tk=0, B=0), do=None, q=None, k=None, v=None, o=None, lse=None, dq=None, dk=None, dv=None, cu_q=None, cu_k=None) == cg.CG_OK


@pytest.mark.parametrize("Tq,Tk,B,Hq,Hkv", [(1, 100, 1, 1, 1), (37, 17000, 8, 16, 4), (1, 1 << 20, 1, 8, 8), (64, 1 << 24, 64, 64, 8), (16384, 16384, 4, 16, 16),
                                            (5, 5, 5, 4, 4), (100000, 100000, 3, 8, 1)])
@pytest.mark.parametrize("buckets", [0, 32])
def test_attention_workspaces_stay_small(Tq, Tk, B, Hq, Hkv, buckets):
    """Partial results take 256 MiB at most, beside two statistics a row and the tables."""
    for which in (cg.CG_PASS_FWD, cg.CG_PASS_BWD_DATA):
        n = cg.cg_attn_workspace_bytes(attn(Tq=Tq, Tk=Tk, B=B, Hq=Hq, Hkv=Hkv, buckets=buckets, far=128 if buckets else 0), which)
        tiles = Tq * Hq // 128 + B * Hq
        assert n <= (2 * 256 << 20) + 8 * Tq * Hq + 64 * tiles * 4 * buckets + Hq * 4 * 300 + 4096


def test_the_binding_refuses_what_does_not_fit():
    x = torch.zeros(4, 8)
    with pytest.raises(TypeError):
        cg.cg_dropout_fwd(cg.drop(0.5, 1), x, None, torch.zeros(4, 8))          # not on a device
    with pytest.raises(TypeError):
        cg.layernorm_desc(x.double())
    with pytest.raises(ValueError):
        cg.cg_layernorm_fwd(cg.layernorm_desc(x), torch.zeros(4, 9), None, None, None)
    q = torch.zeros(5, 4, 8)
    with pytest.raises(ValueError):
        cg.attn_desc(q, q[:, :2], q, q, 1, 1.0)
    with pytest.raises(TypeError):
        cg.attn_desc(q, q, q.bfloat16(), q, 1, 1.0)
    with pytest.raises(ValueError):
        cg.attn_desc(q, q, q, torch.zeros(5, 4, 16)[..., ::2], 1, 1.0)
    d = cg.attn_desc(q, q, q, q, 1, 1.0)
    with pytest.raises(TypeError):
        cg.cg_attn_fwd(d, q, q, q, None, None, None, q, None)


def test_sizes_whose_loops_would_pass_32_bits_are_refused():
    """A loop's step behind the last row has to fit as well: 2^16 below the largest number is the limit."""
    L = cg.lib()
    most = (1 << 31) - (1 << 16)
    for rows, cols in ((most + 1, 1), (1, most + 1), ((1 << 31) - 1, 1)):
        d = cg.cg_layernorm_desc(0, rows, cols, 1e-5)
        assert L.cg_layernorm_fwd(d, 64, cols, 64, 64, 64, cols, None, None, None) == cg.CG_EUNSUPPORTED
        assert cg.cg_layernorm_workspace_bytes(d) == 0
    assert cg.cg_layernorm_workspace_bytes(cg.cg_layernorm_desc(0, most, 1, 1e-5)) > 0
    for d in (attn(Tk=most + 1, Hkv=1, Hq=1, D=1), attn(Tq=most + 1, Hkv=1, Hq=1, D=1), attn(Tk=(1 << 31) - 1, Hkv=1, Hq=1, D=1)):
        assert fwd(d) == cg.CG_EUNSUPPORTED and bwd(d) == cg.CG_EUNSUPPORTED
    assert cg.cg_attn_workspace_bytes(attn(Tk=most, Hkv=1, Hq=1, D=1, B=1, Tq=1), cg.CG_PASS_FWD) > 0
