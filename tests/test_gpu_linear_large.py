"""Tiles of 256 in all three passes of a linear layer: the loop between the first and the last steps, every epilogue, rows of wider tensors, x in 8 bits
that is unpacked first beside the bias's sums in the same workspace."""
import pytest
import torch

import block_util as bu
from linear_plan_util import LARGE
from test_gpu_linear import Layer, _cg, _ws, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,K,N", LARGE)
@pytest.mark.parametrize("pack", [False, True])
def test_whole_numbers(M, K, N, pack):
    """Every sum is a whole number below 2^24 (3128 products of at most 9, and 6 more): bit for bit."""
    L = Layer("bf16", M, K, N, bias=True, residual=True, pad=8, values=lambda s, i: bu.whole(s, 3, M + i))
    h = {k: None if v is None else v.float() for k, v in L.h.items()}
    y, z = L.fwd()
    want = h["x"] @ h["w"].T + h["bias"]
    assert torch.equal(z.cpu(), want.bfloat16()) and torch.equal(y.cpu(), (want + h["residual"]).bfloat16())
    assert torch.equal(L.dx().cpu(), (h["dz"] @ h["w"] + h["add"]).bfloat16())
    for bias in (True, False):
        dw, db = L.dw(L.packed("x") if pack else None, bias)
        assert torch.equal(dw.cpu(), h["dz"].T @ h["x"])
        assert torch.equal(db.cpu(), h["dz"].sum(0)) if bias else bool((db == 7.0).all())


@pytest.mark.parametrize("act,act_in,residual,pack", [("gelu", "silu", True, False), ("silu", "gelu", True, True), ("relu", "gelu", False, False), ("none", "relu", False, True)])
def test_epilogues(act, act_in, residual, pack):
    """Every activation and its slope (of a tensor, and of one in 8 bits), with and without a residual and an added gradient."""
    check(Layer("bf16", *LARGE[2], act, act_in, True, residual, 8, seed=31), pack)


@pytest.mark.parametrize("pack", [False, True])
def test_in_a_graph(pack):
    """Captured, all passes in one workspace, and replayed between eager calls: the same bits."""
    M, K, N = LARGE[2]
    L = Layer("bf16", M, K, N, "gelu", "silu", True, True, seed=32)
    cg, d = _cg(), L.d
    y, z, dx = (torch.empty(s, dtype=L.dt, device="cuda") for s in ((M, N), (M, N), (M, K)))
    dw, db = torch.empty(N, K, device="cuda"), torch.empty(N, device="cuda")
    x, z_in = (L.packed("x"), L.packed("z_in")) if pack else (d["x"], d["z_in"])
    ws = _ws(max(cg.cg_linear_workspace_bytes(L.desc, p) for p in range(3)))
    results = (y, z, dx, dw, db)

    def into():
        cg.cg_linear_fwd(L.desc, d["x"], d["w"], d["bias"], d["residual"], y, z, ws)
        cg.cg_linear_bwd_data(L.desc, d["dz"], d["w"], z_in, d["add"], dx, ws)
        cg.cg_linear_bwd_weight(L.desc, d["dz"], x, dw, db, ws)

    into()
    first = [t.clone() for t in results]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        into()
    for _ in range(3):
        for t in results:
            t.fill_(3.0)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, results))
        into()


@pytest.mark.parametrize("K", [1 << 21, (1 << 21) + 8])
def test_widest_rows_in_8_bits(K):
    """x in 8 bits with the widest rows that are unpacked, and the next: whole numbers, bit for bit where columns begin and end."""
    cg, M, N = _cg(), 1024, 256
    g = torch.Generator("cuda").manual_seed(3)
    codes = torch.randint(-3, 4, (M, K), generator=g, device="cuda", dtype=torch.int8)
    x = cg.Packed8(codes, torch.full((M, (K + 31) // 32), 133, dtype=torch.uint8, device="cuda"))
    dz = torch.randint(-3, 4, (M, N), generator=g, device="cuda").bfloat16()
    d = cg.cg_linear_desc(cg.CG_TYPE_BF16, M, N, K, 0, 0)
    dw, db = torch.full((N, K), 7.0, device="cuda"), torch.full((N,), 7.0, device="cuda")
    cg.cg_linear_bwd_weight(d, dz, x, dw, db, _ws(cg.cg_linear_workspace_bytes(d, cg.CG_PASS_BWD_WEIGHT)))
    h = dz.float().cpu()
    assert torch.equal(db.cpu(), h.sum(0))
    for part in (slice(0, 520), slice(K // 2 - 300, K // 2 + 300), slice(K - 520, K)):
        assert torch.equal(dw[:, part].cpu(), h.T @ codes[:, part].float().cpu())
