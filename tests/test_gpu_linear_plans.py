"""The linear layers' products, kernel by kernel, whole and with a k that is cut in parts: every sum is a whole number below 2^24, so that results are the
same bits in whatever order they are added."""
import pytest
import torch

import block_util as bu
from linear_plan_util import CASES
from test_gpu_linear import Layer

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,which,whole,packed,tile,cut,M,K,N", CASES)
def test_whole_numbers(dtype, which, whole, packed, tile, cut, M, K, N):
    # rows of wider tensors, NaN between them, whole 16 bytes apart or not; backward-data through the slope of relu, which is 0 or 1
    L = Layer(dtype, M, K, N, "none", "relu" if which == 1 else "none", True, True, 8 if whole else 3, values=lambda s, i: bu.whole(s, 3, M + 3 * K + i))
    h = {k: None if v is None else v.float() for k, v in L.h.items()}
    if which == 0:
        y, z = L.fwd()
        want = h["x"] @ h["w"].T + h["bias"]
        assert torch.equal(z.cpu(), want.to(L.dt)) and torch.equal(y.cpu(), (want + h["residual"]).to(L.dt))
    elif which == 1:
        want = ((h["dz"] @ h["w"]) * (h["z_in"] > 0) + h["add"]).to(L.dt)
        for z_in in (None, L.packed("z_in")):
            assert torch.equal(L.dx(z_in).cpu(), want)
    else:
        want = h["dz"].T @ h["x"]
        for bias in (True, False):
            dw, db = L.dw(L.packed("x") if packed else None, bias)
            assert torch.equal(dw.cpu(), want)
            assert torch.equal(db.cpu(), h["dz"].sum(0)) if bias else bool((db == 7.0).all())
