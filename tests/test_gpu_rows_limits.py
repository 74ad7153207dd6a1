"""Layer norm of rows so long that a thread of one launch for each of their columns would be too many."""
import pytest
import torch

import paper_1706_00095_amd as cg

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("rows,cols", [(1, (1 << 27) + 5), (3, (1 << 19) + 9), (2, 1 << 20)])
def test_gradients_of_the_weights_of_long_rows(rows, cols):
    """dbeta is a sum of `rows` numbers, dgamma one of their products with (x - mean) rstd, in fewer than rows + 4 roundings each of
    the products' magnitudes; mean and rstd are given."""
    g = torch.Generator(device="cuda").manual_seed(1)
    x, dy = (torch.empty(rows, cols, device="cuda").normal_(0, 1, generator=g) for _ in range(2))
    gamma = torch.ones(cols, device="cuda")
    mean, rstd = torch.full((rows,), 0.25, device="cuda"), torch.full((rows,), 1.5, device="cuda")
    d = cg.layernorm_desc(x)
    ws = torch.empty(cg.cg_layernorm_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    dx = torch.empty_like(x)
    dgamma, dbeta = (torch.full((cols,), float("nan"), device="cuda") for _ in range(2))
    cg.cg_layernorm_bwd(d, dy, x, gamma, mean, rstd, None, dx, dgamma, dbeta, ws)
    for got, terms, size in ((dbeta, dy.double(), dy.double().abs()), (dgamma, dy.double() * ((x.double() - 0.25) * 1.5), dy.double().abs() * (x.double().abs() + 0.25) * 1.5)):
        assert bool(((got.double() - terms.sum(0)).abs() <= (rows + 4) * U * size.sum(0)).all())
