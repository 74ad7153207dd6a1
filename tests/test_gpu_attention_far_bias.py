"""Attention whose bias lies far from zero: softmax does not change with a constant, and neither do the gradients, however little of
log l a row's lse = m + log l then holds.

Scores are a constant plus a few whole eighths, exact in 24 bits, and what else a product adds is lost beside the constant.  The
library may then be off by what it may be off by without the constant (sublayer_util.Attention), and lse by its own last place."""
import pytest
import torch

from sublayer_util import DTYPES, U, Attention
from test_gpu_attention import call, check, inputs, lengths

pytestmark = pytest.mark.gpu
LOWEST = torch.finfo(torch.float32).min
TINY = 2.0 ** -40


def put(x, i, values):
    """Replaces the values of a device tensor, exact in its type."""
    x[i].copy_(values.to(x[i].dtype))
    assert torch.equal(x[i].double().cpu(), values)


def with_bias(dtype, lens_q, lens_k, Hq, Hkv, D, causal, constant, steps, shift=0):
    dt = DTYPES[dtype]
    x, vals = inputs(dtype, lens_q, lens_k, Hq, Hkv, D, shift=shift)
    vals[0] = vals[0] * TINY
    put(x, 0, vals[0])
    n, far, both = 16, 40, not causal
    eighths = torch.randint(0, steps + 1, (Hq, n), generator=torch.Generator().manual_seed(7)).double() / 8
    table = (constant + eighths).float()
    if steps:
        assert torch.equal(table.double() - constant, eighths)
    a = Attention(*vals, lens_q, lens_k, 0.125, causal, eighths, n, far, both, dt, dtype == "bf16")
    r = call(x, len(lens_q), lengths(lens_q), lengths(lens_k), 0.125, causal, table.cuda(), far, both, dtype == "bf16")
    a.lse += constant
    a.tol_lse = a.tol_lse.nan_to_num(posinf=0.0) + 2 * U * abs(constant)
    check(r, a, dt)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("constant,steps", [(LOWEST, 0), (2.0 ** 20, 31), (-2.0 ** 20, 31), (1024.0, 7), (-1100.0, 7)])
def test_a_constant_in_the_bias(dtype, causal, constant, steps):
    with_bias(dtype, [150, 1, 33], [150, 1, 33], 2, 2, 64, causal, constant, steps)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D,shift", [(32, 0), (96, 0), (128, 0), (77, 1), (128, 1)])
def test_a_constant_in_the_bias_of_other_widths(dtype, D, shift):
    with_bias(dtype, [70, 129], [90, 129], 2, 1, D, True, LOWEST, 0, shift)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("Hq,Hkv", [(2, 2), (4, 1)])
def test_a_constant_in_the_bias_of_axes_that_are_cut(dtype, Hq, Hkv):
    with_bias(dtype, [5, 140, 0], [3000, 777, 9], Hq, Hkv, 64, True, LOWEST, 0)
    with_bias(dtype, [1300], [1300], Hq, Hkv, 32, False, -2.0 ** 20, 31)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("causal", [False, True])
def test_the_types_lowest_value_as_a_mask(dtype, causal):
    """Where another distance is seen it masks; where nothing else is, all it masks is seen equally.  A bias of -200 does the same to 64
    bits, and leaves the tolerances finite."""
    lens, dt = [150, 33], DTYPES[dtype]
    x, vals = inputs(dtype, lens, lens, 3, 3, 64)
    table = torch.zeros(3, 8)
    table[0, 3:] = LOWEST            # head 0 sees three distances
    table[1, 0] = LOWEST             # head 1 does not see itself, but for a sequence's first query, which sees nothing else
    table[2, :3] = LOWEST            # head 2 sees no distance below 3: three queries see masked keys only
    soft = torch.where(table == LOWEST, -200.0, table.double())
    vals[0] = vals[0] * TINY
    put(x, 0, vals[0])
    a = Attention(*vals, lens, lens, 0.125, causal, soft, 8, 20, False, dt, dtype == "bf16")
    r = call(x, 2, lengths(lens), lengths(lens), 0.125, causal, table.cuda(), 20, False, dtype == "bf16")
    low = a.lse < -100
    assert bool(low.any())
    assert bool((r["lse"].cpu()[low] == LOWEST).all())
    r["lse"][low.cuda()] = 0.0
    a.lse[low] = 0.0
    check(r, a, dt)
