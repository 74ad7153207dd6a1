"""CPU-only: the bounds that attention's differences are held to on the GPU are met by the plain forms, and not by results whose
probabilities, or whose o, have fewer bits."""
import pytest
import torch

from precision_util import BF, RMS, dq_with, few_keys_bounds, few_keys_values, outer_differences, pieces, three_tokens, unrounded_bounds
from sublayer_util import half_step


@pytest.mark.parametrize("causal", [False, True])
def test_few_keys_need_more_than_8_bits(causal):
    lens = [5, 64, 1, 33, 2, 40]
    vals = few_keys_values(lens, 2, 64)
    a = few_keys_bounds(vals, lens, 0.125, causal)

    def outside(dq):
        return ((dq - a.dq).abs() > half_step(BF) * (a.dq.abs() + a.tol_dq) + a.tol_dq).any(2).any(1).split(lens)
    assert not any(bool(x.any()) for n in (2, 3) for x in outside(dq_with(vals, lens, 0.125, causal, n)))
    for n, x in zip(lens, outside(dq_with(vals, lens, 0.125, causal, 1))):
        assert n < 5 or bool(x.any()), n


@pytest.mark.parametrize("causal", [False, True])
def test_few_keys_need_more_than_8_bits_of_the_scores_gradients(causal):
    lens = [5, 64, 33, 2, 40]
    g = torch.Generator().manual_seed(1)
    vals = [torch.empty(sum(lens), 2, 64, dtype=torch.float64).normal_(0, 1, generator=g).to(BF).double() for _ in range(4)]
    a = unrounded_bounds(vals, lens, lens, 0.125, causal)

    def outside(n):
        dq = dq_with(vals, lens, 0.125, causal, 3, n)
        return ((dq - a.dq).abs() > half_step(BF) * (a.dq.abs() + a.tol_dq) + a.tol_dq).any(2).any(1).split(lens)
    assert not any(bool(x.any()) for x in outside(2))
    assert all(bool(x.any()) for n, x in zip(lens, outside(1)) if n >= 5)


@pytest.mark.parametrize("D", [8, 64])
@pytest.mark.parametrize("seed", range(4))
def test_the_gradient_of_a_bias_needs_24_bits(D, seed):
    vals, bias = three_tokens(D, seed)
    exact, size = outer_differences(vals, bias)

    def off(**how):
        return float((((outer_differences(vals, bias, **how)[0] - exact) / size) ** 2).mean().sqrt())
    assert off(p_of=lambda p: pieces(p, 3), o_of=lambda o: o.float().double()) < RMS / 4
    assert off(p_of=lambda p: pieces(p, 2)) > 1.4 * RMS
    assert off(p_of=lambda p: pieces(p, 1)) > 100 * RMS
    assert off(o_of=lambda o: pieces(o, 2)) > 1.4 * RMS         # o_rest as a bf16 number
