"""What attention's gradients of differences keep of the probabilities and of o on the GPU, against bounds that fewer bits would not
meet (test_sublayer_precision_host.py)."""
import pytest
import torch

from precision_util import BF, BUCKETS, FAR, RMS, TOKENS, few_keys_bounds, few_keys_values, outer_differences, three_tokens, unrounded_bounds
from sublayer_util import Attention
from test_gpu_attention import call, inputs, lengths, near

pytestmark = pytest.mark.gpu
SHORT, LONG = [5, 64, 1, 33, 2, 40], 1500


def device(vals):
    return [t.to(BF).cuda() for t in vals]


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("D", [32, 64, 77, 96, 128])
@pytest.mark.parametrize("with_long", [False, True])
def test_few_keys_whatever_else_is_in_the_batch(causal, D, with_long):
    H, scale, n = 2, 0.125, sum(SHORT)
    vals = few_keys_values(SHORT, H, D)
    a = few_keys_bounds(vals, SHORT, scale, causal)
    more = few_keys_values([LONG], H, D, 6)
    lens = SHORT + [LONG] if with_long else SHORT
    x = device([torch.cat([s, m]) if with_long else s for s, m in zip(vals, more)])
    r = call(x, len(lens), lengths(lens), lengths(lens), scale, causal, None, 0, False, True)
    for name in ("o", "dq", "dk", "dv"):
        tol = getattr(a, "tol_" + name)
        near(name, r[name][:n], getattr(a, name), tol, BF)
    if with_long:
        b = Attention(*more, [LONG], [LONG], scale, causal, None, 0, 0, False, BF, True)
        for name in ("o", "dq", "dk", "dv"):
            near(name, r[name][n:], getattr(b, name), getattr(b, "tol_" + name), BF)
        alone = call(device(vals), len(SHORT), lengths(SHORT), lengths(SHORT), scale, causal, None, 0, False, True)
        assert all(torch.equal(alone[name], r[name][:n]) for name in ("o", "dq"))


@pytest.mark.parametrize("D", [8, 64, 96, 128])
def test_the_gradient_of_a_bias_keeps_24_bits(D):
    for seed in range(4):
        vals, bias = three_tokens(D, seed)
        exact, size = outer_differences(vals, bias)
        r = call(device(vals), 1, lengths([TOKENS]), lengths([TOKENS]), 1.0, False, bias.float().cuda(), FAR, True, True)
        got = torch.stack([r["dbias"][:, BUCKETS // 2 + 2], r["dbias"][:, 2]]).double().cpu()
        assert float((((got - exact) / size) ** 2).mean().sqrt()) < RMS, seed


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("D", [32, 64, 77, 96, 128])
@pytest.mark.parametrize("Hq,Hkv,bias", [(2, 2, 0), (4, 1, 0), (4, 2, 16)])
def test_few_keys_and_few_rows_lose_nothing_to_rounding_within(causal, D, Hq, Hkv, bias):
    """dq of sequences of 64 keys or fewer; dk and dv of those of 32 rows (of the packed heads) or fewer, dk where o keeps 24 bits too."""
    lens_q, lens_k = [5, 40, 1, 32, 2, 8, 150, 3], [5, 64, 33, 32, 1, 60, 150, 900]
    x, vals = inputs("bf16", lens_q, lens_k, Hq, Hkv, D, shift=D % 2)
    far = 50
    table = torch.empty(Hq, bias).normal_(0, 0.5, generator=torch.Generator().manual_seed(3)) if bias else None
    a = unrounded_bounds(vals, lens_q, lens_k, 0.125, causal, table.double() if bias else None, far)
    r = call(x, len(lens_q), lengths(lens_q), lengths(lens_k), 0.125, causal, table.cuda() if bias else None, far, not causal, True)

    def part(name, lens, which):
        for i, (got, ref, tol) in enumerate(zip(r[name].split(lens), getattr(a, name).split(lens), getattr(a, "tol_" + name).split(lens))):
            if which(lens_q[i] * (1 if bias else Hq // Hkv), lens_k[i]):
                near((name, lens_q[i], lens_k[i]), got, ref, tol, BF)
    part("dq", lens_q, lambda rows, keys: keys <= 64)
    part("dv", lens_k, lambda rows, keys: rows <= 32)
    part("dk", lens_k, lambda rows, keys: rows <= 32 and (bias or keys <= 64))
