"""The training loop that runs the sublayer's operators together: its gradients against a plain 64-bit form differentiated by
torch, its losses, and that a run repeats bit for bit."""
import math

import pytest
import torch

from paper_1706_00095_amd import attention_sublayer as sub
from sublayer_util import buckets_of, keep_factors, norm

pytestmark = pytest.mark.gpu


def plain_loss(x, target, w, layer):
    """The sublayer's loss in 64 bits, of tensors that torch can differentiate."""
    h = norm(x, w["g1"], w["b1"], 1e-5)[0]
    q, k, v = (h @ w["qkv"]).view(layer.T, 3, layer.H, layer.D).unbind(1)
    outs, at = [], 0
    for n in sub.LENGTHS:
        delta = torch.arange(n)[None, :] - torch.arange(n)[:, None]
        b = w["bias"][:, buckets_of(delta, sub.BUCKETS, sub.FAR, True)]
        Q, K, V = (t[at:at + n].transpose(0, 1) for t in (q, k, v))
        outs.append((torch.softmax(Q @ K.transpose(1, 2) * layer.D ** -0.5 + b, 2) @ V).transpose(0, 1).reshape(n, layer.N))
        at += n
    f = keep_factors(layer.T, layer.N, layer.p, layer.seed, layer.step_count)
    y = norm(x + f * (torch.cat(outs) @ w["o"]), w["g2"], w["b2"], 1e-5)[0]
    return ((y @ w["z"] - target) ** 2).mean()


def test_gradients_of_the_whole_sublayer():
    """fp32: some twenty operators in a row, each within 2^-17 of its largest terms: 1e-4 of a tensor's largest gradient."""
    layer = sub.Sublayer(torch.float32)
    layer.w["bias"].normal_(0, 0.5, generator=torch.Generator("cuda").manual_seed(1))
    layer.step_count = 3
    x, target = sub.batch(torch.float32, 5)
    loss, dx = layer.loss_and_gradients(x, target)
    w = {k: t.double().cpu().requires_grad_() for k, t in layer.w.items()}
    x64 = x.double().cpu().requires_grad_()
    ref = plain_loss(x64, target.double().cpu(), w, layer)
    ref.backward()
    assert abs(float(loss) - float(ref.detach())) < 1e-5 * float(ref.detach())
    for name, got in [*layer.grad.items(), ("x", dx)]:
        want = x64.grad if name == "x" else w[name].grad
        assert float((got.double().cpu() - want).abs().max()) < 1e-4 * float(want.abs().max()), name


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_the_loss_falls_and_the_run_repeats(dtype):
    losses = sub.main(["--steps", "120", "--dtype", dtype])
    assert all(math.isfinite(x) for x in losses)
    assert sum(losses[-10:]) < 0.6 * sum(losses[:10])
    assert sub.main(["--steps", "20", "--dtype", dtype]) == losses[:20]
