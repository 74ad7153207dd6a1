"""The training loop that runs the operators of a block over tokens together: its gradients against a plain 64-bit form, and that a run
repeats bit for bit."""
import math

import pytest
import torch

import block_util as bu
from paper_1706_00095_amd import token_block as tb
from sublayer_util import norm

pytestmark = pytest.mark.gpu


class Kept(torch.autograd.Function):
    """A linear layer (of an activation) whose backward pass reads its input, and the activation's, as 8 bits keep them."""

    @staticmethod
    def forward(ctx, x, w, z_in, packed):
        keep = (lambda t: bu.packed(t.float().double())[2]) if packed else (lambda t: t)
        ctx.save_for_backward(keep(x), w, keep(z_in) if z_in is not None else None)
        return x @ w.T

    @staticmethod
    def backward(ctx, g):
        x, w, z_in = ctx.saved_tensors
        dx = g @ w
        return (None if z_in is not None else dx), g.T @ x, (dx * bu.slope(z_in, "gelu") if z_in is not None else None), None


def plain_loss(tokens, target, w, packed):
    t = tokens.long()
    x = torch.where((t >= 0)[:, None], w["table"][t.clamp(min=0)] * tb.WIDTH ** 0.5, 0.0)
    h = norm(x, w["gamma"], w["beta"], 1e-5)[0]
    z = Kept.apply(h, w["w1"], None, packed) + w["b1"]
    r = Kept.apply(bu.act(z, "gelu").detach(), w["w2"], z, packed) + w["b2"] + x
    logp = torch.log_softmax(r @ w["wo"].T + w["bo"], 1)
    some = target >= 0
    return -logp[some].gather(1, target[some].long()[:, None]).mean()


@pytest.mark.parametrize("keep", ["8bit", "tensors"])
def test_gradients_of_the_whole_block(keep):
    """fp32: a dozen operators in a row, each within 2^-17 of its largest terms: 1e-4 of a tensor's largest gradient.  In 8 bits a value that lies
    within a rounding of the border between two codes may get either: one step, 1/64 of its block's largest value at most, which at
    480 tokens is 1/64 of a term of a sum of 480 such terms; a handful of them (values are off by some 2^-22, one in 2^13 is that near a border, of
    480 x 448 of them: 26, over 64 to 192 columns) leave 2e-3 of the largest gradient."""
    block = tb.Block(torch.float32, keep)
    g = torch.Generator("cuda").manual_seed(1)
    for n in ("b1", "b2", "bo", "beta"):
        block.w[n].normal_(0, 0.3, generator=g)
    tokens, target = tb.batch(5)
    loss = block.loss_and_gradients(tokens, target)
    w = {k: t.double().cpu().requires_grad_() for k, t in block.w.items()}
    ref = plain_loss(tokens.cpu(), target.cpu(), w, keep == "8bit")
    ref.backward()
    assert abs(float(loss) - float(ref.detach())) < 1e-5 * float(ref.detach())
    for name, got in block.grad.items():
        want = w[name].grad
        assert float((got.double().cpu() - want).abs().max()) < (2e-3 if keep == "8bit" else 1e-4) * float(want.abs().max()), name


@pytest.mark.parametrize("dtype,keep", [("fp32", "8bit"), ("bf16", "8bit"), ("bf16", "tensors")])
def test_a_run_repeats(dtype, keep):
    losses = tb.main(["--steps", "30", "--dtype", dtype, "--keep", keep])
    assert all(math.isfinite(x) for x in losses)
    assert tb.main(["--steps", "10", "--dtype", dtype, "--keep", keep]) == losses[:10]


@pytest.mark.parametrize("keep", ["8bit", "tensors"])
def test_gradients_of_the_whole_block_in_bf16(keep):
    """bf16: a gradient has passed at most twelve tensors that were rounded (x, h, z, a, r, the logits, their gradient, dr, dz, dh, dx and a weight), each
    off by 2^-8 of its length at most, and a product with a random matrix makes an error at most twice as long as what it belongs to: 24 / 256
    of a gradient's length.  8 bits add half a step, 1/128 of a block's largest, in the two kept tensors that a gradient reads (h or a, and z), whose
    length is at least a third of that: 6 / 256 at most."""
    block = tb.Block(torch.bfloat16, keep, seed=3)
    g = torch.Generator("cuda").manual_seed(2)
    for n in ("b1", "b2", "bo", "beta"):
        block.w[n].normal_(0, 0.3, generator=g)
    tokens, target = tb.batch(6)
    loss = block.loss_and_gradients(tokens, target)
    w = {k: (t.bfloat16() if k in ("w1", "w2", "wo") else t).double().cpu().requires_grad_() for k, t in block.w.items()}
    ref = plain_loss(tokens.cpu(), target.cpu(), w, False)
    ref.backward()
    assert abs(float(loss) - float(ref.detach())) < 24 / 256 * float(ref.detach())
    for name, got in block.grad.items():
        want = w[name].grad
        assert float((got.double().cpu() - want).norm()) < (30 if keep == "8bit" else 24) / 256 * float(want.norm()), name
