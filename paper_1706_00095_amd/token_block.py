"""A small training loop through the operators of a block over tokens:

    x = s E[token];  h = layer norm(x);  z = h W1^T + b1,  a = gelu(z);  r = a W2^T + b2 + x;  logits = r Wo^T + bo
    loss = mean of -log softmax(logits)[next token]

with z, h and a kept for the backward pass in 8 bits (or, with --keep tensors, as they are), and the update by cg_grad_reduce_sgd_multi.  The
texts are walks through a fixed permutation of the vocabulary with some noise, so that the next token follows from the last one; every third text
is cut short (token -1: no token, no loss).  Softmax and its gradient are torch's.

    python -m paper_1706_00095_amd.token_block [--steps 200] [--dtype bf16] [--keep tensors]
"""
import argparse

import torch

import paper_1706_00095_amd as cg

TEXTS, LENGTH, VOCAB, WIDTH, INNER = 12, 40, 96, 64, 192


class Block:
    def __init__(self, dtype=torch.float32, keep="8bit", seed=0):
        self.dtype, self.keep, T = dtype, keep, TEXTS * LENGTH
        g = torch.Generator().manual_seed(seed)

        def weight(*shape):
            return torch.empty(shape).normal_(0, shape[1] ** -0.5, generator=g).cuda()

        zeros = lambda n: torch.zeros(n, device="cuda")  # noqa: E731
        self.w = dict(table=weight(VOCAB, WIDTH), gamma=torch.ones(WIDTH, device="cuda"), beta=zeros(WIDTH), w1=weight(INNER, WIDTH), b1=zeros(INNER),
                      w2=weight(WIDTH, INNER), b2=zeros(WIDTH), wo=weight(VOCAB, WIDTH), bo=zeros(VOCAB))
        self.history = {k: torch.zeros_like(t) for k, t in self.w.items()}
        self.grad = {k: torch.empty_like(t) for k, t in self.w.items()}
        # activations, kept tensors and a workspace, kept from step to step
        def rows(n):
            return torch.empty(T, n, dtype=dtype, device="cuda")

        self.x, self.h, self.r, self.dr, self.dh, self.dx = (rows(WIDTH) for _ in range(6))
        self.z, self.a, self.dz = (rows(INNER) for _ in range(3))
        self.logits = rows(VOCAB)
        self.kept = {n: cg.packed8_like(t) for n, t in (("h", self.h), ("z", self.z), ("a", self.a))}
        self.mean, self.rstd = (torch.empty(T, device="cuda") for _ in range(2))
        self.lookup, self.norm = cg.embedding_desc(self.w["table"], self.x, WIDTH ** 0.5), cg.layernorm_desc(self.x)
        like = lambda n, k: torch.empty(n, k, dtype=dtype, device="cuda")  # noqa: E731
        self.first = cg.linear_desc(self.h, like(INNER, WIDTH), "gelu")
        self.second = cg.linear_desc(self.a, like(WIDTH, INNER), act_in="gelu")
        self.last = cg.linear_desc(self.r, like(VOCAB, WIDTH))
        need = max(cg.cg_embedding_workspace_bytes(self.lookup), cg.cg_layernorm_workspace_bytes(self.norm),
                   *(cg.cg_linear_workspace_bytes(d, p) for d in (self.first, self.second, self.last) for p in range(3)))
        self.ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")

    def keeps(self, name, t):
        """What the backward pass reads of a tensor."""
        if self.keep != "8bit":
            return t
        cg.cg_pack8(t, self.kept[name])
        return self.kept[name]

    def loss_and_gradients(self, tokens, target):
        """tokens, target [TEXTS * LENGTH] int32, -1 where there is none; the gradients go to self.grad."""
        w, d, ws = self.w, self.grad, self.ws
        w1, w2, wo = (w[n].to(self.dtype) for n in ("w1", "w2", "wo"))
        cg.cg_embedding_fwd(self.lookup, tokens, w["table"], self.x)
        cg.cg_layernorm_fwd(self.norm, self.x, w["gamma"], w["beta"], self.h, self.mean, self.rstd)
        cg.cg_linear_fwd(self.first, self.h, w1, w["b1"], None, self.a, self.z, ws)
        cg.cg_linear_fwd(self.second, self.a, w2, w["b2"], self.x, self.r, None, ws)
        cg.cg_linear_fwd(self.last, self.r, wo, w["bo"], None, self.logits, None, ws)
        h, z, a = self.keeps("h", self.h), self.keeps("z", self.z), self.keeps("a", self.a)

        some = target >= 0
        logp = torch.log_softmax(self.logits.float(), 1)
        at = target.clamp(min=0).long()[:, None]
        count = some.sum()
        loss = -(logp.gather(1, at)[:, 0] * some).sum() / count
        dlogits = logp.exp()
        dlogits.scatter_add_(1, at, torch.full_like(dlogits[:, :1], -1.0))
        dlogits = (dlogits * (some[:, None] / count)).to(self.dtype)

        cg.cg_linear_bwd_weight(self.last, dlogits, self.r, d["wo"], d["bo"], ws)
        cg.cg_linear_bwd_data(self.last, dlogits, wo, None, None, self.dr, ws)
        cg.cg_linear_bwd_weight(self.second, self.dr, a, d["w2"], d["b2"], ws)
        cg.cg_linear_bwd_data(self.second, self.dr, w2, z, None, self.dz, ws)          # through the activation too
        cg.cg_linear_bwd_weight(self.first, self.dz, h, d["w1"], d["b1"], ws)
        cg.cg_linear_bwd_data(self.first, self.dz, w1, None, None, self.dh, ws)
        cg.cg_layernorm_bwd(self.norm, self.dh, self.x, w["gamma"], self.mean, self.rstd, self.dr, self.dx, d["gamma"], d["beta"], ws)
        cg.cg_embedding_bwd(self.lookup, tokens, self.dx, d["table"], ws)
        return loss

    def step(self, tokens, target, lr=0.2, mu=0.9):
        loss = self.loss_and_gradients(tokens, target)
        names = list(self.w)
        cg.cg_grad_reduce_sgd_multi([self.w[n] for n in names], [self.history[n] for n in names], [self.grad[n] for n in names], [[] for _ in names],
                                    [self.w[n].numel() for n in names], cg.cg_sgd(lr, mu, 0.0, 1.0))
        return loss


def batch(seed):
    """Tokens and the ones behind them."""
    g = torch.Generator().manual_seed(seed)
    follows = torch.randperm(VOCAB, generator=torch.Generator().manual_seed(12345))
    t = torch.empty(TEXTS, LENGTH + 1, dtype=torch.int64)
    t[:, 0] = torch.randint(0, VOCAB, (TEXTS,), generator=g)
    for i in range(LENGTH):
        other = torch.randint(0, VOCAB, (TEXTS,), generator=g)
        t[:, i + 1] = torch.where(torch.rand(TEXTS, generator=g) < 0.1, other, follows[t[:, i]])
    t[::3, LENGTH // 2:] = -1
    tokens, target = t[:, :-1].clone(), t[:, 1:].clone()
    target[tokens < 0] = -1
    return tokens.reshape(-1).int().cuda(), target.reshape(-1).int().cuda()


def main(argv=None):
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--dtype", choices=["fp32", "bf16"], default="fp32")
    ap.add_argument("--keep", choices=["8bit", "tensors"], default="8bit")
    args = ap.parse_args(argv)
    block, losses = Block(torch.bfloat16 if args.dtype == "bf16" else torch.float32, args.keep), []
    for i in range(args.steps):
        losses.append(block.step(*batch(i)))
        if i % 20 == 0 or i == args.steps - 1:
            print(f"step {i:4d}  loss {float(losses[-1]):.4f}", flush=True)
    return [float(x) for x in losses]


if __name__ == "__main__":
    main()
