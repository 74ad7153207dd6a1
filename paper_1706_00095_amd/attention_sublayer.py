"""A small training loop through the operators of an attention sublayer:

    h = layer norm(x);  q, k, v = h Wqkv;  a = attention(q, k, v, bias by distance);  b = a Wo
    s = x + drop(b);  y = layer norm(s);  z = y Wz;   loss = mean (z - target)^2

over packed sequences of different lengths, every token's target being the input two tokens before it (so that the sublayer has to
learn whom to look at from the distance alone), and the update by cg_grad_reduce_sgd_multi.  The projections are torch's products.

    python -m paper_1706_00095_amd.attention_sublayer [--steps 200] [--dtype bf16]
"""
import argparse

import torch

import paper_1706_00095_amd as cg

LENGTHS, WIDTH, HEADS, BUCKETS, FAR = (40, 7, 96, 1, 64), 64, 4, 16, 32


class Sublayer:
    def __init__(self, dtype=torch.float32, p=0.1, seed=0):
        self.dtype, self.p, self.seed, self.step_count = dtype, p, seed, 0
        g = torch.Generator().manual_seed(seed)
        T, N, H, D = sum(LENGTHS), WIDTH, HEADS, WIDTH // HEADS

        def weight(*shape):
            return torch.empty(shape).normal_(0, shape[0] ** -0.5, generator=g).cuda()

        self.w = dict(g1=torch.ones(N, device="cuda"), b1=torch.zeros(N, device="cuda"), qkv=weight(N, 3 * N), bias=torch.zeros(H, BUCKETS, device="cuda"),
                      o=weight(N, N), g2=torch.ones(N, device="cuda"), b2=torch.zeros(N, device="cuda"), z=weight(N, N))
        self.history = {k: torch.zeros_like(t) for k, t in self.w.items()}
        self.grad = {k: torch.empty_like(t) for k, t in self.w.items()}
        self.cu = torch.tensor([0, *LENGTHS]).cumsum(0).int().cuda()
        self.T, self.N, self.H, self.D = T, N, H, D
        # activations and workspaces, kept from step to step
        like = dict(dtype=dtype, device="cuda")
        self.h, self.s, self.y, self.dh, self.ds, self.db = (torch.empty(T, N, **like) for _ in range(6))
        self.a, self.rest = torch.empty(T, H, D, **like), torch.empty(T, H, D, **like) if dtype == torch.bfloat16 else None
        self.dqkv = torch.empty(T, 3 * H, D, **like)
        self.lse = torch.empty(H, T, device="cuda")
        self.stats = [torch.empty(T, device="cuda") for _ in range(4)]
        self.norm = cg.layernorm_desc(self.h)
        q = self.dqkv[:, :H]
        self.attn = cg.attn_desc(q, q, q, self.a, len(LENGTHS), D ** -0.5, False, BUCKETS, FAR, True)
        need = max(cg.cg_layernorm_workspace_bytes(self.norm), *(cg.cg_attn_workspace_bytes(self.attn, p) for p in (cg.CG_PASS_FWD, cg.CG_PASS_BWD_DATA)))
        self.ws = torch.empty(need, dtype=torch.uint8, device="cuda")

    def loss_and_gradients(self, x, target):
        """x, target [T][N] of self.dtype; the gradients go to self.grad."""
        w, d, H, dt = self.w, self.grad, self.H, self.dtype
        m1, r1, m2, r2 = self.stats
        drop = cg.drop(self.p, self.seed, self.step_count)       # another offset, other elements, every step
        cg.cg_layernorm_fwd(self.norm, x, w["g1"], w["b1"], self.h, m1, r1)
        qkv = (self.h @ w["qkv"].to(dt)).view(self.T, 3 * H, self.D)
        q, k, v = qkv[:, :H], qkv[:, H:2 * H], qkv[:, 2 * H:]
        cg.cg_attn_fwd(self.attn, q, k, v, self.cu, self.cu, w["bias"], self.a, self.lse, self.rest, self.ws)
        a = self.a.view(self.T, self.N)
        branch = a @ w["o"].to(dt)
        cg.cg_dropout_add_layernorm_fwd(self.norm, drop, branch, x, w["g2"], w["b2"], self.s, self.y, m2, r2)
        z = self.y @ w["z"].to(dt)
        diff = z.float() - target.float()
        loss = (diff * diff).mean()

        dz = (diff * (2.0 / diff.numel())).to(dt)
        d["z"].copy_(self.y.t() @ dz)
        dy = dz @ w["z"].to(dt).t()
        cg.cg_dropout_add_layernorm_bwd(self.norm, drop, dy, None, self.s, w["g2"], m2, r2, self.ds, self.db, d["g2"], d["b2"], self.ws)
        d["o"].copy_(a.t() @ self.db)
        da = (self.db @ w["o"].to(dt).t()).view(self.T, H, self.D)
        dq, dk, dv = self.dqkv[:, :H], self.dqkv[:, H:2 * H], self.dqkv[:, 2 * H:]
        cg.cg_attn_bwd(self.attn, da, q, k, v, self.cu, self.cu, w["bias"], self.a, self.rest, self.lse, dq, dk, dv, d["bias"], self.ws)
        dqkv = self.dqkv.view(self.T, 3 * self.N)
        d["qkv"].copy_(self.h.t() @ dqkv)
        torch.matmul(dqkv, w["qkv"].to(dt).t(), out=self.dh)
        dx = torch.empty_like(x)
        cg.cg_layernorm_bwd(self.norm, self.dh, x, w["g1"], m1, r1, self.ds, dx, d["g1"], d["b1"], self.ws)
        return loss, dx

    def step(self, x, target, lr=0.2, mu=0.9):
        loss, _ = self.loss_and_gradients(x, target)
        names = list(self.w)
        cg.cg_grad_reduce_sgd_multi([self.w[n] for n in names], [self.history[n] for n in names], [self.grad[n] for n in names], [[] for _ in names],
                                    [self.w[n].numel() for n in names], cg.cg_sgd(lr, mu, 0.0, 1.0))
        self.step_count += 1
        return loss


def batch(dtype, seed):
    """Inputs, and as targets the inputs two tokens before (zeros where a sequence has none)."""
    g = torch.Generator().manual_seed(seed)
    x = torch.empty(sum(LENGTHS), WIDTH).normal_(0, 1, generator=g)
    parts = [torch.cat([torch.zeros(min(2, n), WIDTH), t[:max(0, n - 2)]]) for n, t in zip(LENGTHS, x.split(list(LENGTHS)))]
    return x.to(dtype).cuda(), torch.cat(parts).to(dtype).cuda()


def main(argv=None):
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--dtype", choices=["fp32", "bf16"], default="fp32")
    args = ap.parse_args(argv)
    dtype = torch.bfloat16 if args.dtype == "bf16" else torch.float32
    layer, losses = Sublayer(dtype), []
    for i in range(args.steps):
        losses.append(layer.step(*batch(dtype, i)))
        if i % 20 == 0 or i == args.steps - 1:
            print(f"step {i:4d}  loss {float(losses[-1]):.4f}", flush=True)
    return [float(x) for x in losses]


if __name__ == "__main__":
    main()
