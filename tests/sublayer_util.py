"""Plain 64-bit forms of the operators of an attention sublayer (dropout, layer norm, attention), written from their
definitions for the tests: numpy and torch on the CPU, nothing of the library."""
import math

import numpy as np
import torch

LOW = np.uint64(0xFFFFFFFF)
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def half_step(dtype):
    """What one rounding to a type is off by, relative to the value."""
    return torch.finfo(dtype).eps / 2


def philox(counter, key, rounds=10):
    """Philox4x32 of counters [n][4] with key (k0, k1); uint32 [n][4]."""
    c = [counter[:, i].astype(np.uint64) for i in range(4)]
    k0, k1 = int(key[0]), int(key[1])
    for _ in range(rounds):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), b & LOW, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), a & LOW]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return np.stack(c, 1).astype(np.uint32)


def threshold(p):
    return min(65535, int(math.floor(65536.0 * p + 0.5)))


def keep_factors(rows, cols, p, seed, offset):
    """0 or 65536 / (65536 - t) for every element, float64 [rows][cols]."""
    n = rows * cols
    blk = np.arange((n + 7) // 8, dtype=np.uint64)
    ctr = np.stack([blk & LOW, blk >> np.uint64(32), np.full_like(blk, offset & 0xFFFFFFFF), np.full_like(blk, offset >> 32)], 1)
    w = philox(ctr, (seed & 0xFFFFFFFF, seed >> 32))
    halves = np.stack([w & 0xFFFF, w >> 16], 2).reshape(-1)[:n]
    t = threshold(p)
    return torch.from_numpy((halves >= t).astype(np.float64).reshape(rows, cols)) * (65536.0 / (65536 - t))


def norm(x, gamma, beta, eps):
    """(y, xhat, mean, rstd) of float64 rows."""
    mean = x.mean(1)
    var = ((x - mean[:, None]) ** 2).mean(1)
    rstd = 1.0 / torch.sqrt(var + eps)
    xh = (x - mean[:, None]) * rstd[:, None]
    return xh * gamma + beta, xh, mean, rstd


def norm_bwd(dy, xh, rstd, gamma):
    g = dy * gamma
    dx = rstd[:, None] * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    return dx, (dy * xh).sum(0), dy.sum(0)


def rows_of(shape, pad, dtype, seed, std=1.0, mean=0.0):
    """A device tensor whose rows lie `pad` elements apart (NaN between them), and the same in float64 on the host."""
    g = torch.Generator().manual_seed(seed)
    v = torch.empty(shape, dtype=torch.float64).normal_(mean, std, generator=g).to(dtype)
    wide = torch.full((shape[0], shape[1] + pad), float("nan"), dtype=dtype, device="cuda")
    wide[:, :shape[1]] = v.cuda()
    return wide[:, :shape[1]], v.double()


def bucket_of(dist, n, far):
    """The bucket of a distance, in whole numbers: step t is reached where dist^m E^t >= E^m far^t, m steps in all."""
    E = n // 2
    if dist < E:
        return dist
    dist, m, t = min(dist, far), n - E, 0
    while t < m - 1 and dist ** m * E ** (t + 1) >= E ** m * far ** (t + 1):
        t += 1
    return E + t


def buckets_of(delta, buckets, max_distance, both):
    """Buckets of key position minus query position, whole numbers of any shape."""
    n = buckets // 2 if both else buckets
    table = torch.tensor([bucket_of(d, n, max_distance) for d in range(max_distance + 1)])
    dist = (delta.abs() if both else (-delta).clamp(min=0)).clamp(max=max_distance)
    b = table[dist]
    return torch.where(delta > 0, b + n, b) if both else b


U = 2.0 ** -24


class Attention:
    """One call's plain form in 64 bits on the host, and how far the library's results may be from it.

    u = 2^-24.  A score is a sum of D products in at most D / 16 * 6 + 8 <= 56 roundings of the products' magnitudes; an
    exponential's argument is off by that and by 4 u of itself, so a probability is off by `R` relative, with another
    (m / 32 + 64) u for the sums of a row.  bf16: the probabilities, and the gradients of the scores, are rounded once for their
    products (half a step each).  Everything else follows by the products' magnitudes; results are rounded once more (near)."""

    def __init__(self, q, k, v, do, lens_q, lens_k, scale, causal, bias, buckets, max_distance, both, dtype, rest):
        Tq, Hq, D = q.shape
        G = Hq // k.shape[1]
        z = torch.zeros
        self.o, self.tol_o = z(Tq, Hq, D, dtype=torch.float64), z(Tq, Hq, D, dtype=torch.float64)
        self.lse, self.tol_lse = z(Hq, Tq, dtype=torch.float64), z(Hq, Tq, dtype=torch.float64)
        self.dq, self.tol_dq = torch.zeros_like(q), torch.zeros_like(q)
        self.dk, self.tol_dk, self.dv, self.tol_dv = (torch.zeros_like(k) for _ in range(4))
        self.dbias, self.tol_dbias = (z(Hq, max(buckets, 1), dtype=torch.float64) for _ in range(2))
        hs = half_step(dtype)
        pr = hs if dtype == torch.bfloat16 else 0.0
        # with a bias and o_rest the probabilities of the forward product are held in two bf16 numbers
        pr_o = pr * pr if rest and buckets else pr
        q0 = k0 = 0
        for n, m in zip(lens_q, lens_k):
            delta = torch.arange(m)[None, :] - torch.arange(n)[:, None] - (m - n)
            b = buckets_of(delta, buckets, max_distance, both) if buckets else None
            sees = delta <= 0 if causal else torch.ones(n, m, dtype=torch.bool)
            for h in range(Hq if n else 0):
                Q, K, V, dO = q[q0:q0 + n, h], k[k0:k0 + m, h // G], v[k0:k0 + m, h // G], do[q0:q0 + n, h]
                S = Q @ K.T * scale + (bias[h][b] if buckets else 0)
                S = torch.where(sees, S, -math.inf)
                size = Q.abs() @ K.abs().T * scale + (torch.nan_to_num(bias[h], neginf=0.0).abs()[b] if buckets else 0)
                big = size.amax(1, keepdim=True) if m else z(n, 1, dtype=torch.float64)
                lse = torch.logsumexp(S, 1) if m else torch.full((n,), -math.inf, dtype=torch.float64)
                P = torch.where(lse[:, None] == -math.inf, 0.0, torch.exp(S - torch.where(lse == -math.inf, 0.0, lse)[:, None]))
                e = 56 * U * big + 8 * U * (big + lse.nan_to_num(neginf=0.0).abs()[:, None])
                R = 2 * e + (m / 32 + 64) * U
                O, PV = P @ V, P @ V.abs()
                self.o[q0:q0 + n, h], self.lse[h, q0:q0 + n] = O, lse
                to = (pr_o + R) * PV
                self.tol_o[q0:q0 + n, h], self.tol_lse[h, q0:q0 + n] = to, (e + R)[:, 0]
                dP = dO @ V.T
                D_ = (dO * O).sum(1, keepdim=True)
                dS = P * (dP - D_)
                # the o that delta is formed with: rounded once, or in two numbers
                eD = (dO.abs() * (to + (hs * hs if rest else hs if pr else 2 * U) * O.abs())).sum(1, keepdim=True) + 64 * U * (dO.abs() * O.abs()).sum(1, keepdim=True)
                eS = P * (56 * U * (dO.abs() @ V.abs().T) + eD) + (R + 4 * U) * P * (dP.abs() + D_.abs())
                eSr = eS + pr * dS.abs() + (m + n) / 32 * U * dS.abs()
                self.dq[q0:q0 + n, h] = dS @ K * scale
                self.tol_dq[q0:q0 + n, h] = (eSr + (m / 32 + 64) * U * dS.abs()) @ K.abs() * scale
                kk = slice(k0, k0 + m)
                self.dk[kk, h // G] += dS.T @ Q * scale
                self.tol_dk[kk, h // G] += (eSr + (n * G / 32 + 64) * U * dS.abs()).T @ Q.abs() * scale
                self.dv[kk, h // G] += P.T @ dO
                self.tol_dv[kk, h // G] += ((pr + R + (n * G / 32 + 64) * U) * P).T @ dO.abs()
                if buckets:
                    flat = b.reshape(-1)
                    self.dbias[h].scatter_add_(0, flat, dS.reshape(-1))
                    self.tol_dbias[h].scatter_add_(0, flat, (eS + 256 * U * dS.abs()).reshape(-1))
            q0, k0 = q0 + n, k0 + m
