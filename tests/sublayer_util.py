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
