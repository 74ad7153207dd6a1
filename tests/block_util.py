"""Plain 64-bit forms of the operators of a block over tokens (embedding, linear layers, tensors in 8 bits), written from their
definitions for the tests, and how far the library's results may be from them: torch on the CPU, nothing of the library."""
import math

import torch

from sublayer_util import DTYPES, U, half_step  # noqa: F401


def wide(values, pad, dtype, fill=float("nan")):
    """A device tensor of these values whose rows lie `pad` elements apart (`fill` between them), and the whole of it."""
    t = torch.full((values.shape[0], values.shape[1] + pad), fill, dtype=dtype, device="cuda")
    t[:, :values.shape[1]] = values.to(dtype).cuda()
    return t[:, :values.shape[1]], t


def normal(shape, dtype, seed, std=1.0):
    """Values of a type, in float64 on the host."""
    g = torch.Generator().manual_seed(seed)
    return torch.empty(shape, dtype=torch.float64).normal_(0.0, std, generator=g).to(dtype).double()


def whole(shape, most, seed):
    """Whole numbers -most .. most, in float64 on the host."""
    g = torch.Generator().manual_seed(seed)
    return torch.randint(-most, most + 1, shape, generator=g).double()


def act(z, name):
    if name == "relu":
        return z.clamp(min=0)
    if name == "gelu":
        return z * torch.special.ndtr(z)
    if name == "silu":
        return z / (1 + torch.exp(-z))
    return z


def slope(z, name):
    if name == "relu":
        return (z > 0).double()
    if name == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "silu":
        p = 1 / (1 + torch.exp(-z))
        return p * (1 + z * (1 - p))
    return torch.ones_like(z)


def sum_error(a, b):
    """How far a product of K terms may be off: an addition every 16 terms or more, each off by at most 2 u of the magnitudes (an instruction
    may cut what lies below its sum's last place), sums of waves and of parts of K (24 more), products dropped by cutting in pieces (4 u)."""
    K = a.shape[1]
    return (2 * (K / 16 + 24) + 4) * U * (a.abs() @ b.abs())


# act is off by at most this much relative to |z| (slopes: to 1): a polynomial within 2 u and ten roundings of what is below 1; an exponential whose
# argument z^2 / 2 is off by 2 u of itself, where it is not below 2^-24 anyway (z^2 / 2 < 17: 34 u of it), and the reciprocal's and exponential's own error
ACT = 64 * U
STEEP = 1.13          # no activation's slope is above it


def linear(x, w, bias, residual, act_name, dtype):
    """(y, its tolerance, z, its tolerance)"""
    z = x @ w.T + (0 if bias is None else bias)
    ez = sum_error(x, w.T) + 2 * U * (z.abs() + (0 if bias is None else bias.abs()))
    y = act(z, act_name)
    ey = STEEP * ez + (ACT * z.abs() if act_name != "none" else 0)
    if residual is not None:
        y = y + residual
    return y, ey + (half_step(dtype) + U) * y.abs() + U * y.abs(), z, ez + (half_step(dtype) + U) * z.abs()


def linear_dx(dz, w, z_in, act_in, add, dtype):
    g = dz @ w
    e = sum_error(dz, w)
    if act_in != "none":
        e = STEEP * e + ACT * g.abs()
        g = g * slope(z_in, act_in)
    if add is not None:
        g = g + add
    return g, e + (half_step(dtype) + 2 * U) * g.abs()


def linear_dw(dz, x):
    return dz.T @ x, sum_error(dz.T, x)


def packed(x):
    """(codes, scales, values) of 8 bits, from the definition: the smallest power of two, 2^-133 to 2^121, at which the block's largest
    magnitude rounds to 127 or less, or is above 127 * 2^121 and made that.  x: float64, finite."""
    rows, cols = x.shape
    blocks = (cols + 31) // 32
    v = torch.zeros(rows, blocks * 32, dtype=torch.float64)
    v[:, :cols] = x
    v = v.view(rows, blocks, 32)
    top = v.abs().amax(2)
    scales = torch.zeros(rows, blocks, dtype=torch.int64)
    for _ in range(254):
        scales += (torch.round(top * torch.exp2(133.0 - scales.double())) > 127).long()
    step = torch.exp2(scales.double() - 133)[..., None]
    codes = torch.round(v / step).clamp(-127, 127)
    return codes.view(rows, -1)[:, :cols].to(torch.int8), scales.to(torch.uint8), (codes * step).view(rows, -1)[:, :cols]


def embedding_grad(tokens, dy, vocab, scale):
    """(dtable, its tolerance): a run of n places is summed with at most n + 8 roundings of the magnitudes."""
    out, size = (torch.zeros(vocab, dy.shape[1], dtype=torch.float64) for _ in range(2))
    there = (tokens >= 0) & (tokens < vocab)
    t = tokens[there].long()
    out.index_add_(0, t, dy[there])
    size.index_add_(0, t, dy[there].abs())
    count = torch.bincount(t, minlength=vocab).double()[:, None]
    return out * scale, (count + 8) * U * size * abs(scale)


def near(got, want, tol, what):
    got = got.detach().double().cpu()
    assert got.shape == want.shape, what
    bad = ~((got - want).abs() <= tol)
    if bad.any():
        i = tuple(int(j) for j in torch.nonzero(bad)[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off, the first at {i}: {got[i]} instead of {want[i]}, allowed {torch.as_tensor(tol).expand_as(want)[i]}")
