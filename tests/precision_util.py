"""Inputs and bounds for the precision that attention's differences need, and what the results would be with fewer bits (for the tests
of the tests).  Plain 64-bit forms on the host, nothing of the library."""
import torch

from sublayer_util import U, Attention

BF = torch.bfloat16


def few_keys_values(lens, H, D, seed=5):
    """q, k, v, do of packed sequences (float64, exact in bf16): v lies about 256, so that what a row's dP differ by is a small part of them,
    and do has one element a row."""
    g = torch.Generator().manual_seed(seed)
    T = sum(lens)
    q, k, v = (torch.empty(T, H, D, dtype=torch.float64).normal_(m, s, generator=g).to(BF).double() for m, s in ((0, 1), (0, 1), (256, 4)))
    return q, k, v, one_element((T, H, D), g)


def one_element(shape, g):
    return torch.zeros(shape, dtype=torch.float64).scatter_(2, torch.randint(0, shape[2], (*shape[:2], 1), generator=g), 1.0)


def few_keys_bounds(vals, lens, scale, causal):
    """The plain form with the tolerances of probabilities that keep 16 bits or more in o, and of an o of 16 bits or more in delta: those
    that sublayer_util.Attention gives a call with a bias (here of zeros)."""
    return Attention(*vals, lens, lens, scale, causal, torch.zeros(vals[0].shape[1], 4, dtype=torch.float64), 4, 3, True, BF, True)


def pieces(x, n):
    """x cut to n bf16 numbers, each the nearest of what the ones before it left."""
    got = torch.zeros_like(x)
    for _ in range(n):
        got = got + (x - got).float().to(BF).double()
    return got


def unrounded_bounds(vals, lens_q, lens_k, scale, causal, bias=None, far=0):
    """The plain form with the tolerances of probabilities and dS that keep 16 bits or more in all products (2^-18 of themselves, the 64
    roundings of 2^-24 that sublayer_util.Attention allows a product's sum in fp32), where only results are rounded to bf16."""
    n = bias.shape[1] if bias is not None else 0
    return Attention(*vals, lens_q, lens_k, scale, causal, bias, n, far, not causal, torch.float32, False)


def dq_with(vals, lens, scale, causal, p_pieces, ds_pieces=9):
    """dq (before its own rounding) where the probabilities of the forward product, and dS, have so many bf16 numbers; the rest in 64 bits."""
    q, k, v, do = vals
    dq, at = torch.zeros_like(q), 0
    for n in lens:
        s = slice(at, at + n)
        sees = torch.arange(n)[None, :] <= torch.arange(n)[:, None] if causal else torch.ones(n, n, dtype=torch.bool)
        for h in range(q.shape[1]):
            S = torch.where(sees, q[s, h] @ k[s, h].T * scale, -torch.inf)
            p = torch.exp(S - S.amax(1, keepdim=True))
            l = p.sum(1, keepdim=True)
            delta = (do[s, h] * (pieces(p, p_pieces) @ v[s, h] / l)).sum(1, keepdim=True)
            dq[s, h] = pieces(p / l * (do[s, h] @ v[s, h].T - delta), ds_pieces) @ k[s, h] * scale
        at += n
    return dq


# A head's three tokens, each of which sees all three.  v about 64, do with one element: delta is one element of o.  Scores are the
# bias alone, 0 for a token and itself and of -1 .. 0 for the others, such that their probabilities lose much without a third piece.
TOKENS, HEADS, BUCKETS, FAR = 3, 64, 16, 20


def three_tokens(D, seed):
    g = torch.Generator().manual_seed(seed)
    q, k = (torch.empty(TOKENS, HEADS, D, dtype=torch.float64).normal_(0, 2.0 ** -40, generator=g).to(BF).double() for _ in range(2))
    v = torch.empty(TOKENS, HEADS, D, dtype=torch.float64).normal_(64, 1, generator=g).to(BF).double()
    bias = -torch.rand(HEADS * BUCKETS * 64, generator=g).double()
    p = torch.exp(bias)
    bias = bias[(p - pieces(p, 2)) / p > 40 * U][:HEADS * BUCKETS].reshape(HEADS, BUCKETS).contiguous()
    bias[:, 0] = 0.0
    return (q, k, v, one_element((TOKENS, HEADS, D), g)), bias


def outer_differences(vals, bias, p_of=lambda p: p, o_of=lambda o: o):
    """dS of the first query and the last key and of the last query and the first key, [2][heads], which are sums of their own in the
    bias's gradient (buckets 8 + 2 and 2); and what an error of o's relative size 1 in delta would change them by."""
    _, _, v, do = vals
    distance = torch.arange(TOKENS)[None, :] - torch.arange(TOKENS)[:, None]
    bucket = torch.where(distance > 0, distance + BUCKETS // 2, -distance)
    p = torch.exp(bias[:, bucket])                                     # [heads][query][key]
    p = p / p.amax(2, keepdim=True)
    l = p.sum(2, keepdim=True)
    vh, dh = v.transpose(0, 1), do.transpose(0, 1)
    o = o_of(p_of(p) @ vh / l)
    dS = p / l * (dh @ vh.transpose(1, 2) - (dh * o).sum(2, keepdim=True))
    size = p / l * (dh * o).sum(2, keepdim=True)
    return torch.stack([dS[:, 0, 2], dS[:, 2, 0]]), torch.stack([size[:, 0, 2], size[:, 2, 0]])


# Root mean square of (dS - exact) / size.  Roundings of at most a step each (2 U, U = 2^-24), taken as independent and even: exp of the
# probability and of the row's sum 2 U each and three more in their arguments (2 U at sizes up to 1), six additions inside and between
# three matrix products (2 U), eleven others of U (l, 1 / l, their product, o_rest, delta, the differences): squares 4 (8 + 6) + 11 = 67 and
# 67 / 3 for even distributions, 4.7 U.  Twice that, and a quarter more for roundings that are cut off instead of to nearest.
RMS = 12 * U
