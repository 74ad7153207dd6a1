"""The operators of a block over tokens in training and at single tokens, as a user of the library has them computed: embedding
lookup with scaling and its gradient by sorted tokens; linear layers (the matrix product with bias, activation and residual
in its epilogue, and their backward passes, the gradient through the activation that made the input in the epilogue too);
and activations kept for the backward pass in 8 bits, alone and as what a linear layer's backward pass reads.

A case is a plain dict.  `listed()` names the cases, `draw(rng)` makes one more of the same ranges, `prepare` makes what
a program holds before the call, `run` is one pass -- through the library's entry points where `own` is true, in plain
torch operations where it is false --, `work` what a pass cannot do without and `exact` the same results in 64 bits.
"""
import math

import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
BLOCK = 32      # neighbours of a row that share a scale in 8 bits


# ---- cases ------------------------------------------------------------------------------------------------------------

def _embed(table, dtype, vocab, cols, tokens, train=False, none=0.0):
    """`none`: the share of places that hold no token (-1: a row of zeros, no gradient)."""
    return dict(op="embed", table=table, dtype=dtype, vocab=vocab, cols=cols, tokens=tokens, train=train, none=none)


def _linear(dtype, M, K, N, act="none", act_in="none", bias=True, residual=False, pad=0, train=False, packed=False):
    """M tokens, K inputs, N outputs; act: of the outputs, act_in: what made the inputs (its gradient is the backward pass's last step);
    pad: elements between rows (slices of wider tensors); packed: the backward pass reads what was kept of the inputs in 8 bits."""
    return dict(op="linear", dtype=dtype, M=M, K=K, N=N, act=act, act_in=act_in, bias=bias, residual=residual, pad=pad, train=train, packed=packed)


def _pack(dtype, rows, cols, pad=0):
    return dict(op="pack", dtype=dtype, rows=rows, cols=cols, pad=pad)


def listed():
    return [
        # the next token of eight sequences: nothing but latency
        dict(name="embed_next_tokens", **_embed("bf16", "bf16", 50000, 1024, 8)),
        # a training step over a batch of texts, the table in fp32 as the update keeps it, tokens as often as words are
        dict(name="embed_train_texts", **_embed("fp32", "bf16", 50000, 1024, 16384, train=True)),
        # a small vocabulary, odd sizes, padded texts
        dict(name="embed_train_ragged", **_embed("fp32", "fp32", 10007, 769, 3001, train=True, none=0.2)),
        # a single token through a block's first layer: the weights are read once
        dict(name="linear_one_token", **_linear("bf16", 1, 4096, 4096, act="gelu")),
        # the next token of thirteen sequences through a block's second layer
        dict(name="linear_few_tokens", **_linear("bf16", 13, 10240, 4096, residual=True)),
        # the widest fully-connected layer of the AlexNet-shaped net, batch 256, as a layer of its own in a training step
        dict(name="linear_train_fc_b256", **_linear("fp32", 256, 9216, 4096, act="relu", train=True)),
        # odd sizes, rows of wider tensors, a training step in fp32
        dict(name="linear_train_ragged", **_linear("fp32", 1500, 771, 515, act="gelu", act_in="silu", residual=True, pad=13, train=True)),
        # a block's first layer over a long prompt
        dict(name="linear_prompt", **_linear("bf16", 8192, 4096, 16384, act="gelu")),
        # the largest: a training step of a block's layer over a batch of texts
        dict(name="linear_train_wide", **_linear("bf16", 16384, 4096, 4096, act_in="gelu", residual=True, train=True)),
        # a block's second layer in a training step that keeps its inputs in 8 bits
        dict(name="linear_train_packed", **_linear("bf16", 8192, 8192, 2048, act_in="gelu", residual=True, train=True, packed=True)),
        # a batch's activations into 8 bits and out of them
        dict(name="pack_texts", **_pack("bf16", 16384, 4096)),
        # a few odd rows of a wider tensor
        dict(name="pack_ragged", **_pack("fp32", 257, 1001, pad=5)),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_embed(rng):
    train = rng.random() < 0.6
    cols = _log_int(rng, 1, 4096)
    if rng.random() < 0.5:
        cols = max(8, cols // 8 * 8)
    tokens = _log_int(rng, 1, max(2, min(100000, (1 << 25) // cols)))
    vocab = _log_int(rng, 1, max(2, min(250000, (1 << 26) // cols)))
    return _embed(rng.choice(["fp32", "fp32", "bf16"]), rng.choice(["fp32", "bf16"]), vocab, cols, tokens, train, rng.choice([0.0, 0.0, 0.1, 0.5]))


def _draw_linear(rng):
    dtype = rng.choice(["fp32", "bf16", "bf16"])
    train, packed = rng.random() < 0.5, rng.random() < 0.3
    K, N = _log_int(rng, 8, 16384), _log_int(rng, 8, 16384)
    if rng.random() < 0.6:
        K, N = max(8, K // 8 * 8), max(8, N // 8 * 8)
    most = 3e10 if dtype == "fp32" else 1e11
    M = _log_int(rng, 1, max(2, min(16384, int(most / (K * N)))))
    acts = ["none", "none", "relu", "gelu", "silu"]
    return _linear(dtype, M, K, N, rng.choice(acts), rng.choice(acts) if train else "none", rng.random() < 0.7, rng.random() < 0.5,
                   rng.choice([0, 0, 0, 8, 13]), train, train and packed)


def _draw_pack(rng):
    cols = _log_int(rng, 1, 16384)
    rows = _log_int(rng, 1, max(2, min(40000, (1 << 25) // cols)))
    if rng.random() < 0.5:
        cols = max(8, cols // 8 * 8)
    return _pack(rng.choice(["fp32", "bf16"]), rows, cols, rng.choice([0, 0, 8, 13]))


def draw(rng):
    return {"embed": _draw_embed, "linear": _draw_linear, "pack": _draw_pack}[rng.choice(["embed", "embed", "linear", "linear", "linear", "pack"])](rng)


# ---- what a program has in hand ---------------------------------------------------------------------------------------

class State:
    pass


def _rows_of(g, dt, rows, cols, pad, std):
    return torch.empty(rows, cols + pad, device="cuda").normal_(0.0, std, generator=g).to(dt)[:, :cols]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = TYPES[case["dtype"]]
    s = State()
    s.case = case
    if case["op"] == "embed":
        V, N, T = case["vocab"], case["cols"], case["tokens"]
        s.table = torch.empty(V, N, device="cuda").normal_(0.0, N ** -0.5, generator=g).to(TYPES[case["table"]])
        s.scale = N ** 0.5
        # the r-th most frequent token about 1 / r as often as the first; which ones are frequent differs from seed to seed
        u = torch.rand(T, device="cuda", generator=g, dtype=torch.float64)
        rank = torch.exp(u * math.log(V + 1)).long().sub_(1).clamp_(0, V - 1)
        s.tokens = torch.randperm(V, device="cuda", generator=g)[rank].int()
        if case["none"]:
            s.tokens[torch.rand(T, device="cuda", generator=g) < case["none"]] = -1
        s.dy = torch.empty(T, N, device="cuda").normal_(0.0, 0.01, generator=g).to(dt) if case["train"] else None
        return s
    if case["op"] == "pack":
        s.x = _rows_of(g, dt, case["rows"], case["cols"], case["pad"], 1.0)
        s.x[:, :: max(1, case["cols"] // 5)] *= 8.0      # a few channels are much larger than the others
        return s
    M, K, N, pad = case["M"], case["K"], case["N"], case["pad"]
    s.x = _rows_of(g, dt, M, K, pad, 1.0)
    s.w = _rows_of(g, dt, N, K, pad, K ** -0.5)
    s.bias = torch.empty(N, device="cuda").normal_(0.0, 0.1, generator=g) if case["bias"] else None
    s.residual = _rows_of(g, dt, M, N, pad, 1.0) if case["residual"] else None
    s.dz = _rows_of(g, dt, M, N, pad, 0.01) if case["train"] else None
    s.z_in = _rows_of(g, dt, M, K, pad, 1.0) if case["train"] and case["act_in"] != "none" else None
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------------

def run(s):
    if own:
        return {"embed": _own_embed, "linear": _own_linear, "pack": _own_pack}[s.case["op"]](s)
    return {"embed": _plain_embed, "linear": _plain_linear, "pack": _plain_pack}[s.case["op"]](s)


def _own_workspace(nbytes):
    return torch.empty(nbytes, dtype=torch.uint8, device="cuda") if nbytes else None


def _own_embed(s):
    import paper_1706_00095_amd as cg
    y = torch.empty(s.case["tokens"], s.case["cols"], dtype=TYPES[s.case["dtype"]], device="cuda")
    d = cg.embedding_desc(s.table, y, s.scale)
    cg.cg_embedding_fwd(d, s.tokens, s.table, y)
    if s.dy is None:
        return {"y": y}
    dtable = torch.empty(s.table.shape, device="cuda")
    cg.cg_embedding_bwd(d, s.tokens, s.dy, dtable, _own_workspace(cg.cg_embedding_workspace_bytes(d)))
    return {"y": y, "dtable": dtable}


def _own_linear(s):
    import paper_1706_00095_amd as cg
    c = s.case
    d = cg.linear_desc(s.x, s.w, c["act"], c["act_in"])
    y = torch.empty(c["M"], c["N"], dtype=s.x.dtype, device="cuda")
    z = torch.empty_like(y) if c["train"] and c["act"] != "none" else None
    cg.cg_linear_fwd(d, s.x, s.w, s.bias, s.residual, y, z, _own_workspace(cg.cg_linear_workspace_bytes(d, cg.CG_PASS_FWD)))
    if not c["train"]:
        return {"y": y}
    x, z_in = s.x, s.z_in
    if c["packed"]:
        x = cg.packed8_like(s.x)
        cg.cg_pack8(s.x, x)
        if z_in is not None:
            z_in = cg.packed8_like(s.z_in)
            cg.cg_pack8(s.z_in, z_in)
    dx = torch.empty(c["M"], c["K"], dtype=s.x.dtype, device="cuda")
    cg.cg_linear_bwd_data(d, s.dz, s.w, z_in, None, dx, _own_workspace(cg.cg_linear_workspace_bytes(d, cg.CG_PASS_BWD_DATA)))
    dw = torch.empty(c["N"], c["K"], device="cuda")
    dbias = torch.empty(c["N"], device="cuda") if c["bias"] else None
    cg.cg_linear_bwd_weight(d, s.dz, x, dw, dbias, _own_workspace(cg.cg_linear_workspace_bytes(d, cg.CG_PASS_BWD_WEIGHT)))
    r = {"y": y, "dx": dx, "dw": dw}
    if z is not None:
        r["z"] = z
    if dbias is not None:
        r["dbias"] = dbias
    return r


def _own_pack(s):
    import paper_1706_00095_amd as cg
    p = cg.packed8_like(s.x)
    cg.cg_pack8(s.x, p)
    y = torch.empty(s.x.shape, dtype=s.x.dtype, device="cuda")
    cg.cg_unpack8(p, y)
    return {"y": y}


# ---- the plain forms --------------------------------------------------------------------------------------------------

def _plain_embed(s):
    dt = TYPES[s.case["dtype"]]
    there = (s.tokens >= 0)[:, None]
    rows = s.tokens.long().clamp(min=0)
    y = torch.where(there, s.table[rows].float() * s.scale, 0.0).to(dt)
    if s.dy is None:
        return {"y": y}
    dtable = torch.zeros(s.table.shape, device="cuda")
    dtable.index_add_(0, rows, torch.where(there, s.dy.float(), 0.0))
    return {"y": y, "dtable": dtable.mul_(s.scale)}


def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, 0.0)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * 0.5 ** 0.5))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).float()
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (2.0 * math.pi) ** -0.5
    p = 1.0 / (1.0 + torch.exp(-z))
    return p * (1.0 + z * (1.0 - p))


def _plain_8bit(x):
    """The values that 8 bits keep of x: blocks of 32 neighbours of a row are whole numbers up to 127 times the smallest power of
    two that allows it, rounded to the nearest, halves to even."""
    rows, cols = x.shape
    f = torch.nn.functional.pad(x.float(), (0, -cols % BLOCK)).view(rows, -1, BLOCK)
    top, e = torch.frexp(f.abs().amax(2, keepdim=True))        # top in [1/2, 1): top 128 < 127.5 rounds to 127 at most
    e = (e - 7 + (top * 128.0 >= 127.5).int()).clamp(min=-133)
    # in two steps: 2^-e alone may lie outside the type's range
    half = e // 2
    q = torch.ldexp(torch.ldexp(f, -half), half - e)
    q = torch.round(q)
    return torch.ldexp(torch.ldexp(q, half), e - half).view(rows, -1)[:, :cols]


def _plain_linear(s):
    c, dt = s.case, s.x.dtype
    x, w = s.x.float(), s.w.float()
    z = torch.matmul(x, w.t())
    if s.bias is not None:
        z += s.bias
    y = _act(z, c["act"])
    if s.residual is not None:
        y = y + s.residual.float()
    r = {"y": y.to(dt)}
    if not c["train"]:
        return r
    if c["act"] != "none":
        r["z"] = z.to(dt)
    dz = s.dz.float()
    dx = torch.matmul(dz, w)
    if s.z_in is not None:
        z_in = _plain_8bit(s.z_in) if c["packed"] else s.z_in.float()
        dx *= _act_slope(z_in, c["act_in"])
    r["dx"] = dx.to(dt)
    r["dw"] = torch.matmul(dz.t(), _plain_8bit(s.x) if c["packed"] else x)
    if s.bias is not None:
        r["dbias"] = dz.sum(0)
    return r


def _plain_pack(s):
    return {"y": _plain_8bit(s.x).to(s.x.dtype)}


# ---- what a pass cannot do without --------------------------------------------------------------------------------------

def work(c):
    size = 4 if c["dtype"] == "fp32" else 2
    if c["op"] == "embed":
        V, N, T = c["vocab"], c["cols"], c["tokens"]
        rows = min(V, T)       # of the table that are read, at most
        b = T * N * size + rows * N * (4 if c["table"] == "fp32" else 2) + 4 * T
        return {"bytes": b + (T * N * size + 4 * V * N if c["train"] else 0), "flops": T * N * (2 if c["train"] else 1)}
    if c["op"] == "pack":
        n = c["rows"] * c["cols"]
        return {"bytes": 2 * n * size + 2 * n * (1 + 1 / BLOCK), "flops": 4 * n}
    M, K, N = c["M"], c["K"], c["N"]
    b = (M * K + N * K + M * N * (1 + c["residual"])) * size + 4 * N * c["bias"]
    f = 2 * M * K * N
    if c["train"]:
        b += M * N * size * (1 + (c["act"] != "none")) + M * K * size * (1 + (c["act_in"] != "none")) + 4 * N * K + 4 * N * c["bias"]
        f *= 3
    return {"bytes": b, "flops": f}


# ---- the same in 64 bits ------------------------------------------------------------------------------------------------

def _exact_embed(case, s):
    E = s.table.double()
    t = s.tokens.long()
    y = torch.zeros(case["tokens"], case["cols"], dtype=torch.float64, device="cuda")
    some = torch.nonzero(t >= 0)[:, 0]
    y[some] = E.index_select(0, t[some]) * s.scale
    if s.dy is None:
        return {"y": y}
    # tokens in order: a run's sum is a difference of running sums within a stretch of at most 1024 places
    order = some[torch.argsort(t[some], stable=True)]
    grad = torch.zeros(case["vocab"], case["cols"], dtype=torch.float64, device="cuda")
    for part in order.split(1024):
        of = t[part]
        run = torch.cumsum(s.dy[part].double(), 0)
        last = torch.nonzero(torch.cat([of[1:] != of[:-1], torch.ones(1, dtype=torch.bool, device="cuda")]))[:, 0]
        sums = run[last]
        grad[of[last]] += torch.cat([sums[:1], sums[1:] - sums[:-1]])
    return {"y": y, "dtable": grad * s.scale}


def _exact_8bit(x):
    """By whole exponents: the step of a block is the first power of two at which its largest value rounds to 127 or less."""
    rows, cols = x.shape
    v = torch.zeros(rows, (cols + BLOCK - 1) // BLOCK * BLOCK, dtype=torch.float64, device="cuda")
    v[:, :cols] = x.double()
    v = v.view(rows, -1, BLOCK)
    top = v.abs().max(2, keepdim=True).values
    step = torch.exp2(torch.floor(torch.log2(top.clamp(min=2.0 ** -200))) - 7.0)
    for _ in range(3):
        step = torch.where(torch.round(top / step) > 127, 2.0 * step, step)
    step = step.clamp(min=2.0 ** -133)
    return (torch.round(v / step) * step).view(rows, -1)[:, :cols]


def _exact_act(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "gelu":
        return z * torch.special.ndtr(z)
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def _exact_slope(z, act):
    if act == "relu":
        return torch.sign(z).clamp(min=0)
    if act == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z.square() / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        p = torch.sigmoid(z)
        return p + z * p * torch.sigmoid(-z)
    return torch.ones_like(z)


def _exact_linear(case, s):
    x, w = s.x.double(), s.w.double()
    z = torch.nn.functional.linear(x, w, None if s.bias is None else s.bias.double())
    r = {"y": _exact_act(z, case["act"]) + (0.0 if s.residual is None else s.residual.double())}
    if not case["train"]:
        return r
    if case["act"] != "none":
        r["z"] = z
    g = s.dz.double()
    kept, kept_z = s.x.double(), None if s.z_in is None else s.z_in.double()
    if case["packed"]:
        kept, kept_z = _exact_8bit(s.x), None if s.z_in is None else _exact_8bit(s.z_in)
    r["dx"] = (g @ w) * (1.0 if kept_z is None else _exact_slope(kept_z, case["act_in"]))
    r["dw"] = g.T @ kept
    if s.bias is not None:
        r["dbias"] = torch.ones(1, g.shape[0], dtype=torch.float64, device="cuda").mm(g)[0]
    return r


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "embed":
        return _exact_embed(case, s)
    if case["op"] == "pack":
        return {"y": _exact_8bit(s.x)}
    return _exact_linear(case, s)
