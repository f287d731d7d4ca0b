"""Timed cases of the stand-alone operators around a sampled verification step, through the package's
public entry points, beside their plain forms.

A case is a dict of plain values. Its "op" says which operator it is:

  norm    rmsnorm_q8: residual add, RMSNorm and rounding to 8 bits with one scale per row
  linear  linear: act(X W^T + bias) + residual, of 16-bit operands or of 8-bit codes with their scales
  verify  verify_sampled: drafted trees against the target's probabilities, by given random numbers

`run` computes the plain form (elementary torch operations) unless `own` is set, when it makes the calls
that a user makes. Sizes are those of this repository's workloads: 27 and 50 rows of a tree, a 290-row
prefix, sixteen ragged prefixes of 4764 rows, a 4096-wide decoder with an 11008-wide feed-forward layer,
32064 token ids of which 256 are action bins.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "i8": torch.int8,
         "e4m3": torch.float8_e4m3fn}
BYTES = {"f32": 4, "bf16": 2, "f16": 2, "i8": 1, "e4m3": 1}
TOP = {"i8": 127.0, "e4m3": 448.0}          # the largest code
EPS = 1e-6


# ------------------------------------------------------------------------------------ the cases
def _norm(**kw):
    return dict(dict(op="norm", rows=27, d=4096, type="bf16", to="i8", residual=True), **kw)


def _linear(**kw):
    return dict(dict(op="linear", t=27, n=4096, k=4096, type="bf16", out="bf16", bias=False, act="none",
                     residual=False), **kw)


def _verify(**kw):
    return dict(dict(op="verify", trees=1, rows=27, vocab=32064, lo=0, hi=32064, type="f32", draft="tree",
                     probs=False, ragged=False, temperature=1.0), **kw)


def listed():
    return [
        # before the head of one verification step: the rows of a 26-node tree and its root
        _norm(name="norm-27"),
        # before a layer of a batched prefill: sixteen prefixes, the residual stream in 32 bits
        _norm(name="norm-4764-e4m3", rows=4764, type="f32", to="e4m3"),
        # activations of an odd width, without a residual
        _norm(name="norm-777-odd", rows=777, d=4095, type="f16", residual=False),
        # output projection of an autoregressive step: one row, added to the residual stream
        _linear(name="linear-1", t=1, residual=True),
        # the language-model head over a tree, 8-bit codes, logits in 32 bits
        _linear(name="head-27-int8", n=32064, type="i8", out="f32"),
        # a feed-forward layer with bias and GELU over one prefix
        _linear(name="linear-290-gelu", t=290, n=11008, bias=True, act="gelu"),
        # gate and up rows of a feed-forward layer over sixteen prefixes, in 8-bit floats
        _linear(name="linear-4764-e4m3", t=4764, n=22016, type="e4m3", act="silu"),
        # every size off the tile: the rows of a batch, an odd number of outputs, a short last K block
        _linear(name="linear-1001-odd", t=1001, n=4331, k=2056, type="f16", out="f16", bias=True,
                act="gelu_tanh", residual=True),
        # one tree whose tokens are action bins: 256 of the ids take part
        _verify(name="verify-27-actions", lo=31744, hi=32000),
        # the 50-node dynamic tree over the whole vocabulary
        _verify(name="verify-50", rows=51, temperature=0.7),
        # sixteen ragged trees drawn from a draft model whose probabilities are given
        _verify(name="verify-16x50-probs", trees=16, rows=51, probs=True, ragged=True),
        # a server's batch of chains of five drafted tokens, logits in 16 bits
        _verify(name="verify-64-chains", trees=64, rows=6, type="bf16", draft="chain", probs=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("norm", "linear", "linear", "verify"))
    if op == "norm":
        return _norm(rows=_log_int(rng, 1, 4764), d=_log_int(rng, 64, 4096), type=rng.choice(("f32", "bf16", "f16")),
                     to=rng.choice(("i8", "e4m3")), residual=rng.random() < 0.6)
    if op == "linear":
        kind = rng.choice(("bf16", "f16", "i8", "e4m3"))
        t, n = _log_int(rng, 1, 4764), _log_int(rng, 64, 22016)
        k = 16 * _log_int(rng, 4, 256)                              # rows of a whole number of 16 bytes
        return _linear(t=t, n=n, k=k, type=kind, out=rng.choice(("f32", "bf16", "f16")), bias=rng.random() < 0.5,
                       act=rng.choice(("none", "relu", "gelu", "gelu_tanh", "silu")), residual=rng.random() < 0.5)
    vocab = _log_int(rng, 256, 32064)
    rows = _log_int(rng, 2, 64)
    trees = max(1, min(_log_int(rng, 1, 64), 16 * 51 * 32064 // (rows * vocab)))
    lo = rng.choice((0, 0, rng.randint(0, vocab // 2)))
    hi = rng.choice((vocab, vocab, rng.randint(lo + 64, vocab)))
    return _verify(trees=trees, rows=rows, vocab=vocab, lo=lo, hi=hi, type=rng.choice(("f32", "bf16", "f16")),
                   draft=rng.choice(("tree", "tree", "chain")), probs=rng.random() < 0.5, ragged=rng.random() < 0.5,
                   temperature=round(rng.uniform(0.3, 1.5), 3))


# ------------------------------------------------------------------------------------ inputs
def _randn(g, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32).to(dtype)


def _codes(x, to):
    """Codes and scales of a matrix's rows, as a program has them that quantised its weights."""
    amax = x.abs().amax(1)
    y = x * (TOP[to] / amax)[:, None]
    return (y.round() if to == "i8" else y).to(TYPES[to]), amax / TOP[to]


def _tree(rows, draft, rng):
    """parent, sibling rank: a chain, or a random tree of up to eight levels and eight children a node."""
    parent, rank, depth, kids = [-1], [0], [0], [0]
    for i in range(1, rows):
        p = i - 1
        if draft == "tree":
            p = int(rng.integers(0, i))
            while depth[p] >= 8 or kids[p] >= 8:
                p = int(rng.integers(0, i))
        parent.append(p), rank.append(kids[p]), depth.append(depth[p] + 1), kids.append(0)
        kids[p] += 1
    return parent, rank


def _prepare_verify(c, g, seed):
    B, R, V, lo, hi = c["trees"], c["rows"], c["vocab"], c["lo"], c["hi"]
    rng = np.random.default_rng(seed)
    built = [_tree(R, c["draft"], rng) for _ in range(B)]
    parent = torch.tensor([b[0] for b in built], dtype=torch.int32, device="cuda")
    rank = torch.tensor([b[1] for b in built], device="cuda")
    logits = _randn(g, B, R, V) * 4
    guess = logits + _randn(g, B, R, V)                             # what the draft model makes of the same rows
    logits = logits.to(TYPES[c["type"]])
    at = parent.long().clamp(min=0)
    if c["probs"]:                                                  # children are drawn from the draft's distribution
        if lo > 0 or hi < V:
            guess[..., :lo], guess[..., hi:] = -math.inf, -math.inf
        probs = torch.softmax(guess / c["temperature"], -1)
        rows = torch.arange(B, device="cuda")[:, None] * R + at
        tokens = torch.multinomial(probs.view(B * R, V), R, replacement=True, generator=g)
        tokens = tokens[rows, torch.arange(R, device="cuda")]
    else:                                                           # children are its best tokens
        probs = None
        best = torch.topk(guess[..., lo:hi], 8, dim=-1).indices + lo
        tokens = best[torch.arange(B, device="cuda")[:, None], at, rank]
    n_rows = torch.full((B,), R, dtype=torch.int32, device="cuda")
    if c["ragged"]:
        n_rows = torch.randint(1, R + 1, (B,), generator=g, device="cuda").int()
    u = torch.rand(B, R, generator=g, device="cuda")
    return dict(logits=logits, tokens=tokens.int(), parent=parent, n_rows=n_rows, probs=probs, u=u)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    c = case
    s = {"case": c}
    if c["op"] == "norm":
        dt = TYPES[c["type"]]
        s["x"] = _randn(g, c["rows"], c["d"], dtype=dt)
        # a few wide channels, as a residual stream has them
        s["x"][:, :: max(1, c["d"] // 8)] *= 8
        s["r"] = (_randn(g, c["rows"], c["d"]) * 2).to(dt) if c["residual"] else None
        s["gain"] = 1 + 0.1 * _randn(g, c["d"])
    elif c["op"] == "linear":
        x, w = _randn(g, c["t"], c["k"]), _randn(g, c["n"], c["k"]) * (1 / math.sqrt(c["k"]))
        if c["type"] in TOP:
            s["x"], s["x_scale"] = _codes(x, c["type"])
            s["w"], s["w_scale"] = _codes(w, c["type"])
        else:
            s["x"], s["w"], s["x_scale"], s["w_scale"] = x.to(TYPES[c["type"]]), w.to(TYPES[c["type"]]), None, None
        s["bias"] = _randn(g, c["n"]) if c["bias"] else None
        s["r"] = _randn(g, c["t"], c["n"], dtype=TYPES[c["out"]]) if c["residual"] else None
    else:
        s.update(_prepare_verify(c, g, seed))
    return s


# ------------------------------------------------------------------------------------ one pass
def _e4m3(v):
    """Rounds 64-bit values to the nearest e4m3 value, ties to the even one."""
    step = torch.ldexp(torch.ones_like(v), torch.frexp(v).exponent.clamp(min=-5) - 4)
    return (torch.round(v / step) * step).clamp(-448.0, 448.0)


def _plain_norm(s):
    c, x = s["case"], s["x"]
    if s["r"] is not None:
        x = (x.float() + s["r"].float()).to(x.dtype)
    # codes are decided next to borders: 64 bits
    t = x.double() * s["gain"].double()
    amax = t.abs().amax(1, keepdim=True)
    v = t * TOP[c["to"]] / amax
    codes = (torch.round(v) if c["to"] == "i8" else _e4m3(v).float()).to(TYPES[c["to"]])
    xf = x.float()
    rstd = torch.rsqrt((xf * xf).mean(1) + EPS)
    scale = amax[:, 0].float() * rstd / TOP[c["to"]]
    return (codes, scale) if s["r"] is None else (codes, scale, x)


def _act(y, act):
    if act == "relu":
        return torch.clamp(y, min=0)
    if act == "gelu":
        return 0.5 * y * (1 + torch.erf(y * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * y * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y * y * y)))
    if act == "silu":
        return y / (1 + torch.exp(-y))
    return y


def _plain_linear(s):
    c = s["case"]
    y = s["x"].float() @ s["w"].float().T
    if s["x_scale"] is not None:
        y = y * s["x_scale"][:, None] * s["w_scale"]
    if s["bias"] is not None:
        y = y + s["bias"]
    y = _act(y, c["act"])
    if s["r"] is not None:
        y = y + s["r"].float()
    return y.to(TYPES[c["out"]])


def _plain_verify(s):
    # 64 bits: a random number may fall next to a border of the cumulative sum
    c = s["case"]
    B, R, lo, hi, probs = c["trees"], c["rows"], c["lo"], c["hi"], s["probs"]
    kids, levels = (1, R - 1) if c["draft"] == "chain" else (8, min(8, R - 1))
    z = s["logits"][..., lo:hi].double()
    p = torch.exp((z - z.amax(-1, keepdim=True)) / c["temperature"])
    p = p / p.sum(-1, keepdim=True)
    q = None if probs is None else probs[..., lo:hi].double()
    # child[b, i, k]: row of the k-th child of row i, 0 where there is none
    b, row = torch.arange(B, device="cuda")[:, None], torch.arange(R, device="cuda")
    up = s["parent"].long()
    rank = ((up[:, :, None] == up[:, None, :]) & (row[None, :] < row[:, None])).sum(-1)
    there = (row > 0) & (row < s["n_rows"][:, None])
    child = torch.zeros(B, R, kids, dtype=torch.long, device="cuda")
    child.index_put_((b.expand(B, R), up.clamp(min=0), rank.clamp(max=kids - 1)), torch.where(there, row, 0), accumulate=True)
    # of every row: the child that is accepted when the walk stands there, and what is left when none is
    left, total = p.clone(), torch.ones(B, R, dtype=torch.float64, device="cuda")
    beta, step = torch.zeros_like(total), torch.zeros(B, R, dtype=torch.long, device="cuda")
    for k in range(kids):
        i = child[..., k]
        x = torch.gather(s["tokens"].long(), 1, i)
        inside = (x >= lo) & (x < hi)
        x = (x - lo).clamp(0, hi - lo - 1)[..., None]
        r = torch.gather(left, 2, x)[..., 0]
        draft = 1.0 if q is None else torch.gather(q, 2, x)[..., 0]
        turn = (i > 0) & (step == 0)
        yes = turn & inside & (torch.gather(s["u"], 1, i).double() * draft * total < r)
        no = turn & ~yes
        step = torch.where(yes, i, step)
        if q is None:
            left.scatter_(2, x, torch.where(no & inside, 0.0, r)[..., None])
        else:
            beta = torch.where(no, beta + total, beta)
            left = (p - beta[..., None] * q).clamp(min=0)
        total = left.sum(-1)
    b = b[:, 0]
    cur = torch.zeros(B, dtype=torch.long, device="cuda")
    way = [cur]
    for _ in range(levels):
        cur = torch.where(step[b, cur] > 0, step[b, cur], cur)
        way.append(cur)
    way = torch.stack(way, 1)
    fresh = torch.ones_like(way, dtype=torch.bool)
    fresh[:, 1:] = way[:, 1:] != way[:, :-1]
    m = fresh.sum(1) - 1
    path = torch.full((B, R), -1, dtype=torch.long, device="cuda")
    path[:, :levels + 1] = torch.where(fresh, way, -1)
    out = torch.full((B, R), -1, dtype=torch.long, device="cuda")
    out[:, :R - 1] = torch.where(path[:, 1:] >= 0, torch.gather(s["tokens"].long(), 1, path[:, 1:].clamp(min=0)), -1)
    # the token after them, from what is left of the last row's distribution
    w = torch.where((total[b, cur] > 0)[:, None], left[b, cur], p[b, cur])
    edge = w.cumsum(-1)
    over = edge > s["u"][:, :1].double() * edge[:, -1:]
    last = torch.where(w > 0, torch.arange(hi - lo, device="cuda"), -1).argmax(-1)
    out[b, m] = lo + torch.where(over.any(-1), over.to(torch.uint8).argmax(-1), last)
    return m.int(), path.int(), out.int()


def run(state):
    s = state
    c = s["case"]
    if own:
        from paper_2507_22424_b200 import binding as B
        if c["op"] == "norm":
            codes, scale, total = B.rmsnorm_q8(s["x"], s["gain"], residual=s["r"], eps=EPS, dtype=TYPES[c["to"]])
            return (codes, scale) if total is None else (codes, scale, total)
        if c["op"] == "linear":
            return B.linear(s["x"], s["w"], bias=s["bias"], act=c["act"], residual=s["r"], x_scale=s["x_scale"],
                            w_scale=s["w_scale"], dtype=TYPES[c["out"]])
        return B.verify_sampled(s["logits"], s["tokens"], s["parent"], s["u"], n_rows=s["n_rows"],
                                temperature=c["temperature"], draft_probs=s["probs"], lo=c["lo"], hi=c["hi"])
    return {"norm": _plain_norm, "linear": _plain_linear, "verify": _plain_verify}[c["op"]](s)


# ------------------------------------------------------------------------------------ work
def work(case):
    c = case
    if c["op"] == "norm":
        e, b = c["rows"] * c["d"], BYTES[c["type"]]
        return {"bytes": e * (b + 1 + (2 * b if c["residual"] else 0)) + 4 * (c["d"] + c["rows"]), "flops": 6 * e}
    if c["op"] == "linear":
        t, n, k = c["t"], c["n"], c["k"]
        scales = 4 * (t + n) if c["type"] in TOP else 0
        io = t * n * BYTES[c["out"]] * (2 if c["residual"] else 1)
        return {"bytes": (t + n) * k * BYTES[c["type"]] + io + scales + (4 * n if c["bias"] else 0), "flops": 2 * t * n * k}
    # every row's logits once, the draft's probabilities where the walk ends, the trees and the answers
    rows, v = c["trees"] * c["rows"], c["hi"] - c["lo"]
    return {"bytes": rows * v * BYTES[c["type"]] + (c["trees"] * v * 4 if c["probs"] else 0) + rows * 20,
            "flops": 4 * rows * v}


# ------------------------------------------------------------------------------------ in 64 bits
def _exact_norm(s):
    c = s["case"]
    x = s["x"].double()
    if s["r"] is not None:
        x = (x + s["r"].double()).to(s["x"].dtype).double()         # the sum is rounded where it is stored
    rms = torch.sqrt((x ** 2).sum(1) / c["d"] + EPS)
    biggest = (x * s["gain"].double()).abs().max(1).values
    out = (None, biggest / rms / TOP[c["to"]])
    return out if s["r"] is None else (*out, x)


def _exact_linear(s):
    c = s["case"]
    y = torch.nn.functional.linear(s["x"].double(), s["w"].double())
    if s["x_scale"] is not None:
        y *= torch.outer(s["x_scale"].double(), s["w_scale"].double())
    if s["bias"] is not None:
        y += s["bias"].double()
    f = {"none": lambda v: v, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu,
         "gelu_tanh": lambda v: torch.nn.functional.gelu(v, approximate="tanh")}[c["act"]]
    y = f(y)
    return y if s["r"] is None else y + s["r"].double()


def exact(case, seed):
    if case["op"] == "verify":
        return None                                                 # whole numbers only
    s = prepare(case, seed)
    return _exact_norm(s) if case["op"] == "norm" else _exact_linear(s)
