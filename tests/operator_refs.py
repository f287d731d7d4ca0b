"""Plain 64-bit implementations of the stand-alone operators (test infrastructure, CPU)."""
import math

import numpy as np
import torch

TOP = {torch.int8: 127.0, torch.float8_e4m3fn: 448.0}
E4M3 = np.array(sorted({(-1) ** s * (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
                        for s in (0, 1) for e in range(16) for m in range(8) if not (e == 15 and m == 7)}))


def round_e4m3(v):
    """Nearest e4m3 value by search; ties to the value with an even last mantissa bit."""
    i = np.clip(np.searchsorted(E4M3, v), 1, len(E4M3) - 1)
    lo, hi = E4M3[i - 1], E4M3[i]
    dl, dh = v - lo, hi - v

    def last_bit(x):
        e = max(math.floor(math.log2(abs(x))), -6) if x else -6
        return int(round(abs(x) / 2.0 ** (e - 3))) & 1
    pick_hi = dh < dl
    for k in np.flatnonzero(dh == dl):
        pick_hi.flat[k] = last_bit(lo.flat[k]) == 1
    return np.where(pick_hi, hi, lo)


def norm_q8(x, gain=None, residual=None, eps=1e-6, dtype=torch.int8, norm=True):
    """codes (as float64), scale, sum: s is rounded to x's type where it is stored."""
    s = x if residual is None else (x.double() + residual.double()).to(x.dtype)
    s64 = s.double().numpy()
    g = np.ones(s64.shape[1]) if gain is None else gain.double().numpy()
    t = s64 * g
    codes, scales = np.zeros_like(t), np.zeros(len(t))
    c = TOP[dtype]
    for i in range(len(t)):
        if not (np.isfinite(s64[i]).all() and np.isfinite(g).all()):
            scales[i] = np.nan
            continue
        amax = np.abs(t[i]).max()
        if amax == 0:
            scales[i] = 1.0
            continue
        v = t[i] * c / amax
        codes[i] = np.rint(v) if dtype == torch.int8 else round_e4m3(v)
        scales[i] = amax / c / (math.sqrt((s64[i] ** 2).mean() + eps) if norm else 1.0)
    return torch.from_numpy(codes), torch.from_numpy(scales), s


def act(v, name):
    if name == "relu":
        return torch.clamp(v, min=0)
    if name == "gelu":
        return 0.5 * v * (1 + torch.erf(v / math.sqrt(2)))
    if name == "gelu_tanh":
        return 0.5 * v * (1 + torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)))
    if name == "silu":
        return v / (1 + torch.exp(-v))
    return v


def linear(x, w, bias=None, act_name="none", residual=None, x_scale=None, w_scale=None):
    """(Y, sum of |terms| of the product with its scales), in 64 bits."""
    x, w = x.double(), w.double()
    y, mag = x @ w.T, x.abs() @ w.abs().T
    for s, shape in ((x_scale, (-1, 1)), (w_scale, (1, -1))):
        if s is not None:
            y, mag = y * s.double().view(shape), mag * s.double().view(shape)
    if bias is not None:
        y = y + bias.double()
    y = act(y, act_name)
    return (y if residual is None else y + residual.double()), mag


def softmax_row(z, temperature):
    """Weights of one row (numpy float64): a NaN counts as -inf, equal infinities share, nothing: the first id."""
    z = np.where(np.isnan(z), -np.inf, z)
    m = z.max()
    if m == -np.inf:
        p = np.zeros(len(z))
        p[0] = 1.0
        return p
    with np.errstate(invalid="ignore"):
        p = np.where(z == m, 1.0, np.exp((z - m) / temperature))
    return p / p.sum()


def verify_sampled(logits, tokens, parent, u, n_rows=None, temperature=1.0, draft_probs=None, lo=0, hi=None):
    """One tree after the other, one child after the other."""
    n, rows, vocab = logits.shape
    hi = vocab if hi is None else hi
    out_m, out_path, out_tok = [], np.full((n, rows), -1), np.full((n, rows), -1)
    temperature = float(np.float32(temperature))
    for b in range(n):
        z = logits[b].double().numpy()
        q = None if draft_probs is None else draft_probs[b].double().numpy()
        t, p_of, r = tokens[b].tolist(), parent[b].tolist(), u[b].double().tolist()
        count = rows if n_rows is None else min(max(int(n_rows[b]), 1), rows)
        cur, path = 0, [0]
        while True:
            p = softmax_row(z[cur][lo:hi], temperature)
            left, S, beta = p.copy(), 1.0, 0.0
            nxt = None
            for c in range(cur + 1, count):
                if p_of[c] != cur:
                    continue
                x = t[c] - lo
                ok = 0 <= x < hi - lo
                qx = 1.0 if q is None else (q[cur][t[c]] if ok and q[cur][t[c]] > 0 else 0.0)      # (a NaN counts as 0)
                if ok and left[x] > 0 and r[c] * qx * S < left[x]:
                    nxt = c
                    break
                if q is None:
                    if ok:
                        left[x] = 0.0
                else:
                    beta += S
                    left = np.maximum(p - beta * np.nan_to_num(np.maximum(q[cur][lo:hi], 0.0)), 0.0)
                S = left.sum()
            if nxt is None:
                break
            cur = nxt
            path.append(cur)
        w = left if left.sum() > 0 else p
        over = np.flatnonzero(np.cumsum(w) > r[0] * np.cumsum(w)[-1])
        last = over[0] if len(over) else np.flatnonzero(w > 0)[-1]
        m = len(path) - 1
        out_m.append(m)
        out_path[b, :m + 1] = path
        out_tok[b, :m + 1] = [t[i] for i in path[1:]] + [lo + last]
    return (torch.tensor(out_m, dtype=torch.int32), torch.from_numpy(out_path).int(), torch.from_numpy(out_tok).int())
