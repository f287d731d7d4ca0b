"""The stand-alone operators against plain 64-bit implementations (operator_refs.py)."""
import math

import numpy as np
import pytest
import torch

import operator_refs as ref

pytestmark = pytest.mark.gpu

BF, HF, F32, I8, E4 = torch.bfloat16, torch.float16, torch.float32, torch.int8, torch.float8_e4m3fn


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _randn(g, *shape):
    return torch.randn(*shape, generator=g)


def _b():
    from paper_2507_22424_b200 import binding
    return binding


# ------------------------------------------------------------------------------------ norm
def check_norm(x, gain, residual, eps, dtype, got, norm=True):
    codes, scale, total = got
    rc, rs, rt = ref.norm_q8(x, gain, residual, eps, dtype, norm)
    assert codes.dtype == dtype
    assert torch.equal(codes.cpu().float().double(), rc)
    # 64-bit scale rounded to f32; the sum of squares is fp32: each of d terms is off by 2^-24 of itself, and a
    # thread's 16 or more, then a tree of at most 10 + 16 levels, add 2^-24 each; the root halves it
    tol = (1 + 64 + x.shape[1] / 512) * 2.0 ** -24
    s = scale.cpu().double()
    ok = torch.isfinite(rs)
    assert torch.equal(torch.isnan(s), torch.isnan(rs))
    assert ((s[ok] - rs[ok]).abs() <= tol * rs[ok].abs() + 2.0 ** -149).all()
    if residual is not None:
        assert torch.equal(total.cpu(), rt) or torch.equal(torch.nan_to_num(total.cpu()), torch.nan_to_num(rt))


@pytest.mark.parametrize("rows,d", [(1, 1), (1, 8), (3, 17), (27, 4096), (5, 4095), (150, 256), (2, 33000), (1, 11008)])
@pytest.mark.parametrize("dtype", [I8, E4])
@pytest.mark.parametrize("kind", [F32, BF, HF])
def test_norm_codes_are_exact(rows, d, dtype, kind):
    g = _gen(rows * 7919 + d)
    x, r = (_randn(g, rows, d) * 3).to(kind), _randn(g, rows, d).to(kind)
    gain = 1 + 0.2 * _randn(g, d)
    got = _b().rmsnorm_q8(x.cuda(), gain.cuda(), residual=r.cuda(), dtype=dtype)
    check_norm(x, gain, r, 1e-6, dtype, got)
    got = _b().rmsnorm_q8(x.cuda(), dtype=dtype)
    check_norm(x, None, None, 1e-6, dtype, got)
    assert got[2] is None


@pytest.mark.parametrize("dtype", [I8, E4])
def test_norm_codes_next_to_borders(dtype):
    """Values that fall on, or one 64-bit step beside, the middle between two codes."""
    c = ref.TOP[dtype]
    mids = np.arange(-126.5, 127) if dtype == I8 else (ref.E4M3[1:] + ref.E4M3[:-1]) / 2
    amax = 3.25
    v = torch.from_numpy(mids * amax / c).float()
    v = torch.cat([v, torch.nextafter(v, v + 1), torch.nextafter(v, v - 1)])
    x = torch.cat([v, torch.tensor([amax])])[None].repeat(3, 1)
    gain = torch.ones(x.shape[1])
    check_norm(x, gain, None, 1e-6, dtype, _b().rmsnorm_q8(x.cuda(), gain.cuda(), dtype=dtype))
    gain = 1 + 0.1 * _randn(_gen(3), x.shape[1])
    check_norm(x, gain, None, 1e-6, dtype, _b().rmsnorm_q8(x.cuda(), gain.cuda(), dtype=dtype))


@pytest.mark.parametrize("dtype", [I8, E4])
@pytest.mark.parametrize("d", [24, 23])
def test_norm_rows_that_are_not_ordinary(dtype, d):
    g = _gen(d)
    x = _randn(g, 12, d)
    x[0] = 0
    x[1] *= 1e30            # squares past fp32
    x[2] *= 1e-30           # and below it
    x[3] = 0
    x[3, 5] = 1e-45
    x[4, 7] = math.inf
    x[5, 1] = math.nan
    x[6] = 3e38             # the product with a gain of 2 passes fp32
    x[7, 0] = -3e38
    x[8] = -0.0
    x[9, 3] = -math.inf
    gain = torch.full((d,), 2.0)
    for eps in (1e-6, 0.0):
        check_norm(x, gain, None, eps, dtype, _b().rmsnorm_q8(x.cuda(), gain.cuda(), eps=eps, dtype=dtype))
    gain[2] = 0
    check_norm(x, gain, None, 1e-6, dtype, _b().rmsnorm_q8(x.cuda(), gain.cuda(), dtype=dtype))
    # two infinities of opposite sign in the sum
    r = torch.zeros_like(x)
    r[9, 3] = math.inf
    check_norm(x, gain, r, 1e-6, dtype, _b().rmsnorm_q8(x.cuda(), gain.cuda(), residual=r.cuda(), dtype=dtype))


@pytest.mark.parametrize("kind", [F32, BF])
@pytest.mark.parametrize("rows,d", [(5, 64), (3, 20000), (7, 61)])
def test_norm_sum_in_place_and_strided_rows(kind, rows, d):
    g = _gen(11)
    x, r = _randn(g, rows, d).to(kind), _randn(g, rows, d).to(kind)
    gain = 1 + 0.1 * _randn(g, d)
    for which in (0, 1):
        wide = torch.full((rows, 2 * d + 8), 7.0, dtype=kind, device="cuda")
        wide[:, :d], wide[:, d + 8:] = x.cuda(), r.cuda()
        xs, rs = wide[:, :d], wide[:, d + 8:]
        got = _b().rmsnorm_q8(xs, gain.cuda(), residual=rs, out_sum=(xs, rs)[which])
        check_norm(x, gain, r, 1e-6, I8, got)
        assert torch.equal((rs, xs)[which].cpu(), (r, x)[which])      # the other one stays
        assert (wide[:, d:d + 8] == 7).all()


@pytest.mark.parametrize("rows", [3, 700])
def test_norm_sum_without_a_residual_is_x(rows):
    """Through the C entry point (the binding has no such call): the sum receives x, codes and scale are those of x."""
    B = _b()
    x = _randn(_gen(8), rows, 64).half()
    xc, s = x.cuda(), torch.zeros(rows, 64, dtype=HF, device="cuda")
    codes, scale = torch.zeros(rows, 64, dtype=I8, device="cuda"), torch.zeros(rows, device="cuda")
    assert B.lib.specvla_rmsnorm_q8(B.NORM_ARGS.pack(rows, 64, 2, 3, xc.data_ptr(), 64, 0, 0, 0, s.data_ptr(), 64, codes.data_ptr(), 64,
                                                     scale.data_ptr(), 1e-6), B._stream()) == 0
    assert torch.equal(s, xc)
    check_norm(x, None, None, 1e-6, I8, (codes, scale, None))


@pytest.mark.parametrize("kind", [F32, BF, HF])
@pytest.mark.parametrize("d", [64, 1024, 4096, 4104, 8192, 9000, 16384])
@pytest.mark.parametrize("dtype", [I8, E4])
def test_norm_of_many_rows(kind, d, dtype):
    """The kernel that copies ahead: every width of its CTAs, full and partly filled, rows of every sort among ordinary ones."""
    g = _gen(d)
    rows = 650
    x, r = (_randn(g, rows, d) * 2).to(kind), _randn(g, rows, d).to(kind)
    x[7] = r[7] = 0
    x[8, 3], x[600, d - 1] = math.nan, math.inf
    x[9], r[9] = 1e-4, 0
    gain = 1 + 0.2 * _randn(g, d)
    gain[: d // 2] = 1                                                # exact products: ties with the middle between two codes
    check_norm(x, gain, r, 1e-6, dtype, _b().rmsnorm_q8(x.cuda(), gain.cuda(), residual=r.cuda(), dtype=dtype))
    codes, scale = _b().quantize_rows(x.cuda(), dtype)
    check_norm(x, None, None, 0.0, dtype, (codes, scale, None), norm=False)
    xc, rc = x.cuda(), r.cuda()
    check_norm(x, gain, r, 1e-6, dtype, _b().rmsnorm_q8(xc, gain.cuda(), residual=rc, dtype=dtype, out_sum=xc))


@pytest.mark.parametrize("kind", [F32, BF, HF])
@pytest.mark.parametrize("dtype", [I8, E4])
def test_quantize_rows(kind, dtype):
    x = (_randn(_gen(5), 9, 300) * 2).to(kind)
    codes, scale = _b().quantize_rows(x.cuda(), dtype)
    check_norm(x, None, None, 0.0, dtype, (codes, scale, None), norm=False)


# ------------------------------------------------------------------------------------ linear
def operands(g, T, N, K, kind):
    x, w = _randn(g, T, K), _randn(g, N, K) / math.sqrt(K)
    if kind in (BF, HF):
        return x.to(kind), w.to(kind), None, None
    (xc, xs, _), (wc, ws, _) = ref.norm_q8(x, dtype=kind, norm=False), ref.norm_q8(w, dtype=kind, norm=False)
    return xc.float().to(kind), wc.float().to(kind), xs.float(), ws.float()


def check_linear(y, want, mag, K, kind, dtype, act, bias, residual):
    """Error bound: fp32 products are summed with at most K roundings (2^-23 each, were the adder to cut off) of the sum of
    their magnitudes (int8: exact); scales and bias round up to four times, an activation of slope < 1.2 up to eight
    times (argument and result), the residual once: 2^-24 of the largest value met each; then half a step of the type."""
    m = mag.double()
    acc = (0 if kind == I8 else K * 2.0 ** -23) * m
    big = m + (bias.abs().double() if bias is not None else 0) + (residual.abs().double() if residual is not None else 0)
    tol = 1.2 * acc + 16 * 2.0 ** -24 * big
    tol = tol + torch.finfo(dtype).eps / 2 * (want.abs() + tol) + torch.finfo(dtype).tiny
    err = (y.cpu().double() - want).abs()
    assert (err <= tol).all(), float((err - tol).max())


@pytest.mark.parametrize("kind", [BF, HF, I8, E4])
@pytest.mark.parametrize("T,N,K", [(1, 1, 16), (1, 128, 64), (3, 300, 208), (16, 129, 1040), (33, 4, 32), (129, 640, 400),
                                   (257, 257, 144), (300, 1000, 96), (64, 2000, 2064), (700, 384, 512)])
def test_linear_shapes(kind, T, N, K):
    g = _gen(T * 31 + N * 7 + K)
    x, w, xs, ws = operands(g, T, N, K, kind)
    cu = lambda t: None if t is None else t.cuda()  # noqa: E731
    for dtype in (F32, BF, HF):
        y = _b().linear(cu(x), cu(w), x_scale=cu(xs), w_scale=cu(ws), dtype=dtype)
        want, mag = ref.linear(x, w, x_scale=xs, w_scale=ws)
        assert y.dtype == dtype and y.shape == (T, N)
        check_linear(y, want, mag, K, kind, dtype, "none", None, None)
    _b().linear_status()


@pytest.mark.parametrize("kind", [BF, HF, I8, E4])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("T,N,K", [(5, 131, 272), (280, 256, 160), (40, 4096, 1024)])
def test_linear_epilogue(kind, act, T, N, K):
    g = _gen(T + N)
    x, w, xs, ws = operands(g, T, N, K, kind)
    bias = _randn(g, N)
    cu = lambda t: None if t is None else t.cuda()  # noqa: E731
    for dtype in (F32, BF):
        r = _randn(g, T, N).to(dtype)
        want, mag = ref.linear(x, w, bias, act, r, xs, ws)
        y = _b().linear(cu(x), cu(w), cu(bias), act, cu(r), cu(xs), cu(ws), dtype=dtype)
        check_linear(y, want, mag, K, kind, dtype, act, bias, r)
        # in place of the residual, in rows further apart than they are long
        wide = torch.full((T, N + 6), 5.0, dtype=dtype, device="cuda")
        wide[:, 1:N + 1] = r.cuda()
        got = _b().linear(cu(x), cu(w), cu(bias), act, wide[:, 1:N + 1], cu(xs), cu(ws), out=wide[:, 1:N + 1])
        assert torch.equal(got, y)
        assert (wide[:, 0] == 5).all() and (wide[:, N + 1:] == 5).all()
    _b().linear_status()


@pytest.mark.parametrize("kind", [BF, I8])
def test_linear_of_more_tiles_than_fit_at_once(kind):
    """Persistent CTAs take several tiles each, over both accumulator buffers."""
    g = _gen(12)
    T, N, K = 1500, 5001, 272
    x, w, xs, ws = operands(g, T, N, K, kind)
    bias, r = _randn(g, N), _randn(g, T, N)
    cu = lambda t: None if t is None else t.cuda()  # noqa: E731
    y = _b().linear(cu(x), cu(w), cu(bias), "silu", cu(r), cu(xs), cu(ws), dtype=F32)
    want, mag = ref.linear(x, w, bias, "silu", r, xs, ws)
    check_linear(y, want, mag, K, kind, F32, "silu", bias, r)
    _b().linear_status()


def test_linear_strided_operands_and_odd_k():
    g = _gen(8)
    T, N, K = 19, 70, 333
    for kind, step in ((BF, 8), (I8, 16)):
        x, w, xs, ws = operands(g, T, N, K, kind)
        ld = (K + step - 1) // step * step + step
        xb = torch.full((T, ld), 99, dtype=kind, device="cuda")      # what lies past K must not count
        wb = torch.full((N, ld), 77, dtype=kind, device="cuda")
        xb[:, :K], wb[:, :K] = x.cuda(), w.cuda()
        y = _b().linear(xb[:, :K], wb[:, :K], x_scale=None if xs is None else xs.cuda(),
                        w_scale=None if ws is None else ws.cuda(), dtype=F32)
        want, mag = ref.linear(x, w, x_scale=xs, w_scale=ws)
        check_linear(y, want, mag, K, kind, F32, "none", None, None)


@pytest.mark.parametrize("T", [7, 300])
def test_linear_non_finite_values_stay_where_they_belong(T):
    g = _gen(2)
    N, K = 260, 128
    x, w, _, _ = operands(g, T, N, K, BF)
    x[3, 5], w[17, 9] = math.nan, math.inf
    r = torch.zeros(T, N)
    r[0, 0] = -math.inf
    y = _b().linear(x.cuda(), w.cuda(), residual=r.cuda(), dtype=F32).cpu()
    bad = torch.zeros(T, N, dtype=torch.bool)
    bad[3], bad[:, 17], bad[0, 0] = True, True, True
    assert torch.equal(~torch.isfinite(y), bad)


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("dtype", [F32, BF, HF])
@pytest.mark.parametrize("T", [3, 200])
def test_linear_activations_far_out(act, dtype, T):
    """Infinities, NaN and the tails, by a bias: as the formula gives them, tails within what their fp32 form rounds."""
    vals = torch.tensor([math.inf, -math.inf, math.nan, 60.0, -60.0, 12.0, -12.0, 6.0, -6.0, 4.0, -4.0, 1e-3, -1e-3, 0.0, -88.0, 100.0, -100.0, 1e30, -1e30])
    x, w = torch.zeros(T, 16, dtype=HF), torch.zeros(len(vals), 16, dtype=HF)
    y = _b().linear(x.cuda(), w.cuda(), vals.cuda(), act, dtype=dtype).cpu()
    want = ref.act(vals.double(), act).to(dtype).double()
    for row in y.double():
        fin = torch.isfinite(want)
        assert torch.equal(torch.isnan(row), torch.isnan(want)) and torch.equal(row[~fin & ~torch.isnan(want)], want[~fin & ~torch.isnan(want)])
        # 1 + erf and 1 + tanh are off by 2^-23 where they are near 0 (fp32), the 16-bit form of erf by 1.5e-7 in all
        tol = 2.0 ** -22 * vals.abs().double()[fin] + torch.finfo(dtype).eps * want[fin].abs() + torch.finfo(dtype).tiny
        assert ((row[fin] - want[fin]).abs() <= tol).all()


def test_linear_int8_sums_are_exact():
    """The largest products an int8 row can make: the sum is a 32-bit integer, rounded once."""
    K = 131056
    x = torch.full((2, K), -128, dtype=I8)
    w = torch.full((3, K), -128, dtype=I8)
    w[1] = 127
    w[2, ::2] = 1
    y = _b().linear(x.cuda(), w.cuda(), dtype=F32).cpu()
    want = (x.double() @ w.double().T).float()
    assert torch.equal(y, want)


def test_linear_wait_that_gives_up_is_reported_once():
    """A K block that never comes: every wait runs out, the status says so, and the next call is right."""
    B = _b()
    g = _gen(4)
    for T, N, K in ((5, 256, 1024), (400, 512, 1024)):
        x, w, _, _ = operands(g, T, N, K, BF)
        xc, wc = x.cuda(), w.cuda()
        assert B.lib.specvla_linear_fault_test(2_000_000, 1) == 0
        B.linear(xc, wc)
        with pytest.raises(B.SpecVLAError) as e:
            B.linear_status()
        assert e.value.code == -6
        B.linear_status()
        want, mag = ref.linear(x, w)
        check_linear(B.linear(xc, wc), want, mag, K, BF, BF, "none", None, None)
        B.linear_status()


# ------------------------------------------------------------------------------------ verification
def trees(rng, n, rows, chain=False):
    parent = np.full((n, rows), -1)
    for b in range(n):
        for i in range(1, rows):
            parent[b, i] = i - 1 if chain else rng.integers(0, i)
    return torch.from_numpy(parent).int()


def drafted(rng, logits, parent, probs, lo, hi):
    """Tokens: drawn from the parent's draft distribution, or likely under the target."""
    n, rows, _ = logits.shape
    tok = np.zeros((n, rows), dtype=np.int64)
    for b in range(n):
        for i in range(1, rows):
            p = int(parent[b, i])
            w = probs[b, p].double().numpy() if probs is not None else ref.softmax_row(
                logits[b, p].double().numpy()[lo:hi] * 0.7, 1.0)
            w = np.maximum(w, 0)
            tok[b, i] = rng.choice(len(w), p=w / w.sum()) + (0 if probs is not None else lo)
    return torch.from_numpy(tok).int()


def check_verify(logits, tokens, parent, u, **kw):
    cu = {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in kw.items()}
    got = _b().verify_sampled(logits.cuda(), tokens.cuda(), parent.cuda(), u.cuda(), **cu)
    want = ref.verify_sampled(logits, tokens, parent, u, **kw)
    for a, b in zip(got, want):
        assert torch.equal(a.cpu(), b)
    return want


@pytest.mark.parametrize("with_probs", [False, True])
@pytest.mark.parametrize("kind", [F32, BF, HF])
@pytest.mark.parametrize("n,rows,vocab,lo,hi", [(1, 1, 5, 0, 5), (1, 27, 1024, 768, 1024), (3, 51, 700, 0, 700), (40, 6, 513, 1, 512),
                                                (2, 128, 5000, 17, 4990), (2, 33, 32064, 0, 32064)])
def test_verify_trees(with_probs, kind, n, rows, vocab, lo, hi):
    rng = np.random.default_rng(n * 1000 + rows)
    g = _gen(vocab)
    logits = (_randn(g, n, rows, vocab) * 4).to(kind)
    parent = trees(rng, n, rows, chain=rows == 6)
    probs = None
    if with_probs:
        q = logits.float() + _randn(g, n, rows, vocab)
        q[..., :lo], q[..., hi:] = -math.inf, -math.inf
        probs = torch.softmax(q / 0.8, -1)
    tokens = drafted(rng, logits, parent, probs, lo, hi)
    n_rows = torch.from_numpy(rng.integers(1, rows + 1, n)).int()
    met = 0
    if n > 2:
        n_rows[0], n_rows[1] = -3, 1000                              # taken as 1 and as all
    for seed in range(4):
        u = torch.rand(n, rows, generator=_gen(seed))
        kw = dict(temperature=(1.0, 0.8, 0.3, 1.7)[seed], draft_probs=probs, lo=lo, hi=hi)
        met += int(check_verify(logits, tokens, parent, u, **kw)[0].sum())
        check_verify(logits, tokens, parent, u, n_rows=n_rows, **kw)
    # (drafted from the flattened target: over 32064 ids a token is likely only with draft probabilities)
    assert met > 0 or rows == 1 or (vocab == 32064 and not with_probs)


@pytest.mark.parametrize("with_probs", [False, True])
@pytest.mark.parametrize("kind,n,rows,vocab,lo,hi", [(F32, 6, 64, 32064, 0, 32064), (BF, 64, 64, 3000, 3, 2999), (HF, 400, 60, 600, 0, 600),
                                                     (F32, 1500, 24, 500, 0, 500), (BF, 32, 128, 2100, 1, 2099)])
def test_verify_many_rows(with_probs, kind, n, rows, vocab, lo, hi):
    """More rows than are summed at once: rows are summed as the walk comes to them, by clusters of eight CTAs down to one."""
    rng = np.random.default_rng(n + rows)
    g = _gen(vocab)
    logits = (_randn(g, n, rows, vocab) * 4).to(kind)
    logits[0, 0] = math.nan                                          # nothing to draw from
    logits[1, 0, lo + 5], logits[1, 0, hi - 1] = math.inf, math.inf
    logits[2, 0, lo:hi] = -math.inf
    logits[2, 0, hi - 1] = 1.0
    parent = trees(rng, n, rows)
    parent[3] = torch.tensor([-1] + list(range(rows - 1)))          # a chain
    probs = None
    if with_probs:
        q = logits.float() + _randn(g, n, rows, vocab)
        q[..., :lo], q[..., hi:] = -math.inf, -math.inf
        probs = torch.softmax(q / 0.8, -1)                          # (NaN and zeros in the first trees' roots)
    tokens = torch.zeros(n, rows, dtype=torch.int32)
    top = torch.topk(torch.nan_to_num(logits[..., lo:hi].float(), nan=0.0), 6, dim=-1).indices + lo
    for i in range(1, rows):
        tokens[:, i] = top[torch.arange(n), parent[:, i].long(), torch.from_numpy(rng.integers(0, 6, n))]
    n_rows = torch.from_numpy(rng.integers(1, rows + 1, n)).int()
    met = 0
    for seed in range(3):
        u = torch.rand(n, rows, generator=_gen(seed))
        kw = dict(temperature=(0.2, 1.0, 0.5)[seed], draft_probs=probs, lo=lo, hi=hi)
        met += int(check_verify(logits, tokens, parent, u, **kw)[0].sum())
        check_verify(logits, tokens, parent, u, n_rows=n_rows, **kw)
    for fill in (0.0, 1.0 - 2.0 ** -24):
        check_verify(logits, tokens, parent, torch.full((n, rows), fill), draft_probs=probs, lo=lo, hi=hi)
    assert met > n


@pytest.mark.parametrize("n", [3, 6])
@pytest.mark.parametrize("kind", [F32, BF, HF])
def test_verify_deep_paths_over_the_whole_vocabulary(kind, n):
    """Each row's likely tokens as its children, low temperatures: paths of many rows."""
    rows, vocab = 64, 32064
    g = _gen(77)
    logits = (_randn(g, n, rows, vocab) * 4).to(kind)
    parent = torch.tensor([-1] + [i // 2 * 2 for i in range(rows - 1)], dtype=torch.int32).repeat(n, 1)   # two children each
    tokens = torch.zeros(n, rows, dtype=torch.int32)
    for i in range(1, rows):
        top = torch.topk(logits[:, int(parent[0, i])].float(), 2, dim=-1).indices
        tokens[:, i] = top[:, i % 2]
    met = 0
    for seed in range(4):
        u = torch.rand(n, rows, generator=_gen(seed))
        met += int(check_verify(logits, tokens, parent, u, temperature=0.1 + 0.1 * seed)[0].sum())
    assert met > 12


def test_verify_keeps_the_targets_distribution():
    """40,000 trees of the same three siblings: the first emitted token is distributed as the target, with and without
    draft probabilities (chi-square over 6 ids: 5 degrees of freedom, 99.9 % quantile 20.5)."""
    n = 40000
    g = _gen(1)
    z = torch.tensor([1.0, 0.2, -0.5, 0.7, -2.0, 0.1])
    q = torch.tensor([0.1, 0.3, 0.2, 0.1, 0.25, 0.05])
    p = torch.softmax(z.double(), 0)
    logits = z.repeat(n, 4, 1)
    parent = torch.tensor([-1, 0, 0, 0], dtype=torch.int32).repeat(n, 1)
    u = torch.rand(n, 4, generator=g)
    drawn = torch.multinomial(q, n * 4, replacement=True, generator=g).view(n, 4).int()
    best = torch.tensor([0, 4, 3, 1], dtype=torch.int32).repeat(n, 1)
    for tokens, probs in ((drawn, q.repeat(n, 4, 1)), (best, None)):
        _, _, out = _b().verify_sampled(logits.cuda(), tokens.cuda(), parent.cuda(), u.cuda(),
                                        draft_probs=None if probs is None else probs.cuda())
        count = torch.bincount(out[:, 0].cpu().long(), minlength=6).double()
        chi = ((count - n * p) ** 2 / (n * p)).sum()
        assert chi < 20.5, (chi, count)


def test_verify_rows_and_numbers_that_are_not_ordinary():
    vocab = 1100
    g = _gen(6)
    base = _randn(g, 12, 4, vocab) * 2
    base[0, 0] = math.nan                       # nothing to draw from: the lowest id
    base[1, 0] = -math.inf
    base[2, 0, 5], base[2, 0, 700] = math.inf, math.inf      # infinities share the row
    base[3, 0, ::2] = math.nan
    base[4, 0] = -math.inf
    base[4, 0, 1099] = -3.0                     # one id has all
    base[5, 0] = torch.finfo(torch.float32).min
    base[6, 0, 9] = 1e30
    base[7, 0] = 0.0
    parent = torch.tensor([-1, 0, 0, 1], dtype=torch.int32).repeat(12, 1)
    tokens = torch.randint(0, vocab, (12, 4), generator=g).int()
    tokens[2, 1], tokens[4, 1], tokens[6, 1] = 700, 1099, 9
    tokens[8, 1], tokens[8, 2] = -1, vocab      # outside the ids
    tokens[9, 1] = tokens[9, 2] = 3             # the same token twice
    parent[10] = torch.tensor([5, 3, 2, 100])   # no row's children
    parent[11] = torch.tensor([0, 0, -7, 0])
    probs = torch.softmax(_randn(g, 12, 4, vocab), -1)
    probs[3, 0, 7:90] = math.nan
    probs[5, 0] = 0.0
    probs[6, 0] = -1.0
    u = torch.rand(12, 4, generator=g)
    for fill in (None, 0.0, 1.0 - 2.0 ** -24):
        if fill is not None:
            u = torch.full((12, 4), fill)
        for q in (None, probs):
            for lo, hi in ((0, vocab), (3, 1000)):
                check_verify(base, tokens, parent, u, draft_probs=q, lo=lo, hi=hi)


def test_verify_strided_rows():
    g = _gen(9)
    wide, wq = _randn(g, 3, 5, 801), torch.rand(3, 5, 640, generator=g)
    parent = trees(np.random.default_rng(0), 3, 5)
    tokens = torch.randint(1, 601, (3, 5), generator=g).int()
    u = torch.rand(3, 5, generator=g)
    z, q = wide[..., 1:601], wq[..., 3:603]
    want = ref.verify_sampled(z, tokens, parent, u, draft_probs=q, lo=1)
    got = _b().verify_sampled(wide.cuda()[..., 1:601], tokens.cuda(), parent.cuda(), u.cuda(), draft_probs=wq.cuda()[..., 3:603], lo=1)
    for a, b in zip(got, want):
        assert torch.equal(a.cpu(), b)
