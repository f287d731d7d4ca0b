"""The stand-alone operators as they are used together: the tail of a sampled verification step, eagerly, in captured graphs
and on several streams; and the context's own verification by random numbers."""
import pytest
import torch

import gpu_helpers as G
import operator_refs as ref
from synth_inputs import configs as C, data

pytestmark = pytest.mark.gpu


def _b():
    from paper_2507_22424_b200 import binding
    return binding


# ------------------------------------------------------------------------------------ norm -> head -> verification
ROWS, D, VOCAB = 27, 264, 1000


class Tail:
    """Residual add and norm to 8 bits, an 8-bit head with bias, verification of one tree."""

    def __init__(self, code=torch.int8, rows=ROWS):
        B = _b()
        g = torch.Generator().manual_seed(5)
        self.rows, self.code = rows, code
        self.gain = (1 + 0.1 * torch.randn(D, generator=g)).cuda()
        self.w, self.w_scale = B.quantize_rows(torch.randn(VOCAB, D, generator=g).cuda() * 0.4, code)
        self.bias = torch.randn(VOCAB, generator=g).cuda()
        self.parent = torch.tensor([[-1] + [i // 3 for i in range(rows - 1)]], dtype=torch.int32).cuda()
        self.x, self.r, self.tokens, self.u = self.inputs(0)

    def inputs(self, seed):
        g = torch.Generator().manual_seed(seed)
        return ((torch.randn(self.rows, D, generator=g) * 2).bfloat16().cuda(), torch.randn(self.rows, D, generator=g).bfloat16().cuda(),
                torch.randint(0, VOCAB, (1, self.rows), generator=g).int().cuda(), torch.rand(1, self.rows, generator=g).cuda())

    def load(self, seed):
        for mine, new in zip((self.x, self.r, self.tokens, self.u), self.inputs(seed)):
            mine.copy_(new)

    def __call__(self):
        B = _b()
        codes, scale, total = B.rmsnorm_q8(self.x, self.gain, residual=self.r, dtype=self.code)
        logits = B.linear(codes, self.w, self.bias, x_scale=scale, w_scale=self.w_scale, dtype=torch.float32)
        return (codes, scale, total, logits, *B.verify_sampled(logits[None], self.tokens, self.parent, self.u, temperature=0.5))


def check_tail(t, out):
    codes, scale, total, logits, m, path, tok = [o.cpu() for o in out]
    rc, rs, rt = ref.norm_q8(t.x.cpu(), t.gain.cpu(), t.r.cpu(), 1e-6, t.code)
    assert torch.equal(codes.float().double(), rc) and torch.equal(total, rt)
    assert ((scale.double() - rs) / rs).abs().max() < (1 + 64 + D / 512) * 2.0 ** -24
    want, mag = ref.linear(codes, t.w.cpu(), t.bias.cpu(), x_scale=scale, w_scale=t.w_scale.cpu())
    # exact integers (int8) or at most D roundings of 2^-23, then four of 2^-24 with the scales and the bias
    tol = (0 if t.code == torch.int8 else D * 2.0 ** -23) * mag + 16 * 2.0 ** -24 * (mag + t.bias.cpu().abs())
    assert ((logits.double() - want).abs() <= tol).all()
    for a, b in zip((m, path, tok), ref.verify_sampled(logits[None], t.tokens.cpu(), t.parent.cpu(), t.u.cpu(), temperature=0.5)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("code", [torch.int8, torch.float8_e4m3fn])
@pytest.mark.parametrize("rows", [1, ROWS, 128])
def test_tail_of_a_verification_step(code, rows):
    t = Tail(code, rows)
    for seed in range(3):
        t.load(seed)
        check_tail(t, t())
    _b().linear_status()


def test_tail_in_captured_graphs():
    """Two graphs of the same calls, replayed with other inputs, in turn with eager calls."""
    tails = [Tail(), Tail(torch.float8_e4m3fn)]
    for t in tails:
        t()
    torch.cuda.synchronize()
    graphs, outs = [], []
    for t in tails:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(t())
        graphs.append(g)
    for seed in range(3, 7):
        for t, g, o in zip(tails, graphs, outs):
            t.load(seed)
            g.replay()
        for t, o in zip(tails, outs):
            check_tail(t, o)
            check_tail(t, t())
    _b().linear_status()


def test_operators_on_two_streams_at_once():
    B = _b()
    g = torch.Generator().manual_seed(1)
    streams = [torch.cuda.Stream() for _ in range(2)]
    tails = [Tail(), Tail(torch.float8_e4m3fn)]
    big = [((torch.randn(700, 512, generator=g)).bfloat16().cuda(), (torch.randn(3000, 512, generator=g)).bfloat16().cuda()) for _ in range(2)]
    want = [B.linear(x, w) for x, w in big]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for k, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[k].append((B.linear(*big[k]), tails[k]()))
    torch.cuda.synchronize()
    for k, s in enumerate(streams):
        for y, out in got[k]:
            assert torch.equal(y, want[k])
        check_tail(tails[k], got[k][-1][1])
        for _, out in got[k][:-1]:
            assert all(torch.equal(a, b) for a, b in zip(out, got[k][-1][1]))
        with torch.cuda.stream(s):
            B.linear_status()


def test_results_do_not_depend_on_timing():
    """Split sums are added in a fixed order: the same bits every time."""
    B = _b()
    g = torch.Generator().manual_seed(2)
    for T, N, K in ((5, 700, 4096), (300, 2000, 1024)):
        x, w = torch.randn(T, K, generator=g).half().cuda(), torch.randn(N, K, generator=g).half().cuda()
        first = B.linear(x, w, dtype=torch.float32)
        for _ in range(10):
            assert torch.equal(B.linear(x, w, dtype=torch.float32), first)


def test_rows_behind_the_last_one_are_left_alone():
    B = _b()
    x = torch.randn(9, 64, device="cuda").half()
    w = torch.randn(70, 64, device="cuda").half()
    room = torch.full((20, 70), 3.0, dtype=torch.float16, device="cuda")
    B.linear(x, w, out=room[4:13])
    assert (room[:4] == 3).all() and (room[13:] == 3).all()
    total = torch.full((20, 64), 3.0, dtype=torch.float16, device="cuda")
    B.rmsnorm_q8(x, residual=x, out_sum=total[4:13])
    assert (total[:4] == 3).all() and (total[13:] == 3).all()


def test_empty_calls():
    B = _b()
    x = torch.zeros(0, 64, device="cuda", dtype=torch.float16)
    w = torch.zeros(7, 64, device="cuda", dtype=torch.float16)
    assert B.linear(x, w).shape == (0, 7) and B.linear(w, x).shape == (7, 0)
    codes, scale, _ = B.rmsnorm_q8(x)
    assert codes.shape == (0, 64) and scale.shape == (0,)
    m, path, out = B.verify_sampled(torch.zeros(0, 3, 9, device="cuda"), *[torch.zeros(0, 3, dtype=torch.int32, device="cuda")] * 2,
                                    torch.zeros(0, 3, device="cuda"))
    assert m.shape == (0,) and path.shape == out.shape == (0, 3)
    with pytest.raises(ValueError):
        B.linear(torch.zeros(3, 64).half(), w)


# ------------------------------------------------------------------------------------ the context's call
@pytest.fixture(scope="module")
def wcuda(c0):
    return G.to_cuda(c0["weights"])


def _ctx(c0, wcuda, **kw):
    return G.make_gpu(c0["desc"], wcuda, **{**dict(max_seq=256, max_episodes=2, max_rows=256, action_only=True), **kw})


def _tree(n, seed, root):
    tok, par, dep = data.random_tree(n, C.TINY, seed=seed, max_depth=4, root_token=root)
    return dict(tokens=tok, parent=par, depth=dep)


def _likely(gpu, episode, n, seed, root, chain=False):
    """A random tree (or a chain) whose nodes are the target's own greedy tokens or neighbours, so that paths are accepted."""
    t = _tree(n, seed, root)
    if chain:
        t["parent"], t["depth"] = list(range(-1, n - 1)), list(range(n))
    for level in range(1, max(t["depth"]) + 1):
        g = gpu.score_tree([episode], [t])
        for i in range(n):
            if t["depth"][i] == level:
                t["tokens"][i] = g[t["parent"][i]] if i % 3 else min(g[t["parent"][i]] + 1, C.TINY.action_base + C.TINY.n_bins - 1)
    return t


@pytest.mark.parametrize("action_only", [True, False])
@pytest.mark.parametrize("persistent", [False, True])
def test_context_verifies_by_random_numbers(c0, wcuda, action_only, persistent):
    """(m, tokens, path, state) as the operator's definition says on the logits that the call returns, several steps long."""
    from paper_2507_22424_b200.binding import OPT_PERSISTENT_FORWARD
    gpu = _ctx(c0, wcuda, action_only=action_only)
    gpu.set_option(OPT_PERSISTENT_FORWARD, int(persistent))
    d = c0["desc"]
    lo, hi = (d.action_base, d.action_base + d.n_bins) if action_only else (0, d.vocab)
    root = gpu.prefill([0], c0["embeds"].cuda(), c0["ids"].tolist(), [len(c0["ids"])])[0]
    P, met = len(c0["ids"]), 0
    for step in range(6):
        n = (15, 1, 27, 8, 15, 27)[step]
        t = _likely(gpu, 0, n, 40 + step, root) if action_only else _tree(n, 40 + step, root)
        u = torch.rand(n, generator=torch.Generator().manual_seed(step))
        T = (0.05, 1.0, 0.1, 0.02, 0.5, 0.05)[step]
        m, emitted, logits = gpu.verify_tree_sampled([0], [t], u.cuda(), T)
        rm, rp, rt = ref.verify_sampled(logits.cpu()[None], torch.tensor([t["tokens"]]).int(), torch.tensor([t["parent"]]).int(), u[None],
                                        temperature=T, lo=lo, hi=hi)
        assert m == rm.tolist() and emitted[0] == rt[0, :m[0] + 1].tolist()
        assert gpu.read_buffer(4, 9, torch.int32).tolist()[:m[0] + 1] == rp[0, :m[0] + 1].tolist()
        P += 1 + m[0]
        root = emitted[0][-1]
        met += m[0]
        assert gpu.read_buffer(5, 4, torch.int32).tolist()[0] == P
        assert gpu.read_buffer(5, 4, torch.int32).tolist()[2:] == [root, m[0] + 1]
    assert met > 0 or not action_only
    gpu.close()


def test_cold_sampling_is_greedy_verification(c0, wcuda):
    """Next to temperature 0 the most likely token has all the weight: the call equals strict verification (r = 0), caches and
    draft state included, over the caller's chains and the draft model's trees. (Not over trees with twins: of siblings with
    the same token the walk takes the first, strict verification the one with the longest path.)"""
    from paper_2507_22424_b200.binding import make_shape
    a, b = _ctx(c0, wcuda), _ctx(c0, wcuda)
    for gpu in (a, b):
        root = gpu.prefill([1], c0["embeds"].cuda(), c0["ids"].tolist(), [len(c0["ids"])])[0]
    met = 0
    for step in range(6):
        if step % 2:
            trees = [_likely(a, 1, 8, step, root, chain=True)]
            n = 8
        else:
            shape = make_shape((2, 2, 2), (1, 2, 4))
            n = len(a.draft_tree([1], shape)[0]["tokens"])
            assert len(b.draft_tree([1], shape)[0]["tokens"]) == n
            trees = None
        u = torch.rand(n, generator=torch.Generator().manual_seed(step)).cuda()
        m, emitted, _ = a.verify_tree_sampled([1], trees, u, 1e-12)
        assert (m, emitted) == b.verify_tree([1], trees, 0)
        met += m[0]
        root = emitted[0][-1]
    P = a.read_buffer(5, 8, torch.int32).tolist()[4]
    assert a.read_buffer(5, 8, torch.int32).tolist() == b.read_buffer(5, 8, torch.int32).tolist() and met > 0
    for layer in range(c0["desc"].n_layers):
        for which in (0, 1):
            assert torch.equal(a.read_kv(1, layer, which, 0, P), b.read_kv(1, layer, which, 0, P))
    a.close()
    b.close()


def test_context_verifies_two_ragged_trees_at_once(c0, wcuda):
    gpu = _ctx(c0, wcuda)
    ids = c0["ids"].tolist()
    both = torch.cat([c0["embeds"], c0["embeds"][:40]]).cuda()
    roots = gpu.prefill([0, 1], both, ids + ids[:40], [len(ids), 40])
    trees = [_likely(gpu, 0, 15, 3, roots[0]), _likely(gpu, 1, 27, 4, roots[1])]
    u = torch.rand(42, generator=torch.Generator().manual_seed(9))
    m, emitted, logits = gpu.verify_tree_sampled([0, 1], trees, u.cuda(), 0.1)
    d, at = c0["desc"], 0
    for e, t in enumerate(trees):
        n = len(t["tokens"])
        rm, _, rt = ref.verify_sampled(logits.cpu()[None, at:at + n], torch.tensor([t["tokens"]]).int(), torch.tensor([t["parent"]]).int(),
                                       u[None, at:at + n], temperature=0.1, lo=d.action_base, hi=d.action_base + d.n_bins)
        assert m[e] == int(rm[0]) and emitted[e] == rt[0, :m[e] + 1].tolist()
        at += n
    gpu.close()


def test_context_call_refuses(c0, wcuda):
    from paper_2507_22424_b200.binding import SpecVLAError
    gpu = _ctx(c0, wcuda)
    t = _tree(5, 1, C.TINY.action_base)
    u = torch.rand(5).cuda()
    with pytest.raises(SpecVLAError) as e:
        gpu.verify_tree_sampled([0], [t], u)                          # not prefilled
    assert e.value.code == -4
    gpu.prefill([0], c0["embeds"].cuda(), c0["ids"].tolist(), [len(c0["ids"])])
    for T in (0.0, -1.0, float("nan"), 2e30):
        with pytest.raises(SpecVLAError) as e:
            gpu.verify_tree_sampled([0], [t], u, T)
        assert e.value.code == -1
    with pytest.raises(ValueError):
        gpu.verify_tree_sampled([0], [t], u[:4])
    with pytest.raises(ValueError):
        gpu.verify_tree_sampled([0], [t], u.cpu())
    from paper_2507_22424_b200.binding import make_shape
    n = len(gpu.draft_tree([0], make_shape((2, 2), (1, 2)))[0]["tokens"])
    for other in (n - 1, n + 1):                                      # numbers for more or fewer rows than the device's tree has
        with pytest.raises(SpecVLAError) as e:
            gpu.verify_tree_sampled([0], None, torch.rand(other).cuda())
        assert e.value.code == -1
    gpu.verify_tree_sampled([0], [t], u)                              # the context is as it was
    gpu.close()


def test_rows_further_apart_than_32_bits_count():
    """Two rows 2^31 elements apart, in every operand whose rows have a distance."""
    B = _b()
    far = 2 ** 31
    big = torch.empty(far + 128, dtype=torch.float16, device="cuda")
    rows = big.as_strided((2, 96), (far, 1))
    g = torch.Generator().manual_seed(3)
    x, w = torch.randn(2, 96, generator=g).half().cuda(), torch.randn(80, 96, generator=g).half().cuda()
    rows.copy_(x)
    want = B.rmsnorm_q8(x, residual=x, dtype=torch.float8_e4m3fn)
    got = B.rmsnorm_q8(rows, residual=rows, dtype=torch.float8_e4m3fn)
    assert all(torch.equal(a.float(), b.float()) for a, b in zip(got, want))
    y = B.linear(x, w)
    assert torch.equal(B.linear(rows, w), y)
    assert torch.equal(B.linear(w, rows), B.linear(w, x))
    out = big.as_strided((2, 80), (far, 1))
    rows.copy_(x)
    out.copy_(y)
    assert torch.equal(B.linear(x, w, residual=out, out=out), B.linear(x, w, residual=y))
    parent, u = torch.tensor([[-1, 0]], dtype=torch.int32).cuda(), torch.tensor([[0.7, 0.0]]).cuda()
    rows.copy_(x)
    tokens = torch.tensor([[0, 17]], dtype=torch.int32).cuda()
    assert all(torch.equal(a, b) for a, b in zip(B.verify_sampled(rows[None], tokens, parent, u), B.verify_sampled(x[None], tokens, parent, u)))
    del big, rows, out
    torch.cuda.empty_cache()


def test_two_host_threads_at_once():
    import threading
    B = _b()
    tails = [Tail(), Tail(torch.float8_e4m3fn)]
    for t in tails:
        t()
    torch.cuda.synchronize()
    outs, errors = [[], []], []

    def work(k):
        try:
            s = torch.cuda.Stream()
            with torch.cuda.stream(s):
                for _ in range(30):
                    outs[k].append(tails[k]())
                B.linear_status()
        except Exception as e:                                        # reported by the main thread
            errors.append(e)

    threads = [threading.Thread(target=work, args=(k,)) for k in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    for k in range(2):
        check_tail(tails[k], outs[k][0])
        for out in outs[k][1:]:
            assert all(torch.equal(a, b) for a, b in zip(out, outs[k][0]))


def test_very_many_rows():
    """More rows than 65535 chunks of 256."""
    T = 65536 * 256 + 77
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randint(-3, 4, (T, 8), generator=g, device="cuda").half()
    w = torch.randint(-3, 4, (3, 8), generator=g, device="cuda").half()
    y = _b().linear(x, w, dtype=torch.float32)
    assert all(torch.equal(y[:, n], (x.float() * w[n].float()).sum(1)) for n in range(3))      # small whole numbers: exact


@pytest.mark.parametrize("T,N,K,kind", [(290, 11008, 160, "bf16"), (600, 10212, 96, "int8"), (1358, 10211, 264, "f16"),
                                        (290, 11008, 130, "e4m3"), (4096, 4096, 512, "bf16")])
def test_linear_over_several_rounds_of_tiles(T, N, K, kind):
    """Sizes whose tiles do not fill their last round on 148 SMs; every element against 64 bits."""
    g = torch.Generator().manual_seed(T + N)
    x, w = (torch.randint(-4, 5, s, generator=g) for s in ((T, K), (N, K)))
    dt = {"bf16": torch.bfloat16, "f16": torch.float16, "int8": torch.int8, "e4m3": torch.float8_e4m3fn}[kind]
    bias, res = torch.randint(-9, 10, (N,), generator=g).float(), torch.randint(-9, 10, (T, N), generator=g).float()
    codes = kind in ("int8", "e4m3")
    xs = 2.0 ** torch.randint(-2, 3, (T,), generator=g) if codes else None
    ws = 2.0 ** torch.randint(-2, 3, (N,), generator=g) if codes else None
    pad = torch.zeros(T + N, (K + 15) // 16 * 16)                       # rows on 16 bytes
    pad[:T, :K], pad[T:, :K] = x, w
    pad = pad.to(dt).cuda()
    y = _b().linear(pad[:T, :K], pad[T:, :K], bias.cuda(), residual=res.cuda(), dtype=torch.float32,
                    x_scale=None if xs is None else xs.cuda(), w_scale=None if ws is None else ws.cuda()).cpu()
    want = x.double() @ w.double().T
    if codes:
        want = want * xs.double()[:, None] * ws.double()[None]
    assert torch.equal(y.double(), want + bias.double() + res.double())  # whole sixteenths below 2^24: exact


def test_context_call_with_another_number_of_rows_leaves_the_drafted_tree(c0, wcuda):
    import ctypes as C_
    from paper_2507_22424_b200.binding import Tree, _ints, lib, make_shape
    host = _tree(5, 1, C.TINY.action_base)
    results = []
    for refused in (False, True):
        gpu = _ctx(c0, wcuda)
        gpu.prefill([0], c0["embeds"].cuda(), c0["ids"].tolist(), [len(c0["ids"])])
        n = len(gpu.draft_tree([0], make_shape((2, 2), (1, 2)))[0]["tokens"])
        u = torch.linspace(0.05, 0.95, n).cuda()
        if refused:
            tree = (Tree * 1)()
            keep = [_ints(host[k]) for k in ("tokens", "parent", "depth")]
            tree[0].n_rows, tree[0].score = 5, None
            tree[0].tokens, tree[0].parent, tree[0].depth = keep
            logits = torch.empty(8, gpu.model.vocab, device="cuda")
            m, toks = (C_.c_int * 1)(), (C_.c_int * 64)()
            for rows in (4, 6, 0, -1):
                assert lib.specvla_verify_tree_sampled(gpu.h, 1, _ints([0]), tree, 1.0, C_.c_void_p(u.data_ptr()),
                                                       C_.c_void_p(logits.data_ptr()), rows, m, toks, None) == -1
        results.append(gpu.verify_tree_sampled([0], None, u))
        gpu.close()
    (ma, ea, la), (mb, eb, lb) = results
    assert ma == mb and ea == eb and torch.equal(la, lb)


@pytest.mark.parametrize("T,N,K,kind", [(44, 20011, 64, "bf16"), (36, 30020, 24, "f16"), (1674, 4870, 96, "int8"), (17, 40000, 640, "e4m3"),
                                        (67, 24344, 320, "f16"), (16, 20011, 64, "bf16"), (1, 40000, 48, "int8")])
def test_linear_of_many_columns_and_few_products(T, N, K, kind):
    """More tiles of 128 columns than run at once, K of one to five blocks: pairs' many short tiles, slices' rounds up to 16 rows."""
    g = torch.Generator().manual_seed(T + K)
    dt = {"bf16": torch.bfloat16, "f16": torch.float16, "int8": torch.int8, "e4m3": torch.float8_e4m3fn}[kind]
    x, w = (torch.randint(-4, 5, s, generator=g) for s in ((T, K), (N, K)))
    y = _b().linear(x.float().to(dt).cuda(), w.float().to(dt).cuda(), dtype=torch.float32).cpu()
    assert torch.equal(y.double(), x.double() @ w.double().T)          # whole numbers below 2^24: exact
