"""Arguments that the stand-alone operators refuse: on the CPU, before anything reaches a GPU (pointers are made up and are
never followed: every call here returns an error)."""
import ctypes as C

import pytest

INVALID, CAPACITY = -1, -2
P = 1 << 20                                 # an aligned address


@pytest.fixture(scope="module")
def B():
    from paper_2507_22424_b200.build import build
    build()
    from paper_2507_22424_b200 import binding
    return binding


NORM = dict(rows=4, d=32, type=1, code_type=3, x=P, ldx=32, residual=P, ld_residual=32, gain=P, sum=P, ld_sum=32, codes=P, ld_codes=32,
            scale=P, eps=1e-6)
LINEAR = dict(T=4, N=64, K=64, type=1, out_type=1, act=0, X=P, ldx=64, x_scale=0, W=P, ldw=64, w_scale=0, bias=P, residual=P,
              ld_residual=64, Y=P, ldy=64, status=P)
VERIFY = dict(n_seq=2, rows=8, vocab=100, lo=0, hi=100, logits_type=0, logits=P, ld_logits=100, draft_probs=P, ld_draft=100,
              temperature=1.0, tokens=P, parent=P, n_rows=P, u=P, accept_len=P, path=P, tokens_out=P)


@pytest.mark.parametrize("change", [
    dict(rows=0), dict(rows=-1), dict(d=0), dict(d=(1 << 30) + 1, **{k: 1 << 31 for k in ("ldx", "ld_residual", "ld_sum", "ld_codes")}), dict(type=3), dict(type=4), dict(type=7), dict(code_type=0), dict(code_type=5), dict(x=0), dict(codes=0),
    dict(scale=0), dict(ldx=31), dict(ld_codes=31), dict(ld_residual=31), dict(ld_sum=31), dict(eps=-1e-6), dict(eps=float("nan")),
    dict(x=P + 1), dict(residual=P + 1), dict(sum=P + 1), dict(gain=P + 2), dict(scale=P + 2)])
def test_norm_refuses(B, change):
    assert B.lib.specvla_rmsnorm_q8(B.NORM_ARGS.pack(*{**NORM, **change}.values()), None) == INVALID


def test_norm_refuses_null(B):
    assert B.lib.specvla_rmsnorm_q8(None, None) == INVALID


@pytest.mark.parametrize("args", [
    (0, 0, 4, 32, 32, P, 3, 32, P), (P, 3, 4, 32, 32, P, 3, 32, P), (P, 0, 0, 32, 32, P, 3, 32, P), (P, 0, 4, 0, 32, P, 3, 32, P),
    (P, 0, 4, 32, 31, P, 3, 32, P), (P, 0, 4, 32, 32, 0, 3, 32, P), (P, 0, 4, 32, 32, P, 1, 32, P), (P, 0, 4, 32, 32, P, 3, 31, P),
    (P, 0, 4, 32, 32, P, 3, 32, 0), (P + 2, 0, 4, 32, 32, P, 3, 32, P)])
def test_quantize_rows_refuses(B, args):
    assert B.lib.specvla_quantize_rows(*args, None) == INVALID


@pytest.mark.parametrize("change", [
    dict(T=0), dict(N=0), dict(K=0), dict(T=-3), dict(type=0), dict(type=5), dict(out_type=3), dict(act=-1), dict(act=5), dict(X=0), dict(W=0),
    dict(Y=0), dict(status=0), dict(ldx=63), dict(ldw=63), dict(ldx=65), dict(ldw=68), dict(X=P + 8), dict(W=P + 2), dict(ldy=63),
    dict(ld_residual=63), dict(x_scale=P), dict(w_scale=P), dict(Y=P + 1), dict(residual=P + 1), dict(bias=P + 1), dict(status=P + 2),
    dict(type=3, K=131072, ldx=131072, ldw=131072), dict(K=(1 << 29) + 8, ldx=1 << 30, ldw=1 << 30), dict(type=3, ldx=72), dict(type=4, x_scale=P + 2)])
def test_linear_refuses(B, change):
    assert B.lib.specvla_linear(B.LINEAR_ARGS.pack(*{**LINEAR, **change}.values()), None) == INVALID


def test_linear_refuses_null_and_bad_hooks(B):
    assert B.lib.specvla_linear(None, None) == INVALID
    assert B.lib.specvla_linear_fault_test(999, 0) == INVALID
    assert B.lib.specvla_linear_fault_test(1000, -2) == INVALID


@pytest.mark.parametrize("change", [
    dict(n_seq=0), dict(rows=0), dict(rows=129), dict(lo=-1), dict(hi=0), dict(lo=100), dict(hi=101), dict(vocab=99), dict(logits_type=3),
    dict(logits=0), dict(tokens=0), dict(parent=0), dict(u=0), dict(accept_len=0), dict(path=0), dict(tokens_out=0), dict(ld_logits=99),
    dict(ld_draft=99), dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=float("nan")), dict(temperature=float("inf")),
    dict(temperature=2e30), dict(logits=P + 2), dict(draft_probs=P + 2), dict(tokens=P + 1), dict(n_rows=P + 2), dict(u=P + 2),
    dict(hi=(1 << 20) + 1, vocab=1 << 21, ld_logits=1 << 21, ld_draft=1 << 21)])
def test_verify_refuses(B, change):
    args = {**VERIFY, **change}
    assert B.lib.specvla_verify_sampled(B.VERIFY_ARGS.pack(*args.values()), P, 1 << 30, None) == INVALID


def test_verify_refuses_scratch(B):
    pack = B.VERIFY_ARGS.pack(*VERIFY.values())
    need = B.lib.specvla_verify_sampled_scratch_bytes(2, 8, 0, 100)
    assert need > 0
    assert B.lib.specvla_verify_sampled(pack, None, need, None) == INVALID
    assert B.lib.specvla_verify_sampled(pack, P + 4, need, None) == INVALID
    assert B.lib.specvla_verify_sampled(pack, P, need - 1, None) == CAPACITY
    assert B.lib.specvla_verify_sampled(None, P, need, None) == INVALID
    for bad in ((0, 8, 0, 100), (2, 0, 0, 100), (2, 129, 0, 100), (2, 8, -1, 100), (2, 8, 5, 5), (2, 8, 0, (1 << 20) + 1), (1 << 22, 128, 0, 9)):
        assert B.lib.specvla_verify_sampled_scratch_bytes(*bad) == 0


def test_context_call_refuses_null(B):
    assert B.lib.specvla_verify_tree_sampled(None, 1, None, None, 1.0, None, None, 5, None, None, None) == INVALID


def test_argument_blocks_have_the_sizes_of_the_structures(B):
    """The packed blocks against the header, by a compiler."""
    import os
    import subprocess
    import tempfile
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = '#include "include/specvla.h"\n#include <stddef.h>\n#include <stdio.h>\nint main(void) { printf("%zu %zu %zu %zu %zu %zu", ' \
          "offsetof(specvla_norm_args, eps), offsetof(specvla_linear_args, status), offsetof(specvla_verify_args, tokens_out), " \
          "offsetof(specvla_norm_args, gain), offsetof(specvla_linear_args, residual), offsetof(specvla_verify_args, temperature)); }\n"
    with tempfile.TemporaryDirectory() as d:
        open(os.path.join(d, "a.c"), "w").write(src)
        subprocess.check_call(["gcc", "-I", root, os.path.join(d, "a.c"), "-o", os.path.join(d, "a")])
        got = list(map(int, subprocess.check_output([os.path.join(d, "a")]).split()))
    assert got == [B.NORM_ARGS.size - 4, B.LINEAR_ARGS.size - 8, B.VERIFY_ARGS.size - 8, 48, 80, 56]


def test_binding_refuses_host_tensors_and_shapes(B):
    import torch
    x = torch.zeros(4, 32)
    for call in (lambda: B.rmsnorm_q8(x.int()), lambda: B.rmsnorm_q8(x, dtype=torch.float16), lambda: B.rmsnorm_q8(x[0]),
                 lambda: B.rmsnorm_q8(x.t()), lambda: B.rmsnorm_q8(x, torch.ones(31)), lambda: B.rmsnorm_q8(x, residual=x[:3]),
                 lambda: B.rmsnorm_q8(x, residual=x.half()), lambda: B.rmsnorm_q8(x, out_sum=x), lambda: B.quantize_rows(x.double()),
                 lambda: B.linear(x, x), lambda: B.linear(x.bfloat16(), x.half()), lambda: B.linear(x.half(), x.half(), act="elu"),
                 lambda: B.linear(x.half(), x.half(), x_scale=torch.ones(4)), lambda: B.linear(x.half(), x.half(), torch.ones(5)),
                 lambda: B.linear(x.half(), x[:, :16].half()), lambda: B.linear(x.half(), x.half(), dtype=torch.int8),
                 lambda: B.verify_sampled(x, x, x, x), lambda: B.verify_sampled(x[None], x[None].int()[..., 0], x[None].int()[..., 0], x[:1, :3])):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("kind,k,step", [("bfloat16", 5, 8), ("float16", 12, 8), ("int8", 24, 16), ("float8_e4m3fn", 8, 16)])
def test_binding_names_operands_whose_rows_do_not_start_on_16_bytes(B, kind, k, step):
    import torch
    kind = getattr(torch, kind)
    good = torch.zeros(6, step * 4).to(kind)[:, :k]
    for x, w, name in ((torch.zeros(6, k).to(kind), good, "x"), (good, torch.zeros(6, k).to(kind), "w"),
                       (torch.zeros(6, step * 4 + 1).to(kind)[:, :k], good, "x"), (torch.zeros(6, step * 4).to(kind)[:, 1:k + 1], good, "x"),
                       (good, torch.zeros(6 * step * 4 + 1).to(kind)[1:].view(6, step * 4)[:, :k], "w")):
        with pytest.raises(ValueError, match=f"{name}.*16 bytes"):
            B.linear(x, w)
