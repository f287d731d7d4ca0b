"""Verification by random numbers where it can go wrong: against the 64-bit definition (operator_refs.py)."""
import numpy as np
import pytest
import torch

import operator_refs as ref

pytestmark = pytest.mark.gpu

BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32


def _b():
    from paper_2507_22424_b200 import binding
    return binding


def check(logits, tokens, parent, u, **kw):
    cu = {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in kw.items()}
    got = _b().verify_sampled(logits.cuda(), tokens.cuda(), parent.cuda(), u.cuda(), **cu)
    want = ref.verify_sampled(logits, tokens, parent, u, **kw)
    for a, b in zip(got, want):
        assert torch.equal(a.cpu(), b), (a.cpu()[(a.cpu() != b).view(len(b), -1).any(1)], b[(a.cpu() != b).view(len(b), -1).any(1)])
    return want


def check_little_left(n, rows, vocab):
    """Two siblings with nearly all of the weight are refused; the third is decided by a random number 2^-20 beside its share of
    what is left (1e-14 of the row): what is left has to be right relative to itself."""
    g = torch.Generator().manual_seed(vocab)
    logits = torch.full((n, rows, vocab), -60.0)
    logits[:, 0, 3] = 0.0
    logits[:, 0, vocab - 2] = -16.0 - torch.rand(n, generator=g)
    logits[:, 0, 7] = logits[:, 0, vocab - 2] - 16.0 - torch.rand(n, generator=g)
    logits[:, 0, vocab // 2] = logits[:, 0, 7] + torch.randn(n, generator=g)
    parent = torch.full((n, rows), -1, dtype=torch.int32)
    parent[:, 1:4] = 0
    tokens = torch.zeros(n, rows, dtype=torch.int32)
    tokens[:, 1], tokens[:, 2], tokens[:, 3] = 3, vocab - 2, 7
    u = torch.rand(n, rows, generator=g)
    u[:, 1] = u[:, 2] = 1 - 2.0 ** -24
    w = torch.exp(logits[:, 0].double())
    left = w.clone()
    left[:, 3] = left[:, vocab - 2] = 0
    share = w[:, 7] / left.sum(1)
    up = torch.arange(n) % 2 == 1
    u[:, 3] = (share * torch.where(up, 1 + 2.0 ** -20, 1 - 2.0 ** -20)).float()
    m = check(logits, tokens, parent, u)[0]
    # (a first token with more than 1 - 2^-24 of the weight is accepted)
    third = (w[:, 3] / w.sum(1) <= u[:, 1].double()) & (w[:, vocab - 2] / (w.sum(1) - w[:, 3]) <= u[:, 2].double())
    assert torch.equal(m[third], (~up).int()[third]) and third.sum() > n // 4


@pytest.mark.parametrize("n,rows", [(64, 4), (400, 60)])            # all rows at once; as the walk comes to them
@pytest.mark.parametrize("vocab", [40, 700])
def test_little_is_left_after_refused_tokens(n, rows, vocab):
    check_little_left(n, rows, vocab)


def test_little_is_left_where_a_cluster_shares_a_row():
    """Row by row over the whole vocabulary: every CTA of a cluster comes to the same decision."""
    check_little_left(8, 64, 32064)


@pytest.mark.parametrize("with_probs", [False, True])
@pytest.mark.parametrize("kind", [F32, BF])
def test_trees_of_one_row_at_any_distance(kind, with_probs):
    """The last row of every sequence's logits, padded rows with a dimension of one between, and ids of one: a distance of a
    dimension of one is no distance."""
    g = torch.Generator().manual_seed(5)
    n, vocab = 7, 300
    wide = (torch.randn(n, 4, vocab + 20, generator=g) * 3).to(kind)
    probs = torch.softmax(torch.randn(n, 3, vocab + 4, generator=g), -1)
    tokens, parent = torch.zeros(n, 1, dtype=torch.int32), torch.full((n, 1), -1, dtype=torch.int32)
    u = torch.rand(n, 1, generator=g)
    z, q = wide[:, -1:, :vocab], probs[:, 1:2, :vocab] if with_probs else None
    want = ref.verify_sampled(z, tokens, parent, u, draft_probs=q)
    cw, cp = wide.cuda(), probs.cuda()
    for zc in (cw[:, -1:, :vocab], cw[:, -1].unsqueeze(1)[..., :vocab], cw.as_strided((n, 1, vocab), (4 * (vocab + 20), 3, 1), 3 * (vocab + 20))):
        got = _b().verify_sampled(zc, tokens.cuda(), parent.cuda(), u.cuda(), draft_probs=cp[:, 1:2, :vocab] if with_probs else None)
        for a, b in zip(got, want):
            assert torch.equal(a.cpu(), b)
    one = cw[:, :, 5:6]                                              # a vocabulary of one id
    tokens, parent = torch.zeros(n, 4, dtype=torch.int32), torch.tensor([[-1, 0, 1, 2]], dtype=torch.int32).repeat(n, 1)
    u = torch.rand(n, 4, generator=g)
    want = ref.verify_sampled(wide[:, :, 5:6], tokens, parent, u)
    for zc in (one, one.contiguous(), one.contiguous().as_strided((n, 4, 1), (4, 1, 9))):
        got = _b().verify_sampled(zc, tokens.cuda(), parent.cuda(), u.cuda())
        for a, b in zip(got, want):
            assert torch.equal(a.cpu(), b)


def test_rows_that_overlap_are_refused():
    z = torch.zeros(40, device="cuda")
    i, u = torch.zeros(3, 1, dtype=torch.int32, device="cuda"), torch.zeros(3, 1, device="cuda")
    for zc in (z.as_strided((3, 1, 10), (9, 1, 1)), z.as_strided((3, 1, 10), (0, 10, 1)), z.as_strided((3, 1, 10), (10, 10, 2))):
        with pytest.raises(ValueError):
            _b().verify_sampled(zc, i, i, u)


@pytest.mark.parametrize("with_probs", [False, True])
@pytest.mark.parametrize("kind,n,rows,vocab,lo,hi", [
    (F32, 1, 8, 70000, 0, 70000),               # more pieces than the warps of a cluster keep: a refused child's pass starts from the logits
    (BF, 2, 12, 70001, 1, 69990),               # the same, rows off every boundary
    (F32, 1, 6, 1 << 20, 0, 1 << 20),           # as many ids as there may be, all rows at once
    (BF, 1, 20, (1 << 20) + 3, 2, (1 << 20) + 2),   # row by row
    (HF, 3, 40, 40000, 5, 39999),               # all rows at once, more than 64 pieces
    (HF, 3, 100, 40000, 5, 39999),              # row by row
])
def test_many_ids(kind, n, rows, vocab, lo, hi, with_probs):
    """Two children at every other row, several at the root: tokens that are likely, and some that are refused."""
    g = torch.Generator().manual_seed(vocab + rows)
    logits = (torch.randn(n, rows, vocab, generator=g) * 4).to(kind)
    parent = torch.tensor([-1, 0, 0, 0, 0] + [i // 2 * 2 for i in range(3, rows - 2)], dtype=torch.int32)[:rows].repeat(n, 1)
    probs = torch.softmax((logits.float() + torch.randn(n, rows, vocab, generator=g)), -1) if with_probs else None
    top = torch.topk(logits[..., lo:hi].float(), 8, dim=-1).indices + lo
    tokens = torch.zeros(n, rows, dtype=torch.int32)
    for i in range(1, rows):
        tokens[:, i] = top[:, int(parent[0, i]), i % 8]
    met = 0
    for seed in range(4):
        u = torch.rand(n, rows, generator=torch.Generator().manual_seed(seed))
        met += int(check(logits, tokens, parent, u, temperature=(0.1, 1.0, 0.3, 0.2)[seed], draft_probs=probs, lo=lo, hi=hi)[0].sum())
    u[:, 1:] = 1 - 2.0 ** -24                                        # (nearly) everything is refused
    for last in (0.0, 0.5, 1 - 2.0 ** -24):
        u[:, 0] = last
        check(logits, tokens, parent, u, draft_probs=probs, lo=lo, hi=hi)
    assert met > 0
