"""The linear layer on whole numbers whose sums every type on the way holds exactly: one product lost, doubled or misplaced shows."""
import pytest
import torch

pytestmark = pytest.mark.gpu

BF, HF, F32, I8, E4 = torch.bfloat16, torch.float16, torch.float32, torch.int8, torch.float8_e4m3fn


def _b():
    from paper_2507_22424_b200 import binding
    return binding


def whole(g, top, *shape):
    return torch.randint(-top, top + 1, shape, generator=g)


def rows(t, kind):
    """On the GPU, rows on 16 bytes."""
    wide = torch.zeros(t.shape[0], (t.shape[1] + 15) // 16 * 16)
    wide[:, :t.shape[1]] = t
    return wide.to(kind).cuda()[:, :t.shape[1]]


@pytest.mark.parametrize("kind", [BF, HF, I8, E4])
@pytest.mark.parametrize("T,N,K", [(1, 4096, 4096), (5, 256, 4096), (27, 4096, 11008), (16, 130, 8200), (64, 1000, 2064), (100, 384, 11008),
                                   (200, 4096, 2056), (290, 4096, 4096), (290, 11008, 1032), (600, 512, 11008), (1001, 4331, 2056)])
def test_long_rows(T, N, K, kind):
    """|x|, |w| <= 4: |sum| <= 16 K < 2^24. The rings turn many times; few rows are cut into slices of K."""
    g = torch.Generator().manual_seed(T + N + K)
    x, w = whole(g, 4, T, K), whole(g, 4, N, K)
    bias, res = whole(g, 9, N).float(), whole(g, 99, T, N).float()
    want = (x.cuda().double() @ w.cuda().double().T).cpu()
    y = _b().linear(rows(x, kind), rows(w, kind), bias.cuda(), residual=res.cuda(), dtype=F32).cpu()
    assert torch.equal(y.double(), want + bias.double() + res.double())


@pytest.mark.parametrize("kind", [BF, HF, I8, E4])
@pytest.mark.parametrize("dtype,K", [(HF, 512), (BF, 64), (F32, 512)])
@pytest.mark.parametrize("T,N", [(1, 64), (3, 130), (7, 131), (27, 512), (64, 1000), (129, 640), (200, 257), (257, 514), (300, 1000), (700, 384)])
def test_residual_and_bias_go_where_they_belong(T, N, dtype, K, kind):
    """16-bit results hold whole numbers up to 2048 (f16) and 256 (bf16): products of -1, 0 and 1 and a small residual stay below.
    The residual is another at every element; in its place too, in rows that are even and odd numbers of elements apart."""
    g = torch.Generator().manual_seed(T * 7 + N)
    x, w = whole(g, 1, T, K), whole(g, 1, N, K)
    bias, res = whole(g, 20, N), whole(g, 100 if dtype == BF else 900, T, N)
    want = (x.double() @ w.double().T + bias + res)
    assert want.abs().max() <= (256 if dtype == BF else 2048)
    xc, wc, bc = rows(x, kind), rows(w, kind), bias.float().cuda()
    y = _b().linear(xc, wc, bc, residual=res.to(dtype).cuda(), dtype=dtype).cpu()
    assert torch.equal(y.double(), want)
    for gap in (6, 7):
        wide = torch.full((T, N + gap), 5.0, dtype=dtype, device="cuda")
        wide[:, 1:N + 1] = res.to(dtype).cuda()
        _b().linear(xc, wc, bc, residual=wide[:, 1:N + 1], out=wide[:, 1:N + 1])
        assert torch.equal(wide[:, 1:N + 1].cpu().double(), want)
        assert (wide[:, 0] == 5).all() and (wide[:, N + 1:] == 5).all()
    _b().linear_status()
