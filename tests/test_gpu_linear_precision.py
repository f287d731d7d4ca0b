"""fp32 results of the linear layer are as good as fp32 arithmetic makes them, whatever the length of a row."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

BF, HF, F32, E4 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn


@pytest.mark.parametrize("kind", [BF, HF, E4])
@pytest.mark.parametrize("T,N,K", [(1, 4096, 11008), (16, 20000, 11008), (27, 4096, 4096), (27, 4096, 11008), (27, 11008, 4096), (64, 2000, 8192),
                                   (100, 1024, 8192), (130, 5000, 4096), (200, 512, 16384), (290, 4096, 4096), (290, 512, 11008),
                                   (290, 11008, 4096), (700, 1000, 4096), (1500, 4331, 2064), (3, 19000, 16400)])
def test_fp32_results(T, N, K, kind):
    """The tensor cores' fp32 additions cut off. A step of MMA loses half a unit in the last place on average, 0.36 * 2^-23 of an
    accumulator that is at 2/3 of its final size on average: 0.24 * 2^-23 of it per MMA. Of at most 48 MMAs' parts of a row, which
    are independent, the whole loses 12 * 2^-23 of its size (root mean square over random rows)."""
    from paper_2507_22424_b200 import binding as B
    g = torch.Generator(device="cuda").manual_seed(T + N + K)
    x = torch.randn(T, K, generator=g, device="cuda").to(kind)
    w = (torch.randn(N, K, generator=g, device="cuda") * (1 if kind == E4 else 1 / math.sqrt(K))).to(kind)
    y = B.linear(x, w, dtype=F32).double()
    want = x.double() @ w.double().T
    off = ((y - want).pow(2).mean() / want.pow(2).mean()).sqrt()
    assert off <= 12 * 2.0 ** -23, float(off) * 2 ** 23
    assert torch.equal(B.linear(x, w, dtype=F32).double(), y)
    B.linear_status()


@pytest.mark.parametrize("kind", [BF, HF])
@pytest.mark.parametrize("K", [64, 200, 256, 512, 1024, 2048])
@pytest.mark.parametrize("T,N", [(5, 2000), (300, 2000)])
def test_fp32_results_of_short_rows(T, N, K, kind):
    """A quarter of a row in each accumulator, one K block (4 MMAs of 16) at least and 8 at most: at 0.24 * 2^-23 per MMA of a part, as
    above, and half a unit at most (2^-24) for each of the up to four additions of parts and for the result, over its size."""
    from paper_2507_22424_b200 import binding as B
    g = torch.Generator(device="cuda").manual_seed(T + K)
    x = torch.randn(T, K, generator=g, device="cuda").to(kind)
    w = torch.randn(N, K, generator=g, device="cuda").to(kind)
    y, want = B.linear(x, w, dtype=F32).double(), x.double() @ w.double().T
    off = ((y - want).pow(2).mean() / want.pow(2).mean()).sqrt()
    mmas = 4 * min(8, max(1, (K + 63) // 64 // 4))
    assert off <= (0.24 * mmas + 2.5) * 2.0 ** -23, float(off) * 2 ** 23
