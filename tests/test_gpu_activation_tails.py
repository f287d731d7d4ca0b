"""The linear layer's activations over their whole range, relative to the value: arguments come in through the bias, so that
nothing but the activation and its rounding is left. Bounds: f32 steps are 2^-23, a rounding half of one."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32


def activated(vals, act, dtype, T):
    """act(vals) from a product of zeros, by the kernel of few rows (T = 3) or of many (T = 200)."""
    from paper_2507_22424_b200 import binding as B
    x, w = torch.zeros(T, 16, dtype=HF, device="cuda"), torch.zeros(len(vals), 16, dtype=HF, device="cuda")
    y = B.linear(x, w, vals.cuda(), act, dtype=dtype).cpu()
    assert torch.equal(y, y[:1].expand_as(y))
    return y[0].double()


def arguments(least):
    v = torch.cat([torch.linspace(least, -least, 4001), torch.logspace(-30, 0, 200), -torch.logspace(-30, 0, 200)])
    return torch.cat([v, torch.tensor([-4.0, -4.5, -5.0, -5.5, -6.0, 4.0, 6.0])])


def gelu(v):
    """v / 2 erfc(-v / sqrt 2): 1 + erf would cancel in 64 bits too."""
    return 0.5 * v * torch.erfc(-v * math.sqrt(0.5))


@pytest.mark.parametrize("T", [3, 200])
def test_gelu_in_f32_keeps_its_tail(T):
    """Polynomial 1 step and its evaluation 3, reciprocal and exponential 1 and 2, products 2: 9 steps of the tail's own
    value; 10 are allowed. Down to -13, where the result is 8e-38."""
    v = arguments(-13.0)
    want = gelu(v.double())
    err = (activated(v, "gelu", F32, T) - want).abs()
    assert (err <= 10 * 2.0 ** -23 * want.abs() + 2.0 ** -149).all(), float((err / want.abs().clamp(min=1e-300)).max())


@pytest.mark.parametrize("T", [3, 200])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_gelu_in_16_bits_is_off_by_its_rounding(dtype, T):
    """Before the result's own half step: polynomial, reciprocals, exponential and products as above, 12 * 2^-23 in all; three
    roundings of the exponent v^2 / 2, each 2^-24 of it. Below half a step of f16 (2^-25) nothing but the rounding counts."""
    v = arguments(-13.0)
    want = gelu(v.double())
    least = 2.0 ** -25 if dtype == HF else 2.0 ** -134
    before = 12 * 2.0 ** -23 + 3 * 2.0 ** -24 * v.double() ** 2 / 2
    err = (activated(v, "gelu", dtype, T) - want).abs()
    tol = (before + torch.finfo(dtype).eps / 2 * (1 + before)) * want.abs() + least
    assert (err <= tol).all(), float((err / want.abs().clamp(min=1e-300))[want.abs() > 1e-4].max())


def silu(v):
    return v * torch.sigmoid(v)


def gelu_tanh(v):
    """v / 2 (1 + tanh z) = v sigmoid(2 z)"""
    return v * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3))


@pytest.mark.parametrize("T", [3, 200])
@pytest.mark.parametrize("act,least", [("silu", -103.0), ("gelu_tanh", -10.7)])
@pytest.mark.parametrize("dtype", [F32, BF, HF])
def test_sigmoids_keep_their_tail(dtype, act, least, T):
    """exp(-z), z the sigmoid's argument: five roundings of z (SiLU: one) and the constant's, 2^-24 each of |z|, the exponential
    2^-22, the reciprocal (or the division) and products 2^-22; then half a step. As far as exp(-|z|) is a number, which below 2^-126 is
    one in steps of 2^-149 that the factor v scales."""
    v = arguments(least)
    f = silu if act == "silu" else gelu_tanh
    want = f(v.double())
    z = v.double().abs() if act == "silu" else 2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v.double() ** 3).abs()
    before = 2.0 ** -20 + 6 * 2.0 ** -24 * z
    err = (activated(v, act, dtype, T) - want).abs()
    small = {F32: 2.0 ** -149, BF: 2.0 ** -134, HF: 2.0 ** -25}[dtype] + 2.0 ** -149 * v.abs().double()
    tol = (before + torch.finfo(dtype).eps / 2 * (1 + before)) * want.abs() + small
    assert (err <= tol).all(), v[err > tol]
