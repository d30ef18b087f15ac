"""The activations and their slopes far from zero, where what is left of them is small: relative to their own size.

One input of weight 1 makes Z the input itself (bf16, exact), so Y is the activation alone and dX the slope alone, each
rounded to bf16 once (2^-8 of it).  Evaluation in fp32: the argument of the complementary error function is z / sqrt(2)
rounded twice, and its value moves by 2 x^2 times that relative error (x = z / sqrt(2), below 2^-16 for |z| <= 12); the
exponential's own error grows with its argument to about 100 units of 2^-23 at -72.  Together below 2^-14 of the value.
The slopes of gelu and silu cross zero near -0.75 and -1.28, where their two terms cancel: 2^-20 of the terms, which are
below 1 there.
"""
import pytest
import torch

from paper_2504_06323_b200 import api

pytestmark = pytest.mark.gpu
DEV = "cuda"
REL = 2.0 ** -8 + 2.0 ** -14


def values(lo, hi):
    """Every bf16 number between lo and hi."""
    bits = torch.arange(0, 1 << 16, device=DEV, dtype=torch.int32).to(torch.int16)
    z = bits.view(torch.bfloat16)
    z = z[torch.isfinite(z)]
    return z[(z >= lo) & (z <= hi) & ((z.abs() > 1e-6) | (z == 0))]


def gelu64(z):
    return 0.5 * z * torch.erfc(-z * 0.5 ** 0.5)


def gelu_slope64(z):
    return 0.5 * torch.erfc(-z * 0.5 ** 0.5) + z * torch.exp(-0.5 * z * z) / (2.0 * torch.pi) ** 0.5


def silu64(z):
    return torch.where(z < 0, z * torch.exp(z), z) / (1.0 + torch.exp(-z.abs()))


def silu_slope64(z):
    s = torch.where(z < 0, torch.exp(z), 1.0) / (1.0 + torch.exp(-z.abs()))
    return s * (1.0 + z * torch.exp(-z.clamp(min=0)) / (1.0 + torch.exp(-z.abs())))


CASES = [("gelu", gelu64, gelu_slope64, -12.0, 12.0), ("silu", silu64, silu_slope64, -80.0, 80.0)]


@pytest.mark.parametrize("tokens", ["one", "two", "all"])
@pytest.mark.parametrize("act,f,_,lo,hi", CASES, ids=["gelu", "silu"])
def test_activation_is_right_relative_to_itself(act, f, _, lo, hi, tokens):
    """Along the outputs of one or two tokens (the few-token kernel) and along the tokens (the tensor cores)."""
    z = values(lo, hi)
    one = torch.ones(1, 1, device=DEV, dtype=torch.bfloat16)
    if tokens == "all":
        X, W = z[:, None].contiguous(), one
    else:
        X, W = one.expand(1 if tokens == "one" else 2, 1).contiguous(), z[:, None].contiguous()
    Y = torch.empty(X.shape[0], W.shape[0], device=DEV, dtype=torch.bfloat16)
    api.mosaic_linear(X, W, Y, act=act)
    want = f(z.double())
    for got in ([Y[:, 0]] if tokens == "all" else list(Y)):
        assert ((got.double() - want).abs() <= REL * want.abs()).all()


@pytest.mark.parametrize("act,_,slope,lo,hi", CASES, ids=["gelu", "silu"])
def test_slope_is_right_relative_to_itself(act, _, slope, lo, hi):
    z = values(lo, hi)
    n = z.numel()
    one = torch.ones(1, 1, device=DEV, dtype=torch.bfloat16)
    dY, dX, Z = torch.ones(n, 1, device=DEV, dtype=torch.bfloat16), torch.empty(n, 1, device=DEV, dtype=torch.bfloat16), z[:, None].contiguous()
    api.mosaic_linear_backward(dY, None, one, Z=Z, act=act, dX=dX)
    want = slope(z.double())
    near_zero = torch.where(z.abs() < 2.5, 2.0 ** -20, 0.0).double()
    assert ((dX[:, 0].double() - want).abs() <= REL * want.abs() + near_zero).all()
