"""Matrices of more than 2^31 elements: what lies behind the 32-bit range is where it should be.  Checked at rows spread over the
whole, the last among them; the calls' own bounds as in test_gpu_gated.py and test_gpu_linear.py."""
import pytest
import torch

from paper_2504_06323_b200 import api
from test_gpu_checkpoint import reference, values
from test_gpu_gated import check_gated, check_gated_backward, empty
from test_gpu_linear import check_forward
from test_gpu_weight4 import reference as reference4, unpack

pytestmark = pytest.mark.gpu
DEV = "cuda"


def filled(rows, cols, g, scale=1.0):
    t = empty(rows, cols)
    for r in range(0, rows, 1 << 15):
        t[r:r + (1 << 15)] = torch.randn(min(1 << 15, rows - r), cols, generator=g, device=DEV) * scale
    return t


def some(rows):
    return torch.tensor(sorted({0, 1, rows // 3, rows // 2, rows // 2 + 1, (1 << 31) // 8192, rows - 2, rows - 1}), device=DEV)


def test_checkpoint():
    g = torch.Generator(device=DEV).manual_seed(1)
    rows, cols = 270000, 8192
    X = filled(rows, cols, g)
    c = api.Checkpoint.empty(rows, cols)
    api.mosaic_checkpoint_store(X, c)
    at = some(rows)
    codes, E = reference(X[at])
    assert torch.equal(c.codes[at].cpu(), codes) and torch.equal(c.exponents[at].cpu(), E)
    X.zero_()
    api.mosaic_checkpoint_load(c, X)
    assert torch.equal(X[at].double().cpu(), values(codes, E, cols))


def test_weight4():
    g = torch.Generator(device=DEV).manual_seed(2)
    rows, cols = 1100000, 4096
    W = filled(rows, cols, g, 0.02)
    w4 = api.Weight4.of(W, 64)
    at = some(rows)
    want, s = reference4(W[at], 64)
    assert torch.equal(unpack(w4.codes[at], cols), want.flatten(1)) and torch.equal(w4.scales[at].double().cpu(), s)
    api.mosaic_dequantize4(w4, W)
    assert torch.equal(W[at].double().cpu(), ((want.double() - 8) * s[..., None]).flatten(1))
    for m in (1, 20):
        X, Y = filled(m, cols, g), empty(m, rows)
        api.mosaic_linear4(X, w4, Y)
        check_forward(X, W[at], None, None, "none", Y[:, at], None)


def test_gated_linear():
    g = torch.Generator(device=DEV).manual_seed(3)
    m, n, k = 270000, 8192, 64
    X, Wg, Wu = filled(m, k, g), filled(n, k, g, 0.2), filled(n, k, g, 0.2)
    H, Z, U = empty(m, n), empty(m, n), empty(m, n)
    api.mosaic_gated_linear(X, Wg, Wu, H, Z=Z, U=U)
    at = some(m)
    check_gated(X[at], Wg, Wu, None, None, "silu", H[at], Z[at], U[at])
    dX, again = empty(m, k), empty(m, n)
    api.mosaic_gated_linear_backward(H, None, Wg, Wu, Z, U, dX=dX, H=again)
    check_gated_backward(H[at], X[at], Wg, Wu, Z[at], U[at], "silu", dX=dX[at], H=again[at])
