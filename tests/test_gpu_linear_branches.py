"""The linear calls at sizes that take the branches which small ones do not: the last wave of the paired kernel cut into
quarters, the widest single tiles, and the few-token kernel over rows off 16 bytes.  Bounds as in test_gpu_linear.py,
whose helpers these tests use.

Which kernel a size takes was read off the launches on 148 SMs (forward / dX / dW; "cut" is the paired kernel and the
quarters of its last wave, "wide" the single 128 x 256 tile); on another number of SMs the sizes test what they meet.
"""
import math

import pytest
import torch

from paper_2504_06323_b200 import api
from test_gpu_linear import ACTS, check_backward, check_forward, matrix, run_backward, run_linear

pytestmark = pytest.mark.gpu
DEV = "cuda"

BRANCHES = [
    (1290, 3400, 4120),   # forward cut: the quarters of the last tiles lie inside, across and wholly outside the matrix
    (1300, 3500, 4100),   # forward cut, quarters across the edge in both directions
    (1290, 4120, 3400),   # dX cut
    (4120, 1290, 3400),   # dW cut
    (250, 9473, 264),     # forward wide, dW wide; an odd number of outputs
    (500, 6000, 520),     # forward wide, dW wide
    (250, 9400, 4104),    # dX wide, its contraction shared
    (512, 4100, 11009),   # forward wide, its contraction shared; dX cut
]


@pytest.mark.parametrize("m,n,k", BRANCHES)
def test_forward(m, n, k):
    g = torch.Generator(device=DEV).manual_seed(m + n + k)
    X, W = matrix(m, k, g, -k % 8), matrix(n, k, g, -k % 8, scale=1.0 / math.sqrt(k))
    bias = torch.randn(n, generator=g, device=DEV).to(torch.bfloat16)
    for act, pitch, offset in (("silu", -n % 2, 0), ("gelu", 1 - n % 2, 1)):      # two elements a word, and one by one
        R, Y, Z = matrix(m, n, g, pitch, offset), matrix(m, n, g, pitch, offset), matrix(m, n, g, pitch, offset)
        run_linear(X, W, Y, bias=bias, residual=R, act=act, Z=Z)
        check_forward(X, W, bias, R, act, Y, Z)
        run_linear(X, W, R, bias=bias, residual=R, act=act)
        assert torch.equal(R, Y)


@pytest.mark.parametrize("m,n,k", BRANCHES)
def test_backward(m, n, k):
    g = torch.Generator(device=DEV).manual_seed(m + 2 * n + k)
    act = ACTS[(m + k) % 4]
    X, W = matrix(m, k, g, -k % 8), matrix(n, k, g, -k % 8, scale=0.05)
    dY, Z = matrix(m, n, g, -n % 8), matrix(m, n, g, scale=2.0) if act != "none" else None
    dX, dW, db = matrix(m, k, g, 1), matrix(n, k, g, k % 2), torch.empty(n, device=DEV, dtype=torch.bfloat16)
    run_backward(dY, X, W, Z=Z, act=act, dX=dX, dW=dW, dbias=db)
    check_backward(dY, X, W, Z, act, dX, dW, db)


def test_cut_wave_writes_only_its_matrix():
    g = torch.Generator(device=DEV).manual_seed(5)
    m, n, k = 1290, 3400, 4120
    X, W = matrix(m, k, g), matrix(n, k, g)
    for left, right in ((4, 4), (3, 2)):
        buf = torch.full((m + 2, left + n + right), 3.0, device=DEV, dtype=torch.bfloat16)
        run_linear(X, W, buf[1:m + 1, left:left + n])
        assert (buf[0] == 3).all() and (buf[-1] == 3).all() and (buf[:, :left] == 3).all() and (buf[:, left + n:] == 3).all()


@pytest.mark.parametrize("m", [1, 2, 3, 4])
@pytest.mark.parametrize("n,k", [(1, 1), (5, 7), (203, 333), (1001, 4099), (64, 8192)])
@pytest.mark.parametrize("px,ox,pw,ow", [(0, 0, 0, 0), (0, 1, 0, 3), (3, 0, 1, 0), (8, 8, 5, 1)])
def test_few_tokens_any_alignment(m, n, k, px, ox, pw, ow):
    """Against fp64 at each alignment: the kernels of aligned and unaligned rows add in different orders."""
    g = torch.Generator(device=DEV).manual_seed(m * 7 + n)
    X, W = matrix(m, k, g, px, ox), matrix(n, k, g, pw, ow, scale=1.0 / math.sqrt(k))
    bias = torch.randn(n, generator=g, device=DEV).to(torch.bfloat16)
    act = ACTS[(m + px) % 4]
    R, Y, Z = matrix(m, n, g, 3, 1), matrix(m, n, g, 2, 1), matrix(m, n, g, 1)
    run_linear(X, W, Y, bias=bias, residual=R, act=act, Z=Z)
    check_forward(X, W, bias, R, act, Y, Z)
    run_linear(X, W, R, bias=bias, residual=R, act=act)
    assert torch.equal(R, Y)
    buf = torch.full((m + 2, n + 9), 3.0, device=DEV, dtype=torch.bfloat16)
    run_linear(X, W, buf[1:m + 1, 4:4 + n])
    assert (buf[0] == 3).all() and (buf[-1] == 3).all() and (buf[:, :4] == 3).all() and (buf[:, 4 + n:] == 3).all()
    assert torch.isfinite(buf).all()


def test_few_tokens_nonfinite_stays_in_its_row_and_column():
    g = torch.Generator(device=DEV).manual_seed(6)
    for pad in (0, 1):
        X, W = matrix(4, 333, g, pad), matrix(150, 333, g, pad)
        X[2, 332] = float("inf")
        W[11, 50] = float("nan")
        Y = matrix(4, 150, g)
        run_linear(X, W, Y)
        ok = torch.ones(4, 150, dtype=torch.bool, device=DEV)
        ok[2], ok[:, 11] = False, False
        assert torch.isfinite(Y[ok]).all() and not torch.isfinite(Y[2]).any() and Y[:, 11].isnan().all()


def test_status_is_written_by_every_kernel():
    """A status word that held something is 0 after each kind of call (few tokens, single tiles, pairs with a cut wave)."""
    g = torch.Generator(device=DEV).manual_seed(2)
    for m, n, k in ((1, 40, 64), (3, 40, 63), (50, 40, 64), (1290, 3400, 4120)):
        status = torch.full((1,), 9, device=DEV, dtype=torch.int32)
        api.mosaic_linear(matrix(m, k, g), matrix(n, k, g), matrix(m, n, g), status=status)
        assert int(status.item()) == 0
