"""Products with 4-bit weights over many stages a CTA, and of prompts.  The bounds are test_gpu_linear.py's and test_gpu_gated.py's
for the unpacked matrix, whose values the products use exactly."""
import math

import pytest
import torch

from paper_2504_06323_b200 import api
from test_gpu_gated import check_gated, empty, vector
from test_gpu_linear import ACTS, check_forward, matrix
from test_gpu_weight4 import DEV, weight4

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m", [12, 20, 33, 48, 64, 100, 128, 200])
@pytest.mark.parametrize("n,k", [(300, 9000), (4096, 8807), (9600, 4096)])
def test_many_stages(m, n, k):
    """Every tile width over contractions of up to 36 stages: the first result against the formula, twenty more for its bits."""
    g = torch.Generator(device=DEV).manual_seed(m + n)
    w4, W = weight4(n, k, g, 64, 1.0 / math.sqrt(k))
    u4, U = weight4(n, k, g, 128, 1.0 / math.sqrt(k))
    X, bias = matrix(m, k, g, -k % 8), vector(n, g)
    status = torch.full((2,), 7, device=DEV, dtype=torch.int32)

    def both():
        Y, H = empty(m, n), empty(m, n)
        api.mosaic_linear4(X, w4, Y, bias=bias, status=status[0:1])
        api.mosaic_gated_linear4(X, w4, u4, H, bias_gate=bias, status=status[1:2])
        return Y, H

    Y, H = both()
    check_forward(X, W, bias, None, "none", Y, None)
    check_gated(X, W, U, bias, None, "silu", H, None, None)
    for _ in range(20):
        more = both()
        assert torch.equal(more[0], Y) and torch.equal(more[1], H)
    assert not bool(status.any())


@pytest.mark.parametrize("m,n,k", [(2049, 2500, 136), (260, 5000, 4100), (4100, 4200, 264), (2304, 2305, 64), (2560, 2050, 1500), (300, 8807, 1001)])
def test_prompts(m, n, k):
    """Tokens of a whole prompt: tiles of pairs of CTAs, a last wave cut up, X off 16 bytes beside the unpacked weights."""
    g = torch.Generator(device=DEV).manual_seed(m + n + k)
    act, group = ACTS[(m + n) % 4], (32, 64, 128)[k % 3]
    w4, W = weight4(n, k, g, group, 1.0 / math.sqrt(k))
    X, R, Y = matrix(m, k, g, m % 3), matrix(m, n, g), matrix(m, n, g, 1)
    bias = vector(n, g) if n % 2 else None
    status = torch.full((1,), 7, device=DEV, dtype=torch.int32)
    api.mosaic_linear4(X, w4, Y, bias=bias, residual=R if k % 2 == 0 else None, act=act, status=status)
    assert int(status.item()) == 0
    check_forward(X, W, bias, R if k % 2 == 0 else None, act, Y, None)


@pytest.mark.parametrize("m,n,k", [(2049, 1250, 136), (260, 5000, 4100), (4100, 2100, 264), (2304, 1153, 64), (2560, 1050, 1500), (300, 4403, 1001)])
def test_gated_prompts(m, n, k):
    g = torch.Generator(device=DEV).manual_seed(m + n + k)
    act = ACTS[(m + k) % 4]
    g4, Wg = weight4(n, k, g, 128, 1.0 / math.sqrt(k))
    u4, Wu = weight4(n, k, g, 32, 1.0 / math.sqrt(k))
    X, H = matrix(m, k, g, m % 3), matrix(m, n, g, 1)
    bg, bu = vector(n, g) if n % 2 else None, vector(n, g) if k % 2 else None
    status = torch.full((1,), 7, device=DEV, dtype=torch.int32)
    api.mosaic_gated_linear4(X, g4, u4, H, bias_gate=bg, bias_up=bu, act=act, status=status)
    assert int(status.item()) == 0
    check_gated(X, Wg, Wu, bg, bu, act, H, None, None)
