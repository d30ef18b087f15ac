"""Weights in 4 bits: codes and scales bit for bit against the definition, and the products that read them.

Packing divides once and rounds twice, both decided by small whole numbers (a bf16 value over a scale of five bits), so codes,
scales and values are compared for equality.  The products multiply by the values exactly, which are bf16 numbers: their
bounds are those of test_gpu_linear.py and test_gpu_gated.py for the unpacked matrix."""
import math

import pytest
import torch

from paper_2504_06323_b200 import api
from test_gpu_gated import check_gated, empty, vector
from test_gpu_linear import ACTS, check_forward, matrix

pytestmark = pytest.mark.gpu
DEV = "cuda"


def reference(W, group):
    """(codes + 8 [rows, groups, group], scales) from the definition, in fp64 on the host."""
    w = W.double().cpu()
    rows, cols = w.shape
    w = torch.nn.functional.pad(w, (0, -cols % group)).view(rows, -(-cols // group), group)
    ideal = w.abs().amax(2) / 7.0
    mantissa, exponent = torch.frexp(torch.nan_to_num(ideal, nan=1.0, posinf=1.0))
    s = torch.round(mantissa * 32.0) * torch.pow(2.0, (exponent - 5).double())
    s = torch.where(ideal < 2.0 ** -126, 0.0, torch.clamp(s, max=2.0 ** 123))
    bad = ~torch.isfinite(ideal)
    code = torch.where((s > 0)[..., None], torch.nan_to_num(w) / torch.where(s > 0, s, 1.0)[..., None], 0.0)
    code = torch.where(bad[..., None], 0.0, torch.round(code).clamp(-7, 7))
    return (code + 8).to(torch.uint8), torch.where(bad, float("nan"), s)


def unpack(codes, cols):
    c = codes.cpu()
    return torch.stack([c & 15, c >> 4], 2).flatten(1)[:, :cols]


def check_pack(W, group, pitch=0, width=0):
    rows, cols = W.shape
    n, groups = -(-cols // 32) * 16, -(-cols // group)
    codes = torch.full((rows, n + 16 * width), 7, dtype=torch.uint8, device=DEV)
    scales = torch.full((rows, groups + width), 3.0, dtype=torch.bfloat16, device=DEV)
    w4 = api.Weight4(codes, scales, cols, group)
    api.mosaic_quantize4(W, w4)
    want, s = reference(W, group)
    assert torch.equal(unpack(codes, cols), want.flatten(1)[:, :cols])
    assert torch.equal(torch.nan_to_num(scales[:, :groups].double().cpu(), nan=1e300), torch.nan_to_num(s, nan=1e300))
    assert (codes[:, n:] == 7).all() and (scales[:, groups:] == 3).all()
    buf = torch.full((rows * (cols + pitch) + 8,), 5.0, device=DEV, dtype=torch.bfloat16)
    out = buf[pitch:pitch + rows * (cols + pitch)].view(rows, cols + pitch) if pitch < 8 else buf[:rows * (cols + pitch)].view(rows, cols + pitch)
    api.mosaic_dequantize4(w4, out[:, :cols])
    values = ((want.double() - 8) * s[..., None]).flatten(1)[:, :cols]
    assert torch.equal(torch.nan_to_num(out[:, :cols].double().cpu(), nan=1e300), torch.nan_to_num(values, nan=1e300))
    assert (out[:, cols:] == 5).all()
    return w4


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 31), (3, 32), (2, 33), (5, 127), (4, 129), (7, 255), (3, 2049), (37, 8807), (301, 96)])
@pytest.mark.parametrize("pitch,width", [(0, 0), (5, 1), (8, 2)])
def test_packing(group, rows, cols, pitch, width):
    g = torch.Generator(device=DEV).manual_seed(rows + cols + group)
    W = matrix(rows, cols, g, pitch, pitch if pitch < 8 else 8, 0.02)
    W *= torch.rand(rows, cols, generator=g, device=DEV) < 0.5
    w4 = check_pack(W, group, pitch, width)
    back = empty(rows, cols)
    api.mosaic_dequantize4(w4, back)
    assert (back[W == 0] == 0).all()


@pytest.mark.parametrize("group", [32, 128])
def test_packing_ties_and_extremes(group):
    """Every bf16 magnitude under every kind of scale: ties among the codes, all sizes, subnormals, infinities, NaN."""
    g = torch.Generator(device=DEV).manual_seed(group)
    bits = torch.randint(0, 1 << 16, (2048, 256), generator=g, device=DEV, dtype=torch.int32).to(torch.int16)
    W = bits.view(torch.bfloat16).clone()
    big = torch.exp2(torch.randint(-130, 128, (2048, 1), generator=g, device=DEV).double()) * 1.25
    W = torch.where(W.double().abs() <= big, W, torch.zeros_like(W))
    W[::9, ::50] = float("inf")
    W[1::9, ::70] = float("nan")
    check_pack(W, group)
    # whole and half multiples of a scale: 7 s is the largest, so the scale is s itself
    s = torch.tensor([16, 17, 19, 24, 29, 31], dtype=torch.float64)[:, None] * 2.0 ** -9
    halves = torch.arange(-14, 15, dtype=torch.float64)[None] / 2
    T = (s * halves).to(torch.bfloat16)
    check_pack(torch.nn.functional.pad(T, (0, 32 - T.shape[1])).to(DEV), 32)
    check_pack(torch.zeros(4, 70, device=DEV, dtype=torch.bfloat16), group)
    check_pack(empty(0, 40), group)


@pytest.mark.parametrize("power", [-120, -99, -12, 0, 60, 118])
def test_every_value_under_every_scale(power):
    """A group's largest is 7 s, so its scale is s: every bf16 number up to 7 s beside it, for all 16 significands of s."""
    rows = []
    for s in range(16, 32):
        v = torch.arange(1, 1 << 15, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).double()
        v = v[(v >= s * 0.2) & (v <= 7.0 * s)]
        v = torch.nn.functional.pad(v, (0, -v.numel() % 31)).view(-1, 31)
        rows.append(torch.cat([torch.full((v.shape[0], 1), 7.0 * s, dtype=torch.float64), v], 1))
    W = (torch.cat(rows) * 2.0 ** power).to(torch.bfloat16)
    W[1::2, 1:] *= -1
    check_pack(W.to(DEV), 32)


def weight4(n, k, g, group, scale):
    """(packed, the values it stands for)"""
    w4 = api.Weight4.of(matrix(n, k, g, scale=scale), group)
    W = empty(n, k)
    api.mosaic_dequantize4(w4, W)
    return w4, W


TOKENS = [1, 2, 7, 8, 9, 16, 17, 24, 33, 65, 129, 256, 257]


@pytest.mark.parametrize("m", TOKENS)
@pytest.mark.parametrize("n,k,group", [(1, 1, 32), (15, 33, 32), (17, 127, 64), (130, 1000, 128), (257, 2049, 32), (640, 4096, 128), (100, 8807, 64)])
def test_linear4(m, n, k, group):
    g = torch.Generator(device=DEV).manual_seed(m + n + k)
    act = ACTS[(m + n) % 4]
    w4, W = weight4(n, k, g, group, 1.0 / math.sqrt(k))
    X, R, Y = matrix(m, k, g, m % 3), matrix(m, n, g), matrix(m, n, g, 1)
    bias = vector(n, g) if m % 2 else None
    status = torch.full((1,), 7, device=DEV, dtype=torch.int32)
    api.mosaic_linear4(X, w4, Y, bias=bias, residual=R if n % 2 else None, act=act, status=status)
    assert int(status.item()) == 0
    check_forward(X, W, bias, R if n % 2 else None, act, Y, None)
    if n % 2:   # added in place
        before = R.clone()
        api.mosaic_linear4(X, w4, R, bias=bias, residual=R, act=act)
        assert torch.equal(R, Y)
        check_forward(X, W, bias, None, act, R, None, y_ref_residual=before)


@pytest.mark.parametrize("m", TOKENS)
@pytest.mark.parametrize("n,k,groups", [(1, 1, (32, 32)), (7, 33, (32, 64)), (9, 127, (64, 64)), (130, 1000, (128, 32)), (257, 2049, (32, 32)), (640, 4096, (128, 128))])
def test_gated_linear4(m, n, k, groups):
    g = torch.Generator(device=DEV).manual_seed(m + n + k)
    act = ACTS[(m + n) % 4]
    g4, Wg = weight4(n, k, g, groups[0], 1.0 / math.sqrt(k))
    u4, Wu = weight4(n, k, g, groups[1], 1.0 / math.sqrt(k))
    X, H = matrix(m, k, g, -k % 8), matrix(m, n, g, 3, 1)
    bg, bu = vector(n, g) if m % 2 else None, vector(n, g) if n % 2 else None
    api.mosaic_gated_linear4(X, g4, u4, H, bias_gate=bg, bias_up=bu, act=act)
    check_gated(X, Wg, Wu, bg, bu, act, H, None, None)


@pytest.mark.parametrize("m", [1, 8, 20, 70, 200])
def test_gated_weights_lie_anywhere(m):
    """Gate before up in memory or behind it, of equal or unequal pitch and group, or one and the same: the same bits."""
    g = torch.Generator(device=DEV).manual_seed(m)
    n, k = 200, 1200
    Wg, Wu, X = matrix(n, k, g, scale=0.05), matrix(n, k, g, scale=0.05), matrix(m, k, g)
    width, seen = 608, []
    for gate_at, up_at, gate_w, up_w in ((0, 1, width, width), (1, 0, width, width), (0, 1, width + 16, width), (1, 0, width, width + 32)):
        buf, scales = torch.full((2, n * (width + 32)), 0xA5, dtype=torch.uint8, device=DEV), torch.zeros(2, n, 40, dtype=torch.bfloat16, device=DEV)
        pair = [api.Weight4(buf[at, :n * w].view(n, w), scales[at, :, :38], k, 32) for at, w in ((gate_at, gate_w), (up_at, up_w))]
        for w4, W in zip(pair, (Wg, Wu)):
            api.mosaic_quantize4(W, w4)
        H = empty(m, n)
        api.mosaic_gated_linear4(X, *pair, H)
        seen.append(H)
    assert all(torch.equal(seen[0], other) for other in seen[1:])
    values = [empty(n, k), empty(n, k)]
    for w4, v in zip(pair, values):
        api.mosaic_dequantize4(w4, v)
    check_gated(X, *values, None, None, "silu", seen[0], None, None)
    api.mosaic_gated_linear4(X, pair[0], pair[0], H)
    check_gated(X, values[0], values[0], None, None, "silu", H, None, None)


@pytest.mark.parametrize("m", [1, 8, 16, 40, 128, 256])
@pytest.mark.parametrize("n,k", [(300, 9000), (4096, 4096), (130, 300)])
def test_calls_repeat_their_bits(m, n, k):
    """Fifty calls in a row over contractions of one stage to many: no wait lets a stage of another turn through."""
    g = torch.Generator(device=DEV).manual_seed(m + n)
    w4, _ = weight4(n, k, g, 64, 0.02)
    u4, _ = weight4(n, k, g, 128, 0.02)
    X = matrix(m, k, g)
    first = None
    for _ in range(50):
        Y, H = empty(m, n), empty(m, n)
        api.mosaic_linear4(X, w4, Y)
        api.mosaic_gated_linear4(X, w4, u4, H)
        if first is None:
            first = Y, H
        assert torch.equal(Y, first[0]) and torch.equal(H, first[1])


@pytest.mark.parametrize("m", [1, 20, 40])
def test_nothing_behind_the_last_column_or_row_is_used(m):
    """Codes behind the last column hold anything, scales around the matrix NaN; outputs end where they should."""
    g = torch.Generator(device=DEV).manual_seed(4)
    n, k, group = 45, 173, 64
    W = matrix(n, k, g, scale=0.1)
    codes = torch.randint(0, 256, (n, 128), generator=g, device=DEV, dtype=torch.int32).to(torch.uint8)
    scales = torch.full((n, 5), float("nan"), device=DEV, dtype=torch.bfloat16)
    w4 = api.Weight4(codes, scales, k, group)
    api.mosaic_quantize4(W, w4)
    codes[:, 87:] = 0xEE
    codes[:, 86] |= 0xF0
    values = empty(n, k)
    api.mosaic_dequantize4(w4, values)
    X, Y, H = matrix(m, k, g, 3), matrix(m, n, g, 2, 1), matrix(m, n, g, 2, 1)
    before = Y._base.clone(), H._base.clone()
    api.mosaic_linear4(X, w4, Y)
    api.mosaic_gated_linear4(X, w4, w4, H, act="none")
    check_forward(X, values, None, None, "none", Y, None)
    check_gated(X, values, values, None, None, "none", H, None, None)
    for t, b in zip((Y, H), before):
        outside = torch.ones_like(b, dtype=torch.bool)
        outside.as_strided(t.shape, t.stride(), t.storage_offset()).fill_(False)
        assert torch.equal(t._base[outside].view(torch.int16), b[outside].view(torch.int16))


@pytest.mark.parametrize("m", [0, 1, 12, 50])
def test_values_that_are_no_numbers(m):
    """A row with a NaN weight gives NaN in its output alone; a NaN token stays in its row; no tokens is legal."""
    g = torch.Generator(device=DEV).manual_seed(5)
    W = matrix(40, 200, g, scale=0.1)
    W[3, 100] = float("inf")
    w4 = api.Weight4.of(W, 64)
    X, Y = matrix(m, 200, g), empty(m, 40)
    if m > 1:
        X[1, 7] = float("nan")
    api.mosaic_linear4(X, w4, Y)
    bad = torch.zeros(m, 40, dtype=torch.bool, device=DEV)
    bad[:, 3] = True
    if m > 1:
        bad[1] = True
    assert torch.equal(torch.isnan(Y), bad)


def test_refusals():
    g = torch.Generator(device=DEV).manual_seed(1)
    W, X, Y = matrix(24, 40, g), matrix(4, 40, g), empty(4, 24)
    w4 = api.Weight4.of(W, 32)
    u8 = lambda *s: torch.empty(*s, dtype=torch.uint8, device=DEV)  # noqa: E731
    for args, error in (((u8(24, 31), empty(24, 2), 40, 32), ValueError), ((u8(24, 32), empty(24, 1), 40, 32), ValueError), ((u8(24, 32), empty(23, 2), 40, 32), ValueError),
                        ((u8(24, 32), empty(24, 2), 40, 48), ValueError), ((u8(24, 32).cpu(), empty(24, 2), 40, 32), TypeError),
                        ((u8(24, 32), empty(24, 2).float(), 40, 32), TypeError), ((u8(32, 24).T, empty(24, 2), 40, 32), ValueError), ((u8(24, 32), empty(24, 2), 0, 32), ValueError)):
        with pytest.raises(error):
            api.Weight4(*args)
    for call, error in ((lambda: api.mosaic_linear4(X, W, Y), TypeError), (lambda: api.mosaic_linear4(X[:, :39], w4, Y), ValueError), (lambda: api.mosaic_linear4(X, w4, None), TypeError),
                        (lambda: api.mosaic_linear4(X, w4, empty(4, 23)), ValueError), (lambda: api.mosaic_linear4(X.float(), w4, Y), TypeError),
                        (lambda: api.mosaic_linear4(X, w4, Y, act="tanh"), ValueError), (lambda: api.mosaic_linear4(X, w4, Y, bias=empty(23)), ValueError),
                        (lambda: api.mosaic_gated_linear4(X, w4, api.Weight4.of(W[:23], 32), Y), ValueError), (lambda: api.mosaic_gated_linear4(X, w4, None, Y), TypeError),
                        (lambda: api.mosaic_quantize4(W.float(), w4), TypeError), (lambda: api.mosaic_quantize4(W[:, :39], w4), ValueError),
                        (lambda: api.mosaic_dequantize4(w4, W[:23]), ValueError)):
        with pytest.raises(error):
            call()
    for call, status in ((lambda: api.mosaic_linear4(X, w4, X[:, :24]), -6), (lambda: api.mosaic_gated_linear4(X, w4, w4, X[:, :24]), -6), (lambda: api.mosaic_linear4(X, w4, Y, act=7), -1),
                         (lambda: api.mosaic_quantize4(W, api.Weight4(u8(24, 40), empty(24, 2), 40, 32)), -4)):
        with pytest.raises(api.MosaicError) as e:
            call()
        assert e.value.status == status
