"""mosaic_linear / mosaic_linear_backward against the plain formulas in fp64.

Tolerances, element by element, from the arithmetic:
  * a bf16 rounding is at most half a unit in the last place: 2^-8 of the value's magnitude;
  * the tensor cores add 16 exact products to an fp32 running sum per step and truncate: at most
    (C/4 + 4) 2^-24 of the sum of absolute products (C the contraction length; tests/test_gpu_gram.py),
    a split contraction adds at most 8 more roundings of partial sums, bias and residual one each;
  * the activations have slopes below 1.2 in magnitude and are evaluated to 2^-18 of their argument;
  * backward with an activation: dZ is rounded once to bf16 before the products - 2^-8 of the sum of absolute
    products in the worst case.  As a whole (2-norm) two independent roundings of rms below 2^-9 each stay
    below 2^-8 of the result.
"""
import math

import pytest
import torch

from paper_2504_06323_b200 import api

pytestmark = pytest.mark.gpu
DEV = "cuda"
ACTS = ["none", "relu", "gelu", "silu"]


def act64(z, act):
    return {"none": lambda v: v, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}[act](z)


def matrix(rows, cols, g, pitch=0, offset=0, scale=1.0):
    """bf16 [rows, cols] with a leading dimension of cols + pitch, `offset` elements into its buffer; NaN around it."""
    ld = cols + pitch
    buf = torch.full((rows * ld + offset + 8,), float("nan"), device=DEV, dtype=torch.bfloat16)
    m = buf[offset:offset + rows * ld].view(rows, ld)[:, :cols]
    m.copy_(torch.randn(rows, cols, generator=g, device=DEV) * scale)
    return m


def sum_bound(c, abs_sum):
    return (c / 4.0 + 12.0) * 2.0 ** -24 * abs_sum


def forward_ref(X, W, bias, residual, act):
    Xd, Wd = X.double(), W.double()
    z = Xd @ Wd.T + (0 if bias is None else bias.double())
    z_abs = Xd.abs() @ Wd.abs().T + (0 if bias is None else bias.double().abs())
    y = act64(z, act) + (0 if residual is None else residual.double())
    return z, z_abs, y


def check_forward(X, W, bias, residual, act, Y, Z, y_ref_residual=None):
    z, z_abs, y = forward_ref(X, W, bias, residual if y_ref_residual is None else y_ref_residual, act)
    dz = sum_bound(X.shape[1], z_abs)
    bound = 1.2 * dz + 2.0 ** -18 * z.abs() + 2.0 ** -8 * y.abs() + 2.0 ** -23 * (y.abs() + z.abs()) + 1e-37
    assert torch.isfinite(Y).all()
    assert ((Y.double() - y).abs() <= bound).all()
    if Z is not None:
        assert ((Z.double() - z).abs() <= dz + 2.0 ** -8 * z.abs() + 1e-37).all()


def run_linear(X, W, Y, **kw):
    status = torch.full((1,), 7, device=DEV, dtype=torch.int32)
    api.mosaic_linear(X, W, Y, status=status, **kw)
    torch.cuda.synchronize()
    assert int(status.item()) == 0, "a bounded wait of the kernel ran out"
    return Y


SHAPES = [  # tokens, out, in: one token to many, around tile edges (16 / 32 / 64 / 128 tokens, 128 outputs, 64 inputs), odd ones
    (1, 1, 1), (1, 128, 64), (1, 1000, 4096), (3, 130, 65), (15, 257, 129), (16, 128, 2048), (17, 127, 63), (32, 640, 320), (33, 300, 1031),
    (64, 513, 777), (65, 96, 64), (100, 1, 500), (127, 200, 8), (128, 688, 256), (129, 129, 129), (257, 385, 1000), (500, 260, 4100),
    (1000, 1025, 96), (2049, 300, 200),
    (2049, 2500, 136), (260, 5000, 4100), (4100, 4200, 264), (2304, 2305, 64), (2560, 2050, 1500), (1000, 4096, 2048),   # pairs of CTAs, a last wave cut up
]


@pytest.mark.parametrize("m,n,k", SHAPES)
def test_linear_shapes(m, n, k):
    g = torch.Generator(device=DEV).manual_seed(m * 31 + n * 7 + k)
    pad = -k % 8
    X, W = matrix(m, k, g, pad), matrix(n, k, g, pad, scale=1.0 / math.sqrt(k))
    bias = torch.randn(n, generator=g, device=DEV).to(torch.bfloat16)
    R, Y, Z = matrix(m, n, g), matrix(m, n, g), matrix(m, n, g)
    run_linear(X, W, Y, bias=bias, residual=R, act=ACTS[(m + n) % 4], Z=Z)
    check_forward(X, W, bias, R, ACTS[(m + n) % 4], Y, Z)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("m", [2, 300])
@pytest.mark.parametrize("bias_on,res_on,z_on", [(False, False, False), (True, False, True), (False, True, False), (True, True, True)])
def test_linear_epilogues(act, m, bias_on, res_on, z_on):
    g = torch.Generator(device=DEV).manual_seed(m + len(act))
    n, k = 200, 520
    X, W = matrix(m, k, g), matrix(n, k, g, scale=0.1)
    bias = torch.randn(n, generator=g, device=DEV).to(torch.bfloat16) if bias_on else None
    R = matrix(m, n, g, 3, 1) if res_on else None
    Y, Z = matrix(m, n, g, 5, 3), matrix(m, n, g, 1) if z_on else None
    run_linear(X, W, Y, bias=bias, residual=R, act=act, Z=Z)
    check_forward(X, W, bias, R, act, Y, Z)
    if res_on:   # the residual added in place
        before = R.clone()
        run_linear(X, W, R, bias=bias, residual=R, act=act)
        assert torch.equal(R, Y)
        check_forward(X, W, bias, None, act, R, None, y_ref_residual=before)


@pytest.mark.parametrize("px,ox,pw,ow", [(0, 0, 0, 0), (0, 1, 0, 3), (3, 0, 1, 0), (8, 8, 16, 16), (5, 7, 0, 8)])
@pytest.mark.parametrize("m", [1, 5, 140])
def test_linear_any_alignment(m, px, ox, pw, ow):
    """Dense odd rows, odd bases, wide rows: the same bits as with aligned copies, NaN around the matrices never read."""
    g = torch.Generator(device=DEV).manual_seed(m)
    n, k = 203, 333
    X, W = matrix(m, k, g, px, ox), matrix(n, k, g, pw, ow)
    Y, Y2 = matrix(m, n, g, 2, 1), matrix(m, n, g)
    run_linear(X, W, Y, act="silu")
    Xa, Wa = matrix(m, k, g, -k % 8), matrix(n, k, g, -k % 8)
    Xa.copy_(X)
    Wa.copy_(W)
    run_linear(Xa, Wa, Y2, act="silu")
    assert torch.equal(Y, Y2)
    check_forward(X, W, None, None, "silu", Y, None)


def test_linear_writes_only_its_matrix():
    g = torch.Generator(device=DEV).manual_seed(5)
    for m, n, k in [(3, 130, 200), (131, 131, 72)]:
        X, W = matrix(m, k, g), matrix(n, k, g)
        buf = torch.full((m + 2, n + 9), 3.0, device=DEV, dtype=torch.bfloat16)
        run_linear(X, W, buf[1:m + 1, 4:4 + n])
        assert (buf[0] == 3).all() and (buf[-1] == 3).all() and (buf[:, :4] == 3).all() and (buf[:, 4 + n:] == 3).all()


def test_linear_nonfinite_stays_in_its_row_and_column():
    g = torch.Generator(device=DEV).manual_seed(6)
    X, W = matrix(40, 100, g), matrix(150, 100, g)
    X[7, 3] = float("inf")
    W[11, 50] = float("nan")
    Y = matrix(40, 150, g)
    run_linear(X, W, Y)
    ok = torch.ones(40, 150, dtype=torch.bool, device=DEV)
    ok[7], ok[:, 11] = False, False
    assert torch.isfinite(Y[ok]).all() and not torch.isfinite(Y[7]).any() and Y[:, 11].isnan().all()


def test_linear_large_values_saturate_as_the_formula():
    """Activations far out on both sides: relu, gelu and silu of -/+ 1e4 are 0 and z."""
    X = torch.tensor([[1e4], [-1e4], [0.0]], device=DEV).to(torch.bfloat16)
    W = torch.ones(130, 1, device=DEV, dtype=torch.bfloat16)
    for act in ("relu", "gelu", "silu"):
        Y = torch.empty(3, 130, device=DEV, dtype=torch.bfloat16)
        run_linear(X, W, Y, act=act)
        assert (Y[0] == X[0]).all() and (Y[1:] == 0).all()


def test_linear_no_tokens_and_offsets_past_32_bits():
    g = torch.Generator(device=DEV).manual_seed(8)
    W = matrix(64, 64, g)
    api.mosaic_linear(torch.empty(0, 64, device=DEV, dtype=torch.bfloat16), W, torch.empty(0, 64, device=DEV, dtype=torch.bfloat16))
    ld = 1 << 30   # rows two gigabytes apart: element offsets beyond 2^31
    big = torch.empty(3 * ld, device=DEV, dtype=torch.bfloat16)
    X = big.view(3, ld)[:, 8:72]
    Y = big.view(3, ld)[:, 1024:1088]
    X.copy_(torch.randn(3, 64, generator=g, device=DEV))
    Xs = X.clone()
    run_linear(Xs, W, Y)
    check_forward(Xs, W, None, None, "none", Y, None)
    Y2 = torch.empty(3, 64, device=DEV, dtype=torch.bfloat16)
    run_linear(X, W, Y2)
    assert torch.equal(Y2, Y)


def test_linear_deterministic_and_on_another_stream():
    g = torch.Generator(device=DEV).manual_seed(9)
    X, W = matrix(37, 4096, g), matrix(1000, 4096, g, scale=0.02)
    Y = [matrix(37, 1000, g) for _ in range(3)]
    run_linear(X, W, Y[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        api.mosaic_linear(X, W, Y[1])
    api.mosaic_linear(X, W, Y[2], stream=side)
    side.synchronize()
    assert torch.equal(Y[0], Y[1]) and torch.equal(Y[0], Y[2])


def test_linear_llama_width_against_fp64():
    """The projections of the 7B shape (and a compacted one) at one token, a few, and a sequence's worth."""
    for m, n, k in [(1, 11008, 4096), (37, 4096, 8807), (700, 4096, 4096), (2048, 1024, 4096)]:
        g = torch.Generator(device=DEV).manual_seed(m)
        X, W = matrix(m, k, g, -k % 8), matrix(n, k, g, -k % 8, scale=0.02)
        Y = matrix(m, n, g)
        run_linear(X, W, Y)
        check_forward(X, W, None, None, "none", Y, None)


# ------------------------------------------------------------------ backward
def backward_ref(dY, X, W, Z, act):
    z = None if Z is None else Z.double().requires_grad_(True)
    d = dY.double()
    if act != "none":
        d, = torch.autograd.grad(act64(z, act), z, d)
    return d, d @ W.double(), d.T @ X.double(), d.sum(0)


def check_backward(dY, X, W, Z, act, dX, dW, db):
    d, rx, rw, rb = backward_ref(dY, X, W, Z, act)
    slope = 2.0 ** -17 * (dY.double().abs() + 0 * d) if act != "none" else 0 * d     # the slope's own evaluation
    rounded = 2.0 ** -8 * d.abs() + slope if act != "none" else 0 * d
    for got, ref, a, b, err_a in ((dX, rx, d, W.double(), rounded), (dW, rw, d.T, X.double(), rounded.T)):
        if got is None:
            continue
        assert torch.isfinite(got).all()
        bound = err_a @ b.abs() + sum_bound(a.shape[1], a.abs() @ b.abs()) * 1.01 + 2.0 ** -8 * ref.abs() * 1.01 + 1e-37
        assert ((got.double() - ref).abs() <= bound).all()
        if ref.numel() >= 64:
            assert (got.double() - ref).norm() <= 2.0 ** -8 * ref.norm()
    if db is not None:
        m = dY.shape[0]
        bound = 2.0 ** -8 * rb.abs() * 1.01 + (m + 2) * 2.0 ** -24 * d.abs().sum(0) + (slope.sum(0) if act != "none" else 0) + 1e-37
        assert ((db.double() - rb).abs() <= bound).all()


def run_backward(dY, X, W, **kw):
    status = torch.full((1,), 7, device=DEV, dtype=torch.int32)
    api.mosaic_linear_backward(dY, X, W, status=status, **kw)
    torch.cuda.synchronize()
    assert int(status.item()) == 0, "a bounded wait of the kernel ran out"


@pytest.mark.parametrize("m,n,k", SHAPES)
def test_backward_shapes(m, n, k):
    g = torch.Generator(device=DEV).manual_seed(m * 3 + n * 5 + k)
    act = ACTS[(m + k) % 4]
    X, W = matrix(m, k, g, -k % 8), matrix(n, k, g, -k % 8, scale=0.05)
    dY, Z = matrix(m, n, g, -n % 8), matrix(m, n, g, 1, scale=2.0) if act != "none" else None
    dX, dW, db = matrix(m, k, g), matrix(n, k, g), torch.empty(n, device=DEV, dtype=torch.bfloat16)
    run_backward(dY, X, W, Z=Z, act=act, dX=dX, dW=dW, dbias=db)
    check_backward(dY, X, W, Z, act, dX, dW, db)


@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("off", [0, 1])
def test_backward_any_alignment_and_any_subset(act, off):
    g = torch.Generator(device=DEV).manual_seed(3)
    m, n, k = 77, 131, 205
    X, W, dY = matrix(m, k, g, off, off), matrix(n, k, g, 2 * off, 3 * off), matrix(m, n, g, 0, off)
    Z = matrix(m, n, g, 2, 5) if act != "none" else None
    dX, dW, db = matrix(m, k, g, 1, 3), matrix(n, k, g, 4, 1), torch.empty(n, device=DEV, dtype=torch.bfloat16)
    run_backward(dY, X, W, Z=Z, act=act, dX=dX, dW=dW, dbias=db)
    check_backward(dY, X, W, Z, act, dX, dW, db)
    for keep in (("dX",), ("dW",), ("dbias",), ("dX", "dbias")):
        out = {"dX": torch.empty_like(dX), "dW": torch.empty_like(dW), "dbias": torch.empty_like(db)}
        run_backward(dY, X if "dW" in keep else None, W, Z=Z, act=act, **{q: out[q] for q in keep})
        for q, want in (("dX", dX), ("dW", dW), ("dbias", db)):
            if q in keep:
                assert torch.equal(out[q], want)


def test_backward_no_tokens_gives_zero():
    W = torch.randn(40, 24, device=DEV).to(torch.bfloat16)
    e = lambda *s: torch.empty(*s, device=DEV, dtype=torch.bfloat16)  # noqa: E731
    dW, db = torch.full((40, 30), 5.0, device=DEV, dtype=torch.bfloat16), e(40)
    api.mosaic_linear_backward(e(0, 40), e(0, 24), W, dX=e(0, 24), dW=dW[:, :24], dbias=db)
    assert (dW[:, :24] == 0).all() and (dW[:, 24:] == 5).all() and (db == 0).all()


@pytest.mark.parametrize("act", ACTS)
def test_gradients_against_differences(act):
    """Directional differences of f(X, W, b) = sum(G * act(X W^T + b)) in fp64 against the kernel's gradients
    (Z as the forward call stored it).  The differences' own error is O(h^2); the kernel's is bounded by its
    roundings: 2^-8 for dZ (worst case over the products), 2^-8 for the result, and the slope's change over
    half a unit of the stored Z (second derivatives below 1.2; relu is kept away from its kink)."""
    g = torch.Generator(device=DEV).manual_seed(11)
    m, n, k = 33, 70, 48
    X, W, b = matrix(m, k, g), matrix(n, k, g, scale=0.3), torch.randn(n, generator=g, device=DEV).to(torch.bfloat16)
    G = matrix(m, n, g)
    Y, Z = matrix(m, n, g), matrix(m, n, g)
    run_linear(X, W, Y, bias=b, act=act, Z=Z)
    if act == "relu":
        G = torch.where(Z.abs() < 0.05, torch.zeros_like(G), G)
    dX, dW, db = matrix(m, k, g), matrix(n, k, g), torch.empty(n, device=DEV, dtype=torch.bfloat16)
    run_backward(G, X, W, Z=Z, act=act, dX=dX, dW=dW, dbias=db)
    f = lambda x, w, c: (G.double() * act64(x @ w.T + c, act)).sum()  # noqa: E731
    x, w, c, h = X.double(), W.double(), b.double(), 1e-5
    dz_err = G.double().abs() * (2.0 ** -8 * 1.2 + 1.2 * 2.0 ** -8 * Z.double().abs())
    for which, grad, base in (("x", dX, x), ("w", dW, w), ("c", db, c)):
        d = torch.randn(base.shape, generator=g, device=DEV, dtype=torch.float64)
        args = lambda s: [t + (s * h * d if nm == which else 0) for nm, t in (("x", x), ("w", w), ("c", c))]  # noqa: E731
        diff = (f(*args(1)) - f(*args(-1))) / (2 * h)
        if which == "x":
            err = (dz_err @ w.abs() * d.abs()).sum()
        elif which == "w":
            err = (dz_err.T @ x.abs() * d.abs()).sum()
        else:
            err = (dz_err.sum(0) * d.abs()).sum()
        err = err + 2.0 ** -8 * (grad.double().abs() * d.abs()).sum() + 1e-6 * (1 + diff.abs())
        assert (diff - (grad.double() * d).sum()).abs() <= err


# ------------------------------------------------------------------ refusals
def test_linear_refusals():
    L = api.lib()
    g = torch.Generator(device=DEV).manual_seed(1)
    X, W, Y = matrix(8, 16, g), matrix(24, 16, g), matrix(8, 24, g)
    with pytest.raises(TypeError):
        api.mosaic_linear(X.float(), W, Y)
    with pytest.raises(TypeError):
        api.mosaic_linear(X, W, Y.float())
    with pytest.raises(TypeError):
        api.mosaic_linear(X.cpu(), W, Y)
    with pytest.raises(ValueError):
        api.mosaic_linear(X, W, Y[:, :23])
    with pytest.raises(ValueError):
        api.mosaic_linear(X, W, matrix(24, 8, g).T)
    with pytest.raises(ValueError):
        api.mosaic_linear(X, W, Y, act="tanh")
    with pytest.raises(ValueError):
        api.mosaic_linear(X, W, Y, bias=torch.zeros(23, device=DEV, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        api.mosaic_linear_backward(Y, X, W, act="silu", dX=torch.empty_like(X))
    with pytest.raises(api.MosaicError) as e:
        api.mosaic_linear(X, W, Y, act=9)
    assert e.value.status == -1
    both = torch.zeros(8 * 40, device=DEV, dtype=torch.bfloat16)
    with pytest.raises(api.MosaicError) as e:
        api.mosaic_linear(both[:128].view(8, 16), W, both[64:256].view(8, 24))
    assert e.value.status == -6
    with pytest.raises(api.MosaicError) as e:
        api.mosaic_linear_backward(Y, X, W, dX=X, dW=torch.empty_like(W))   # X is still needed for dW
    assert e.value.status == -6
    # a misaligned operand needs scratch: too little, and none
    Xo = matrix(8, 16, g, 1)
    need = L.mosaic_linear_workspace_bytes(Xo.data_ptr(), 17, W.data_ptr(), 16, 8, 24, 16)
    assert need == 256
    call = lambda ws, n: L.mosaic_linear(Xo.data_ptr(), 17, W.data_ptr(), 16, 8, 24, 16, api.BF16, None, None, 24, 0, Y.data_ptr(), 24, None, 24, None, ws, n, None)  # noqa: E731
    assert call(None, 0) == -2
    ws = torch.empty(1024, dtype=torch.uint8, device=DEV)
    assert call(ws.data_ptr(), 128) == -5 and call(ws.data_ptr() + 16, 512) == -4
    assert call(ws.data_ptr(), 256) == 0
    torch.cuda.synchronize()
