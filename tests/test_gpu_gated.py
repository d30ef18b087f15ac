"""mosaic_gated_linear / mosaic_gated_linear_backward against the plain formulas in fp64.

Tolerances, element by element, from the arithmetic (those of test_gpu_linear.py, whose sum_bound is used):
  * Z and U are off by their sums' bound; H = act(Z) U from the unrounded sums, so by |U| (1.2 dZ + 2^-18 |Z|) + (|act(Z)| +
    1.2 dZ + 2^-18 |Z|) dU, the product's own 2^-24 and one rounding, 2^-8 of it;
  * backward: act and its slope are evaluated to 2^-17 (in units of 1 + |Z|) and to 2^-17, two or three multiplications round
    to 2^-24 each; dZ and dU are rounded once to bf16, 2^-8 in the worst case over the sum of absolute products, and as a
    whole (2-norm) two independent roundings of rms below 2^-9 stay below 2^-8 of the result.
"""
import math

import pytest
import torch

from paper_2504_06323_b200 import api
from test_gpu_linear import ACTS, act64, matrix, sum_bound

pytestmark = pytest.mark.gpu
DEV = "cuda"


def empty(*s):
    return torch.empty(*s, device=DEV, dtype=torch.bfloat16)


def vector(n, g):
    return torch.randn(n, generator=g, device=DEV).to(torch.bfloat16)


def check_gated(X, Wg, Wu, bg, bu, act, H, Z, U):
    parts = []
    for W, b in ((Wg, bg), (Wu, bu)):
        x, w = X.double(), W.double()
        s = x @ w.T + (0 if b is None else b.double())
        parts.append((s, sum_bound(X.shape[1], x.abs() @ w.abs().T + (0 if b is None else b.double().abs()))))
    (z, dz), (u, du) = parts
    a = act64(z, act)
    da = 1.2 * dz + 2.0 ** -18 * z.abs()
    h = a * u
    bound = (u.abs() * da + (a.abs() + da) * du) * 1.01 + 2.0 ** -8 * h.abs() * 1.01 + 2.0 ** -23 * h.abs() + 1e-37
    assert torch.isfinite(H).all()
    assert ((H.double() - h).abs() <= bound).all()
    for got, want, d in ((Z, z, dz), (U, u, du)):
        if got is not None:
            assert ((got.double() - want).abs() <= d + 2.0 ** -8 * want.abs() * 1.01 + 1e-37).all()


def run_gated(X, Wg, Wu, H, **kw):
    status = torch.full((1,), 7, device=DEV, dtype=torch.int32)
    api.mosaic_gated_linear(X, Wg, Wu, H, status=status, **kw)
    torch.cuda.synchronize()
    assert int(status.item()) == 0, "a bounded wait of the kernel ran out"


SHAPES = [  # tokens, channels, in: around the tiles' edges (16 / 32 / 64 / 128 tokens, 16 and 64 channels, 64 inputs), odd ones
    (1, 1, 1), (1, 128, 64), (1, 1000, 4096), (2, 15, 200), (3, 130, 65), (4, 17, 2000), (15, 257, 129), (16, 128, 2048), (17, 63, 63), (32, 640, 320),
    (33, 300, 1031), (64, 513, 777), (65, 96, 64), (100, 1, 500), (127, 200, 8), (128, 688, 256), (129, 65, 129), (257, 385, 1000), (500, 260, 4100),
    (1000, 1025, 96), (2049, 300, 200),
    (2049, 1250, 136), (260, 5000, 4100), (4100, 2100, 264), (2304, 1153, 64), (2560, 1050, 1500), (1000, 4096, 2048),   # pairs of CTAs, a last wave cut up
]


@pytest.mark.parametrize("m,n,k", SHAPES)
def test_gated_shapes(m, n, k):
    g = torch.Generator(device=DEV).manual_seed(m * 31 + n * 7 + k)
    act, kept = ACTS[(m + n) % 4], (m + k) % 4
    X, Wg, Wu = matrix(m, k, g, -k % 8), matrix(n, k, g, -k % 8, scale=1.0 / math.sqrt(k)), matrix(n, k, g, -k % 8, scale=1.0 / math.sqrt(k))
    bg, bu = vector(n, g) if n % 2 else None, vector(n, g) if k % 2 == 0 else None
    H = matrix(m, n, g, -n % 8)
    Z, U = matrix(m, n, g, -n % 8) if kept & 1 else None, matrix(m, n, g, -n % 8) if kept & 2 else None
    run_gated(X, Wg, Wu, H, bias_gate=bg, bias_up=bu, act=act, Z=Z, U=U)
    check_gated(X, Wg, Wu, bg, bu, act, H, Z, U)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("m", [1, 4, 19, 300])
@pytest.mark.parametrize("off", [0, 1])
def test_gated_any_alignment(act, m, off):
    """Dense odd rows and odd bases: NaN around the matrices never read, nothing outside the outputs written."""
    g = torch.Generator(device=DEV).manual_seed(m + off)
    n, k = 203, 519
    X, Wg, Wu = matrix(m, k, g, off, off), matrix(n, k, g, 2 * off, 3 * off, 0.1), matrix(n, k, g, off, 5 * off, 0.1)
    H, Z, U = (matrix(m, n, g, p, o) for p, o in ((0, off), (5 * off, 1), (off, 0)))
    before = [t._base.clone() for t in (H, Z, U)]
    bias = vector(n, g)
    run_gated(X, Wg, Wu, H, bias_gate=bias, bias_up=None, act=act, Z=Z, U=U)
    check_gated(X, Wg, Wu, bias, None, act, H, Z, U)
    for t, b in zip((H, Z, U), before):
        outside = torch.ones_like(t._base, dtype=torch.bool)
        outside.as_strided(t.shape, t.stride(), t.storage_offset()).fill_(False)
        assert torch.equal(t._base[outside].view(torch.int16), b[outside].view(torch.int16))


@pytest.mark.parametrize("m", [1, 2, 5, 40, 600])
def test_gated_alignment_changes_no_bit(m):
    """What is kept and where it lies does not change H; Z and U are those of mosaic_linear up to their sums."""
    g = torch.Generator(device=DEV).manual_seed(m)
    n, k = 331, 264
    X, Wg, Wu, bg, bu = matrix(m, k, g), matrix(n, k, g, scale=0.1), matrix(n, k, g, scale=0.1), vector(n, g), vector(n, g)
    H = empty(m, n)
    run_gated(X, Wg, Wu, H, bias_gate=bg, bias_up=bu, act="silu")
    check_gated(X, Wg, Wu, bg, bu, "silu", H, None, None)
    for pitch, kept in ((5, True), (5, False), (1, True), (0, True)):
        H2 = matrix(m, n, g, pitch, pitch)
        Z, U = (matrix(m, n, g, pitch, 1), matrix(m, n, g, 0, 3)) if kept else (None, None)
        run_gated(X, Wg, Wu, H2, bias_gate=bg, bias_up=bu, act="silu", Z=Z, U=U)
        assert torch.equal(H2, H)
        check_gated(X, Wg, Wu, bg, bu, "silu", H2, Z, U)


@pytest.mark.parametrize("m,n,k", [(1, 40, 72), (5, 100, 264), (300, 1000, 520), (2049, 1256, 136), (600, 4104, 2048)])
def test_gated_weights_lie_anywhere(m, n, k):
    """Gate before up in memory or behind it, of equal or unequal pitch, far apart, or one and the same: the same bits."""
    g = torch.Generator(device=DEV).manual_seed(m + n)
    X, Wg, Wu, bg = matrix(m, k, g, -k % 8), matrix(n, k, g, scale=0.1), matrix(n, k, g, scale=0.1), vector(n, g)
    ld = k + -k % 8
    H, Z, U = empty(m, n), empty(m, n), empty(m, n)
    seen = []
    for gate_at, up_at, gate_ld, up_ld in ((0, 1, ld, ld), (1, 0, ld, ld), (0, 1, ld + 8, ld), (1, 0, ld, ld + 16), (0, 5, ld, ld)):
        room = n * (ld + 16) + 64
        buf = torch.full((6 * room,), float("nan"), device=DEV, dtype=torch.bfloat16)
        place = lambda at, pitch, W: buf[at * room:at * room + n * pitch].view(n, pitch)[:, :k].copy_(W)  # noqa: E731
        run_gated(X, place(gate_at, gate_ld, Wg), place(up_at, up_ld, Wu), H, bias_gate=bg, act="silu", Z=Z, U=U)
        seen.append((H.clone(), Z.clone(), U.clone()))
    check_gated(X, Wg, Wu, bg, None, "silu", *seen[0])
    for other in seen[1:]:
        assert all(torch.equal(a, b) for a, b in zip(seen[0], other))
    W = matrix(n, k, g, -k % 8, scale=0.1)
    run_gated(X, W, W, H, bias_gate=bg, act="silu", Z=Z, U=U)
    check_gated(X, W, W, bg, None, "silu", H, Z, U)


@pytest.mark.parametrize("m", [0, 1, 3, 50])
def test_gated_extremes(m):
    """Infinite and NaN inputs stay in their token; rows of zeros give zero; no tokens is legal."""
    g = torch.Generator(device=DEV).manual_seed(2)
    n, k = 150, 96
    X, Wg, Wu, H = matrix(m, k, g), matrix(n, k, g, scale=0.1), matrix(n, k, g, scale=0.1), empty(m, n)
    if m > 1:
        X[0, 5], X[1] = float("nan"), 0.0
    run_gated(X, Wg, Wu, H, act="silu")
    if m > 1:
        assert torch.isnan(H[0]).all() and (H[1] == 0).all()
        check_gated(X[1:], Wg, Wu, None, None, "silu", H[1:], None, None)


def backward_terms(dH, Z, U, act):
    z = Z.double().requires_grad_(True)
    a = act64(z, act)
    a.sum().backward()
    slope, a, u, dh = z.grad, a.detach(), U.double(), dH.double()
    z = z.detach()
    e_a, e_s = (2.0 ** -17 * (1 + z.abs()), 2.0 ** -17) if act != "none" else (0 * z, 0.0)
    dz, du, h = dh * u * slope, dh * a, a * u
    own = [((dh * u).abs() * e_s + 2.0 ** -22 * dz.abs()), (dh.abs() * e_a + 2.0 ** -22 * du.abs()), u.abs() * e_a + 2.0 ** -22 * h.abs()]
    return (dz, du, h), own


def check_gated_backward(dH, X, Wg, Wu, Z, U, act, dX=None, dWg=None, dWu=None, dbg=None, dbu=None, H=None):
    (dz, du, h), (ez, eu, eh) = backward_terms(dH, Z, U, act)
    if H is not None:
        assert ((H.double() - h).abs() <= 1.01 * 2.0 ** -8 * h.abs() + eh + 1e-37).all()
    rz, ru = 1.01 * 2.0 ** -8 * dz.abs() + ez, 1.01 * 2.0 ** -8 * du.abs() + eu
    if dX is not None:
        g, u = Wg.double(), Wu.double()
        ref = dz @ g + du @ u
        bound = rz @ g.abs() + ru @ u.abs() + 1.01 * sum_bound(2 * dz.shape[1], dz.abs() @ g.abs() + du.abs() @ u.abs()) + 1.01 * 2.0 ** -8 * ref.abs() + 1e-37
        assert torch.isfinite(dX).all() and ((dX.double() - ref).abs() <= bound).all()
        if ref.numel() >= 64:
            assert (dX.double() - ref).norm() <= 2.0 ** -8 * ref.norm()
    for got, d, r in ((dWg, dz, rz), (dWu, du, ru)):
        if got is None:
            continue
        x = X.double()
        ref = d.T @ x
        bound = r.T @ x.abs() + 1.01 * sum_bound(d.shape[0], d.abs().T @ x.abs()) + 1.01 * 2.0 ** -8 * ref.abs() + 1e-37
        assert torch.isfinite(got).all() and ((got.double() - ref).abs() <= bound).all()
        if ref.numel() >= 64:
            assert (got.double() - ref).norm() <= 2.0 ** -8 * ref.norm()
    for got, d, e in ((dbg, dz, ez), (dbu, du, eu)):
        if got is None:
            continue
        ref = d.sum(0)
        bound = 1.01 * 2.0 ** -8 * ref.abs() + (d.shape[0] + 2) * 2.0 ** -24 * d.abs().sum(0) + e.sum(0) + 1e-37
        assert ((got.double() - ref).abs() <= bound).all()


def run_back(dH, X, Wg, Wu, Z, U, **kw):
    status = torch.full((1,), 7, device=DEV, dtype=torch.int32)
    api.mosaic_gated_linear_backward(dH, X, Wg, Wu, Z, U, status=status, **kw)
    torch.cuda.synchronize()
    assert int(status.item()) == 0, "a bounded wait of the kernel ran out"


@pytest.mark.parametrize("m,n,k", SHAPES)
def test_gated_backward_shapes(m, n, k):
    g = torch.Generator(device=DEV).manual_seed(m * 3 + n * 5 + k)
    act = ACTS[(m + k) % 4]
    X, Wg, Wu = matrix(m, k, g, -k % 8), matrix(n, k, g, -k % 8, scale=0.05), matrix(n, k, g, -k % 8, scale=0.05)
    dH, Z, U = matrix(m, n, g, -n % 8), matrix(m, n, g, -n % 8, scale=2.0), matrix(m, n, g, -n % 8)
    out = dict(dX=matrix(m, k, g, -k % 8), dW_gate=matrix(n, k, g, -k % 8), dW_up=matrix(n, k, g, -k % 8), dbias_gate=empty(n), dbias_up=empty(n),
               H=matrix(m, n, g, -n % 8))
    run_back(dH, X, Wg, Wu, Z, U, act=act, **out)
    check_gated_backward(dH, X, Wg, Wu, Z, U, act, *out.values())


@pytest.mark.parametrize("m,n,k", [(2560, 1500, 2304), (3000, 1000, 2560), (4096, 700, 2200)])
def test_gated_backward_last_wave_cut_up(m, n, k):
    """dX and dW of more tiles than pairs of SMs, with few left over: their quarters share the contraction."""
    g = torch.Generator(device=DEV).manual_seed(m)
    X, Wg, Wu = matrix(m, k, g), matrix(n, k, g, scale=0.05), matrix(n, k, g, scale=0.05)
    dH, Z, U = matrix(m, n, g), matrix(m, n, g, scale=2.0), matrix(m, n, g)
    out = dict(dX=empty(m, k), dW_gate=empty(n, k), dW_up=empty(n, k))
    run_back(dH, X, Wg, Wu, Z, U, act="silu", **out)
    check_gated_backward(dH, X, Wg, Wu, Z, U, "silu", *out.values())


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("m", [1, 77])
@pytest.mark.parametrize("off", [0, 1])
def test_gated_backward_any_alignment_and_any_subset(act, m, off):
    g = torch.Generator(device=DEV).manual_seed(3)
    n, k = 131, 205
    X, Wg, Wu, dH = matrix(m, k, g, off, off), matrix(n, k, g, 2 * off, 3 * off), matrix(n, k, g, off, 7 * off), matrix(m, n, g, 0, off)
    Z, U = matrix(m, n, g, 2, 5), matrix(m, n, g, 0, off)
    out = dict(dX=matrix(m, k, g, 1, 3), dW_gate=matrix(n, k, g, 4, 1), dW_up=matrix(n, k, g, 0, 1), dbias_gate=empty(n), dbias_up=empty(n), H=matrix(m, n, g, 1))
    before = {q: t._base.clone() for q, t in out.items() if t._is_view()}
    run_back(dH, X, Wg, Wu, Z, U, act=act, **out)
    check_gated_backward(dH, X, Wg, Wu, Z, U, act, *out.values())
    for q, b in before.items():
        t, outside = out[q], torch.ones_like(b, dtype=torch.bool)
        outside.as_strided(t.shape, t.stride(), t.storage_offset()).fill_(False)
        assert torch.equal(t._base[outside].view(torch.int16), b[outside].view(torch.int16))
    whole = {q: t.clone() for q, t in out.items()}
    for names in (["dX"], ["dW_gate"], ["dW_up"], ["dW_gate", "dW_up"], ["dbias_up"], ["dbias_gate", "dX"], ["H"], ["dX", "dW_up", "dbias_up"]):
        some = {q: torch.full_like(out[q], 9.0) for q in names}
        needs_x, needs_w = any(q.startswith("dW") for q in names), "dX" in names
        run_back(dH, X if needs_x or not needs_w else None, Wg if needs_w else None, Wu if needs_w else None, Z, U, act=act, **some)
        for q, t in some.items():
            assert torch.equal(t, whole[q]), q


def test_gated_backward_no_tokens_gives_zero():
    W = torch.randn(40, 24, device=DEV).to(torch.bfloat16)
    dWg, dWu, dbg, dbu = torch.full((40, 30), 5.0, device=DEV, dtype=torch.bfloat16), empty(40, 24), empty(40), empty(40)
    e = empty(0, 40)
    api.mosaic_gated_linear_backward(e, empty(0, 24), W, W, e, e, dX=empty(0, 24), dW_gate=dWg[:, :24], dW_up=dWu, dbias_gate=dbg, dbias_up=dbu, H=empty(0, 40))
    assert (dWg[:, :24] == 0).all() and (dWg[:, 24:] == 5).all() and (dWu == 0).all() and (dbg == 0).all() and (dbu == 0).all()


@pytest.mark.parametrize("act", ACTS)
def test_gated_gradients_against_differences(act):
    """Directional differences of f = sum(G * act(X Wg^T + bg) * (X Wu^T + bu)) in fp64 against the gradients (Z and U as the
    forward call kept them).  The kernel's error: half a unit of the kept Z and U (2^-8 of each) moves dZ by |G| (|U| 1.2 |dZ| +
    1.2 |dU|) and dU by 1.2 |G| |dZ|; 2^-8 for the roundings of dZ and dU, 2^-8 for the result."""
    g = torch.Generator(device=DEV).manual_seed(11)
    m, n, k = 33, 70, 48
    X, Wg, Wu, bg, bu = matrix(m, k, g), matrix(n, k, g, scale=0.3), matrix(n, k, g, scale=0.3), vector(n, g), vector(n, g)
    G, H, Z, U = (matrix(m, n, g) for _ in range(4))
    run_gated(X, Wg, Wu, H, bias_gate=bg, bias_up=bu, act=act, Z=Z, U=U)
    if act == "relu":
        G = torch.where(Z.abs() < 0.05, torch.zeros_like(G), G)
    out = dict(dX=empty(m, k), dW_gate=empty(n, k), dW_up=empty(n, k), dbias_gate=empty(n), dbias_up=empty(n))
    run_back(G, X, Wg, Wu, Z, U, act=act, **out)
    base = dict(dX=X.double(), dW_gate=Wg.double(), dW_up=Wu.double(), dbias_gate=bg.double(), dbias_up=bu.double())
    f = lambda p: (G.double() * act64(p["dX"] @ p["dW_gate"].T + p["dbias_gate"], act) * (p["dX"] @ p["dW_up"].T + p["dbias_up"])).sum()  # noqa: E731
    gd, zd, ud, h = G.double().abs(), Z.double().abs(), U.double().abs(), 1e-5
    dz_err = gd * (1.2 * ud * 2.0 ** -8 + ud * 1.2 * 2.0 ** -8 * zd + 1.2 * 2.0 ** -8 * ud)
    du_err = gd * (2.0 ** -8 * (zd + 0.2) + 1.2 * 2.0 ** -8 * zd)
    for which, grad in out.items():
        d = torch.randn(base[which].shape, generator=g, device=DEV, dtype=torch.float64)
        diff = (f({**base, which: base[which] + h * d}) - f({**base, which: base[which] - h * d})) / (2 * h)
        if which == "dX":
            err = ((dz_err @ base["dW_gate"].abs() + du_err @ base["dW_up"].abs()) * d.abs()).sum()
        else:
            e = dz_err if which.endswith("gate") else du_err
            err = ((e.T @ X.double().abs() if which.startswith("dW") else e.sum(0)) * d.abs()).sum()
        err = err + 2.0 ** -8 * (grad.double().abs() * d.abs()).sum() + 1e-6 * (1 + diff.abs())
        assert (diff - (grad.double() * d).sum()).abs() <= err, which


def test_gated_refusals():
    g = torch.Generator(device=DEV).manual_seed(1)
    X, W, H = matrix(8, 16, g), matrix(24, 16, g), matrix(8, 24, g)
    call = lambda **k: api.mosaic_gated_linear(**{**dict(X=X, W_gate=W, W_up=W, H=H), **k})  # noqa: E731
    for wrong, error in ((dict(X=X.float()), TypeError), (dict(W_up=None), TypeError), (dict(H=None), TypeError), (dict(H=H[:, :23]), ValueError),
                         (dict(W_up=W[:23]), ValueError), (dict(W_gate=matrix(24, 8, g)), ValueError), (dict(act="tanh"), ValueError),
                         (dict(Z=H.float()), TypeError), (dict(bias_up=empty(23)), ValueError), (dict(X=X.cpu()), TypeError),
                         (dict(Z=api.Checkpoint.empty(8, 24)), ValueError), (dict(Z=api.Checkpoint.empty(8, 23), U=api.Checkpoint.empty(8, 24)), ValueError)):
        with pytest.raises(error):
            call(**wrong)
    with pytest.raises(api.MosaicError) as e:
        call(Z=H)
    assert e.value.status == -6
    with pytest.raises(api.MosaicError) as e:
        call(act=9)
    assert e.value.status == -1
    back = lambda **k: api.mosaic_gated_linear_backward(**{**dict(dH=H, X=X, W_gate=W, W_up=W, Z=H, U=H), **k})  # noqa: E731
    for wrong in (dict(Z=None), dict(X=None, dW_up=empty(24, 16)), dict(W_up=None, dX=empty(8, 16)), dict(dX=empty(8, 15)),
                  dict(X=api.Checkpoint.empty(8, 15)), dict(U=api.Checkpoint.empty(8, 24))):
        with pytest.raises(ValueError):
            back(**wrong)
    with pytest.raises(TypeError):
        back(X=None, W_gate=None, W_up=None)
    with pytest.raises(api.MosaicError) as e:
        back(dX=X, dW_up=empty(24, 16))
    assert e.value.status == -6
    back()   # nothing wanted: nothing done
