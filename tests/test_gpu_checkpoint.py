"""Activations in 8 bits: codes and exponents bit for bit against the definition, and their use in the gated calls.

Storing rounds once, everything else is exact (powers of two), so stored codes and loaded values are compared for
equality; a loaded value is within half a code of what was stored.  The gated forward call's checkpoints are those of the
bf16 Z and U that it would have kept; the backward call's results are those of the loaded bf16 matrices.  Both to the bit."""
import pytest
import torch

from paper_2504_06323_b200 import api
from test_gpu_gated import SHAPES, empty, run_back, run_gated, vector
from test_gpu_linear import ACTS, matrix

pytestmark = pytest.mark.gpu
DEV = "cuda"


def reference(X):
    """(codes, exponents) from the definition, in fp64 on the host."""
    x = X.double().cpu()
    rows, cols = x.shape
    x = torch.nn.functional.pad(x, (0, -cols % 16)).view(rows, -1, 16)
    finite = torch.isfinite(x)
    largest = torch.where(finite, x.abs(), 0.0).amax(2)
    E = torch.where(largest > 0, torch.frexp(largest).exponent + 126, 0).clamp(min=1)   # a zero has the exponent 0
    code = torch.round(torch.where(finite, x, 0.0) * torch.pow(2.0, (133 - E).double())[..., None]).clamp(-127, 127)
    return torch.where(finite, code, -128.0).flatten(1).to(torch.int8), E.to(torch.uint8)


def values(codes, E, cols):
    v = codes.double().view(codes.shape[0], -1, 16) * torch.pow(2.0, E.double() - 133)[..., None]
    return torch.where(codes.view(v.shape) == -128, float("nan"), v).flatten(1)[:, :cols]


def same(a, b):
    return torch.equal(torch.nan_to_num(a.double().cpu(), nan=1e300), torch.nan_to_num(b.double().cpu(), nan=1e300))


def check_roundtrip(X, pitch=0, offset=0, width=0):
    rows, cols = X.shape
    groups = -(-cols // 16)
    codes = torch.full((rows, 16 * (groups + width)), 77, dtype=torch.int8, device=DEV)
    exponents = torch.full((rows, groups + width), 99, dtype=torch.uint8, device=DEV)
    c = api.Checkpoint(codes, exponents, cols)
    api.mosaic_checkpoint_store(X, c)
    want, E = reference(X)
    assert torch.equal(codes[:, :16 * groups].cpu(), want) and torch.equal(exponents[:, :groups].cpu(), E)
    assert (codes[:, 16 * groups:] == 77).all() and (exponents[:, groups:] == 99).all()
    buf = torch.full((rows * (cols + pitch) + offset + 8,), 3.0, device=DEV, dtype=torch.bfloat16)
    out = buf[offset:offset + rows * (cols + pitch)].view(rows, cols + pitch)
    api.mosaic_checkpoint_load(c, out[:, :cols])
    assert same(out[:, :cols], values(want, E, cols))
    assert (out[:, cols:] == 3).all() and (buf[:offset] == 3).all() and (buf[offset + rows * (cols + pitch):] == 3).all()
    finite = torch.isfinite(X).cpu()
    step = torch.pow(2.0, E.double() - 133).repeat_interleave(16, 1)[:, :cols]
    off = (values(want, E, cols) - X.double().cpu()).abs()
    assert (off[finite] <= 0.5 * step[finite]).all()


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 15), (1, 16), (1, 17), (2, 255), (3, 256), (4, 257), (5, 2047), (5, 2049), (37, 8807), (300, 96), (1001, 1000)])
@pytest.mark.parametrize("pitch,offset,width", [(0, 0, 0), (5, 3, 1), (8, 8, 0)])
def test_roundtrip(rows, cols, pitch, offset, width):
    g = torch.Generator(device=DEV).manual_seed(rows + cols)
    X = matrix(rows, cols, g, pitch, offset)
    X[:, :: 7] *= 50.0
    check_roundtrip(X, pitch, offset, width)


def test_every_bf16_number():
    """Each next to neighbours of all sizes: alone in its group, and below a larger one."""
    bits = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    X = torch.zeros(1 << 13, 128, dtype=torch.bfloat16)
    X[:, ::16] = bits.view(1 << 13, 8)
    X[::3, 1::16] = 1.0
    X[1::3, 2::16] = float("inf")
    X[2::3, 3::16] = 2.0 ** -120
    X[::5, 4::16] = -3.3895e38
    check_roundtrip(X.to(DEV))
    check_roundtrip(torch.randn(64, 200).mul(1e-39).to(torch.bfloat16).to(DEV))   # subnormal throughout


def test_groups_without_a_value_and_no_rows():
    X = torch.full((3, 40), float("nan"), device=DEV, dtype=torch.bfloat16)
    X[1] = 0.0
    X[2, 16:] = -float("inf")
    check_roundtrip(X)
    c = api.Checkpoint.empty(0, 40)
    api.mosaic_checkpoint_store(empty(0, 40), c)
    api.mosaic_checkpoint_load(c, empty(0, 40))


def loaded(c):
    out = empty(c.rows, c.cols)
    api.mosaic_checkpoint_load(c, out)
    return out


@pytest.mark.parametrize("m,n,k", SHAPES)
def test_gated_forward_keeps_8_bits(m, n, k):
    g = torch.Generator(device=DEV).manual_seed(m + n + k)
    act = ACTS[(m + n) % 4]
    X, Wg, Wu = matrix(m, k, g, -k % 8), matrix(n, k, g, -k % 8, scale=0.1), matrix(n, k, g, -k % 8, scale=0.1)
    b = vector(n, g)
    H, H8, Z, U = (empty(m, n) for _ in range(4))
    Z8, U8 = api.Checkpoint.empty(m, n), api.Checkpoint.empty(m, n)
    run_gated(X, Wg, Wu, H, bias_gate=b, act=act, Z=Z, U=U)
    run_gated(X, Wg, Wu, H8, bias_gate=b, act=act, Z=Z8, U=U8)
    assert torch.equal(H, H8)
    for c, t in ((Z8, Z), (U8, U)):
        codes, E = reference(t)
        assert torch.equal(c.codes.cpu(), codes) and torch.equal(c.exponents.cpu(), E)


@pytest.mark.parametrize("scale", [1.0, 3e-39, 1e37])
@pytest.mark.parametrize("m,n,k", [(2, 40, 64), (16, 100, 64), (128, 688, 256), (64, 513, 777), (300, 1000, 2048), (2304, 1153, 64)])
def test_gated_forward_keeps_what_is_not_finite_and_what_is_tiny(m, n, k, scale):
    """Infinities and NaN on the way, sums that leave bf16's range and sums of subnormals: what the 8 bits keep is what they would keep of
    the bf16 Z and U."""
    g = torch.Generator(device=DEV).manual_seed(m + n + k)
    X, Wg, Wu = matrix(m, k, g, -k % 8), matrix(n, k, g, -k % 8, scale=scale), matrix(n, k, g, -k % 8, scale=scale)
    X[0, 3], X[1, 5] = float("inf"), float("nan")
    Wg[n // 2, 7], Wu[n // 3, 9] = -float("inf"), float("nan")
    H, H8, Z, U = (empty(m, n) for _ in range(4))
    Z8, U8 = api.Checkpoint.empty(m, n), api.Checkpoint.empty(m, n)
    run_gated(X, Wg, Wu, H, act="none", Z=Z, U=U)
    run_gated(X, Wg, Wu, H8, act="none", Z=Z8, U=U8)
    assert same(H, H8)
    for c, t in ((Z8, Z), (U8, U)):
        codes, E = reference(t)
        assert torch.equal(c.codes.cpu(), codes) and torch.equal(c.exponents.cpu(), E)


@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (3, 130, 65), (17, 127, 63), (64, 513, 777), (129, 65, 129), (1000, 1025, 96), (2304, 1153, 64)])
@pytest.mark.parametrize("which", ["x", "zu", "xzu"])
def test_gated_backward_reads_8_bits(m, n, k, which):
    g = torch.Generator(device=DEV).manual_seed(m + n + k)
    act = ACTS[(m + k) % 4]
    X, Z, U, dH = matrix(m, k, g), matrix(m, n, g, scale=2.0), matrix(m, n, g), matrix(m, n, g)
    Wg, Wu = matrix(n, k, g, scale=0.05), matrix(n, k, g, scale=0.05)
    kept = []
    for t in (X, Z, U):
        c = api.Checkpoint.empty(*t.shape)
        api.mosaic_checkpoint_store(t, c)
        kept.append(c)
    out = lambda: dict(dX=empty(m, k), dW_gate=empty(n, k), dW_up=empty(n, k), dbias_gate=empty(n), dbias_up=empty(n), H=empty(m, n))  # noqa: E731
    a, b = out(), out()
    X8, Z8, U8 = (c if q in which else t for q, c, t in zip("xzu", kept, (X, Z, U)))
    run_back(dH, X8, Wg, Wu, Z8, U8, act=act, **a)
    back = lambda t: loaded(t) if isinstance(t, api.Checkpoint) else t  # noqa: E731
    run_back(dH, back(X8), Wg, Wu, back(Z8), back(U8), act=act, **b)
    for q in a:
        assert torch.equal(a[q], b[q]), q


@pytest.mark.parametrize("m,n,k", [(3, 130, 65), (129, 65, 129), (600, 1025, 96)])
def test_gated_backward_of_what_is_not_finite(m, n, k):
    """A NaN or infinity that 8 bits kept is a NaN in its token's gradients, and in the sums over tokens, as from the loaded matrices."""
    g = torch.Generator(device=DEV).manual_seed(m)
    X, Z, U, dH = matrix(m, k, g), matrix(m, n, g), matrix(m, n, g), matrix(m, n, g)
    X[0, 0], Z[1, 1], U[2, n - 1] = float("inf"), float("nan"), -float("inf")
    Wg, Wu = matrix(n, k, g, scale=0.05), matrix(n, k, g, scale=0.05)
    kept = []
    for t in (X, Z, U):
        c = api.Checkpoint.empty(*t.shape)
        api.mosaic_checkpoint_store(t, c)
        kept.append(c)
    out = lambda: dict(dX=empty(m, k), dW_gate=empty(n, k), dW_up=empty(n, k), dbias_gate=empty(n), dbias_up=empty(n), H=empty(m, n))  # noqa: E731
    a, b = out(), out()
    run_back(dH, kept[0], Wg, Wu, kept[1], kept[2], act="silu", **a)
    run_back(dH, loaded(kept[0]), Wg, Wu, loaded(kept[1]), loaded(kept[2]), act="silu", **b)
    for q in a:
        assert same(a[q], b[q]), q
    bad = torch.isnan(a["dX"]).all(1)
    assert bad[1] and bad[2] and not bad[0] and not bad[3:].any()
    assert torch.isnan(a["dW_gate"][:, 0]).all() and torch.isnan(a["dbias_gate"][1]) and torch.isnan(a["dbias_gate"][n - 1])


def test_refusals():
    X = matrix(4, 40, torch.Generator(device=DEV).manual_seed(0))
    good = api.Checkpoint.empty(4, 40)
    i8 = lambda *s: torch.empty(*s, dtype=torch.int8, device=DEV)  # noqa: E731
    u8 = lambda *s: torch.empty(*s, dtype=torch.uint8, device=DEV)  # noqa: E731
    for args, error in (((i8(4, 47), u8(4, 3), 40), ValueError), ((i8(4, 48), u8(4, 2), 40), ValueError), ((i8(4, 48), u8(3, 3), 40), ValueError),
                        ((u8(4, 48), u8(4, 3), 40), TypeError), ((i8(4, 48).cpu(), u8(4, 3), 40), TypeError), ((i8(48, 4).T, u8(4, 3), 40), ValueError),
                        ((i8(4, 48), u8(4, 3), 0), ValueError)):
        with pytest.raises(error):
            api.Checkpoint(*args)
    for call in (lambda: api.mosaic_checkpoint_store(X.float(), good), lambda: api.mosaic_checkpoint_load(good, X.float())):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: api.mosaic_checkpoint_store(X[:3], good), lambda: api.mosaic_checkpoint_load(good, X[:, :39])):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(api.MosaicError) as e:    # rows that are not on 16-byte boundaries
        api.mosaic_checkpoint_store(X, api.Checkpoint(i8(4, 56), u8(4, 3), 40))
    assert e.value.status == -4
    both = i8(4 * 80)
    with pytest.raises(api.MosaicError) as e:
        api.mosaic_checkpoint_store(both[:160].view(torch.bfloat16).view(2, 40), api.Checkpoint(both[96:192].view(2, 48), u8(2, 3), 40))
    assert e.value.status == -6
