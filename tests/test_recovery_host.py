"""CPU-only checks of the recovery calls (linear, top logits, distillation): arguments are refused before any
device call, in the order null / type / sizes / alignment / overlap, and workspaces are sized from the arguments."""
import pytest

from paper_2504_06323_b200 import api, build

INVALID, NULL, DTYPE, MISALIGNED, WS, ALIAS = -1, -2, -3, -4, -5, -6
A = 1 << 20   # addresses that are never touched: every call here is refused first


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return api.lib()


def linear(lib, **k):
    g = k.get
    return lib.mosaic_linear(g("X", A), g("ldx", 64), g("W", 2 * A), g("ldw", 64), g("m", 8), g("n", 32), g("k", 64), g("dtype", api.BF16),
                             g("bias"), g("R"), g("ldr", 32), g("act", 0), g("Y", 4 * A), g("ldy", 32), g("Z"), g("ldz", 32), g("status"),
                             g("ws"), g("ws_bytes", 0), None)


def test_linear_refusals_need_no_device(lib):
    assert linear(lib, dtype=api.F32) == DTYPE and linear(lib, dtype=7) == DTYPE
    assert linear(lib, m=-1) == INVALID and linear(lib, n=0) == INVALID and linear(lib, k=0) == INVALID and linear(lib, m=1 << 31) == INVALID
    assert linear(lib, act=4) == INVALID and linear(lib, act=-1) == INVALID
    assert linear(lib, ldx=63) == INVALID and linear(lib, ldw=63) == INVALID and linear(lib, ldy=31) == INVALID
    assert linear(lib, Z=8 * A, ldz=31) == INVALID and linear(lib, R=8 * A, ldr=31) == INVALID
    assert linear(lib, X=None) == NULL and linear(lib, W=None) == NULL and linear(lib, Y=None) == NULL
    assert linear(lib, X=A + 1) == MISALIGNED and linear(lib, bias=A + 1) == MISALIGNED and linear(lib, status=A + 2) == MISALIGNED
    assert linear(lib, Y=A + 64) == ALIAS and linear(lib, Y=2 * A) == ALIAS and linear(lib, Z=4 * A) == ALIAS
    assert linear(lib, R=4 * A + 64) == ALIAS and linear(lib, R=4 * A, ldr=40) == ALIAS and linear(lib, bias=4 * A) == ALIAS
    assert linear(lib, X=A + 2) == NULL                                    # an odd base needs scratch
    assert linear(lib, X=A + 2, ws=8 * A, ws_bytes=100) == WS and linear(lib, X=A + 2, ws=8 * A + 64, ws_bytes=1 << 20) == MISALIGNED


def test_linear_workspaces(lib):
    q = lib.mosaic_linear_workspace_bytes
    assert q(A, 64, 2 * A, 64, 8, 32, 64) == 0
    assert q(A + 2, 64, 2 * A, 64, 8, 32, 64) == 8 * 64 * 2                # X copied
    assert q(A, 63, 2 * A, 63, 8, 32, 63) == 8 * 64 * 2 + 32 * 64 * 2      # both, rows padded to 64
    assert q(A, 63, 2 * A, 64, 1, 32, 63) == 0                             # one row has no leading dimension to speak of
    b = lib.mosaic_linear_backward_workspace_bytes
    args = (A, 32, 2 * A, 64, 4 * A, 64, 8, 32, 64)
    assert b(*args, api.ACT_NONE, 1, 1, 0) == 0
    assert b(*args, api.ACT_SILU, 1, 1, 0) == 8 * 32 * 2                   # dZ
    assert b(*args, api.ACT_SILU, 0, 0, 1) == 256                          # column sums alone: one band of 32 fp32, rounded up
    assert b(A + 2, 32, 2 * A, 64, 4 * A, 64, 8, 32, 64, api.ACT_NONE, 1, 1, 0) == 8 * 32 * 2


def backward(lib, **k):
    g = k.get
    return lib.mosaic_linear_backward(g("dY", A), g("lddy", 32), g("X", 2 * A), g("ldx", 64), g("W", 3 * A), g("ldw", 64), g("Z"), g("ldz", 32),
                                      g("m", 8), g("n", 32), g("k", 64), g("dtype", api.BF16), g("act", 0), g("dX", 4 * A), g("lddx", 64),
                                      g("dW", 5 * A), g("lddw", 64), g("db"), g("status"), g("ws"), g("ws_bytes", 0), None)


def test_backward_refusals_need_no_device(lib):
    assert backward(lib, dtype=api.F32) == DTYPE
    assert backward(lib, n=0) == INVALID and backward(lib, act=9) == INVALID and backward(lib, lddx=63) == INVALID
    assert backward(lib, dY=None) == NULL and backward(lib, X=None) == NULL and backward(lib, W=None) == NULL
    assert backward(lib, act=api.ACT_RELU) == NULL                         # no stored Z
    assert backward(lib, dX=3 * A) == ALIAS and backward(lib, dW=2 * A) == ALIAS and backward(lib, dW=4 * A) == ALIAS and backward(lib, db=A) == ALIAS
    assert backward(lib, db=6 * A) == NULL                                 # the column sums need scratch
    assert backward(lib, db=6 * A, ws=7 * A, ws_bytes=64) == WS


def top(lib, **k):
    g = k.get
    return lib.mosaic_top_logits(g("L", A), g("rows", 4), g("vocab", 100), g("ld", 100), g("dtype", api.F32), g("top", 10), g("T", 1.0),
                                 g("values", 2 * A), g("indices", 3 * A), g("lse"), g("ws", 8 * A), g("ws_bytes", 1 << 16), None)


def test_top_logits_refusals_need_no_device(lib):
    assert top(lib, dtype=2) == DTYPE
    assert top(lib, rows=-1) == INVALID and top(lib, vocab=0) == INVALID and top(lib, ld=99) == INVALID and top(lib, top=0) == INVALID
    assert top(lib, top=101) == INVALID and top(lib, vocab=5000, ld=5000, top=1025) == INVALID and top(lib, vocab=1 << 31, ld=1 << 31) == INVALID
    assert top(lib, T=0.0) == INVALID and top(lib, T=float("inf")) == INVALID and top(lib, T=1e-40) == INVALID
    assert top(lib, L=None) == NULL and top(lib, values=None) == NULL and top(lib, indices=None) == NULL
    assert top(lib, L=A + 2) == MISALIGNED and top(lib, values=A + 2) == MISALIGNED and top(lib, lse=A + 1) == MISALIGNED
    assert top(lib, values=A) == ALIAS and top(lib, indices=2 * A) == ALIAS and top(lib, lse=3 * A) == ALIAS
    assert top(lib, rows=0, L=None) == 0 and top(lib, vocab=(1 << 20) + 1, ld=1 << 21) == INVALID
    assert top(lib, ws=None) == NULL and top(lib, ws=8 * A + 16) == MISALIGNED and top(lib, rows=100, ws_bytes=64) == WS
    q = lib.mosaic_top_logits_workspace_bytes
    assert q(0, 100, 0, 10) == 0 and q(4, (1 << 20) + 1, 0, 10) == 0 and q(4, 100, 0, 10) == 512
    assert q(4096, 32000, 1, 64) >= 4096 * (500 * 2 + 8)


def test_distill_workspace(lib):
    q = lib.mosaic_distill_workspace_bytes
    assert q(4, 10) == 512 and q(1000, 64) == (1000 * (32 + 512) + 255) // 256 * 256 and q(0, 10) == 0


def distill(lib, which, **k):
    g = k.get
    head = (g("S", A), g("rows", 4), g("vocab", 100), g("ld", 100), g("dtype", api.F32), g("tv", 2 * A), g("ti", 3 * A), g("top", 10), g("t_lse"),
            g("weight"), g("T", 1.0))
    if which == "loss":
        return lib.mosaic_distill_loss(*head, g("loss", 4 * A), g("lse", 5 * A), g("ws", 8 * A), g("ws_bytes", 1 << 16), None)
    if which == "grad":
        return lib.mosaic_distill_grad(*head, g("lse", 5 * A), g("gr"), 1.0, g("dS", 6 * A), g("ldd", 100), g("ws", 8 * A), g("ws_bytes", 1 << 16), None)
    return lib.mosaic_distill_loss_grad(*head, g("loss", 4 * A), g("lse", 5 * A), g("gr"), 1.0, g("dS", 6 * A), g("ldd", 100), g("ws", 8 * A), g("ws_bytes", 1 << 16), None)


@pytest.mark.parametrize("which", ["loss", "grad", "both"])
def test_distill_refusals_need_no_device(lib, which):
    call = lambda **k: distill(lib, which, **k)  # noqa: E731
    assert call(dtype=3) == DTYPE
    assert call(vocab=0) == INVALID and call(ld=99) == INVALID and call(top=0) == INVALID and call(top=1025) == INVALID and call(T=-2.0) == INVALID
    assert call(S=None) == NULL and call(tv=None) == NULL and call(ti=None) == NULL
    assert call(S=A + 2) == MISALIGNED and call(tv=A + 1) == MISALIGNED and call(weight=A + 2) == MISALIGNED
    assert call(rows=0, S=None) == 0
    assert call(ws=None) == NULL and call(ws=8 * A + 64) == MISALIGNED and call(ws_bytes=128) == WS
    if which != "grad":
        assert call(loss=None) == NULL and call(loss=2 * A) == ALIAS and call(lse=4 * A) == ALIAS
    if which != "loss":
        assert call(dS=None) == NULL and call(ldd=99) == INVALID and call(dS=A + 4) == ALIAS and call(dS=A, ldd=101) == ALIAS and call(dS=2 * A) == ALIAS
    if which == "grad":
        assert call(lse=None) == NULL and call(lse=6 * A) == ALIAS


def test_binding_refuses_cpu_tensors_and_unknown_activations(lib):
    import torch
    x = torch.zeros(4, 8, dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        api.mosaic_linear(x, x, x)
    with pytest.raises(TypeError):
        api.mosaic_linear_backward(x, x, x)
    with pytest.raises(TypeError):
        api.mosaic_top_logits(x, x, x)
    with pytest.raises(TypeError):
        api.mosaic_distill_loss(x, x, x, x)
    with pytest.raises(ValueError):
        api._act_code("tanh")
    assert [api._act_code(a) for a in ("none", "relu", "gelu", "silu", api.ACT_SILU)] == [0, 1, 2, 3, 3]
