"""CPU-only checks of the gated and 8-bit calls: arguments are refused before any device call, workspaces are sized from the
arguments."""
import ctypes as C

import pytest

from paper_2504_06323_b200 import api, build

INVALID, NULL, DTYPE, MISALIGNED, WS, ALIAS = -1, -2, -3, -4, -5, -6
A = 1 << 20   # addresses that are never touched: every call here is refused first


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return api.lib()


class Saved(api._CheckpointStruct):
    alive = []   # the library reads the struct during the call

    @property
    def at(self):
        Saved.alive.append(self)
        return C.addressof(self)


def saved(base, ldc=32, lde=2, exponents=None):
    return Saved(base, ldc, base + A // 2 if exponents is None else exponents, lde)


def gated(lib, **k):
    g = k.get
    return lib.mosaic_gated_linear(g("X", A), g("ldx", 64), g("Wg", 2 * A), g("ldwg", 64), g("Wu", 3 * A), g("ldwu", 64), g("m", 8), g("n", 32), g("k", 64),
                                   g("dtype", api.BF16), g("bg"), g("bu"), g("act", 3), g("H", 4 * A), g("ldh", 32), g("Z"), g("ldz", 32), g("U"), g("ldu", 32),
                                   g("z8"), g("u8"), g("status"), g("ws"), g("ws_bytes", 0), None)


def test_gated_refusals_need_no_device(lib):
    assert gated(lib, dtype=api.F32) == DTYPE
    assert gated(lib, m=-1) == INVALID and gated(lib, n=0) == INVALID and gated(lib, k=0) == INVALID and gated(lib, act=4) == INVALID
    assert gated(lib, ldx=63) == INVALID and gated(lib, ldwg=63) == INVALID and gated(lib, ldwu=63) == INVALID and gated(lib, ldh=31) == INVALID
    assert gated(lib, Z=5 * A, ldz=31) == INVALID and gated(lib, U=5 * A, ldu=31) == INVALID
    assert gated(lib, X=None) == NULL and gated(lib, Wg=None) == NULL and gated(lib, Wu=None) == NULL and gated(lib, H=None) == NULL
    assert gated(lib, Wu=3 * A + 1) == MISALIGNED and gated(lib, bu=A + 1) == MISALIGNED and gated(lib, status=A + 2) == MISALIGNED
    for out in ("H", "Z", "U"):
        for at in (A, 2 * A, 3 * A):
            assert gated(lib, **{out: at}) == ALIAS
    assert gated(lib, Z=4 * A) == ALIAS and gated(lib, U=4 * A) == ALIAS and gated(lib, Z=5 * A, U=5 * A) == ALIAS and gated(lib, bg=4 * A) == ALIAS
    assert gated(lib, X=A + 2) == NULL and gated(lib, Wu=3 * A + 2, ws=8 * A, ws_bytes=100) == WS and gated(lib, X=A + 2, ws=8 * A + 64, ws_bytes=1 << 20) == MISALIGNED


def test_gated_checkpoints_are_checked(lib):
    z, u = saved(5 * A), saved(6 * A)
    assert gated(lib, z8=z.at) == INVALID and gated(lib, u8=u.at) == INVALID and gated(lib, z8=z.at, u8=u.at, Z=7 * A) == INVALID
    assert gated(lib, z8=saved(5 * A, ldc=16).at, u8=u.at) == INVALID and gated(lib, z8=z.at, u8=saved(6 * A, lde=1).at) == INVALID
    assert gated(lib, z8=saved(5 * A + 8).at, u8=u.at) == MISALIGNED and gated(lib, z8=saved(5 * A, ldc=40).at, u8=u.at) == MISALIGNED
    assert gated(lib, z8=Saved(None, 32, 5 * A, 2).at, u8=u.at) == NULL
    assert gated(lib, z8=z.at, u8=z.at) == ALIAS and gated(lib, z8=saved(4 * A).at, u8=u.at) == ALIAS and gated(lib, z8=saved(5 * A, exponents=A).at, u8=u.at) == ALIAS


def test_gated_workspaces(lib):
    q = lib.mosaic_gated_linear_workspace_bytes
    assert q(A, 64, 2 * A, 64, 3 * A, 64, 8, 32, 64, 0) == 0
    assert q(A + 2, 64, 2 * A, 64, 3 * A, 64, 8, 32, 64, 0) == 8 * 64 * 2
    assert q(A, 63, 2 * A, 63, 3 * A, 63, 8, 32, 63, 0) == 8 * 64 * 2 + 2 * 32 * 64 * 2
    assert q(A, 63, 2 * A, 63, 3 * A, 63, 4, 32, 63, 0) == 0               # few tokens are read as they are
    assert q(A, 64, 2 * A, 64, 3 * A, 64, 8, 32, 64, 1) == 0               # checkpoints are written by the product itself,
    assert q(A, 64, 2 * A, 64, 3 * A, 64, 2, 32, 64, 1) == 2 * 256         # but of few tokens
    b = lib.mosaic_gated_linear_backward_workspace_bytes
    assert b(A, 64, 0, 2 * A, 64, 3 * A, 64, 8, 32, 64, 1, 1, 0) == 2 * 8 * 32 * 2          # dZ and dU
    assert b(A, 64, 0, 2 * A, 64, 3 * A, 64, 8, 32, 64, 0, 0, 1) == 2 * 256                  # column sums
    assert b(None, 64, 1, 2 * A, 64, 3 * A, 64, 8, 32, 64, 0, 1, 0) == 2 * 8 * 32 * 2 + 8 * 64 * 2   # X, loaded
    assert b(A, 63, 0, 2 * A, 63, 3 * A, 63, 8, 32, 63, 1, 0, 0) == 2 * 8 * 32 * 2 + 2 * 32 * 64 * 2


def back(lib, **k):
    g = k.get
    return lib.mosaic_gated_linear_backward(g("dH", A), g("lddh", 32), g("X", 2 * A), g("ldx", 64), g("x8"), g("Wg", 3 * A), g("ldwg", 64), g("Wu", 4 * A), g("ldwu", 64),
                                            g("Z", 5 * A), g("ldz", 32), g("U", 6 * A), g("ldu", 32), g("z8"), g("u8"), g("m", 8), g("n", 32), g("k", 64),
                                            g("dtype", api.BF16), g("act", 3), g("dX", 7 * A), g("lddx", 64), g("dWg", 8 * A), g("lddwg", 64), g("dWu", 9 * A), g("lddwu", 64),
                                            g("dbg"), g("dbu"), g("H"), g("ldh", 32), g("status"), g("ws"), g("ws_bytes", 0), None)


def test_gated_backward_refusals_need_no_device(lib):
    assert back(lib, dtype=api.F32) == DTYPE and back(lib, n=0) == INVALID and back(lib, act=9) == INVALID and back(lib, lddx=63) == INVALID and back(lib, lddwu=63) == INVALID
    for name in ("dH", "X", "Wg", "Wu", "Z", "U"):
        assert back(lib, **{name: None}) == NULL
    assert back(lib, H=11 * A, ldh=31) == INVALID and back(lib, dbu=11 * A + 1) == MISALIGNED
    z, u, x = saved(11 * A), saved(12 * A), saved(13 * A, ldc=64, lde=4)
    assert back(lib, z8=z.at, u8=u.at) == INVALID and back(lib, Z=None, U=None, z8=z.at) == INVALID and back(lib, x8=x.at) == INVALID
    assert back(lib, X=None, x8=saved(13 * A, ldc=48, lde=4).at) == INVALID and back(lib, X=None, x8=saved(13 * A + 4, ldc=64, lde=4).at) == MISALIGNED
    for out in ("dX", "dWg", "dWu", "dbg", "dbu", "H"):
        for at in (A, 2 * A, 3 * A, 4 * A, 5 * A, 6 * A):
            assert back(lib, **{out: at}) == ALIAS
    assert back(lib, dWg=9 * A) == ALIAS and back(lib, H=7 * A) == ALIAS
    assert back(lib, Z=None, U=None, z8=z.at, u8=u.at, H=12 * A) == ALIAS and back(lib, X=None, x8=x.at, dX=13 * A) == ALIAS
    assert back(lib) == NULL and back(lib, ws=16 * A, ws_bytes=1000) == WS and back(lib, ws=16 * A + 16, ws_bytes=1 << 20) == MISALIGNED


def test_checkpoint_refusals_need_no_device(lib):
    for call in (lambda **k: lib.mosaic_checkpoint_store(k.get("X", A), k.get("rows", 4), k.get("cols", 20), k.get("ld", 20), k.get("dtype", 1), k.get("c", saved(2 * A).at), None),
                 lambda **k: lib.mosaic_checkpoint_load(k.get("c", saved(2 * A).at), k.get("rows", 4), k.get("cols", 20), k.get("X", A), k.get("ld", 20), k.get("dtype", 1), None)):
        assert call(dtype=0) == DTYPE and call(rows=-1) == INVALID and call(cols=0) == INVALID and call(ld=19) == INVALID
        assert call(X=None) == NULL and call(c=None) == NULL and call(c=Saved(2 * A, 32, None, 2).at) == NULL
        assert call(X=A + 1) == MISALIGNED and call(c=saved(2 * A + 1).at) == MISALIGNED and call(c=saved(2 * A, lde=1).at) == INVALID
        assert call(X=2 * A) == ALIAS and call(c=saved(2 * A, exponents=2 * A + 16).at) == ALIAS
        assert call(rows=0, X=None, c=Saved(None, 32, None, 2).at) == 0


def test_binding_refuses_cpu_tensors(lib):
    import torch
    x = torch.zeros(4, 16, dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        api.mosaic_gated_linear(x, x, x, x)
    with pytest.raises(TypeError):
        api.mosaic_gated_linear_backward(x, x, x, x, x, x)
    with pytest.raises(TypeError):
        api.Checkpoint.empty(4, 16, "cpu")


class W4(api._Weight4Struct):
    alive = []

    @property
    def at(self):
        W4.alive.append(self)
        return C.addressof(self)


def w4(codes=2 * A, ldc=32, scales=3 * A, lds=2, group=32):
    return W4(codes, ldc, scales, lds, group).at


def linear4(lib, **k):
    g = k.get
    return lib.mosaic_linear4(g("X", A), g("ldx", 64), g("W", w4()), g("m", 8), g("n", 32), g("k", 64), g("dtype", api.BF16), g("bias"), g("R"), g("ldr", 32),
                              g("act", 0), g("Y", 4 * A), g("ldy", 32), g("status"), g("ws"), g("ws_bytes", 0), None)


def gated4(lib, **k):
    g = k.get
    return lib.mosaic_gated_linear4(g("X", A), g("ldx", 64), g("W", w4()), g("W2", w4(5 * A, scales=6 * A)), g("m", 8), g("n", 32), g("k", 64), g("dtype", api.BF16),
                                    g("bias"), g("bu"), g("act", 3), g("Y", 4 * A), g("ldy", 32), g("status"), g("ws"), g("ws_bytes", 0), None)


@pytest.mark.parametrize("call", [linear4, gated4])
def test_products4_refusals_need_no_device(lib, call):
    assert call(lib, dtype=api.F32) == DTYPE and call(lib, n=0) == INVALID and call(lib, act=5) == INVALID and call(lib, ldx=63) == INVALID and call(lib, ldy=31) == INVALID
    assert call(lib, X=None) == NULL and call(lib, Y=None) == NULL and call(lib, W=None) == NULL
    assert call(lib, W=w4(codes=None)) == NULL and call(lib, W=w4(scales=None)) == NULL
    assert call(lib, W=w4(group=16)) == INVALID and call(lib, W=w4(group=96)) == INVALID and call(lib, W=w4(ldc=16)) == INVALID and call(lib, W=w4(lds=1)) == INVALID
    assert call(lib, W=w4(codes=2 * A + 8)) == MISALIGNED and call(lib, W=w4(ldc=40)) == MISALIGNED and call(lib, W=w4(scales=3 * A + 1)) == MISALIGNED
    assert call(lib, status=A + 2) == MISALIGNED and call(lib, Y=A) == ALIAS and call(lib, Y=2 * A) == ALIAS and call(lib, Y=3 * A) == ALIAS and call(lib, bias=4 * A) == ALIAS
    assert call(lib, X=A + 2) == NULL and call(lib, X=A + 2, ws=8 * A, ws_bytes=100) == WS and call(lib, X=A + 2, ws=8 * A + 8, ws_bytes=1 << 20) == MISALIGNED
    assert call(lib, m=api.FEW4_TOKENS + 1) == NULL and call(lib, m=api.FEW4_TOKENS + 1, ws=8 * A, ws_bytes=32 * 64 * 2 - 1) == WS   # many tokens: the weights in bf16
    if call is linear4:
        assert call(lib, R=4 * A, ldr=40) == ALIAS and call(lib, R=4 * A + 32) == ALIAS
    else:
        assert call(lib, W2=None) == NULL and call(lib, Y=5 * A) == ALIAS and call(lib, bu=4 * A) == ALIAS and call(lib, W2=w4(group=3)) == INVALID


def test_products4_workspaces(lib):
    q, g = lib.mosaic_linear4_workspace_bytes, lib.mosaic_gated_linear4_workspace_bytes
    assert q(A, 64, 1, 32, 64) == 0 and g(A, 64, 1, 32, 64) == 0
    assert q(A, 64, api.FEW4_TOKENS, 32, 64) == 0 and q(A, 64, api.FEW4_TOKENS + 1, 32, 64) == 32 * 64 * 2 and g(A, 64, api.FEW4_TOKENS + 1, 32, 64) == 2 * 32 * 64 * 2
    assert q(A + 2, 64, 8, 32, 64) == 8 * 64 * 2 and q(A, 63, 8, 32, 63) == 8 * 64 * 2 and q(A, 63, 1, 32, 63) == 0


def test_packing_refusals_need_no_device(lib):
    for call in (lambda **k: lib.mosaic_quantize4(k.get("W", A), k.get("rows", 4), k.get("cols", 40), k.get("ld", 40), k.get("dtype", 1), k.get("c", w4()), None),
                 lambda **k: lib.mosaic_dequantize4(k.get("c", w4()), k.get("rows", 4), k.get("cols", 40), k.get("W", A), k.get("ld", 40), k.get("dtype", 1), None)):
        assert call(dtype=0) == DTYPE and call(rows=-1) == INVALID and call(cols=0) == INVALID and call(ld=39) == INVALID
        assert call(W=None) == NULL and call(c=None) == NULL and call(c=w4(scales=None)) == NULL
        assert call(W=A + 1) == MISALIGNED and call(c=w4(codes=2 * A + 4)) == MISALIGNED and call(c=w4(ldc=16)) == INVALID and call(c=w4(group=0)) == INVALID
        assert call(W=2 * A) == ALIAS and call(W=3 * A) == ALIAS and call(c=w4(scales=2 * A + 16)) == ALIAS
        assert call(rows=0, W=None, c=w4(None, 32, None)) == 0
