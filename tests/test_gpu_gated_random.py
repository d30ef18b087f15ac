"""The gated, 8-bit and 4-bit calls one after another at random: sizes, pitches, offsets, activations, formats and which outputs are
wanted.  Each against the formula in fp64 on the host (bounds of test_gpu_linear.py and test_gpu_gated.py); nothing is written
outside an output."""
import math
import random

import pytest
import torch

from paper_2504_06323_b200 import api
from test_gpu_checkpoint import reference
from test_gpu_gated import check_gated, check_gated_backward, vector
from test_gpu_linear import ACTS, check_forward

pytestmark = pytest.mark.gpu
DEV, BF16 = "cuda", torch.bfloat16


class Calls:
    def __init__(self, seed):
        self.rng, self.g, self.outs = random.Random(seed), torch.Generator(device=DEV).manual_seed(seed), []

    def size(self, lo, hi):
        return max(lo, min(hi, round(math.exp(self.rng.uniform(math.log(lo), math.log(hi))))))

    def matrix(self, rows, cols, scale=1.0, out=False):
        ld, offset = cols + self.rng.choice([0, 0, -cols % 8, -cols % 8, 1, 3, 8, 5]), self.rng.choice([0, 0, 0, 1, 2, 3, 4, 8])
        buf = torch.full((rows * ld + offset + 8,), float("nan"), device=DEV, dtype=BF16)
        m = buf[offset:offset + rows * ld].view(rows, ld)[:, :cols]
        if out:
            self.outs.append((m, buf))
        else:
            m.copy_(torch.randn(rows, cols, generator=self.g, device=DEV) * scale)
        return m

    def checkpoint(self, rows, cols):
        groups = -(-cols // 16) + self.rng.choice([0, 0, 1, 3])
        return api.Checkpoint(torch.full((rows, 16 * groups), 77, dtype=torch.int8, device=DEV), torch.full((rows, groups), 99, dtype=torch.uint8, device=DEV), cols)

    def stored(self, X):
        c, back = self.checkpoint(*X.shape), torch.empty(X.shape, device=DEV, dtype=BF16)
        api.mosaic_checkpoint_store(X, c)
        api.mosaic_checkpoint_load(c, back)
        return c, back

    def packed(self, rows, cols):
        group, more = self.rng.choice([32, 64, 128]), self.rng.choice([0, 0, 1, 2])
        w4 = api.Weight4(torch.full((rows, (-(-cols // 32) + more) * 16), 0xA5, dtype=torch.uint8, device=DEV),
                         torch.full((rows, -(-cols // group) + more), float("nan"), dtype=BF16, device=DEV), cols, group)
        api.mosaic_quantize4(self.matrix(rows, cols, cols ** -0.5), w4)
        back = torch.empty(rows, cols, device=DEV, dtype=BF16)
        api.mosaic_dequantize4(w4, back)
        return w4, back

    def nothing_outside(self):
        for m, buf in self.outs:
            outside = torch.ones_like(buf, dtype=torch.bool)
            outside.as_strided(m.shape, m.stride(), m.storage_offset()).fill_(False)
            assert torch.isnan(buf.cpu()[outside.cpu()]).all()
        self.outs.clear()


def host(*ts):
    return [t.cpu() if torch.is_tensor(t) else t for t in ts]


@pytest.mark.parametrize("seed", range(6))
def test_calls_at_random(seed):
    r = Calls(seed)
    rng, done = r.rng, 0
    while done < 60:
        op, m, n, k, act = rng.choice(["gated", "backward", "linear4", "gated4"]), r.size(1, 1500), r.size(1, 2500), r.size(1, 2500), rng.choice(ACTS)
        if op == "backward":   # its bound as a whole takes many independent roundings
            m, n = max(m, 32), max(n, 32)
        if m * n * k > 6e7:
            continue
        done += 1
        b1, b2 = (vector(n, r.g) if rng.random() < 0.4 else None for _ in range(2))
        status = torch.full((1,), 7, device=DEV, dtype=torch.int32)
        if op == "gated":
            X, Wg, Wu, H = r.matrix(m, k), r.matrix(n, k, k ** -0.5), r.matrix(n, k, k ** -0.5), r.matrix(m, n, out=True)
            Z, U = (r.matrix(m, n, out=True), r.matrix(m, n, out=True)) if rng.random() < 0.6 else (None, None)
            api.mosaic_gated_linear(X, Wg, Wu, H, bias_gate=b1, bias_up=b2, act=act, Z=Z, U=U, status=status)
            check_gated(*host(X, Wg, Wu, b1, b2, act, H, Z, U))
            if Z is not None:
                Z8, U8 = r.checkpoint(m, n), r.checkpoint(m, n)
                api.mosaic_gated_linear(X, Wg, Wu, H, bias_gate=b1, bias_up=b2, act=act, Z=Z8, U=U8, status=status)
                for c, t in ((Z8, Z), (U8, U)):
                    codes, E = reference(t)
                    assert torch.equal(c.codes[:, :codes.shape[1]].cpu(), codes) and torch.equal(c.exponents[:, :E.shape[1]].cpu(), E)
                    assert (c.codes[:, codes.shape[1]:] == 77).all() and (c.exponents[:, E.shape[1]:] == 99).all()
        elif op == "backward":
            X, Wg, Wu, dH, Z, U = r.matrix(m, k), r.matrix(n, k, 0.05), r.matrix(n, k, 0.05), r.matrix(m, n), r.matrix(m, n, 2.0), r.matrix(m, n)
            (Zc, Zr), (Uc, Ur) = (r.stored(Z), r.stored(U)) if rng.random() < 0.5 else ((Z, Z), (U, U))
            Xc, Xr = r.stored(X) if rng.random() < 0.5 else (X, X)
            want = [rng.random() < 0.7 for _ in range(6)]
            want[0] |= not any(want)
            dX, dWg, dWu, H = (r.matrix(*s, out=True) if w else None for s, w in zip(((m, k), (n, k), (n, k), (m, n)), want))
            dbg, dbu = (torch.empty(n, device=DEV, dtype=BF16) if w else None for w in want[4:])
            api.mosaic_gated_linear_backward(dH, Xc, Wg, Wu, Zc, Uc, act=act, dX=dX, dW_gate=dWg, dW_up=dWu, dbias_gate=dbg, dbias_up=dbu, H=H, status=status)
            check_gated_backward(*host(dH, Xr, Wg, Wu, Zr, Ur, act, dX, dWg, dWu, dbg, dbu, H))
        else:
            X, Y, (w4, W) = r.matrix(m, k), r.matrix(m, n, out=True), r.packed(n, k)
            if op == "linear4":
                R = r.matrix(m, n) if rng.random() < 0.5 else None
                api.mosaic_linear4(X, w4, Y, bias=b1, residual=R, act=act, status=status)
                check_forward(*host(X, W, b1, R, act, Y, None))
            else:
                u4, U = r.packed(n, k)
                api.mosaic_gated_linear4(X, w4, u4, Y, bias_gate=b1, bias_up=b2, act=act, status=status)
                check_gated(*host(X, W, U, b1, b2, act, Y, None, None))
        assert int(status.item()) == 0
        r.nothing_outside()
