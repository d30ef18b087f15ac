"""Calls in a row on one stream: every launch of a chain may start while the one before it runs, and reads what that one
writes.  A chain issued at once has the bits of the same chain with the device idle between its calls, over contents
that change from round to round (so that what an earlier round left in memory is wrong)."""
import pytest
import torch

from paper_2504_06323_b200 import api

pytestmark = pytest.mark.gpu
DEV = "cuda"


def chain(steps, idle):
    for f in steps:
        f()
        if idle:
            torch.cuda.synchronize()
    torch.cuda.synchronize()


@pytest.mark.parametrize("tokens", [1, 2, 4, 37, 300])
@pytest.mark.parametrize("hidden,width", [(512, 1024), (333, 777)])     # rows on 16-byte boundaries, and dense odd ones
def test_products_read_what_the_call_before_them_wrote(tokens, hidden, width):
    g = torch.Generator(device=DEV).manual_seed(tokens + width)
    r = lambda *s, scale=1.0: (torch.randn(*s, generator=g, device=DEV) * scale).to(torch.bfloat16)  # noqa: E731
    W = [(r(width, hidden, scale=hidden ** -0.5), r(hidden, width, scale=width ** -0.5)) for _ in range(3)]
    ws = api.Workspace(DEV)
    for _ in range(6):
        X, dY = r(tokens, hidden), r(tokens, hidden)
        results = []
        for idle in (True, False):
            e = lambda *s: torch.zeros(*s, device=DEV, dtype=torch.bfloat16)  # noqa: E731
            a, dX = X.clone(), e(tokens, hidden)
            out, steps = [a, dX], []
            for up, down in W:
                H, Z, dH, dup, ddown, db = e(tokens, width), e(tokens, width), e(tokens, width), e(width, hidden), e(hidden, width), e(width)
                out += [H, Z, dH, dup, ddown, db]
                steps += [lambda up=up, H=H, Z=Z: api.mosaic_linear(a, up, H, act="silu", Z=Z, ws=ws),
                          lambda down=down, H=H: api.mosaic_linear(H, down, a, residual=a, ws=ws),
                          lambda down=down, H=H, dH=dH, ddown=ddown: api.mosaic_linear_backward(dY, H, down, dX=dH, dW=ddown, ws=ws),
                          lambda up=up, Z=Z, dH=dH, dup=dup, db=db: api.mosaic_linear_backward(dH, a, up, Z=Z, act="silu", dX=dX, dW=dup,
                                                                                             dbias=db, ws=ws)]
            chain(steps, idle)
            results.append(out)
        assert all(torch.equal(p, q) for p, q in zip(*results))


def test_training_step_reads_what_the_calls_before_it_wrote():
    g = torch.Generator(device=DEV).manual_seed(3)
    r = lambda *s, scale=1.0: (torch.randn(*s, generator=g, device=DEV) * scale).to(torch.bfloat16)  # noqa: E731
    head, tokens, vocab, top = r(5003, 256, scale=1 / 16), 700, 5003, 24
    ws = api.Workspace(DEV)
    for _ in range(6):
        X, T = r(tokens, 256), r(tokens, 256)
        results = []
        for idle in (True, False):
            f = lambda *s, dtype=torch.float32: torch.zeros(*s, device=DEV, dtype=dtype)  # noqa: E731
            L, S, v, i, lse, loss = r(tokens, vocab), r(tokens, vocab), f(tokens, top), f(tokens, top, dtype=torch.int32), f(tokens), f(tokens)
            dX, dW = f(tokens, 256, dtype=torch.bfloat16), f(vocab, 256, dtype=torch.bfloat16)
            chain([lambda: api.mosaic_linear(T, head, L, ws=ws), lambda: api.mosaic_top_logits(L, v, i, lse, ws=ws),
                   lambda: api.mosaic_linear(X, head, S, ws=ws),
                   lambda: api.mosaic_distill_loss_grad(S, v, i, loss, None, S, t_lse=lse, ws=ws),
                   lambda: api.mosaic_linear_backward(S, X, head, dX=dX, dW=dW, ws=ws)], idle)
            results.append([L, S, v, i, lse, loss, dX, dW])
        assert all(torch.equal(p, q) for p, q in zip(*results))
