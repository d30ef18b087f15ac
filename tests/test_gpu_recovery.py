"""The recovery path as a whole: a compacted block against its teacher, one step compared with the plain formulas in fp64.

Tolerances: every tensor that the path passes on (H, Y, logits, their gradients, the weights' gradients) is rounded to
bf16 once, an error of at most 2^-8 of it (rms below 2^-9).  The slopes of a token's loss in its logits, temperature
times a difference of probabilities, add up to at most 2 x temperature in magnitude: it moves by that times the largest
error of a logit, here |logit| times 2^-8 of its own rounding and the errors of H and Y behind it, each 2^-8 of a sum of
absolute products.  A gradient of the weights, in the 2-norm, passes through at most six such roundings (H, Y, logits,
their gradient, dY or dH with dZ, the result): 6 x 2^-8 of it in the worst case where they line up; the error of the
probabilities that the logits' errors cause (at most twice the largest such error over the temperature, relative)
comes on top.
"""
import pytest
import torch

from paper_2504_06323_b200 import driver, recovery, workloads as wl

pytestmark = pytest.mark.gpu
DEV = "cuda"


def block_pair(frac=0.3, vocab=500):
    cfg = wl.CONFIGS["tiny"]
    st = driver.alloc_model(cfg, torch.device(DEV, 0), layers=[0], outputs=False, masks=False)
    driver.accumulate_norms(st, 0, driver.make_activations(cfg, 0, DEV, 256))
    g = torch.Generator(device=DEV).manual_seed(5)
    head = (torch.randn(vocab, cfg.hidden, generator=g, device=DEV) * cfg.hidden ** -0.5).to(torch.bfloat16)
    student, teacher = recovery.compact_mlp(st, 0, frac, head)
    return student, teacher, g


def plain_loss(X, w, bias, targets, T):
    values, indices, lse = targets
    z = X @ w["up"].T + bias
    logits = (X + torch.nn.functional.silu(z) @ w["down"].T) @ w["head"].T
    logq = torch.log_softmax(logits / T, -1).gather(1, indices.long())
    logp = torch.log_softmax(values.double() / T, 1) if lse is None else values.double() / T - lse.double()[:, None]
    return logits, logp, logq


@pytest.mark.parametrize("tokens,renormalise", [(1, True), (37, False), (200, True), (200, False)])
def test_step_matches_plain_formulas(tokens, renormalise):
    student, teacher, g = block_pair()
    assert student.up.shape[0] == 482          # an even width whose rows are not on 16-byte boundaries: down is read through a copy
    X = torch.randn(tokens, 256, generator=g, device=DEV).to(torch.bfloat16)
    run = recovery.Recovery(student, teacher, top=40, temperature=2.0, renormalise=renormalise)
    targets = run.targets(X)
    loss, grads = run.gradients(X, targets)
    student.check()
    teacher.check()
    w = {k: getattr(student, k).double().requires_grad_() for k in ("up", "down", "head")}
    bias = student.bias.double().requires_grad_()
    logits, logp, logq = plain_loss(X.double(), w, bias, targets, 2.0)
    ref = 4.0 * (logp.exp() * (logp - logq)).sum(1)
    with torch.no_grad():
        h = torch.nn.functional.silu(X.double() @ w["up"].T)
        y_err = 2.0 ** -8 * (2 * h.abs() @ w["down"].abs().T + (X.double() + h @ w["down"].T).abs())
        err = float((y_err @ w["head"].abs().T + 2.0 ** -8 * logits.abs()).max())
        assert ((loss.double() - ref).abs() <= 2 * 2.0 * err + 1e-5).all()
    ref.mean().backward()
    for name, want in [(k, v.grad) for k, v in w.items()] + [("bias", bias.grad)]:
        got = grads[name].double()
        share = float((got - want).norm() / want.norm())
        assert share <= 6 * 2.0 ** -8 + 2 * err / 2.0, (name, share)


def test_loss_falls_and_evaluation_agrees():
    student, teacher, g = block_pair()
    X = torch.randn(256, 256, generator=g, device=DEV).to(torch.bfloat16)
    run = recovery.Recovery(student, teacher, top=32, rate=0.5)
    targets = run.targets(X)
    before = run.loss(X, targets)
    first = run.step(X, targets)
    assert torch.equal(before, first)          # the loss is the same with and without its gradient
    for _ in range(40):
        run.step(X, targets)
    after = run.loss(X, targets)
    assert float(after.mean()) < float(before.mean())
    student.check()


def test_command_runs():
    losses = recovery.main(["--steps", "12", "--tokens", "64", "--vocab", "300", "--top", "20"])
    assert losses[-1] < losses[0]


def test_blocks_that_do_not_fit_are_refused():
    student, teacher, _ = block_pair()
    with pytest.raises(ValueError):
        recovery.Block(student.up, teacher.down, student.head)
    with pytest.raises(ValueError):
        recovery.Recovery(student, recovery.Block(teacher.up, teacher.down, teacher.head[:100]))
