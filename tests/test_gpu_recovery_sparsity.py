"""Recovery of a composite-pruned block: what unstructured pruning removed stays removed, and the rest is trained as it
would be without it."""
import pytest
import torch

from paper_2504_06323_b200 import driver, recovery, workloads as wl
from paper_2504_06323_b200.workloads import PROJECTIONS

pytestmark = pytest.mark.gpu
DEV = "cuda"


def composite(gated):
    """(student, teacher) of the tiny block: half of every row removed, then 30 % of the MLP's channels."""
    cfg = wl.CONFIGS["tiny"]
    st = driver.alloc_model(cfg, torch.device(DEV, 0), layers=[0])
    driver.accumulate_norms(st, 0, driver.make_activations(cfg, 0, DEV, 256))
    driver.prune_unstructured_layer(st, 0, [cfg.shape(pr)[1] // 2 for pr in PROJECTIONS])
    g = torch.Generator(device=DEV).manual_seed(5)
    head = (torch.randn(400, cfg.hidden, generator=g, device=DEV) * cfg.hidden ** -0.5).to(torch.bfloat16)
    _, teacher = recovery.compact_mlp(st, 0, 0.0, head, gated=gated)
    W = driver.prune_structured_coupled_layer(st, 0, 0.3, source={pr: st.W_out[0, pr] for pr in PROJECTIONS})["W"]
    W = {pr: W[pr].to(torch.bfloat16) for pr in ("gate", "up", "down")}
    return recovery.Block(W["up"], W["down"], head.clone(), gate=W["gate"] if gated else None), teacher, g


@pytest.mark.parametrize("gated", [False, True])
def test_removed_weights_stay_removed(gated):
    student, teacher, g = composite(gated)
    names = [w for w in ("gate", "up", "down") if getattr(student, w) is not None]
    zero = {w: getattr(student, w) == 0 for w in names}
    assert all(0.3 < float(z.float().mean()) < 0.7 for z in zero.values())
    run = recovery.Recovery(student, teacher, top=32, rate=0.1)
    X = torch.randn(128, 256, generator=g, device=DEV).to(torch.bfloat16)
    targets = run.targets(X)
    before = {w: run.master[w].clone() for w in run.master}
    _, grads = run.gradients(X, targets)
    want = {w: before[w].add_(grads[w], alpha=-0.1) for w in grads}      # a step without anything removed
    run.step(X, targets)
    for w in names:
        assert (getattr(student, w)[zero[w]] == 0).all() and (run.master[w][zero[w]] == 0).all()
        assert (grads[w][zero[w]] != 0).any()                       # they would have moved
        assert torch.equal(run.master[w][~zero[w]], want[w][~zero[w]])
    assert torch.equal(run.master["head"], want["head"])
    first = float(run.loss(X, targets).mean())
    for _ in range(10):
        run.step(X, targets)
    assert all((getattr(student, w)[zero[w]] == 0).all() for w in names)
    assert float(run.loss(X, targets).mean()) < first
    student.check()


def test_a_bias_of_zero_is_trained():
    cfg = wl.CONFIGS["tiny"]
    st = driver.alloc_model(cfg, torch.device(DEV, 0), layers=[0], outputs=False, masks=False)
    driver.accumulate_norms(st, 0, driver.make_activations(cfg, 0, DEV, 256))
    g = torch.Generator(device=DEV).manual_seed(5)
    head = (torch.randn(400, cfg.hidden, generator=g, device=DEV) * cfg.hidden ** -0.5).to(torch.bfloat16)
    student, teacher = recovery.compact_mlp(st, 0, 0.3, head)
    run = recovery.Recovery(student, teacher, top=32, rate=0.1)
    X = torch.randn(128, 256, generator=g, device=DEV).to(torch.bfloat16)
    run.step(X)
    assert (student.bias != 0).any() and not run.removed
