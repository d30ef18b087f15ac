"""One training step of the recovery path, stage by stage: each call's results against the formula in fp64 from the
tensors that the path handed to that call, so that every bound is one call's own (test_gpu_linear.py and
test_gpu_logits.py, whose checks are used here).  Each check is also shown to fail for what a mistake would leave:
gradients that are zero or lack the activation's slope, a missing residual, a loss of zero."""
import pytest
import torch

from paper_2504_06323_b200 import driver, recovery, workloads as wl
from test_gpu_linear import check_backward, check_forward
from test_gpu_logits import distill_ref, grad_bound, loss_bound, top_ref

pytestmark = pytest.mark.gpu
DEV = "cuda"
T = 2.0


def step(tokens, renormalise, gated):
    """A step's tensors by their names: inputs, what the calls stored, and the gradients."""
    cfg = wl.CONFIGS["tiny"]
    st = driver.alloc_model(cfg, torch.device(DEV, 0), layers=[0], outputs=False, masks=False)
    driver.accumulate_norms(st, 0, driver.make_activations(cfg, 0, DEV, 256))
    g = torch.Generator(device=DEV).manual_seed(5)
    head = (torch.randn(500, cfg.hidden, generator=g, device=DEV) * cfg.hidden ** -0.5).to(torch.bfloat16)
    student, teacher = recovery.compact_mlp(st, 0, 0.3, head, gated=gated)
    X = torch.randn(tokens, 256, generator=g, device=DEV).to(torch.bfloat16)
    run = recovery.Recovery(student, teacher, top=40, temperature=T, renormalise=renormalise)
    targets = run.targets(X)
    a = dict(X=X, teacher=teacher._bufs["L"].clone(), targets=targets, logits=student.forward(X).clone(), student=student)
    loss, grads = run.gradients(X, targets)
    student.check()
    teacher.check()
    a |= {k: v.clone() for k, v in student._bufs.items()}
    a |= dict(loss=loss, dL=a.pop("L"), **{"d" + k: v.clone() for k, v in grads.items()})
    return a


def check_targets(a):
    values, indices, lse = a["targets"]
    want = torch.from_numpy(top_ref(a["teacher"], 40)).to(DEV)
    assert torch.equal(indices.long(), want) and torch.equal(values, a["teacher"].float().gather(1, want))
    if lse is not None:
        ref = torch.logsumexp(a["teacher"].double() / T, 1)
        assert ((lse.double() - ref).abs() <= 2.0 ** -17 + 2.0 ** -24 * ref.abs()).all()


def check_forward_pass(a):
    s = a["student"]
    if s.gate is None:
        check_forward(a["X"], s.up, s.bias, None, "silu", a["H"], a["Z"])
    else:
        check_forward(a["X"], s.gate, s.bias, None, "silu", a["G"], a["Z"])
        check_forward(a["X"], s.up, None, None, "none", a["U"], None)
        assert torch.equal(a["H"], a["G"] * a["U"])
    check_forward(a["H"], s.down, None, a["X"], "none", a["Y"], None)
    check_forward(a["Y"], s.head, None, None, "none", a["logits"], None)


def check_loss(a):
    values, indices, lse = a["targets"]
    rows = a["X"].shape[0]
    one = torch.full((rows,), 1.0 / rows, device=DEV, dtype=torch.float64)
    ref = distill_ref(a["logits"], values, indices, lse, None, T, one)
    assert ((a["loss"].double() - ref["loss"]).abs() <= loss_bound(ref, T)).all()
    assert ((a["dL"].double() - ref["dS"]).abs() <= grad_bound(ref, torch.bfloat16, T)).all()


def check_head(a):
    check_backward(a["dL"], a["Y"], a["student"].head, None, "none", a["dY"], a["dhead"], None)


def check_down(a):
    check_backward(a["dY"], a["H"], a["student"].down, None, "none", a["dH"], a["ddown"], None)


def check_mlp(a):
    s, db = a["student"], a.get("dbias")
    if s.gate is None:
        check_backward(a["dH"], a["X"], s.up, a["Z"], "silu", None, a["dup"], db)
    else:
        assert torch.equal(a["dG"], a["dH"] * a["U"]) and torch.equal(a["dU"], a["dH"] * a["G"])
        check_backward(a["dG"], a["X"], s.gate, a["Z"], "silu", None, a["dgate"], db)
        check_backward(a["dU"], a["X"], s.up, None, "none", None, a["dup"], None)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("renormalise", [True, False])
@pytest.mark.parametrize("tokens", [1, 4, 37, 200])
def test_every_stage_of_a_step(tokens, renormalise, gated):
    a = step(tokens, renormalise, gated)
    for check in (check_targets, check_forward_pass, check_loss, check_head, check_down, check_mlp):
        check(a)


def without_slope(a, name):
    into = a["dG"] if a["student"].gate is not None else a["dH"]
    return {name: (into.double().T @ a["X"].double()).to(torch.bfloat16)}


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("renormalise", [True, False])
@pytest.mark.parametrize("tokens", [4, 200])
def test_each_check_fails_for_what_a_mistake_would_leave(tokens, renormalise, gated):
    a = step(tokens, renormalise, gated)
    zero = lambda k: {k: torch.zeros_like(a[k])}  # noqa: E731
    active = "dgate" if gated else "dup"
    mistakes = [
        (check_targets, {"targets": (a["targets"][0], a["targets"][1].flip(1), a["targets"][2])}),
        (check_forward_pass, {"Y": (a["Y"].float() - a["X"].float()).to(torch.bfloat16)}), (check_forward_pass, zero("logits")),
        (check_loss, zero("loss")), (check_loss, zero("dL")),
        (check_head, zero("dhead")), (check_head, zero("dY")), (check_down, zero("ddown")), (check_down, zero("dH")),
        (check_mlp, zero("dup")), (check_mlp, zero(active)), (check_mlp, without_slope(a, active))]
    if a.get("dbias") is not None:
        mistakes.append((check_mlp, zero("dbias")))
    if gated:
        mistakes += [(check_forward_pass, {"H": a["G"]}), (check_mlp, {"dU": a["dH"]})]
    for check, wrong in mistakes:
        check(a)
        with pytest.raises(AssertionError):
            check({**a, **wrong})
