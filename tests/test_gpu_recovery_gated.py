"""The recovery path over the MLP that the LLaMA-shaped models compute, down(silu(gate(X)) * up(X)).

The answer of a block is compared with the formula in fp64 from the tensors that the block stored on the way, so each
bound is one product's: its fp32 sum, and one rounding to bf16 (2^-8 of the value)."""
import pytest
import torch

from paper_2504_06323_b200 import driver, recovery, workloads as wl

pytestmark = pytest.mark.gpu
DEV = "cuda"


def model(config="tiny", vocab=500, tokens=256):
    cfg = wl.CONFIGS[config]
    st = driver.alloc_model(cfg, torch.device(DEV, 0), layers=[0], outputs=False, masks=False)
    driver.accumulate_norms(st, 0, driver.make_activations(cfg, 0, DEV, tokens))
    g = torch.Generator(device=DEV).manual_seed(5)
    head = (torch.randn(vocab, cfg.hidden, generator=g, device=DEV) * cfg.hidden ** -0.5).to(torch.bfloat16)
    return cfg, st, head, g


def near(got, want, abs_sum, c):
    return bool(((got.double() - want).abs() <= 2.0 ** -8 * want.abs() + (c / 4.0 + 12.0) * 2.0 ** -24 * abs_sum + 1e-37).all())


@pytest.mark.parametrize("tokens", [1, 3, 37, 200])
def test_teacher_answers_as_the_layer(tokens):
    cfg, st, head, g = model()
    _, teacher = recovery.compact_mlp(st, 0, 0.3, head, gated=True)
    X = torch.randn(tokens, cfg.hidden, generator=g, device=DEV).to(torch.bfloat16)
    L = teacher.forward(X, keep=False)
    teacher.check()
    W = {pr: st.W[0, pr].to(torch.bfloat16).double() for pr in ("gate", "up", "down")}
    x = X.double()
    z = x @ W["gate"].T
    G, U, H, Y = (teacher._bufs[n].double() for n in ("G", "U", "H", "Y"))
    assert near(G, torch.nn.functional.silu(z), 1.2 * (x.abs() @ W["gate"].abs().T) + 2.0 ** 4 * z.abs(), cfg.hidden)
    assert near(U, x @ W["up"].T, x.abs() @ W["up"].abs().T, cfg.hidden)
    assert near(H, G * U, 0 * H, 1)
    assert near(Y, x + H @ W["down"].T, x.abs() + H.abs() @ W["down"].abs().T, cfg.intermediate)
    assert near(L, Y @ head.double().T, Y.abs() @ head.double().abs().T, cfg.hidden)
    # and as a whole it is the layer's answer, not that of a layer without its gate
    whole = (x + (torch.nn.functional.silu(z) * (x @ W["up"].T)) @ W["down"].T) @ head.double().T
    assert float((L.double() - whole).norm() / whole.norm()) < 4 * 2.0 ** -8


def test_student_keeps_the_rows_that_compaction_kept():
    cfg, st, head, _ = model()
    student, teacher = recovery.compact_mlp(st, 0, 0.3, head, gated=True)
    n = cfg.intermediate - int(0.3 * cfg.intermediate)
    assert student.gate.shape == student.up.shape == (n, cfg.hidden) and student.down.shape == (cfg.hidden, n)
    kept = (teacher.up[:, None, :] == student.up[None]).all(-1).any(1).nonzero()[:, 0]
    assert kept.numel() == n
    assert torch.equal(teacher.gate[kept], student.gate) and torch.equal(teacher.down[:, kept], student.down)


def test_command_trains_the_gated_block(monkeypatch):
    seen = []
    init = recovery.Recovery.__init__
    monkeypatch.setattr(recovery.Recovery, "__init__", lambda self, student, teacher, *a, **k: (seen.append((student, teacher)), init(self, student, teacher, *a, **k))[1])
    losses = recovery.main(["--steps", "12", "--tokens", "64", "--vocab", "300", "--top", "20"])
    assert losses[-1] < losses[0]
    (student, teacher), = seen
    assert student.gate is not None and teacher.gate is not None


def test_gate_of_another_shape_is_refused():
    _, st, head, _ = model()
    student, teacher = recovery.compact_mlp(st, 0, 0.3, head, gated=True)
    with pytest.raises(ValueError):
        recovery.Block(student.up, student.down, student.head, gate=teacher.gate)
