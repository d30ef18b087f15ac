"""Checkpoint and Weight4 objects, and the block that is served from them, over their life: tensors that are put in another
place, arguments that are none, and a student that goes on learning."""
import pytest
import torch

from paper_2504_06323_b200 import api, recovery
from test_gpu_linear import matrix
from test_gpu_recovery_fused import blocks

pytestmark = pytest.mark.gpu
DEV = "cuda"


def test_a_served_block_stays_as_it_was_packed():
    """The bias is packed with the weights: what the student learns afterwards is not in the answer."""
    g = torch.Generator(device=DEV).manual_seed(2)
    W = lambda *s: (torch.randn(*s, generator=g, device=DEV) * 0.1).to(torch.bfloat16)  # noqa: E731
    block = recovery.Block(W(96, 64), W(64, 96), W(50, 64), W(96), gate=W(96, 64), fused=True)
    X = W(9, 64)
    served = block.packed(32)
    before = served.forward(X).clone()
    for w in recovery.Block.WEIGHTS:
        getattr(block, w).mul_(-2.0)
    assert torch.equal(served.forward(X), before)
    again = block.packed(32).forward(X)
    assert not torch.equal(again, before)


def test_the_fused_block_is_served_from_copies():
    student, _, X, _ = blocks(16, fused=True)
    served = student.packed(64)
    before = served.forward(X).clone()
    student.down.zero_()
    assert torch.equal(served.forward(X), before)


def test_no_checkpoint_is_refused():
    X = torch.zeros(5, 96, device=DEV, dtype=torch.bfloat16)
    for call in (lambda: api.mosaic_checkpoint_store(X, X), lambda: api.mosaic_checkpoint_store(X, None), lambda: api.mosaic_checkpoint_load(X, X),
                 lambda: api.mosaic_checkpoint_load(None, X), lambda: api.mosaic_checkpoint_store(X, api.Weight4.empty(5, 96, 32))):
        with pytest.raises(TypeError):
            call()


@pytest.mark.parametrize("how", ["attribute", "data"])
def test_codes_put_in_another_place_are_read_there(how):
    """The calls read the tensors that an object holds now, wherever they lie."""
    g = torch.Generator(device=DEV).manual_seed(3)
    W, X = matrix(40, 96, g, scale=0.2), matrix(5, 96, g)
    w4, c = api.Weight4.of(W, 32), api.Checkpoint.empty(5, 96)
    api.mosaic_checkpoint_store(X, c)
    old = w4.codes, w4.scales, c.codes, c.exponents     # alive, and changed below: no call may still read them

    def put(o, name):
        t = getattr(o, name)
        if how == "attribute":
            setattr(o, name, t.clone())
            t.zero_()
        else:
            first = t.detach()
            t.data = t.clone()
            first.zero_()
            old_data.append(first)

    old_data = []
    want = {}
    for state in ("before", "after"):
        Y, back, x = torch.empty(5, 40, device=DEV, dtype=torch.bfloat16), torch.empty_like(W), torch.empty(5, 96, device=DEV, dtype=torch.bfloat16)
        api.mosaic_linear4(X, w4, Y)
        api.mosaic_dequantize4(w4, back)
        api.mosaic_checkpoint_load(c, x)
        if state == "before":
            want = dict(Y=Y, back=back, x=x)
            for o, name in ((w4, "codes"), (w4, "scales"), (c, "codes"), (c, "exponents")):
                put(o, name)
        else:
            assert torch.equal(Y, want["Y"]) and torch.equal(back, want["back"]) and torch.equal(x, want["x"])
    assert len(old) == 4


def test_what_does_not_fit_any_more_is_refused():
    w4, c = api.Weight4.empty(40, 96, 32), api.Checkpoint.empty(5, 96)
    X, Y = torch.zeros(5, 96, device=DEV, dtype=torch.bfloat16), torch.zeros(5, 40, device=DEV, dtype=torch.bfloat16)
    keep = w4.codes, c.exponents
    w4.codes = w4.codes[:, :32].clone()
    c.exponents = c.exponents.cpu()
    with pytest.raises(ValueError):
        api.mosaic_linear4(X, w4, Y)
    with pytest.raises(TypeError):
        api.mosaic_checkpoint_store(X, c)
    assert len(keep) == 2
