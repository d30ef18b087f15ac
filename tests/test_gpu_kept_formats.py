"""Checkpoint and Weight4 objects, and the block that is served from them, over their life: tensors that are put in another
place, arguments that are none, and a student that goes on learning."""
import pytest
import torch

from paper_2504_06323_b200 import api, recovery
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
