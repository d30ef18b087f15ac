"""How far a value kept in 8 bits may be from what was stored: half a code, 2^(E - 134), which is 2^-7 of the group's largest
magnitude where that is a normal number.  Below the normal numbers a code stays 2^-132, whatever the largest is."""
import pytest
import torch

from paper_2504_06323_b200 import api

pytestmark = pytest.mark.gpu
DEV = "cuda"


def kept(X):
    c = api.Checkpoint.empty(*X.shape)
    api.mosaic_checkpoint_store(X, c)
    out = torch.empty_like(X)
    api.mosaic_checkpoint_load(c, out)
    return out.double(), c.exponents.double()


@pytest.mark.parametrize("top", [1, 2, 3, 17, 126, 127, 128, 129, 200, 0x100, 0x1FF, 0x3F80, 0x7F00, 0x7F7F])
def test_half_a_code(top):
    """Groups whose largest magnitude is one bf16 number (its bits: below 128 no normal one), beside it all that are smaller."""
    bits = torch.arange(max(top - 15 * 64, 0), top, device=DEV, dtype=torch.int32)
    bits = torch.nn.functional.pad(bits, (0, -bits.numel() % 15)).view(-1, 15)
    bits = torch.cat([torch.full((bits.shape[0], 1), top, device=DEV, dtype=torch.int32), bits], 1)
    bits[:, 1::2] |= -32768
    X = bits.to(torch.int16).view(torch.bfloat16)
    back, E = kept(X)
    x, largest = X.double(), X.double().abs().amax(1, keepdim=True)
    off = (back - x).abs()
    assert (off <= torch.exp2(E - 134)).all()
    if top >= 128:
        assert (off <= largest * 2.0 ** -7).all()


def test_the_smallest_number_is_lost():
    X = torch.zeros(1, 16, device=DEV, dtype=torch.bfloat16)
    X[0, 3] = 2.0 ** -133
    back, E = kept(X)
    assert float(E[0, 0]) == 1 and float(back.abs().sum()) == 0
    X[0, 3] = 2.0 ** -132
    assert float(kept(X)[0][0, 3]) == 2.0 ** -132
