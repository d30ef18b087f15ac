"""What the linear calls refuse names the argument and is a TypeError or a ValueError, whichever argument it is."""
import pytest
import torch

from paper_2504_06323_b200 import api

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("name", ["dY", "X", "W", "Z", "dX", "dW", "dbias"])
def test_backward_refuses_what_is_no_matrix(name):
    e = lambda *s: torch.zeros(*s, device=DEV, dtype=torch.bfloat16)  # noqa: E731
    good = dict(dY=e(8, 24), X=e(8, 16), W=e(24, 16), Z=e(8, 24), dX=e(8, 16), dW=e(24, 16), dbias=e(24))

    def call(**k):
        a = {**good, **k}
        api.mosaic_linear_backward(a.pop("dY"), a.pop("X"), a.pop("W"), act="silu", **a)

    call()
    rank = e(1, 24) if name == "dbias" else e(good[name].numel())
    for bad, error in ((3.0, TypeError), (good[name].cpu(), TypeError), (good[name].float(), TypeError), (rank, ValueError)):
        with pytest.raises(error, match=name):
            call(**{name: bad})
    torch.cuda.synchronize()


@pytest.mark.parametrize("only", ["X", "W"])
def test_backward_with_one_operand_refuses_what_is_no_matrix(only):
    e = lambda *s: torch.zeros(*s, device=DEV, dtype=torch.bfloat16)  # noqa: E731
    dY, db = e(8, 24), e(24)
    for bad, error in ((3.0, TypeError), (e(16), ValueError), (e(7, 16), ValueError)):
        with pytest.raises(error, match=only):
            api.mosaic_linear_backward(dY, bad if only == "X" else None, bad if only == "W" else None, dbias=db)
