"""The recovery calls in a captured graph: replayed over new contents of the same tensors they give the bits of the calls
themselves, whatever eager calls did to the workspace in between."""
import pytest
import torch

from paper_2504_06323_b200 import api

pytestmark = pytest.mark.gpu
DEV = "cuda"


def bf16(g, *s, scale=1.0):
    return (torch.randn(*s, generator=g, device=DEV) * scale).to(torch.bfloat16)


@pytest.mark.parametrize("tokens", [1, 3, 37, 1500])
@pytest.mark.parametrize("ws_given", [True, False])
def test_replays_give_the_calls_bits(tokens, ws_given):
    g = torch.Generator(device=DEV).manual_seed(tokens)
    hidden, width, vocab, top = 256, 777, 1201, 20          # down is [hidden, 777]: dense odd rows, read through a copy
    X, up, down, head, bias = (bf16(g, tokens, hidden), bf16(g, width, hidden, scale=0.06), bf16(g, hidden, width, scale=0.04),
                               bf16(g, vocab, hidden, scale=0.06), bf16(g, width))
    teacher = bf16(g, tokens, vocab)
    f = lambda *s, dtype=torch.float32: torch.zeros(*s, device=DEV, dtype=dtype)  # noqa: E731
    e = lambda *s: torch.zeros(*s, device=DEV, dtype=torch.bfloat16)  # noqa: E731
    out = dict(H=e(tokens, width), Z=e(tokens, width), Y=e(tokens, hidden), L=e(tokens, vocab), v=f(tokens, top), i=f(tokens, top, dtype=torch.int32),
               lse=f(tokens), loss=f(tokens), dY=e(tokens, hidden), dH=e(tokens, width), dhead=e(vocab, hidden), ddown=e(hidden, width),
               dup=e(width, hidden), db=e(width), status=f(1, dtype=torch.int32))
    ws = api.Workspace(DEV) if ws_given else None

    def step(o):
        api.mosaic_top_logits(teacher, o["v"], o["i"], o["lse"], ws=ws)
        api.mosaic_linear(X, up, o["H"], bias=bias, act="gelu", Z=o["Z"], status=o["status"], ws=ws)
        api.mosaic_linear(o["H"], down, o["Y"], residual=X, status=o["status"], ws=ws)
        api.mosaic_linear(o["Y"], head, o["L"], ws=ws)
        api.mosaic_distill_loss_grad(o["L"], o["v"], o["i"], o["loss"], None, o["L"], t_lse=o["lse"], grad_scale=1.0 / tokens, ws=ws)
        api.mosaic_linear_backward(o["L"], o["Y"], head, dX=o["dY"], dW=o["dhead"], ws=ws)
        api.mosaic_linear_backward(o["dY"], o["H"], down, dX=o["dH"], dW=o["ddown"], ws=ws)
        api.mosaic_linear_backward(o["dH"], X, None, Z=o["Z"], act="gelu", dW=o["dup"], dbias=o["db"], status=o["status"], ws=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(out)
    for round_ in range(3):
        X.copy_(bf16(g, tokens, hidden))
        teacher.copy_(bf16(g, tokens, vocab))
        want = {k: torch.zeros_like(v) for k, v in out.items()}
        step(want)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[k], want[k]) for k in out)
        if round_ == 0:      # a larger eager call on the captured stream, and new tensors where a freed buffer would be
            big = bf16(g, 700, 3001)
            with torch.cuda.stream(side):
                api.mosaic_linear(big, bf16(g, 900, 3001), e(700, 900), ws=ws)
            torch.cuda.synchronize()
            taken = [torch.full((n,), 7, dtype=torch.uint8, device=DEV) for n in (1 << 12, 1 << 16, 1 << 18, 1 << 20, 1 << 21, 1 << 22) for _ in range(8)]
            with torch.cuda.stream(side):
                taken += [torch.full((n,), 7, dtype=torch.uint8, device=DEV) for n in (1 << 12, 1 << 16, 1 << 18, 1 << 20, 1 << 21, 1 << 22) for _ in range(8)]
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(bool((t == 7).all()) for t in taken)
