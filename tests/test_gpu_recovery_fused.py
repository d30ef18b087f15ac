"""The gated operators together, as the recovery path uses them: a fused block's training step with activations in bf16 and
in 8 bits, and the block served in 4 bits - each stage against the formula in fp64 from the tensors that it was given
(bounds of test_gpu_linear.py and test_gpu_gated.py), the whole against the gradients of the formula."""
import threading

import pytest
import torch

from paper_2504_06323_b200 import api, driver, recovery, workloads as wl
from test_gpu_gated import check_gated, check_gated_backward
from test_gpu_linear import check_backward, check_forward

pytestmark = pytest.mark.gpu
DEV = "cuda"


def blocks(tokens, seed=5, **options):
    cfg = wl.CONFIGS["tiny"]
    st = driver.alloc_model(cfg, torch.device(DEV, 0), layers=[0], outputs=False, masks=False)
    driver.accumulate_norms(st, 0, driver.make_activations(cfg, 0, DEV, 256))
    g = torch.Generator(device=DEV).manual_seed(seed)
    head = (torch.randn(500, cfg.hidden, generator=g, device=DEV) * cfg.hidden ** -0.5).to(torch.bfloat16)
    student, teacher = recovery.compact_mlp(st, 0, 0.3, head, gated=True, **options)
    return student, teacher, torch.randn(tokens, cfg.hidden, generator=g, device=DEV).to(torch.bfloat16), g


def kept(block, name):
    """What the forward pass kept, in bf16."""
    if not block.saved8:
        return block._bufs[name].clone()
    c = block._saved[name]
    out = torch.empty(c.rows, c.cols, device=DEV, dtype=torch.bfloat16)
    api.mosaic_checkpoint_load(c, out)
    return out


@pytest.mark.parametrize("saved8", [False, True])
@pytest.mark.parametrize("tokens", [1, 4, 37, 200])
def test_every_stage_of_a_fused_step(tokens, saved8):
    student, teacher, X, g = blocks(tokens, fused=True, saved8=saved8)
    L = student.forward(X)
    b = {k: v.clone() for k, v in student._bufs.items()}
    Z, U = kept(student, "Z"), kept(student, "U")
    if not saved8:
        check_gated(X, student.gate, student.up, None, None, "silu", b["H"], Z, U)
    check_forward(b["H"], student.down, None, X, "none", b["Y"], None)
    check_forward(b["Y"], student.head, None, None, "none", b["L"], None)
    dL = (torch.randn(tokens, L.shape[1], generator=g, device=DEV) * 0.01).to(torch.bfloat16)
    dX = torch.empty_like(X)
    grads = {k: v.clone() for k, v in student.backward(X, dL, dX).items()}
    student.check()
    a = student._bufs
    check_backward(dL, b["Y"], student.head, None, "none", a["dY"], grads["head"], None)
    check_backward(a["dY"], a["H"], student.down, None, "none", a["dH"], grads["down"], None)
    check_gated_backward(a["dH"], kept(student, "X") if saved8 else X, student.gate, student.up, Z, U, "silu", None, grads["gate"], grads["up"], None, None, a["H"] if saved8 else None)
    inner = torch.empty_like(X)
    api.mosaic_gated_linear_backward(a["dH"], None, student.gate, student.up, Z, U, act="silu", dX=inner)
    assert torch.equal(dX, inner + a["dY"])


@pytest.mark.parametrize("saved8", [False, True])
def test_gradients_of_the_whole_block(saved8):
    """Against the formula's gradients in fp64 (2-norm).  bf16: six tensors between input and gradient are rounded at 2^-8 or
    less each, rms 2^-9.4: within 2^-7 together.  8 bits: X, Z and U are off by half a code, at most 2^-7 of their group's
    largest, in rms about a third of that: within 2^-5 together."""
    student, _, X, g = blocks(150, fused=True, saved8=saved8)
    student.forward(X)
    dL = (torch.randn(150, 500, generator=g, device=DEV) * 0.01).to(torch.bfloat16)
    dX = torch.empty_like(X)
    grads = dict(student.backward(X, dL, dX), X=dX)
    w = {k: getattr(student, k).double().requires_grad_(True) for k in ("gate", "up", "down", "head")}
    w["X"] = X.double().requires_grad_(True)
    y = w["X"] + (torch.nn.functional.silu(w["X"] @ w["gate"].T) * (w["X"] @ w["up"].T)) @ w["down"].T
    ((y @ w["head"].T) * dL.double()).sum().backward()
    for k, v in w.items():
        assert (grads[k].double() - v.grad).norm() <= (2.0 ** -5 if saved8 else 2.0 ** -7) * v.grad.norm(), k


@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("tokens", [1, 6, 40])
def test_trained_pruned_and_served(tokens, group):
    """Steps of a fused block with 8-bit activations keep what pruning removed at zero; so do 4 bits; the served block answers
    as its own weights say."""
    student, teacher, X, g = blocks(64, fused=True, saved8=True)
    for w in ("gate", "up", "down"):
        t = getattr(student, w)
        t.masked_fill_(torch.rand(t.shape, generator=g, device=DEV) < 0.5, 0.0)
    gone = {w: getattr(student, w) == 0 for w in ("gate", "up", "down")}
    run = recovery.Recovery(student, teacher, top=40)
    targets = run.targets(X)
    for _ in range(3):
        loss = run.step(X, targets)
    assert torch.isfinite(loss).all()
    student.check()
    served = student.packed(group)
    x = X[:tokens]
    L = served.forward(x)
    served.check()
    back = {}
    for w in ("gate", "up", "down", "head"):
        q = getattr(served, w)
        back[w] = torch.empty(q.rows, q.cols, device=DEV, dtype=torch.bfloat16)
        api.mosaic_dequantize4(q, back[w])
        if w in gone:
            assert (getattr(student, w)[gone[w]] == 0).all() and (back[w][gone[w]] == 0).all()
    same = recovery.Block(back["up"], back["down"], back["head"], gate=back["gate"], fused=True)
    want = same.forward(x, keep=False)
    # the same weights and formula, fp32 sums in another order: two roundings of H and Y apart at most
    assert (L.double() - want.double()).norm() <= 2.0 ** -7 * want.double().norm()
    assert run.loss(x, tuple(None if t is None else t[:tokens].contiguous() for t in targets), served).shape == (tokens,)


def test_command():
    losses = recovery.main(["--steps", "2", "--tokens", "32", "--vocab", "300", "--top", "20", "--fused", "--saved8", "--serve4", "64"])
    assert len(losses) == 3 and all(l == l for l in losses)


def test_refusals():
    student, teacher, X, _ = blocks(8)
    with pytest.raises(ValueError):
        recovery.Block(student.up, student.down, student.head, fused=True)
    with pytest.raises(ValueError):
        recovery.Block(student.up, student.down, student.head, gate=student.gate, saved8=True)
    student.forward(X)
    with pytest.raises(ValueError):
        student.backward(X, torch.zeros(8, 500, device=DEV, dtype=torch.bfloat16), torch.empty_like(X))


# ------------------------------------------------------------------ graphs, streams, threads
def operands(seed, tokens, n=333, k=264):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = lambda *s: (torch.randn(*s, generator=g, device=DEV) * 0.2).to(torch.bfloat16)  # noqa: E731
    e = lambda *s: torch.zeros(*s, device=DEV, dtype=torch.bfloat16)  # noqa: E731
    d = dict(X=r(tokens, k), Wg=r(n, k), Wu=r(n, k), Wd=r(k, n), bg=r(n), dH=r(tokens, n), H=e(tokens, n), again=e(tokens, n), dX=e(tokens, k), dWg=e(n, k), dWu=e(n, k),
             dbg=e(n), dbu=e(n), Y=e(tokens, k), H4=e(tokens, n), back=e(n, k), X8=api.Checkpoint.empty(tokens, k), Z8=api.Checkpoint.empty(tokens, n),
             U8=api.Checkpoint.empty(tokens, n), g4=api.Weight4.empty(n, k, 64), d4=api.Weight4.empty(k, n, 32), u4=api.Weight4.empty(n, k, 128))
    return d


def chain(o, ws=None):
    """Every new call once, over dense odd rows that need scratch."""
    api.mosaic_checkpoint_store(o["X"], o["X8"])
    api.mosaic_gated_linear(o["X"], o["Wg"], o["Wu"], o["H"], bias_gate=o["bg"], Z=o["Z8"], U=o["U8"], ws=ws)
    api.mosaic_gated_linear_backward(o["dH"], o["X8"], o["Wg"], o["Wu"], o["Z8"], o["U8"], dX=o["dX"], dW_gate=o["dWg"], dW_up=o["dWu"], dbias_gate=o["dbg"],
                                     dbias_up=o["dbu"], H=o["again"], ws=ws)
    for w, q in (("Wg", "g4"), ("Wu", "u4"), ("Wd", "d4")):
        api.mosaic_quantize4(o[w], o[q])
    api.mosaic_dequantize4(o["g4"], o["back"])
    api.mosaic_gated_linear4(o["X"], o["g4"], o["u4"], o["H4"], bias_up=o["bg"], ws=ws)
    api.mosaic_linear4(o["H4"], o["d4"], o["Y"], residual=o["X"], ws=ws)


RESULTS = ("H", "again", "dX", "dWg", "dWu", "dbg", "dbu", "H4", "Y", "back")


def results(o):
    return {k: o[k].clone() for k in RESULTS}


@pytest.mark.parametrize("tokens", [1, 5, 37, 700])
def test_replayed_graphs_give_the_calls_bits(tokens):
    """Two graphs with a workspace each, captured in turn, replayed in turn and at once over new contents."""
    pair = []
    for seed in (1, 2):
        o, ws = operands(seed, tokens), api.Workspace(DEV)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            chain(o, ws)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            chain(o, ws)
        pair.append((o, graph, side, ws))   # a graph uses its Workspace's buffer: both must live
    for (o, *_), seed in zip(pair, (11, 12)):
        fresh = operands(seed, tokens)
        for k in ("X", "Wg", "Wu", "Wd", "bg", "dH"):
            o[k].copy_(fresh[k])
    want = []
    for o, *_ in pair:
        chain(o)
        want.append(results(o))
        for k in RESULTS:
            o[k].zero_()
    torch.cuda.synchronize()
    for _ in range(3):
        for o, graph, side, _ in pair:
            with torch.cuda.stream(side):
                graph.replay()
    torch.cuda.synchronize()
    for (o, *_), w in zip(pair, want):
        for k in RESULTS:
            assert torch.equal(o[k], w[k]), k


@pytest.mark.parametrize("tokens", [1, 37, 300])
def test_two_streams_and_three_threads(tokens):
    """The default workspace serves every stream and thread its own buffer: the bits of one call after another."""
    sets = [operands(20 + i, tokens) for i in range(3)]
    want = []
    for o in sets:
        chain(o)
        want.append(results(o))
        for k in RESULTS:
            o[k].zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream(), torch.cuda.current_stream()]

    def work(i):
        with torch.cuda.stream(streams[i]):
            for _ in range(4):
                chain(sets[i])

    threads = [threading.Thread(target=work, args=(i,)) for i in range(3)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for o, w in zip(sets, want):
        for k in RESULTS:
            assert torch.equal(o[k], w[k]), k
