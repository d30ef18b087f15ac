"""Scratch of the calls: a buffer for every stream and host thread, whoever passes the Workspace and whoever passes none.

The host tests take the buffers from CPU memory; the GPU test issues calls to two streams with nothing between them, as
a program does that asks its teacher on one stream and trains its student on another, and compares bits with calls that
ran one after another.  The order in which the two streams' kernels run is the device's: equal bits in every round do
not prove that the buffers are apart (the host tests do), unequal ones prove that they are not.
"""
import threading

import pytest
import torch

from paper_2504_06323_b200 import api

DEV = "cuda"


def test_a_stream_has_its_own_buffer():
    ws = api.Workspace("cpu")
    a, n = ws.get(1000, 0)
    b, _ = ws.get(1000, 77)
    assert a != b and n >= 1000
    assert ws.get(500, 0) == (a, n) and ws.get(1000, 77)[0] == b      # and keeps it


def test_growth_replaces_one_stream_s_buffer_only():
    ws = api.Workspace("cpu")
    a, b = ws.get(300, 1)[0], ws.get(300, 2)[0]
    grown, n = ws.get(1 << 20, 1)
    assert n >= 1 << 20 and ws.get(300, 1) == (grown, n) and ws.get(300, 2)[0] == b


def test_an_outgrown_buffer_is_kept():
    """(a captured graph may go on using it), and there are few of them however slowly the need grows"""
    ws, seen = api.Workspace("cpu"), []
    for n in range(256, 200_000, 256):
        p, size = ws.get(n, 0)
        assert size >= n
        if p not in (q for q, _ in seen):
            seen.append((p, size))
    kept = {t.data_ptr() for t in ws._outgrown} | {ws.get(1, 0)[0]}
    assert {p for p, _ in seen} == kept and len(seen) <= 11
    assert sum(n for _, n in seen[:-1]) < seen[-1][1] <= 400_000


def test_a_thread_has_its_own_buffer():
    ws, got, hold = api.Workspace("cpu"), {}, threading.Barrier(4)

    def work(i):
        got[i] = ws.get(4096, 5)[0]
        hold.wait(timeout=30)          # all threads alive: no two of them share an identity

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert len(set(got.values())) == 4


def test_default_workspace_is_one_object_for_all_threads():
    found = []
    threads = [threading.Thread(target=lambda: found.append(api._ws(None, 0))) for _ in range(8)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert len({id(w) for w in found}) == 1


@pytest.mark.gpu
def test_buffers_belong_to_their_stream():
    ws, side = api.Workspace(DEV), torch.cuda.Stream()
    ws.get(1000)
    ws.get(1000, side.cuda_stream)
    with torch.cuda.stream(side):
        assert ws.get(1000)[0] == ws.get(1000, side.cuda_stream)[0]
    segments = [s for s in torch.cuda.memory_snapshot() if s["stream"] == side.cuda_stream]
    inside = lambda p: any(s["address"] <= p < s["address"] + s["total_size"] for s in segments)  # noqa: E731
    assert inside(ws.get(1000, side.cuda_stream)[0]) and not inside(ws.get(1000)[0])


@pytest.mark.gpu
def test_two_streams_at_once_give_the_bits_of_one_after_another():
    g = torch.Generator(device=DEV).manual_seed(4)
    teacher = torch.randn(2048, 9001, generator=g, device=DEV)
    student = torch.randn(1500, 7003, generator=g, device=DEV).to(torch.bfloat16)
    tv, ti = (t.contiguous() for t in torch.topk(student.float() + 1.0, 40, dim=1))
    ti = ti.to(torch.int32)
    X = torch.randn(300, 1001, generator=g, device=DEV).to(torch.bfloat16)       # rows off 16 bytes: read through a copy
    W = torch.randn(700, 1001, generator=g, device=DEV).to(torch.bfloat16)

    def buffers():
        f = lambda *s, dtype=torch.float32: torch.full(s, -7, device=DEV, dtype=dtype)  # noqa: E731
        return dict(v=f(2048, 40), i=f(2048, 40, dtype=torch.int32), lse=f(2048), loss=f(1500), l2=f(1500), dS=torch.zeros_like(student),
                    Y=f(300, 700, dtype=torch.bfloat16))

    def ask(o, stream=None):
        api.mosaic_top_logits(teacher, o["v"], o["i"], o["lse"], stream=stream)

    def train(o, stream=None):
        api.mosaic_linear(X, W, o["Y"], stream=stream)
        api.mosaic_distill_loss_grad(student, tv, ti, o["loss"], o["l2"], o["dS"], stream=stream)

    want = buffers()
    ask(want)
    torch.cuda.synchronize()
    train(want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(10):
        got = buffers()
        torch.cuda.synchronize()
        for _ in range(3):
            ask(got, stream=side)
            train(got)
        torch.cuda.synchronize()
        assert all(torch.equal(got[k], want[k]) for k in want)


@pytest.mark.gpu
def test_two_threads_on_one_stream_give_the_bits_of_one_after_another():
    """The launches of two threads' calls interleave on the stream; each call's own order is kept."""
    g = torch.Generator(device=DEV).manual_seed(8)
    logits = [torch.randn(400, 5003 + 10 * i, generator=g, device=DEV).to(torch.bfloat16) for i in range(3)]
    kept = []
    for x in logits:
        v, i = torch.topk(x.float() + 0.5, 30, dim=1)
        kept.append((v.contiguous(), i.to(torch.int32)))

    def buffers(x):
        f = lambda *s, dtype=torch.float32: torch.full(s, -7, device=DEV, dtype=dtype)  # noqa: E731
        return [f(400, 30), f(400, 30, dtype=torch.int32), f(400), f(400), torch.zeros_like(x), torch.zeros_like(x)]

    def calls(x, k, o):
        api.mosaic_top_logits(x, o[0], o[1], o[2])
        api.mosaic_distill_loss_grad(x, *k, o[3], None, o[4])
        api.mosaic_distill_grad(x, *k, o[2], o[5])

    want = [buffers(x) for x in logits]
    for x, k, o in zip(logits, kept, want):
        calls(x, k, o)
        torch.cuda.synchronize()
    got = [buffers(x) for x in logits]
    torch.cuda.synchronize()
    start, failed = threading.Barrier(3), []

    def work(n):
        try:
            start.wait(timeout=30)
            for _ in range(40):
                calls(logits[n], kept[n], got[n])
        except Exception as e:   # noqa: BLE001   (a thread's error is the test's)
            failed.append(e)

    threads = [threading.Thread(target=work, args=(n,)) for n in range(3)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed
    assert all(torch.equal(p, q) for a, b in zip(got, want) for p, q in zip(a, b))
