"""mosaic_top_logits and the distillation calls against their definitions in fp64.

Order and values of the top logits are exact.  Tolerances elsewhere, from the arithmetic:
  * exponentials in fp32: the hardware's 2^x is within 2^-22, its argument (x - m) * log2(e) / T within
    2^-23 |x - m| / T * 1.4427: an entry's relative error is below E(x) = 2^-21.5 + 2^-22.5 |x - m| / T;
  * a row's sum: entries' errors averaged, plus at most 64 + 8 + 16 + 8 additions in sequence and the merging
    factors, together below 2^-17 (all of one sign: no cancellation);  lse = m / T + log(sum), rounded to fp32
    once, so |lse - exact| <= 2^-17 + 2^-24 |lse|;
  * loss: sum of p times differences, each off by at most the lse's 2^-17 (P times), p rounded to fp32;
  * gradient: coef (P q - p): q off by E + 2^-17 relative, p by 2^-23, the products and the difference by 2^-22 of
    their terms, one rounding to the output type (2^-8 for bf16, 2^-24 for fp32).  From a saved lse (fp32, an input)
    the argument x / T - lse carries 2^-22 (|x / T| + |lse|).
"""
import math

import numpy as np
import pytest
import torch

from paper_2504_06323_b200 import api

pytestmark = pytest.mark.gpu
DEV = "cuda"
INF = float("inf")


def logits(rows, cols, dtype, seed, pitch=0, offset=0, kind="normal"):
    """[rows, cols] with NaN around it."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    ld = cols + pitch
    buf = torch.full((rows * ld + offset + 16,), float("nan"), device=DEV, dtype=dtype)
    m = buf[offset:offset + rows * ld].view(rows, ld)[:, :cols]
    x = torch.randn(rows, cols, generator=g, device=DEV) * 3
    if kind == "ties":
        x = torch.randint(-4, 5, (rows, cols), generator=g, device=DEV).float()
    elif kind == "ascending":
        x = torch.arange(cols, device=DEV, dtype=torch.float32).expand(rows, cols) * 0.01
    elif kind == "descending":
        x = -torch.arange(cols, device=DEV, dtype=torch.float32).expand(rows, cols) * 0.01
    elif kind == "peaked":
        x[:, cols // 2] += 40
    elif kind == "large":
        x = x * 1e4
    m.copy_(x)
    return m


def top_ref(x, top):
    """Indices of the largest entries, value descending then index ascending, NaN first, -0 equal to +0."""
    v = x.float().cpu().numpy().astype(np.float64)
    idx = np.arange(v.shape[1])
    return np.stack([np.lexsort((idx, -r, ~np.isnan(r)))[:top] for r in v])


def run_top(x, top, T=1.0):
    rows = x.shape[0]
    values = torch.full((rows, top), -7.0, device=DEV)
    indices = torch.full((rows, top), -7, device=DEV, dtype=torch.int32)
    lse = torch.full((rows,), -7.0, device=DEV)
    api.mosaic_top_logits(x, values, indices, lse, temperature=T)
    torch.cuda.synchronize()
    return values, indices, lse


def check_top(x, top, T=1.0):
    values, indices, lse = run_top(x, top, T)
    want = torch.from_numpy(top_ref(x, top)).to(DEV)
    assert torch.equal(indices.long(), want)
    assert torch.equal(values.view(torch.int32), x.float().contiguous().gather(1, want).view(torch.int32))
    ref = torch.logsumexp(x.double() / T, dim=1)
    fine = torch.isfinite(ref)
    assert ((lse.double() - ref).abs()[fine] <= 2.0 ** -17 + 2.0 ** -24 * ref.abs()[fine]).all()
    assert torch.equal(lse[~fine].isnan(), ref[~fine].isnan())
    rest = ~fine & ~ref.isnan()
    assert torch.equal(lse[rest].double(), ref[rest])
    return values, indices, lse


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols,top", [
    (1, 1, 1), (3, 2, 2), (1, 7, 3), (2, 8, 8), (5, 9, 1), (1, 100, 100), (4, 1000, 64), (2, 1024, 1024), (300, 513, 20), (1, 32000, 20),
    (7, 32000, 64), (200, 32001, 256), (3, 32768, 500), (2, 32769, 300), (1, 50001, 1000), (2, 65536, 64), (150, 65537, 5), (1, 131072, 64),
    (1, 262145, 50), (2, 300001, 256)])
def test_top_shapes(rows, cols, top, dtype):
    check_top(logits(rows, cols, dtype, rows + cols), top, T=1.0 if cols % 2 else 2.5)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", ["ties", "ascending", "descending", "peaked", "large"])
@pytest.mark.parametrize("cols,top", [(3000, 100), (40000, 33), (40000, 700)])
def test_top_distributions(kind, dtype, cols, top):
    check_top(logits(3, cols, dtype, 5, kind=kind), top)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", [70, 5000, 70000])
def test_top_masked_and_nonfinite(dtype, cols):
    x = logits(10, cols, dtype, 2)
    x[0] = -INF                              # nothing left
    x[1, 3:] = -INF                          # three left
    x[2, ::2] = -INF
    x[3, 5] = INF
    x[4, 6] = float("nan")
    x[4, 60] = INF
    x[5, ::3] = float("nan")                 # more NaN than kept
    x[6] = 0.0
    x[6, ::2] = -0.0                         # zeros of both signs are ties
    x[7] = torch.finfo(dtype).min            # masked with the type's lowest value
    x[7, 11] = 1.0
    x[8] = INF
    x[9] = torch.finfo(dtype).max
    for top in (1, 40, 64):
        check_top(x, top)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pitch,offset", [(0, 0), (0, 1), (1, 0), (3, 5), (8, 8), (16, 2)])
def test_top_any_alignment(dtype, pitch, offset):
    for cols in (1, 5, 777, 4003):
        check_top(logits(6, cols, dtype, cols, pitch, offset), min(cols, 30))


def test_top_offsets_past_32_bits():
    ld = (1 << 30) + 3
    big = torch.empty(3 * ld, device=DEV, dtype=torch.bfloat16)
    x = big.view(3, ld)[:, 7:5007]
    x.copy_(torch.randn(3, 5000, device=DEV))
    check_top(x, 64)


def test_top_no_rows_no_lse_other_stream_and_same_bits():
    e = torch.empty(0, 50, device=DEV)
    api.mosaic_top_logits(e, torch.empty(0, 5, device=DEV), torch.empty(0, 5, device=DEV, dtype=torch.int32))
    x = logits(50, 33000, torch.bfloat16, 3)
    a = check_top(x, 64)
    v, i = torch.empty_like(a[0]), torch.empty_like(a[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    api.mosaic_top_logits(x, v, i, stream=side)
    side.synchronize()
    assert torch.equal(v, a[0]) and torch.equal(i, a[1])
    b = run_top(x, 64)
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_top_refusals():
    x = logits(4, 100, torch.float32, 1)
    v, i = torch.empty(4, 10, device=DEV), torch.empty(4, 10, device=DEV, dtype=torch.int32)

    def status(fn):
        with pytest.raises(api.MosaicError) as e:
            fn()
        return e.value.status

    assert status(lambda: api.mosaic_top_logits(x[:, :9], v, i)) == -1                      # more kept than there are
    assert status(lambda: api.mosaic_top_logits(x, v, i, temperature=0.0)) == -1
    assert status(lambda: api.mosaic_top_logits(x, v, i, temperature=float("nan"))) == -1
    y = logits(4, 2000, torch.float32, 1)
    big = (torch.empty(4, 1025, device=DEV), torch.empty(4, 1025, device=DEV, dtype=torch.int32))
    assert status(lambda: api.mosaic_top_logits(y, *big)) == -1                             # above 1024
    flat = torch.zeros(4000, device=DEV)
    assert status(lambda: api.mosaic_top_logits(flat[:400].view(4, 100), flat[390:430].view(4, 10), i)) == -6
    for bad in (lambda: api.mosaic_top_logits(x.cpu(), v, i), lambda: api.mosaic_top_logits(x.half(), v, i),
                lambda: api.mosaic_top_logits(x, v.double(), i), lambda: api.mosaic_top_logits(x, v, i.long())):
        with pytest.raises(TypeError):
            bad()
    with pytest.raises(ValueError):
        api.mosaic_top_logits(x, v, i[:, :9])
    with pytest.raises(ValueError):
        api.mosaic_top_logits(x.T, v, i)


# ------------------------------------------------------------------ distillation
def teacher(S, top, seed, T, given):
    """Kept logits of a teacher near the student, in a shuffled order."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    t = S.float() + torch.randn(S.shape, generator=g, device=DEV)
    values, indices = torch.topk(t, top, dim=1)
    p = torch.randperm(top, generator=g, device=DEV)
    lse = torch.logsumexp(t.double() / T, dim=1).float() if given else None
    return values[:, p].contiguous(), indices[:, p].to(torch.int32).contiguous(), lse


def distill_ref(S, tv, ti, t_lse, weight, T, grad, lse=None):
    """(loss, lse, dS, and the pieces the bounds need) in fp64, from the definition."""
    rows, vocab = S.shape
    x = S.double() / T
    there = (ti >= 0) & (ti < vocab)
    u = torch.where(there, tv.double() / T, -INF)
    if t_lse is None:
        top = u.amax(1, keepdim=True)
        top = torch.where(torch.isfinite(top), top, torch.zeros_like(top))
        norm = top + torch.log(torch.exp(u - top).sum(1, keepdim=True))
    else:
        norm = t_lse.double()[:, None]
    logp = torch.where(u > -INF, u - norm, -INF)
    p = torch.where(u > -INF, torch.exp(logp), 0.0)
    own = torch.logsumexp(x, 1) if lse is None else lse.double()
    at = ti.long().clamp(0, vocab - 1)
    term = torch.where(p > 0, p * (logp - (x.gather(1, at) - own[:, None])), 0.0)
    w = torch.ones(rows, device=DEV, dtype=torch.float64) if weight is None else weight.double()
    mass = p.sum(1)
    live = (w != 0) & (mass != 0)
    loss = torch.where(live, w * T * T * term.sum(1), 0.0)
    coef = grad.double() * w * T
    q = torch.exp(x - own[:, None])
    d = coef[:, None] * (mass[:, None] * q).scatter_add(1, at, -p)
    d = torch.where(live[:, None], d, 0.0)
    return dict(loss=loss, lse=own, dS=d, q=q, p=p, mass=mass, coef=coef, live=live, w=w, x=x, at=at, logp=logp)


def grad_bound(ref, dtype, T, lse=None):
    x, q, p = ref["x"], ref["q"], ref["p"]
    big = torch.where(torch.isfinite(x), x, torch.zeros_like(x)).amax(1, keepdim=True)
    span = torch.where(torch.isfinite(x), (big - x).abs(), torch.zeros_like(x))
    rel = 2.0 ** -21.5 + 2.0 ** -22.5 * span + 2.0 ** -17
    if lse is not None:
        rel = rel + 2.0 ** -22 * (torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x)) + lse.double().abs()[:, None])
    tq = ref["mass"][:, None] * q
    tp = torch.zeros_like(q).scatter_add(1, ref["at"], p)
    b = ref["coef"].abs()[:, None] * (tq * (rel + 2.0 ** -20) + tp * 2.0 ** -20) + ref["dS"].abs() * (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -23)
    return b + 1e-37


def loss_bound(ref, T):
    terms = torch.where(ref["p"] > 0, ref["p"] * (ref["logp"].abs() + ref["x"].gather(1, ref["at"]).abs() + ref["lse"].abs()[:, None]), 0.0).sum(1)
    return ref["w"].abs() * T * T * (2.0 ** -17 * ref["mass"] + 2.0 ** -21 * terms) + 2.0 ** -23 * ref["loss"].abs() + 1e-37


def check_distill(S, tv, ti, t_lse=None, weight=None, T=1.0, grad_rows=None, grad_scale=1.0, dS_like=None):
    rows, vocab = S.shape
    f = lambda: torch.full((rows,), -7.0, device=DEV)  # noqa: E731
    new = (lambda: torch.full_like(S, 5.0, memory_format=torch.contiguous_format)) if dS_like is None else dS_like
    g = torch.full((rows,), grad_scale, device=DEV, dtype=torch.float64)
    if grad_rows is not None:
        g = g * grad_rows.double()
    kw = dict(t_lse=t_lse, row_weight=weight, temperature=T)
    loss, lse = f(), f()
    api.mosaic_distill_loss(S, tv, ti, loss, lse, **kw)
    loss2, lse2, dS2 = f(), f(), new()
    api.mosaic_distill_loss_grad(S, tv, ti, loss2, lse2, dS2, grad_rows=grad_rows, grad_scale=grad_scale, **kw)
    dS = new()
    api.mosaic_distill_grad(S, tv, ti, lse, dS, grad_rows=grad_rows, grad_scale=grad_scale, **kw)
    torch.cuda.synchronize()
    ref = distill_ref(S, tv, ti, t_lse, weight, T, g)
    live = ref["live"]
    ok = torch.isfinite(ref["lse"])
    assert ((lse.double() - ref["lse"]).abs()[ok] <= 2.0 ** -17 + 2.0 ** -24 * ref["lse"].abs()[ok]).all()
    assert torch.equal(loss, loss2) and torch.equal(lse.view(torch.int32), lse2.view(torch.int32))
    assert (loss[~live] == 0).all() and (dS[~live] == 0).all() and (dS2[~live] == 0).all()
    assert ((loss.double() - ref["loss"]).abs()[live] <= loss_bound(ref, T)[live]).all()
    assert ((dS2.double() - ref["dS"]).abs()[live] <= grad_bound(ref, S.dtype, T)[live]).all()
    saved = distill_ref(S, tv, ti, t_lse, weight, T, g, lse=lse)
    assert ((dS.double() - saved["dS"]).abs()[live] <= grad_bound(saved, S.dtype, T, lse)[live]).all()
    return loss, lse, dS2, dS


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("rows,vocab,top,T", [
    (1, 1, 1, 1.0), (2, 5, 5, 1.0), (3, 8, 2, 2.0), (1, 1000, 64, 1.0), (5, 1003, 20, 4.0), (300, 700, 50, 1.0), (4, 32000, 64, 2.0),
    (2, 32769, 256, 1.0), (150, 32003, 33, 1.0), (1, 131072, 1024, 3.0), (2, 300001, 100, 1.0)])
def test_distill_shapes(rows, vocab, top, T, given, dtype):
    S = logits(rows, vocab, dtype, rows + vocab)
    tv, ti, t_lse = teacher(S, top, 1, T, given)
    g = torch.rand(rows, device=DEV, generator=torch.Generator(device=DEV).manual_seed(2)) + 0.1
    check_distill(S, tv, ti, t_lse, T=T, grad_rows=g if rows > 2 else None, grad_scale=0.5)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("vocab", [200, 40001])
def test_distill_rows_that_count_for_nothing(dtype, given, vocab):
    rows, top = 8, 16
    S = logits(rows, vocab, dtype, 3)
    tv, ti, t_lse = teacher(S, top, 4, 1.0, given)
    weight = torch.tensor([1, 0, 0.5, 1, 1, 0, 1, 2.0], device=DEV)
    S[5] = float("nan")              # dropped: its content must not matter
    ti[3] = -1                       # no entry at all
    ti[4, ::2] = vocab + 5           # half of the entries outside the vocabulary
    ti[4, 1] = -2 ** 31
    tv[6] = -INF                     # all kept logits masked
    tv[7, 3:] = -INF                 # some of them
    loss, lse, a, b = check_distill(S, tv, ti, t_lse, weight=weight)
    assert (loss[[1, 3, 5, 6]] == 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_distill_masked_vocabulary(dtype):
    """Entries of -inf in the student (a masked vocabulary) outside the kept ones get gradient 0."""
    S = logits(4, 5000, dtype, 5)
    tv, ti, t_lse = teacher(S, 20, 6, 1.0, True)
    hole = torch.ones(4, 5000, dtype=torch.bool, device=DEV).scatter(1, ti.long(), False)
    hole[:, ::2] = False
    S[hole] = -INF
    _, _, a, b = check_distill(S, tv, ti, t_lse)
    assert (a[hole] == 0).all() and (b[hole] == 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("top", [6, 300])
def test_distill_doubled_entries_add_up(dtype, top):
    S = logits(3, 2000, dtype, 7)
    tv, ti, t_lse = teacher(S, top, 8, 1.0, False)
    ti[0, 1] = ti[0, 0]
    ti[1] = ti[1, 2]
    check_distill(S, tv, ti)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pitch,offset", [(0, 1), (1, 0), (3, 5), (8, 8)])
@pytest.mark.parametrize("vocab", [3, 1001, 33000])
def test_distill_any_alignment_and_in_place(dtype, pitch, offset, vocab):
    S = logits(5, vocab, dtype, vocab, pitch, offset)
    tv, ti, t_lse = teacher(S, min(vocab, 12), 9, 2.0, True)
    other = lambda: logits(5, vocab, dtype, 0, 7, 3)  # noqa: E731   (another alignment than S)
    _, lse, a, b = check_distill(S, tv, ti, t_lse, T=2.0)
    _, _, c, d = check_distill(S, tv, ti, t_lse, T=2.0, dS_like=other)
    assert torch.equal(a, c) and torch.equal(b, d)
    kw = dict(t_lse=t_lse, temperature=2.0)
    for grad in (False, True):
        buf = logits(5, vocab, dtype, vocab, pitch, offset)
        around = buf._base if buf._base is not None else buf
        if grad:
            api.mosaic_distill_grad(buf, tv, ti, lse, buf, **kw)
            assert torch.equal(buf, b)
        else:
            loss, l2 = torch.empty(5, device=DEV), torch.empty(5, device=DEV)
            api.mosaic_distill_loss_grad(buf, tv, ti, loss, l2, buf, **kw)
            assert torch.equal(buf, a) and torch.equal(l2, lse)
        flat = torch.as_strided(around, (5 * (vocab + pitch) + offset + 16,), (1,), 0)
        assert int(torch.isnan(flat).sum()) == flat.numel() - 5 * vocab     # nothing written around the rows


def test_distill_label_is_cross_entropy():
    S = logits(64, 3000, torch.float32, 3)
    label = torch.randint(0, 3000, (64, 1), device=DEV, dtype=torch.int32)
    loss = torch.empty(64, device=DEV)
    api.mosaic_distill_loss(S, torch.zeros(64, 1, device=DEV), label, loss)
    ref = torch.nn.functional.cross_entropy(S.double(), label[:, 0].long(), reduction="none")
    assert ((loss.double() - ref).abs() <= 2.0 ** -17 + 2.0 ** -20 * ref).all()


def test_distill_gradient_against_differences():
    """The sum of the losses moved along random directions, differenced in fp64 from the definition."""
    g = torch.Generator(device=DEV).manual_seed(12)
    rows, vocab, top, T = 6, 400, 20, 2.0
    S = logits(rows, vocab, torch.float32, 1)
    for given in (False, True):
        tv, ti, t_lse = teacher(S, top, 2, T, given)
        w = torch.rand(rows, generator=g, device=DEV) + 0.5
        _, _, dS, _ = check_distill(S, tv, ti, t_lse, weight=w, T=T)
        one = torch.ones(rows, device=DEV, dtype=torch.float64)
        for _ in range(3):
            d, h = torch.randn(rows, vocab, generator=g, device=DEV, dtype=torch.float64), 1e-4
            f = lambda s: distill_ref(S.double() + s * h * d, tv, ti, t_lse, w, T, one)["loss"].sum()  # noqa: E731
            diff = (f(1) - f(-1)) / (2 * h)
            assert abs(float(diff - (dS.double() * d).sum())) <= 1e-5 * (1 + abs(float(diff)))


def test_distill_offsets_past_32_bits():
    ld = (1 << 30) + 8
    big = torch.empty(3 * ld, device=DEV, dtype=torch.bfloat16)
    S = big.view(3, ld)[:, 8:3008]
    dS = big.view(3, ld)[:, 4096:7096]
    S.copy_(torch.randn(3, 3000, device=DEV))
    tv, ti, t_lse = teacher(S, 32, 1, 1.0, True)
    near = S.clone()
    check_distill(near, tv, ti, t_lse)
    loss, lse, want = torch.empty(3, device=DEV), torch.empty(3, device=DEV), torch.empty_like(near)
    api.mosaic_distill_loss_grad(near, tv, ti, loss, lse, want, t_lse=t_lse)
    # rows interleaved with the output's in one buffer: the spans overlap, so the call refuses them
    with pytest.raises(api.MosaicError):
        api.mosaic_distill_loss_grad(S, tv, ti, loss, lse, dS, t_lse=t_lse)
    api.mosaic_distill_loss_grad(S, tv, ti, loss, lse, S, t_lse=t_lse)
    torch.cuda.synchronize()
    assert torch.equal(S, want)


def test_distill_same_bits_and_other_stream():
    S = logits(40, 33000, torch.bfloat16, 3)
    tv, ti, t_lse = teacher(S, 64, 1, 1.0, True)
    a = check_distill(S, tv, ti, t_lse)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    loss, lse, dS = torch.empty(40, device=DEV), torch.empty(40, device=DEV), torch.empty_like(S)
    with torch.cuda.stream(side):
        api.mosaic_distill_loss_grad(S, tv, ti, loss, lse, dS, t_lse=t_lse)
    side.synchronize()
    assert torch.equal(loss, a[0]) and torch.equal(lse, a[1]) and torch.equal(dS, a[2])


def test_distill_no_rows_and_refusals():
    e = torch.empty(0, 50, device=DEV)
    ev, ei, e1 = torch.empty(0, 5, device=DEV), torch.empty(0, 5, device=DEV, dtype=torch.int32), torch.empty(0, device=DEV)
    api.mosaic_distill_loss_grad(e, ev, ei, e1, None, torch.empty_like(e))
    S = logits(4, 100, torch.float32, 1)
    tv, ti, t_lse = teacher(S, 10, 1, 1.0, True)
    loss, lse, dS = torch.empty(4, device=DEV), torch.empty(4, device=DEV), torch.empty_like(S)

    def status(fn):
        with pytest.raises(api.MosaicError) as err:
            fn()
        return err.value.status

    assert status(lambda: api.mosaic_distill_loss(S, tv, ti, loss, temperature=-1.0)) == -1
    assert status(lambda: api.mosaic_distill_loss(S, tv, ti, loss, temperature=INF)) == -1
    assert status(lambda: api.mosaic_distill_loss(S, tv, ti, loss, lse=loss)) == -6
    flat = torch.zeros(900, device=DEV)
    assert status(lambda: api.mosaic_distill_grad(flat[:400].view(4, 100), tv, ti, lse, flat[200:600].view(4, 100))) == -6
    wide = (torch.zeros(4, 1025, device=DEV), torch.zeros(4, 1025, device=DEV, dtype=torch.int32))
    assert status(lambda: api.mosaic_distill_loss(S, *wide, loss)) == -1
    for bad in (lambda: api.mosaic_distill_loss(S.cpu(), tv, ti, loss), lambda: api.mosaic_distill_loss(S.half(), tv, ti, loss),
                lambda: api.mosaic_distill_loss(S, tv, ti.long(), loss), lambda: api.mosaic_distill_grad(S, tv, ti, lse, None),
                lambda: api.mosaic_distill_grad(S, tv, ti, lse, dS.bfloat16())):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: api.mosaic_distill_loss(S, tv, ti[:, :9], loss), lambda: api.mosaic_distill_loss(S, tv[:3], ti, loss),
                lambda: api.mosaic_distill_loss(S, tv, ti, loss[:3]), lambda: api.mosaic_distill_grad(S, tv, ti, lse, dS[:, :99])):
        with pytest.raises(ValueError):
            bad()
