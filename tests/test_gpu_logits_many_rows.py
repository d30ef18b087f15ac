"""Top logits and distillation with so many rows that the calls take other kernels than for a few: a row a warp (from
20 rows an SM on) or a row of 128 threads (above 5 an SM), and CTAs past the first wave of the distillation's pass (three
an SM).  Rows of every kind lie side by side, as four of them share a CTA where a warp has one.  Helpers and bounds of
test_gpu_logits.py."""
import pytest
import torch

from paper_2504_06323_b200 import api
from test_gpu_logits import INF, check_distill, check_top, logits, teacher

pytestmark = pytest.mark.gpu
DEV = "cuda"


def sms():
    return torch.cuda.get_device_properties(0).multi_processor_count


def row_counts():
    n = sms()
    # one row more than the limits, none a multiple of four; one row a CTA of 128 threads and four short of the next
    return {"a CTA a row": 5 * n + 1, "a CTA a row, more": 8 * n + 17, "a warp a row": 20 * n + 1, "a warp a row, more": 27 * n + 3}


def spoil(x, dtype, first, step=5):
    """Every `step`-th row from `first` on is of another kind, so that each kind meets every place in a group of four."""
    rows, cols = x.shape
    g = torch.Generator(device=DEV).manual_seed(cols)
    kinds = ["nan", "all masked", "few left", "one value", "ties", "lowest", "inf", "zeros", "descending", "many nan", "some hundred ties",
             "ascending"]
    for i, r in enumerate(range(first, rows, step)):
        kind = kinds[i % len(kinds)]
        if kind == "nan":
            x[r, (7 * r) % cols] = float("nan")
        elif kind == "all masked":
            x[r] = -INF
        elif kind == "few left":
            x[r, 3:] = -INF
        elif kind == "one value":
            x[r] = torch.finfo(dtype).max
        elif kind == "ties":
            x[r] = torch.randint(-2, 3, (cols,), generator=g, device=DEV).to(dtype)
        elif kind == "lowest":
            x[r] = torch.finfo(dtype).min
            x[r, cols // 2] = 1.0
        elif kind == "inf":
            x[r, ::50] = INF
        elif kind == "zeros":
            x[r] = 0.0
            x[r, ::2] = -0.0
        elif kind == "descending":
            x[r] = -torch.arange(cols, device=DEV, dtype=torch.float32) * 0.01
        elif kind == "many nan":
            x[r, ::3] = float("nan")
        elif kind == "some hundred ties":      # more equal candidates than kept, fewer than the list holds
            x[r, :] = -5.0
            x[r, : min(cols, 300 + r % 200)] = 9.0
        else:
            x[r] = torch.arange(cols, device=DEV, dtype=torch.float32) * 0.01
    return x


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("which", list(row_counts()) if torch.cuda.is_available() else ["a CTA a row"])
@pytest.mark.parametrize("cols,top", [(1003, 1), (1003, 20), (1003, 64), (1003, 128), (1003, 256), (1600, 400), (3001, 1000), (200, 200), (7, 3)])
def test_top_many_rows(which, cols, top, dtype):
    rows = row_counts()[which]
    if cols > 2000:
        rows = min(rows, 8 * sms() + 17)     # the reference sorts on the host
    x = spoil(logits(rows, cols, dtype, rows + cols), dtype, first=rows % 4)
    check_top(x, top)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols,top", [(33001, 64), (33001, 200)])
def test_top_many_long_rows(cols, top, dtype):
    """Groups of 128 bytes (a few kept of many) under each kernel, most rows ordinary; against a sort on the device."""
    for rows in (5 * sms() + 2, 20 * sms() + 2):
        x = spoil(logits(rows, cols, dtype, top), dtype, first=1, step=97)
        values, indices, lse = (torch.full((rows, top), -7.0, device=DEV), torch.full((rows, top), -7, device=DEV, dtype=torch.int32),
                                torch.full((rows,), -7.0, device=DEV))
        api.mosaic_top_logits(x, values, indices, lse)
        for r0 in range(0, rows, 512):
            part = x[r0:r0 + 512].float()
            nan = part.isnan()
            key = torch.where(nan, INF, part)
            # NaN first: sorted by (NaN, value descending), both stable in the index
            order = torch.sort(key, dim=1, descending=True, stable=True).indices
            order = order.gather(1, torch.sort(nan.gather(1, order).int(), dim=1, descending=True, stable=True).indices)[:, :top]
            assert torch.equal(indices[r0:r0 + 512].long(), order)
            assert torch.equal(values[r0:r0 + 512].view(torch.int32), part.gather(1, order).view(torch.int32))
            ref = torch.logsumexp(part.double(), 1)
            fine = torch.isfinite(ref)
            got = lse[r0:r0 + 512].double()
            assert ((got - ref).abs()[fine] <= 2.0 ** -17 + 2.0 ** -24 * ref.abs()[fine]).all()
            assert torch.equal(got[~fine].isnan(), ref[~fine].isnan())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("vocab,top", [(701, 24), (701, 300), (4100, 128)])
def test_distill_past_the_first_wave(dtype, given, vocab, top):
    rows = 7 * sms() + 3
    S = logits(rows, vocab, dtype, vocab)
    tv, ti, t_lse = teacher(S, top, 4, 2.0, given)
    g = torch.Generator(device=DEV).manual_seed(6)
    weight = (torch.rand(rows, generator=g, device=DEV) + 0.25) * (torch.rand(rows, generator=g, device=DEV) > 0.2)
    weight[5::11] = 0.0
    S[5::11] = float("nan")                       # dropped: what they hold must not matter
    ti[1::13] = -1                                # no entry at all
    ti[2::13, ::2] = vocab + 5                    # half of the entries outside the vocabulary
    if not given:
        ti[3::13, 1] = ti[3::13, 0]               # an entry kept twice
    tv[4::13] = -INF                              # all kept logits masked
    gr = torch.rand(rows, generator=g, device=DEV) + 0.1
    loss, lse, a, b = check_distill(S, tv, ti, t_lse, weight, T=2.0, grad_rows=gr, grad_scale=0.5)
    kw = dict(t_lse=t_lse, row_weight=weight, temperature=2.0, grad_rows=gr, grad_scale=0.5)
    for grad, want in ((False, a), (True, b)):    # in place
        buf = S.clone()
        if grad:
            api.mosaic_distill_grad(buf, tv, ti, lse, buf, **kw)
        else:
            l2 = torch.empty_like(loss)
            api.mosaic_distill_loss_grad(buf, tv, ti, l2, None, buf, **kw)
            assert torch.equal(l2, loss)
        assert torch.equal(buf, want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_distill_clusters_past_the_first_wave(dtype):
    """Rows shared by several CTAs, more of them than run at once."""
    rows, vocab = 2 * sms() + 5, 70001
    S = logits(rows, vocab, dtype, 1)
    tv, ti, t_lse = teacher(S, 64, 2, 1.0, True)
    weight = torch.ones(rows, device=DEV)
    weight[3::7] = 0.0
    S[3::7] = float("nan")
    ti[1::13] = -1
    _, lse, a, b = check_distill(S, tv, ti, t_lse, weight)
    buf, l2 = S.clone(), torch.empty(rows, device=DEV)
    api.mosaic_distill_loss_grad(buf, tv, ti, l2, None, buf, t_lse=t_lse, row_weight=weight)
    assert torch.equal(buf, a)
