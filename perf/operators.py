"""The operators that bring a pruned model back, as cases to measure.

Pruning (this framework's path) leaves smaller dense projections and a model whose answers have moved.
What a user does next is run those projections, forward and backward, against what the foundation model
answered:

* ``linear`` / ``linear_backward``: a projection's matrix product with bias, activation and residual in
  its epilogue, ``Y = act(X W^T + b) + R``, and its gradients ``dX``, ``dW``, ``db``;
* ``top_logits``: the k largest logits of every row of the teacher (ties to the lowest index), in order,
  with the log-sum-exp of the whole row - all that has to be kept of the teacher's answer;
* ``distill``: the divergence of the student's distribution from those top logits, per row, and its
  gradient with respect to the student's logits.

`own` false computes them in their plain form (elementary torch operations in 32 bits, rounded once at the
end); `own` true makes the calls a user of the framework makes.  Sizes are the framework's projection shapes
(hidden 256 / 4096 / 5120, intermediate 688 / 11008 / 13824 / 14336, and 8807 = 11008 with a fifth of the
channels compacted away), the rest is generic: vocabularies of about 1000 to 131072, 1 to 4096 rows.
"""
import math

import numpy as np
import torch

own = False

LISTED = [
    # a tiny decoder block's up projection for a short prompt: every call is launch latency
    dict(name="linear_tiny_block", op="linear", m=128, n=688, k=256, act="relu", bias=True, residual=False, save=False, pitch=False),
    # one token through the gate projection of the 7B shape: the weights are read once, for one row
    dict(name="linear_one_token_gate", op="linear", m=1, n=11008, k=4096, act="silu", bias=False, residual=False, save=False, pitch=False),
    # a few dozen sequences' next tokens through a down projection with 20 % of its channels compacted
    # away, added to the residual stream: an odd contraction length
    dict(name="linear_tokens_down_compacted", op="linear", m=37, n=4096, k=8807, act="none", bias=False, residual=True, save=False, pitch=True),
    # a training sequence through a gate projection; the pre-activation is kept for the backward pass
    dict(name="linear_sequence_gate", op="linear", m=2048, n=14336, k=4096, act="silu", bias=True, residual=False, save=True, pitch=False),
    # backward of a compacted gate projection on a ragged batch of tokens
    dict(name="linear_backward_compacted_gate", op="linear_backward", m=1001, n=8807, k=4096, act="silu", bias=True, pitch=True),
    # backward of the widest down projection (13B shape) for two training sequences: the largest products
    dict(name="linear_backward_down", op="linear_backward", m=4096, n=5120, k=13824, act="none", bias=False, pitch=False),
    # the next-token logits of one sequence
    dict(name="top_logits_one_row", op="top_logits", rows=1, vocab=32000, top=20, dtype="f32", masked=0, temperature=1.0),
    # a teacher's answers to two training sequences, stored for distillation
    dict(name="top_logits_sequences", op="top_logits", rows=4096, vocab=32000, top=64, dtype="bf16", masked=0, temperature=2.0),
    # an odd vocabulary in fp32, dense rows of any alignment, the padding entries masked with -inf
    dict(name="top_logits_odd_vocabulary", op="top_logits", rows=301, vocab=50001, top=100, dtype="f32", masked=129, temperature=1.0),
    # the loss alone on a small evaluation batch, probabilities renormalised over the kept logits
    dict(name="distill_loss_evaluation", op="distill_loss", rows=64, vocab=32003, top=50, dtype="f32", renorm=True, dropped=0.1, temperature=1.0),
    # the training step's loss and gradient in one call, at a temperature, with padding tokens
    dict(name="distill_training_step", op="distill_loss_grad", rows=4096, vocab=32000, top=64, dtype="bf16", renorm=False, dropped=0.05, temperature=2.0),
    # the gradient on its own, from the saved log-sum-exp and a gradient per row, over a wide vocabulary
    dict(name="distill_gradient_wide", op="distill_grad", rows=1024, vocab=131072, top=256, dtype="bf16", renorm=True, dropped=0.0, temperature=1.0),
]


def listed():
    return [dict(c) for c in LISTED]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread evenly over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["linear", "linear", "linear_backward", "top_logits", "distill_loss", "distill_loss_grad", "distill_grad"])
    if op in ("linear", "linear_backward"):
        while True:
            m, n, k = _spread(rng, 1, 4096), _spread(rng, 64, 14336), _spread(rng, 64, 14336)
            work = m * n * k * (2 if op == "linear_backward" else 1)
            if 3072 not in (m, n, k) and work <= 2 * 4096 * 5120 * 13824 and (n * k >= 1 << 16):
                break
        case = dict(op=op, m=m, n=n, k=k, act=rng.choice(["none", "relu", "gelu", "silu"]), bias=rng.random() < 0.5, pitch=rng.random() < 0.7)
        if op == "linear":
            case |= dict(residual=rng.random() < 0.5, save=rng.random() < 0.3)
        return case
    dtype = rng.choice(["bf16", "f32"])
    while True:
        rows, vocab = _spread(rng, 1, 4096), _spread(rng, 1000, 131072)
        if 3072 not in (rows, vocab) and rows * vocab * (2 if dtype == "bf16" else 4) <= 4096 * 32000 * 2:
            break
    case = dict(op=op, rows=rows, vocab=vocab, top=_spread(rng, 1, 256), dtype=dtype, temperature=rng.choice([1.0, 1.0, 2.0, 4.0]))
    if op == "top_logits":
        case["masked"] = rng.choice([0, 0, 1, 100])
    else:
        case |= dict(renorm=rng.random() < 0.5, dropped=rng.choice([0.0, 0.05, 0.3]))
    return case


# ------------------------------------------------------------------ what a program has in hand
def _pitched(rows, cols, pitch, dtype=torch.bfloat16):
    """An empty matrix; with `pitch` its rows start on 16-byte boundaries, else they follow one another."""
    ld = (cols + 7) // 8 * 8 if pitch else cols
    return torch.empty(rows, ld, device="cuda", dtype=dtype)[:, :cols]


def _prepare_linear(case, g):
    m, n, k, pitch = case["m"], case["n"], case["k"], case["pitch"]
    randn = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    X, W = _pitched(m, k, pitch), _pitched(n, k, pitch)
    x = randn(m, k)
    x[:, torch.randperm(k, generator=g, device="cuda")[: max(1, k // 200)]] *= 10.0   # outlier channels
    X.copy_(x)
    W.copy_(randn(n, k) * (1.2 / math.sqrt(k)))
    st = dict(case=case, X=X, W=W, bias=None, residual=None, Z=None)
    if case["bias"]:
        st["bias"] = (randn(n) * 0.5).to(torch.bfloat16)
    if case["op"] == "linear":
        st["Y"] = _pitched(m, n, pitch)
        if case["residual"]:
            st["residual"] = _pitched(m, n, pitch)
            st["residual"].copy_(randn(m, n))
        if case["save"]:
            st["Z"] = _pitched(m, n, pitch)
        return st
    st["dY"] = _pitched(m, n, pitch)
    st["dY"].copy_(randn(m, n) * 0.01)
    if case["act"] != "none":
        st["Z"] = _pitched(m, n, pitch)
        st["Z"].copy_(randn(m, n) * 1.5)
    st["dX"], st["dW"] = _pitched(m, k, pitch), _pitched(n, k, pitch)
    st["db"] = torch.empty(n, device="cuda", dtype=torch.bfloat16) if case["bias"] else None
    return st


def _logits(rows, vocab, g):
    """Logits as a model gives them: a broad body, a few likely tokens, rows of different sharpness."""
    x = torch.randn(rows, vocab, generator=g, device="cuda") * 2.0
    x *= 0.6 + torch.rand(rows, 1, generator=g, device="cuda")
    likely = torch.randint(0, vocab, (rows, 8), generator=g, device="cuda")
    x.scatter_add_(1, likely, 6.0 * torch.rand(rows, 8, generator=g, device="cuda"))
    return x


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if case["op"] in ("linear", "linear_backward"):
        return _prepare_linear(case, g)
    rows, vocab, top = case["rows"], case["vocab"], case["top"]
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    teacher = _logits(rows, vocab, g)
    f32 = lambda *shape: torch.empty(*shape, device="cuda")  # noqa: E731
    if case["op"] == "top_logits":
        if case["masked"]:
            teacher[:, vocab - case["masked"]:] = -math.inf
        return dict(case=case, L=teacher.to(dtype), values=f32(rows, top), indices=torch.empty(rows, top, device="cuda", dtype=torch.int32),
                    lse=f32(rows))
    T = case["temperature"]
    values, indices = torch.topk(teacher, top, dim=1)
    t_lse = None if case["renorm"] else torch.logsumexp(teacher / T, dim=1)
    teacher += torch.randn(rows, vocab, generator=g, device="cuda")      # the student: the teacher, moved
    S = teacher.to(dtype)
    st = dict(case=case, S=S, t_values=values.float().contiguous(), t_indices=indices.to(torch.int32), t_lse=t_lse,
              row_weight=(torch.rand(rows, generator=g, device="cuda") >= case["dropped"]).float() if case["dropped"] else None,
              loss=f32(rows), lse=f32(rows), grad_rows=None, dS=None)
    if case["op"] != "distill_loss":
        st["dS"] = torch.empty_like(S)
    if case["op"] == "distill_grad":
        st["lse"].copy_(torch.logsumexp(S.float() / T, dim=1))
        st["grad_rows"] = torch.rand(rows, generator=g, device="cuda") / rows
    return st


# ------------------------------------------------------------------ one pass
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(st):
    from paper_2504_06323_b200 import api
    case = st["case"]
    op = case["op"]
    if op == "linear":
        api.mosaic_linear(st["X"], st["W"], st["Y"], bias=st["bias"], residual=st["residual"], act=case["act"], Z=st["Z"])
        return st["Y"], st["Z"]
    if op == "linear_backward":
        api.mosaic_linear_backward(st["dY"], st["X"], st["W"], Z=st["Z"], act=case["act"], dX=st["dX"], dW=st["dW"], dbias=st["db"])
        return st["dX"], st["dW"], st["db"]
    T = case["temperature"]
    if op == "top_logits":
        api.mosaic_top_logits(st["L"], st["values"], st["indices"], st["lse"], temperature=T)
        return st["values"], st["indices"], st["lse"]
    teacher = dict(t_lse=st["t_lse"], row_weight=st["row_weight"], temperature=T)
    if op == "distill_loss":
        api.mosaic_distill_loss(st["S"], st["t_values"], st["t_indices"], st["loss"], st["lse"], **teacher)
        return st["loss"], st["lse"]
    if op == "distill_loss_grad":
        api.mosaic_distill_loss_grad(st["S"], st["t_values"], st["t_indices"], st["loss"], st["lse"], st["dS"], grad_scale=1.0 / case["rows"], **teacher)
        return st["loss"], st["lse"], st["dS"]
    api.mosaic_distill_grad(st["S"], st["t_values"], st["t_indices"], st["lse"], st["dS"], grad_rows=st["grad_rows"], **teacher)
    return st["dS"]


def _act(z, act):
    if act == "relu":
        return z.clamp(min=0.0)
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    return torch.ones_like(z)


def _top_plain(x, top):
    """The `top` largest of each row, ties to the lowest index: one whole-number key an entry, value first."""
    vocab = x.shape[1]
    bits = (x + 0.0).view(torch.int32)
    order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
    last = torch.arange(vocab - 1, -1, -1, device=x.device)
    keys, _ = torch.topk(order * (1 << 32) + last, top, dim=1)
    indices = vocab - 1 - (keys & 0xFFFFFFFF)
    return x.gather(1, indices), indices.to(torch.int32)


def _teacher_probabilities(values, indices, t_lse, vocab, T):
    """(p, log p, sum of p) of the kept logits; entries outside the vocabulary are absent."""
    u = torch.where((indices >= 0) & (indices < vocab), values / T, -math.inf)
    if t_lse is None:
        top = u.amax(dim=1, keepdim=True).clamp(min=torch.finfo(u.dtype).min)
        norm = top + torch.log(torch.exp(u - top).sum(dim=1, keepdim=True))
    else:
        norm = t_lse[:, None]
    log_p = torch.where(u > -math.inf, u - norm, -math.inf)
    p = torch.exp(log_p)
    return p, log_p, p.sum(dim=1)


def _run_plain(st):
    case = st["case"]
    op = case["op"]
    if op == "linear":
        z = st["X"].float() @ st["W"].float().T
        if st["bias"] is not None:
            z = z + st["bias"].float()
        y = _act(z, case["act"])
        if st["residual"] is not None:
            y = y + st["residual"].float()
        return y.to(torch.bfloat16), (z.to(torch.bfloat16) if case["save"] else None)
    if op == "linear_backward":
        dz = st["dY"].float()
        if case["act"] != "none":
            dz = dz * _act_slope(st["Z"].float(), case["act"])
        dX, dW = dz @ st["W"].float(), dz.T @ st["X"].float()
        db = dz.sum(dim=0).to(torch.bfloat16) if case["bias"] else None
        return dX.to(torch.bfloat16), dW.to(torch.bfloat16), db
    T = case["temperature"]
    if op == "top_logits":
        x = st["L"].float()
        values, indices = _top_plain(x, case["top"])
        m = values[:, :1]
        lse = (m / T)[:, 0] + torch.log(torch.exp((x - m) / T).sum(dim=1))
        return values, indices, lse
    vocab, rows = case["vocab"], case["rows"]
    x = st["S"].float() / T
    p, log_p, mass = _teacher_probabilities(st["t_values"], st["t_indices"], st["t_lse"], vocab, T)
    weight = torch.ones(rows, device=x.device) if st["row_weight"] is None else st["row_weight"]
    at = st["t_indices"].long().clamp(0, vocab - 1)
    out = ()
    if op == "distill_grad":
        lse = st["lse"]
        coef = st["grad_rows"] * weight * T
    else:
        m = x.amax(dim=1)
        lse = m + torch.log(torch.exp(x - m[:, None]).sum(dim=1))
        term = torch.where(p > 0, p * (log_p - (x.gather(1, at) - lse[:, None])), 0.0)
        loss = torch.where(weight != 0, weight * (T * T) * term.sum(dim=1), 0.0)
        out = (loss, lse)
        if op == "distill_loss":
            return out
        coef = weight * (T / rows)
    d = torch.exp(x - lse[:, None]) * mass[:, None]
    d.scatter_add_(1, at, -p)
    d = torch.where((coef != 0)[:, None], d * coef[:, None], 0.0).to(st["S"].dtype)
    return (*out, d) if out else d


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    if case["op"] in ("linear", "linear_backward"):
        m, n, k = case["m"], case["n"], case["k"]
        back = case["op"] == "linear_backward"
        elements = m * k + n * k + m * n + (n if case["bias"] else 0)
        if back:
            elements += m * k + n * k + (m * n if case["act"] != "none" else 0)
        else:
            elements += (m * n if case["residual"] else 0) + (m * n if case["save"] else 0)
        return {"bytes": 2 * elements, "flops": (4 if back else 2) * m * n * k}
    cells, size = case["rows"] * case["vocab"], 2 if case["dtype"] == "bf16" else 4
    kept = case["rows"] * case["top"] * 8
    if case["op"] == "top_logits":
        return {"bytes": cells * size + kept + 4 * case["rows"], "flops": 4 * cells}
    passes = 1 if case["op"] == "distill_loss" else 2
    return {"bytes": passes * cells * size + kept + 16 * case["rows"], "flops": 4 * passes * cells}


# ------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    d = lambda t: None if t is None else t.double()  # noqa: E731
    if case["op"] in ("linear", "linear_backward"):
        X, W = d(st["X"]), d(st["W"])
        act = {"none": lambda z: z, "relu": torch.relu, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu}[case["act"]]
        if case["op"] == "linear":
            z = torch.einsum("mk,nk->mn", X, W) + (0 if st["bias"] is None else d(st["bias"]))
            y = act(z) + (0 if st["residual"] is None else d(st["residual"]))
            return y, (z if case["save"] else None)
        dz = d(st["dY"])
        if case["act"] != "none":
            z = d(st["Z"]).requires_grad_(True)
            dz, = torch.autograd.grad(act(z), z, dz)
        return torch.einsum("mn,nk->mk", dz, W), torch.einsum("mn,mk->nk", dz, X), (dz.sum(0) if case["bias"] else None)
    T = case["temperature"]
    if case["op"] == "top_logits":
        x = d(st["L"])
        values, indices = torch.sort(x, dim=1, descending=True, stable=True)
        return values[:, : case["top"]].clone(), indices[:, : case["top"]].to(torch.int32), torch.logsumexp(x / T, dim=1)
    # row by row groups, from the definition: KL of the student's softmax from the kept part of the teacher's
    rows, vocab = case["rows"], case["vocab"]
    weight = np.ones(rows) if st["row_weight"] is None else st["row_weight"].double().cpu().numpy()
    losses, lses, grads = [], [], []
    for r0 in range(0, rows, 256):
        r = slice(r0, min(rows, r0 + 256))
        w = torch.from_numpy(weight[r]).cuda()
        x = d(st["S"][r]) / T
        dense = torch.zeros_like(x)
        u = d(st["t_values"][r]) / T
        p = torch.softmax(u, dim=1) if st["t_lse"] is None else torch.exp(u - d(st["t_lse"][r])[:, None])
        dense.scatter_add_(1, st["t_indices"][r].long(), p)
        if case["op"] == "distill_grad":
            lse = d(st["lse"][r])
            coef = d(st["grad_rows"][r]) * w * T
        else:
            lse = torch.logsumexp(x, dim=1)
            coef = w * T / rows
        losses.append(w * T * T * (torch.xlogy(dense, dense) - dense * (x - lse[:, None])).sum(1))
        lses.append(lse)
        if case["op"] != "distill_loss":
            grads.append(coef[:, None] * (torch.exp(x - lse[:, None]) * p.sum(1, keepdim=True) - dense))
    if case["op"] == "distill_loss":
        return torch.cat(losses), torch.cat(lses)
    if case["op"] == "distill_grad":
        return torch.cat(grads)
    return torch.cat(losses), torch.cat(lses), torch.cat(grads)
