"""The operators that train and serve a pruned model's gated MLP, as cases to measure.

The models that this framework prunes compute ``down(act(gate(X)) * up(X))``.  What recovery and deployment run of it:

* ``gated`` / ``gated_backward`` / ``gated_step``: ``H = act(X Wg^T + bg) * (X Wu^T + bu)`` as one operator, its
  gradients ``dX``, ``dWg``, ``dWu``, ``dbg``, ``dbu`` (and H once more, from what was kept), and both in a row as a
  training step makes them;
* ``checkpoint``: activations kept in 8 bits between the two passes - 16 adjacent columns share an exponent ``E``, a
  value is a code in -127..127 times ``2^(E - 133)`` - stored and loaded; ``gated_backward`` also reads them as they are;
* ``quantize4``: a weight matrix in 4 bits - `group` adjacent columns share a scale of five significant bits, a value
  is a code in -7..7 times it, zeros stay zeros - packed and unpacked;
* ``linear4`` / ``gated4``: a projection, or the gated pair of them, with such weights, for the next tokens of one
  sequence or many.

`own` false computes them in their plain form (elementary torch operations in 32 bits, rounded once at the end); `own`
true makes the calls a user of the framework makes.  Sizes are the framework's projection shapes (hidden 256 / 4096 /
5120, intermediate 688 / 11008 / 13824 / 14336, and 8807 = 11008 with a fifth of the channels compacted away); tokens
from one to 4096.
"""
import math

import torch

own = False

LISTED = [
    # a tiny decoder block's MLP for a short prompt: every call is launch latency
    dict(name="gated_tiny_prompt", op="gated", m=128, n=688, k=256, act="silu", bias=False, save=False, pitch=True),
    # the next token of one sequence through the 7B shape: two weight matrices are read once, for one row
    dict(name="gated_one_token", op="gated", m=1, n=11008, k=4096, act="silu", bias=False, save=False, pitch=True),
    # a training sequence through the widest MLP; what the backward pass needs is kept as it is
    dict(name="gated_sequence", op="gated", m=2048, n=14336, k=4096, act="silu", bias=False, save=True, pitch=True),
    # backward of a compacted MLP with biases on a ragged batch of tokens; dense rows of an odd width
    dict(name="gated_backward_compacted", op="gated_backward", m=1001, n=8807, k=4096, act="silu", bias=True, saved8=False, again=False, pitch=False),
    # backward of the 13B shape from 8-bit activations, H computed once more for the projection behind it
    dict(name="gated_backward_saved8", op="gated_backward", m=2048, n=13824, k=5120, act="silu", bias=False, saved8=True, again=True, pitch=True),
    # a training step of the 7B shape over two sequences that keeps its activations in 8 bits: the largest work
    dict(name="gated_step_saved8", op="gated_step", m=4096, n=11008, k=4096, act="silu", bias=False, pitch=True),
    # the tokens of two sequences at the widest place of the 13B shape, stored and loaded
    dict(name="checkpoint_sequences", op="checkpoint", m=4096, n=13824, pitch=True),
    # a few dozen tokens of a compacted MLP, dense rows of an odd width
    dict(name="checkpoint_compacted", op="checkpoint", m=37, n=8807, pitch=False),
    # a gate projection of the 7B shape, half of it pruned away, packed for serving
    dict(name="quantize4_gate", op="quantize4", n=11008, k=4096, group=128, pitch=True),
    # a compacted down projection with an odd contraction length, in fine groups
    dict(name="quantize4_down_compacted", op="quantize4", n=4096, k=8807, group=32, pitch=False),
    # the next token of one sequence through gate and up in 4 bits
    dict(name="gated4_one_token", op="gated4", m=1, n=11008, k=4096, act="silu", bias=False, group=128, pitch=True),
    # sixteen sequences' next tokens through a compacted down projection in 4 bits, added to the residual stream
    dict(name="linear4_tokens_down_compacted", op="linear4", m=16, n=4096, k=8807, act="none", bias=False, residual=True, group=64, pitch=True),
]


def listed():
    return [dict(c) for c in LISTED]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread evenly over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["gated", "gated", "gated_backward", "gated_backward", "gated_step", "checkpoint", "quantize4", "linear4", "gated4"])
    act, bias, pitch = rng.choice(["silu", "silu", "gelu", "relu", "none"]), rng.random() < 0.4, rng.random() < 0.7
    if op == "checkpoint":
        return dict(op=op, m=_spread(rng, 1, 4096), n=_spread(rng, 64, 14336), pitch=pitch)
    while True:
        m, n, k = _spread(rng, 1, 512 if op in ("linear4", "gated4") else 4096), _spread(rng, 64, 14336), _spread(rng, 64, 14336)
        passes = {"gated_backward": 2, "gated_step": 3}.get(op, 1)
        if n * k >= 1 << 16 and m * n * k * passes <= 3 * 4096 * 11008 * 4096:
            break
    if op == "quantize4":
        return dict(op=op, n=n, k=k, group=rng.choice([32, 64, 128]), pitch=pitch)
    case = dict(op=op, m=m, n=n, k=k, act=act, bias=bias, pitch=pitch)
    if op == "gated":
        case |= dict(save=rng.random() < 0.4)
    elif op == "gated_backward":
        case |= dict(saved8=rng.random() < 0.5, again=rng.random() < 0.5)
    elif op in ("linear4", "gated4"):
        case |= dict(group=rng.choice([32, 64, 128]))
        if op == "linear4":
            case |= dict(residual=rng.random() < 0.5)
    return case


# ------------------------------------------------------------------ what a program has in hand
def _matrix(rows, cols, pitch, values=None):
    """A bf16 matrix; with `pitch` its rows start on 16-byte boundaries, else they follow one another."""
    ld = (cols + 7) // 8 * 8 if pitch else cols
    m = torch.empty(rows, ld, device="cuda", dtype=torch.bfloat16)[:, :cols]
    if values is not None:
        m.copy_(values)
    return m


def _activations(rows, cols, g):
    """N(0, 1) with half a percent of outlier channels."""
    x = torch.randn(rows, cols, generator=g, device="cuda")
    x[:, torch.randperm(cols, generator=g, device="cuda")[: max(1, cols // 200)]] *= 10.0
    return x


def _weights(rows, cols, g, pruned=0.0):
    """Heavy-tailed weights, a part of them zero."""
    w = torch.randn(rows, cols, generator=g, device="cuda")
    w *= (1.0 + 0.5 * torch.randn(rows, cols, generator=g, device="cuda") ** 2) * (0.7 / math.sqrt(cols))
    if pruned:
        w.masked_fill_(torch.rand(rows, cols, generator=g, device="cuda") < pruned, 0.0)
    return w


def _empty8(rows, cols):
    return (torch.zeros(rows, (cols + 15) // 16 * 16, device="cuda", dtype=torch.int8),
            torch.zeros(rows, (cols + 15) // 16, device="cuda", dtype=torch.uint8))


def _empty4(rows, cols, group):
    return (torch.zeros(rows, (cols + 31) // 32 * 16, device="cuda", dtype=torch.uint8),
            torch.zeros(rows, (cols + group - 1) // group, device="cuda", dtype=torch.bfloat16))


def _own8(state, name, cols):
    if own:
        from paper_2504_06323_b200 import api
        state[name + "_handle"] = api.Checkpoint(*state[name], cols)


def _own4(state, name, cols, group):
    if own:
        from paper_2504_06323_b200 import api
        state[name + "_handle"] = api.Weight4(*state[name], cols, group)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op, n, pitch = case["op"], case["n"], case["pitch"]
    st = dict(case=case)
    if op == "checkpoint":
        st["X"], st["out"] = _matrix(case["m"], n, pitch, _activations(case["m"], n, g)), _matrix(case["m"], n, pitch)
        st["kept"] = _empty8(case["m"], n)
        _own8(st, "kept", n)
        return st
    k = case["k"]
    if op == "quantize4":
        st["W"], st["out"] = _matrix(n, k, pitch, _weights(n, k, g, 0.5)), _matrix(n, k, pitch)
        st["W4"] = _empty4(n, k, case["group"])
        _own4(st, "W4", k, case["group"])
        return st
    m = case["m"]
    st["X"] = _matrix(m, k, pitch, _activations(m, k, g))
    vector = lambda: (torch.randn(n, generator=g, device="cuda") * 0.5).to(torch.bfloat16) if case["bias"] else None  # noqa: E731
    if op in ("linear4", "gated4"):
        for name in ("W",) if op == "linear4" else ("Wg", "Wu"):
            codes, scales = _empty4(n, k, case["group"])
            c, s = _quantize4(_weights(n, k, g, 0.5).to(torch.bfloat16), case["group"])
            codes.copy_(_pack(c, codes.shape[1]))
            scales.copy_(s)
            st[name] = (codes, scales)
            _own4(st, name, k, case["group"])
        st["Y"] = _matrix(m, n, pitch)
        st["residual"] = _matrix(m, n, pitch, torch.randn(m, n, generator=g, device="cuda")) if case.get("residual") else None
        st["bias"] = vector()
        st["bias2"] = vector() if op == "gated4" else None
        return st
    st["Wg"], st["Wu"] = _matrix(n, k, pitch, _weights(n, k, g)), _matrix(n, k, pitch, _weights(n, k, g))
    if op in ("gated", "gated_step"):
        st["bg"], st["bu"] = vector(), vector()
        st["H"] = _matrix(m, n, pitch)
    if op == "gated":
        st["Z"], st["U"] = (_matrix(m, n, pitch), _matrix(m, n, pitch)) if case["save"] else (None, None)
        return st
    st["dH"] = _matrix(m, n, pitch, torch.randn(m, n, generator=g, device="cuda") * 0.01)
    st["dX"], st["dWg"], st["dWu"] = _matrix(m, k, pitch), _matrix(n, k, pitch), _matrix(n, k, pitch)
    st["dbg"], st["dbu"] = ((torch.empty(n, device="cuda", dtype=torch.bfloat16) for _ in range(2)) if case["bias"] else (None, None))
    if op == "gated_step":
        st["X8"], st["Z8"], st["U8"] = _empty8(m, k), _empty8(m, n), _empty8(m, n)
    else:
        st["H"] = _matrix(m, n, pitch) if case["again"] else None
        st["Z"] = _matrix(m, n, pitch, torch.randn(m, n, generator=g, device="cuda") * 1.5)
        st["U"] = _matrix(m, n, pitch, torch.randn(m, n, generator=g, device="cuda") * 1.5)
        if case["saved8"]:
            for name in ("X", "Z", "U"):
                x = st.pop(name)
                kept = st[name + "8"] = _empty8(*x.shape)
                codes, exponents = _encode8(x)
                kept[0].copy_(codes)
                kept[1].copy_(exponents)
    for name, cols in (("X8", k), ("Z8", n), ("U8", n)):
        if name in st:
            _own8(st, name, cols)
    return st


# ------------------------------------------------------------------ one pass
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(st):
    from paper_2504_06323_b200 import api
    case = st["case"]
    op = case["op"]
    if op == "checkpoint":
        api.mosaic_checkpoint_store(st["X"], st["kept_handle"])
        api.mosaic_checkpoint_load(st["kept_handle"], st["out"])
        return st["out"]
    if op == "quantize4":
        api.mosaic_quantize4(st["W"], st["W4_handle"])
        api.mosaic_dequantize4(st["W4_handle"], st["out"])
        return st["out"]
    act = case["act"]
    if op == "linear4":
        api.mosaic_linear4(st["X"], st["W_handle"], st["Y"], bias=st["bias"], residual=st["residual"], act=act)
        return st["Y"]
    if op == "gated4":
        api.mosaic_gated_linear4(st["X"], st["Wg_handle"], st["Wu_handle"], st["Y"], bias_gate=st["bias"], bias_up=st["bias2"], act=act)
        return st["Y"]
    if op == "gated":
        api.mosaic_gated_linear(st["X"], st["Wg"], st["Wu"], st["H"], bias_gate=st["bg"], bias_up=st["bu"], act=act, Z=st["Z"], U=st["U"])
        return st["H"], st["Z"], st["U"]
    if op == "gated_step":
        api.mosaic_checkpoint_store(st["X"], st["X8_handle"])
        api.mosaic_gated_linear(st["X"], st["Wg"], st["Wu"], st["H"], bias_gate=st["bg"], bias_up=st["bu"], act=act,
                                Z=st["Z8_handle"], U=st["U8_handle"])
    X, Z, U = (st[name + "8_handle"] if name + "8" in st else st[name] for name in ("X", "Z", "U"))
    api.mosaic_gated_linear_backward(st["dH"], X, st["Wg"], st["Wu"], Z, U, act=act, dX=st["dX"], dW_gate=st["dWg"], dW_up=st["dWu"],
                                     dbias_gate=st["dbg"], dbias_up=st["dbu"], H=st["H"] if op == "gated_backward" else None)
    return st["dX"], st["dWg"], st["dWu"], st["dbg"], st["dbu"], st["H"]


# the plain forms
def _groups(x, size):
    """[rows, groups, size] in 32 bits, zeros behind the last column."""
    rows, cols = x.shape
    return torch.nn.functional.pad(x.float(), (0, -cols % size)).view(rows, -1, size)


def _power(e):
    """2^e in 32 bits, from its bits: exp2 need not be exact."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _times_power(x, e):
    """x 2^e for |e| up to 250, in two steps that stay in range."""
    half = torch.div(e, 2, rounding_mode="floor")
    return x * _power(half) * _power(e - half)


def _encode8(x):
    g = _groups(x, 16)
    largest = torch.where(torch.isfinite(g), g.abs(), 0.0).amax(dim=2)
    exponent = (torch.frexp(largest).exponent + 126).clamp(min=1)            # the biased exponent of the largest finite value
    code = torch.round(_times_power(g, 133 - exponent[..., None])).clamp(-127, 127)
    code = torch.where(torch.isfinite(g), code, -128.0)
    return code.flatten(1).to(torch.int8), exponent.to(torch.uint8)


def _decode8(kept, cols):
    codes, exponents = kept
    c = codes.float().view(codes.shape[0], -1, 16)
    v = _times_power(c, exponents.int()[..., None] - 133)
    return torch.where(c == -128, math.nan, v).flatten(1)[:, :cols]


def _quantize4(W, group):
    g = _groups(W, group)
    mantissa, exponent = torch.frexp(g.abs().amax(dim=2) / 7.0)
    scale = _times_power(torch.round(mantissa * 32.0), exponent - 5)               # five significant bits
    code = torch.where(scale[..., None] > 0, g / scale[..., None], 0.0)
    return torch.round(code).clamp(-7, 7).flatten(1)[:, : W.shape[1]], scale


def _pack(codes, width):
    """Two codes a byte, the first in the lower half, each with 8 added."""
    c = torch.nn.functional.pad(codes + 8.0, (0, 2 * width - codes.shape[1]), value=8.0).to(torch.uint8)
    return c[:, 0::2] | (c[:, 1::2] << 4)


def _weights4(packed, scales, cols, group):
    c = torch.stack([packed & 15, packed >> 4], dim=2).flatten(1).float()[:, :cols] - 8.0
    return (_groups(c, group) * scales.float()[..., None]).flatten(1)[:, :cols]


def _act(z, act):
    if act == "relu":
        return torch.clamp(z, min=0.0)
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    if act == "gelu":
        return z * 0.5 * torch.erfc(z * -math.sqrt(0.5))
    return z


def _slope(z, act):
    if act == "relu":
        return (z > 0).float()
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    if act == "gelu":
        return 0.5 * torch.erfc(z * -math.sqrt(0.5)) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    return torch.ones_like(z)


def _plus(z, bias):
    return z if bias is None else z + bias.float()


def _run_plain(st):
    case = st["case"]
    op = case["op"]
    bf16 = torch.bfloat16
    if op == "checkpoint":
        return _decode8(_encode8(st["X"]), case["n"]).to(bf16)
    if op == "quantize4":
        codes, scales = _quantize4(st["W"], case["group"])
        return _weights4(_pack(codes, st["W4"][0].shape[1]), scales.to(bf16), case["k"], case["group"]).to(bf16)
    act = case["act"]
    if op in ("linear4", "gated4"):
        x, products = st["X"].float(), []
        for name, bias in (("W", "bias"),) if op == "linear4" else (("Wg", "bias"), ("Wu", "bias2")):
            products.append(_plus(x @ _weights4(*st[name], case["k"], case["group"]).T, st[bias]))
        y = _act(products[0], act)
        if op == "gated4":
            y = y * products[1]
        return (y if st["residual"] is None else y + st["residual"].float()).to(bf16)
    wg, wu = st["Wg"].float(), st["Wu"].float()
    H = None
    if op in ("gated", "gated_step"):
        x = st["X"].float()
        z, u = _plus(x @ wg.T, st["bg"]), _plus(x @ wu.T, st["bu"])
        H = (_act(z, act) * u).to(bf16)
        if op == "gated":
            return (H, z.to(bf16), u.to(bf16)) if case["save"] else (H, None, None)
        x, z, u = (_decode8(_encode8(t.to(bf16)), t.shape[1]) for t in (x, z, u))
    elif case["saved8"]:
        x, z, u = _decode8(st["X8"], case["k"]), _decode8(st["Z8"], case["n"]), _decode8(st["U8"], case["n"])
    else:
        x, z, u = st["X"].float(), st["Z"].float(), st["U"].float()
    dh, a = st["dH"].float(), _act(z, act)
    if op == "gated_backward" and case["again"]:
        H = (a * u).to(bf16)
    dg, du = dh * u * _slope(z, act), dh * a
    out = [(dg @ wg + du @ wu).to(bf16), (dg.T @ x).to(bf16), (du.T @ x).to(bf16)]
    out += [dg.sum(0).to(bf16), du.sum(0).to(bf16)] if case["bias"] else [None, None]
    return (*out, H)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    op, n = case["op"], case["n"]
    if op == "checkpoint":    # two bytes read, a code and a sixteenth of an exponent written; then the way back
        return {"bytes": case["m"] * n * (2 + 1.0625) * 2, "flops": 4 * case["m"] * n}
    k = case["k"]
    if op == "quantize4":
        return {"bytes": n * k * (2 + 0.5 + 2 / case["group"]) * 2, "flops": 4 * n * k}
    m = case["m"]
    vectors = 2 * n if case["bias"] else 0
    if op in ("linear4", "gated4"):
        matrices = 2 if op == "gated4" else 1
        return {"bytes": matrices * n * k * (0.5 + 2 / case["group"]) + 2 * (m * k + m * n + vectors + (m * n if case.get("residual") else 0)),
                "flops": 2 * matrices * m * n * k}
    weights, wide = 2 * n * k, 1.0625 if case.get("saved8") or op == "gated_step" else 2
    forward = 2 * (m * k + weights + vectors + m * n) + (2 * wide * m * n if op == "gated_step" or case.get("save") else 0)
    backward = 2 * (m * n + weights + m * k + weights + vectors + (m * n if case.get("again") else 0)) + wide * (m * k + 2 * m * n)
    if op == "gated":
        return {"bytes": forward, "flops": 4 * m * n * k}
    if op == "gated_backward":
        return {"bytes": backward, "flops": 8 * m * n * k}
    return {"bytes": forward + wide * m * k + backward, "flops": 12 * m * n * k}


# ------------------------------------------------------------------ the definitions in 64 bits
def _kept64(x):
    """What 8 bits keep of bf16 values: multiples of 2^-6 of the power of two below a group's largest, at most 127 of them."""
    rows, cols = x.shape
    out = torch.empty(rows, cols, device=x.device, dtype=torch.float64)
    for c in range(0, cols, 4096):                       # whole groups a time
        part = torch.nn.functional.pad(x[:, c:c + 4096].double(), (0, -(cols - c) % 16 if c + 4096 >= cols else 0)).unflatten(1, (-1, 16))
        largest = part.abs().amax(dim=2, keepdim=True).clamp(min=2.0 ** -126)
        step = ((largest.view(torch.int64) >> 52) - 6 << 52).view(torch.float64)      # its power of two, times 2^-6
        out[:, c:c + 4096] = ((part / step).round().clamp(-127, 127) * step).flatten(1)[:, : min(4096, cols - c)]
    return out


def _values4(packed, scales, cols, group):
    """The matrix that 4-bit codes and scales stand for, column by column group."""
    codes = torch.empty(packed.shape[0], 2 * packed.shape[1], device=packed.device, dtype=torch.float64)
    codes[:, 0::2] = packed.remainder(16).double()
    codes[:, 1::2] = torch.div(packed, 16, rounding_mode="floor").double()
    return (codes[:, :cols] - 8.0) * scales.double().repeat_interleave(group, dim=1)[:, :cols]


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    d = lambda t: None if t is None else t.double()  # noqa: E731
    if op == "checkpoint":
        return _kept64(st["X"])
    if op == "quantize4":
        W, group = st["W"].double(), case["group"]
        out = torch.zeros_like(W)
        for c in range(0, case["k"], group):
            part = W[:, c:c + group]
            ideal = part.abs().amax(dim=1, keepdim=True) / 7.0
            unit = ((ideal.clamp(min=1e-30).view(torch.int64) >> 52) - 4 << 52).view(torch.float64)
            scale = torch.where(ideal > 0, (ideal / unit).round() * unit, 1.0)
            out[:, c:c + group] = (part / scale).round().clamp(-7, 7) * scale
        return out
    act = {"none": lambda z: z, "relu": torch.relu, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu}[case["act"]]
    linear = lambda x, w, b: torch.einsum("mk,nk->mn", x, w) + (0 if b is None else d(b))  # noqa: E731
    if op in ("linear4", "gated4"):
        x = d(st["X"])
        if op == "linear4":
            return act(linear(x, _values4(*st["W"], case["k"], case["group"]), st["bias"])) + (0 if st["residual"] is None else d(st["residual"]))
        return act(linear(x, _values4(*st["Wg"], case["k"], case["group"]), st["bias"])) * \
            linear(x, _values4(*st["Wu"], case["k"], case["group"]), st["bias2"])
    Wg, Wu, H = d(st["Wg"]), d(st["Wu"]), None
    if op in ("gated", "gated_step"):
        x = d(st["X"])
        z, u = linear(x, Wg, st["bg"]), linear(x, Wu, st["bu"])
        H = act(z) * u
        if op == "gated":
            return (H, z, u) if case["save"] else (H, None, None)
        x, z, u = (_kept64(t.to(torch.bfloat16)) for t in (x, z, u))
    elif case["saved8"]:
        back = lambda kept, cols: (kept[0].double().unflatten(1, (-1, 16)) * ((kept[1].long() + 1023 - 133) << 52).view(torch.float64)[..., None]).flatten(1)[:, :cols]  # noqa: E731
        x, z, u = back(st["X8"], case["k"]), back(st["Z8"], case["n"]), back(st["U8"], case["n"])
    else:
        x, z, u = d(st["X"]), d(st["Z"]), d(st["U"])
    z.requires_grad_(True)
    h = act(z)
    dh = d(st["dH"])
    dg, = torch.autograd.grad(h, z, dh * u)
    du = dh * h.detach()
    if op == "gated_backward" and case["again"]:
        H = h.detach() * u
    sums = (dg.sum(0), du.sum(0)) if case["bias"] else (None, None)
    return (torch.einsum("mn,nk->mk", dg, Wg) + torch.einsum("mn,nk->mk", du, Wu), torch.einsum("mn,mk->nk", dg, x),
            torch.einsum("mn,mk->nk", du, x), *sums, H)
