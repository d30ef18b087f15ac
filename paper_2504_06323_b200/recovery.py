"""Recovery of a pruned block: the compacted student is trained on what its unpruned teacher answers.

    teacher   mosaic_linear x 4 -> mosaic_top_logits: the largest logits of every token
    student   mosaic_linear x 4 -> mosaic_distill_loss_grad: the loss, and its gradient in the logits' place
              mosaic_linear_backward x 4, and a step of plain gradient descent on fp32 copies of the weights
(gate, up, down and head; the elementwise product of gate and up, and its gradient, are plain tensor operations.)

The teacher runs once per batch: its targets are `top` values and indices a token instead of `vocab` logits.
Every call goes to the current stream; one workspace serves them all.  `python -m paper_2504_06323_b200.recovery`
prunes the MLP of the tiny configuration and prints the loss as it falls.
"""
from __future__ import annotations

import argparse

import torch

from . import api, driver, workloads as wl


class Block:
    """logits = (X + down(mlp(X))) head^T with bf16 up and gate [channels, hidden], down [hidden, channels], head
    [vocab, hidden] and bias [channels] or None:
        mlp(X) = act(gate(X) + bias) * up(X)      the gated MLP of the LLaMA-shaped models
        mlp(X) = act(up(X) + bias)                without a gate
    Buffers are kept for the last number of tokens; a block serves one stream at a time."""

    WEIGHTS = ("gate", "up", "down", "head", "bias")

    def __init__(self, up: torch.Tensor, down: torch.Tensor, head: torch.Tensor, bias: torch.Tensor | None = None, act: str = "silu",
                 ws: api.Workspace | None = None, gate: torch.Tensor | None = None):
        if up.shape != down.shape[::-1] or head.shape[1] != up.shape[1]:
            raise ValueError(f"up {tuple(up.shape)}, down {tuple(down.shape)} and head {tuple(head.shape)} do not fit together")
        if gate is not None and gate.shape != up.shape:
            raise ValueError(f"gate {tuple(gate.shape)} and up {tuple(up.shape)} do not fit together")
        self.gate, self.up, self.down, self.head, self.bias, self.act = gate, up, down, head, bias, act
        self.ws = ws if ws is not None else api.Workspace(up.device)
        self.status = torch.zeros(8, dtype=torch.int32, device=up.device)   # a word for each product, which its call resets
        self._bufs: dict[str, torch.Tensor] = {}

    def _buf(self, name: str, rows: int, cols: int) -> torch.Tensor:
        # rows on 16-byte boundaries, whatever width compaction left: the next product reads them without a copy
        t = self._bufs.get(name)
        if t is None or t.shape != (rows, cols):
            t = self._bufs[name] = torch.empty(rows, -(-cols // 8) * 8, dtype=torch.bfloat16, device=self.up.device)[:, :cols]
        return t

    def forward(self, X: torch.Tensor, keep: bool = True) -> torch.Tensor:
        """The logits [tokens, vocab], in a buffer that the next call reuses; with `keep`, backward() may follow."""
        t, (channels, hidden) = X.shape[0], self.up.shape
        H, Y, L = self._buf("H", t, channels), self._buf("Y", t, hidden), self._buf("L", t, self.head.shape[0])
        Z = self._buf("Z", t, channels) if keep else None
        if self.gate is None:
            api.mosaic_linear(X, self.up, H, bias=self.bias, act=self.act, Z=Z, status=self.status[0:1], ws=self.ws)
        else:
            G, U = self._buf("G", t, channels), self._buf("U", t, channels)
            api.mosaic_linear(X, self.gate, G, bias=self.bias, act=self.act, Z=Z, status=self.status[6:7], ws=self.ws)
            api.mosaic_linear(X, self.up, U, status=self.status[0:1], ws=self.ws)
            torch.mul(G, U, out=H)
        api.mosaic_linear(H, self.down, Y, residual=X, status=self.status[1:2], ws=self.ws)
        api.mosaic_linear(Y, self.head, L, status=self.status[2:3], ws=self.ws)
        return L

    def backward(self, X: torch.Tensor, dL: torch.Tensor) -> dict:
        """Gradients of the weights from that of the logits, after forward(X)."""
        t, (channels, hidden) = X.shape[0], self.up.shape
        b = self._bufs
        g = {w: self._buf("d" + w, *getattr(self, w).shape) for w in ("gate", "up", "down", "head") if getattr(self, w) is not None}
        if self.bias is not None:
            g["bias"] = self._buf("dbias", 1, channels)[0]
        dY, dH = self._buf("dY", t, hidden), self._buf("dH", t, channels)
        api.mosaic_linear_backward(dL, b["Y"], self.head, dX=dY, dW=g["head"], status=self.status[3:4], ws=self.ws)
        api.mosaic_linear_backward(dY, b["H"], self.down, dX=dH, dW=g["down"], status=self.status[4:5], ws=self.ws)
        if self.gate is not None:
            dG, dU = self._buf("dG", t, channels), self._buf("dU", t, channels)
            torch.mul(dH, b["U"], out=dG)
            torch.mul(dH, b["G"], out=dU)
            api.mosaic_linear_backward(dG, X, None, Z=b["Z"], act=self.act, dW=g["gate"], dbias=g.get("bias"), status=self.status[7:8],
                                       ws=self.ws)
            api.mosaic_linear_backward(dU, X, None, dW=g["up"], status=self.status[5:6], ws=self.ws)
        else:
            api.mosaic_linear_backward(dH, X, None, Z=b["Z"], act=self.act, dW=g["up"], dbias=g.get("bias"), status=self.status[5:6],
                                       ws=self.ws)
        return g

    def check(self) -> None:
        """Raise if a wait of the last products ran out (reads the status words from the device)."""
        if bool(self.status.any()):
            raise api.MosaicError(api.ERR_TIMEOUT, "a product of the block")


class Recovery:
    """Trains `student` to answer as `teacher` does: gradient descent on the mean distillation loss over the tokens.
    With `renormalise` the kept logits are the teacher's whole answer (the loss is then never negative); without, they
    keep the probabilities that they have among all.  Entries of gate, up and down that are 0 when training begins, the ones
    that unstructured pruning removed, stay 0."""

    def __init__(self, student: Block, teacher: Block, top: int = 64, temperature: float = 2.0, rate: float = 0.1, renormalise: bool = True):
        if student.head.shape[0] != teacher.head.shape[0]:
            raise ValueError("student and teacher must share a vocabulary")
        self.student, self.teacher, self.top, self.temperature, self.rate = student, teacher, top, temperature, rate
        self.renormalise = renormalise
        self.master = {w: getattr(student, w).float() for w in Block.WEIGHTS if getattr(student, w) is not None}
        zeros = {w: self.master[w] == 0 for w in ("gate", "up", "down") if w in self.master}
        self.removed = {w: z for w, z in zeros.items() if bool(z.any())}

    def targets(self, X: torch.Tensor) -> tuple:
        """(values [tokens, top], indices, log of the whole sum or None) of the teacher's logits."""
        t, dev = X.shape[0], X.device
        values, indices = torch.empty(t, self.top, device=dev), torch.empty(t, self.top, dtype=torch.int32, device=dev)
        lse = None if self.renormalise else torch.empty(t, device=dev)
        api.mosaic_top_logits(self.teacher.forward(X, keep=False), values, indices, lse, self.temperature, ws=self.teacher.ws)
        return values, indices, lse

    def loss(self, X: torch.Tensor, targets: tuple) -> torch.Tensor:
        """Each token's loss, without a step."""
        values, indices, lse = targets
        out = torch.empty(X.shape[0], device=X.device)
        api.mosaic_distill_loss(self.student.forward(X, keep=False), values, indices, out, t_lse=lse, temperature=self.temperature,
                                ws=self.student.ws)
        return out

    def gradients(self, X: torch.Tensor, targets: tuple) -> tuple[torch.Tensor, dict]:
        """Each token's loss, and the gradients of their mean."""
        values, indices, lse = targets
        out = torch.empty(X.shape[0], device=X.device)
        L = self.student.forward(X)
        api.mosaic_distill_loss_grad(L, values, indices, out, None, L, t_lse=lse, grad_scale=1.0 / X.shape[0], temperature=self.temperature,
                                     ws=self.student.ws)
        return out, self.student.backward(X, L)

    def step(self, X: torch.Tensor, targets: tuple | None = None) -> torch.Tensor:
        """One step on a batch (its targets are made if they are not given); each token's loss before it."""
        loss, grads = self.gradients(X, targets if targets is not None else self.targets(X))
        for w, g in grads.items():
            self.master[w].add_(g, alpha=-self.rate)
            if w in self.removed:
                self.master[w].masked_fill_(self.removed[w], 0.0)
            getattr(self.student, w).copy_(self.master[w])
        return loss


def compact_mlp(st: driver.ModelState, layer: int, frac: float, head: torch.Tensor, gated: bool = False) -> tuple[Block, Block]:
    """(student, teacher): the MLP of a layer with `frac` of its channels removed, and as it is.  `gated`: the MLP that the
    model computes, down(silu(gate(X)) * up(X)).  Otherwise up and down alone, with a bias for the student to learn: not
    the model's answer, but what a model without a gate would have."""
    def block(W: dict, head: torch.Tensor, learns_bias: bool) -> Block:
        W = {pr: W[pr].to(torch.bfloat16) for pr in ("gate", "up", "down")}
        bias = torch.zeros(W["up"].shape[0], dtype=torch.bfloat16, device=head.device) if learns_bias else None
        return Block(W["up"], W["down"], head, bias, ws=st.ws, gate=W["gate"] if gated else None)

    pruned = driver.prune_structured_coupled_layer(st, layer, frac)["W"]
    whole = {pr: st.W[layer, pr] for pr in ("gate", "up", "down")}
    return block(pruned, head.clone(), not gated), block(whole, head, False)


def main(argv=None) -> list[float]:
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--config", default="tiny", choices=sorted(wl.CONFIGS))
    ap.add_argument("--frac", type=float, default=0.3, help="part of the MLP's channels to remove")
    ap.add_argument("--tokens", type=int, default=512)
    ap.add_argument("--vocab", type=int, default=2000)
    ap.add_argument("--top", type=int, default=64)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--rate", type=float, default=0.1)
    args = ap.parse_args(argv)
    cfg, dev = wl.CONFIGS[args.config], torch.device("cuda", torch.cuda.current_device())
    gen = torch.Generator(device=dev).manual_seed(cfg.seed)
    st = driver.alloc_model(cfg, dev, layers=[0], outputs=False, masks=False)
    X = torch.randn(args.tokens, cfg.hidden, generator=gen, device=dev)
    driver.accumulate_norms(st, 0, driver.make_activations(cfg, 0, dev, args.tokens))
    head = (torch.randn(args.vocab, cfg.hidden, generator=gen, device=dev) * cfg.hidden ** -0.5).to(torch.bfloat16)
    student, teacher = compact_mlp(st, 0, args.frac, head, gated=True)
    run = Recovery(student, teacher, min(args.top, args.vocab), rate=args.rate)
    X = X.to(torch.bfloat16)
    targets, losses = run.targets(X), []
    for i in range(args.steps):
        losses.append(float(run.step(X, targets).mean()))
        if i % 10 == 0:
            print(f"step {i:4d}  loss {losses[-1]:.5f}", flush=True)
    losses.append(float(run.loss(X, targets).mean()))
    student.check()
    teacher.check()
    print(f"{cfg.name}: {student.up.shape[0]} of {teacher.up.shape[0]} channels, loss {losses[0]:.5f} -> {losses[-1]:.5f}", flush=True)
    return losses


if __name__ == "__main__":
    main()
