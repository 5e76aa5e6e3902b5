"""A language-model head trained through the compressed step: norm, loss, top_K messages, AdamW.

    python -m paper_2209_15203_b200.train_head [--workers 4] [--tokens 256] [--vocab 4096] [--dim 256]
        [--keep 0.01] [--steps 60] [--states 32|8] [--update adamw|sgd] [--lr ...]

The parameters (gain and bias of a layer norm, and the head's matrix) lie in one flat fp32 vector w, as
tk_step takes it; every worker's gradient is one row of G, and the operators write into the row's slices.  A step is

    worker q   y = norm(x_q; gain, bias);  loss = cross entropy of y head^T;  gradients into row q of G
    exchange   bidirectional Top_K with the error memories (tk_step on a zero vector: the dense message)
    update     AdamW on the message (--update adamw), or the paper's own w -= message (--update sgd)

The data is synthetic (seeded): the hidden state of a token is its target's fixed vector plus noise.
"""
from __future__ import annotations

import argparse
from typing import List

import torch

from . import binding as B


class Head:
    """The flat parameter vector and its views, and one worker's loss and gradient."""

    def __init__(self, dim: int, vocab: int, device, seed: int = 0):
        self.dim, self.vocab = dim, vocab
        self.sizes = [dim, dim, vocab * dim]
        g = torch.Generator(device=device).manual_seed(seed)
        self.w = torch.zeros(sum(self.sizes), device=device)
        self.gain, self.bias, self.matrix = self.split(self.w)
        self.gain.fill_(1.0)
        self.matrix.copy_(torch.randn((vocab, dim), generator=g, device=device) * 0.02)

    def split(self, flat: torch.Tensor) -> List[torch.Tensor]:
        """A flat vector's views of the shapes of gain, bias and the head's matrix."""
        gain, bias, matrix = torch.split(flat, self.sizes)
        return [gain, bias, matrix.view(self.vocab, self.dim)]

    def gradient(self, x: torch.Tensor, target: torch.Tensor, row: torch.Tensor) -> torch.Tensor:
        """Writes the gradient of the mean loss over the tokens that take part into `row`; the loss of each token."""
        dgain, dbias, dmatrix = self.split(row)
        y, mean, rstd = B.tk_layernorm_forward(x, self.gain, self.bias)
        loss, lse = B.tk_xent_loss(y, self.matrix, target)
        held = (target >= 0).float()
        dloss = held / held.sum().clamp(min=1)
        dy, _ = B.tk_xent_grad(y, self.matrix, target, lse, dloss, dw=dmatrix)
        B.tk_layernorm_backward(dy, x, self.gain, mean, rstd, dgain=dgain, dbias=dbias, need_dx=False)
        return loss


class Data:
    """Hidden states that point, through noise, at their next token."""

    def __init__(self, dim: int, vocab: int, device, seed: int = 1):
        self.g = torch.Generator(device=device).manual_seed(seed)
        self.centre = torch.randn((vocab, dim), generator=self.g, device=device)
        self.device = device

    def batch(self, tokens: int):
        target = torch.randint(0, self.centre.shape[0], (tokens,), generator=self.g, device=self.device)
        x = self.centre[target] + torch.randn((tokens, self.centre.shape[1]), generator=self.g, device=self.device)
        skip = torch.rand(tokens, generator=self.g, device=self.device) < 0.05        # tokens without a target
        return x, torch.where(skip, torch.full_like(target, -100), target).to(torch.int32)


def train(workers: int = 4, tokens: int = 256, vocab: int = 4096, dim: int = 256, keep: float = 0.01, steps: int = 60,
          states: int = 32, update: str = "adamw", lr: float = 0.0, device="cuda:0", report=None) -> List[float]:
    """The mean loss of every step."""
    head, data = Head(dim, vocab, device), Data(dim, vocab, device)
    d = head.w.numel()
    k = max(1, int(keep * d))
    ctx = B.Context(d, workers, k, k, torch.full((workers,), 1.0 / workers), device=torch.device(device))
    ctx.tk_ef_attach()
    mode = B.TK_MODE_BIDIR | B.TK_MODE_EF
    G = torch.empty((workers, d), device=device)
    message = torch.zeros(d, device=device)
    opt = B.AdamW(head.split(head.w), state_bits=states, lr=lr or 1e-2, weight_decay=[0.0, 0.0, 0.01])
    losses = []
    for step in range(steps):
        total = 0.0
        for q in range(workers):
            x, target = data.batch(tokens)
            loss = head.gradient(x, target, G[q])
            total += float(loss.sum() / (target >= 0).sum().clamp(min=1))
        losses.append(total / workers)
        if update == "adamw":
            # with -1 for the step size the "parameters" handed over become the dense message itself
            message.zero_()
            ctx.tk_step(message, G, -1.0, mode)
            opt.tk_adamw_step(head.split(message))
        else:
            ctx.tk_step(head.w, G, lr or 3.0, mode)
        if report and (step % 10 == 0 or step == steps - 1):
            report("step %4d  loss %.4f" % (step, losses[-1]))
    if ctx.tk_status().device_status != 0 or B.tk_xent_status() != 0:
        raise RuntimeError("a kernel reported an error")
    ctx.close()
    return losses


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--tokens", type=int, default=256)
    ap.add_argument("--vocab", type=int, default=4096)
    ap.add_argument("--dim", type=int, default=256)
    ap.add_argument("--keep", type=float, default=0.01, help="share of the entries a message keeps")
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--states", type=int, default=32, choices=(8, 32), help="bits of the AdamW states")
    ap.add_argument("--update", default="adamw", choices=("adamw", "sgd"))
    ap.add_argument("--lr", type=float, default=0.0, help="0: 1e-2 for AdamW, 3 for SGD")
    a = ap.parse_args()
    if not torch.cuda.is_available():
        raise SystemExit("needs a CUDA device: the library has no CPU path")
    train(a.workers, a.tokens, a.vocab, a.dim, a.keep, a.steps, a.states, a.update, a.lr, report=print)


if __name__ == "__main__":
    main()
