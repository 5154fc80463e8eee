"""Fine-tuning on the library's entry points without logits: the last part of a model as a training program runs it.

  * supervised_step trains what lies behind the last block on text: dropout onto the residual stream (gs_dropout), layer norm (gs_layer_norm), cross entropy of the
    head (gs_head_cross_entropy), and the way back (gs_layer_norm_grad, gs_dropout) down to the gradients that the block below takes;
  * preference_step_without_logits takes the place of post_training.py's preference_step (gs_head_logp, gs_preference_loss, gs_head_logp_grad).

One step takes k micro-batches, whose bf16 gradients are added into fp32 sums (gs_accum_add), then norm, clip and step as in post_training.py.  Nothing in a
step waits for the GPU.  PyTorch supplies memory.

    python -m paper_2512_17570_amd.fine_tuning
"""
from __future__ import annotations

from dataclasses import dataclass

import torch

from . import gs
from .post_training import DEV, Head, Pairs, Parameter, ranked_pairs


def preference_step_without_logits(head: Head, micro_batches: list[Pairs], beta: float, lr: float, max_norm: float = 1.0):
    """preference_step, with neither the logits nor their gradient in memory."""
    pairs = sum((len(b.offsets) - 1) // 2 for b in micro_batches)
    hp = gs.PreferenceHParams(beta=beta, scale=1.0 / pairs)
    w, bias = head.weight.w, head.bias.w
    dw, db = torch.empty_like(w), torch.empty_like(bias)
    loss, margins = torch.empty(1, device=DEV), []
    for j, b in enumerate(micro_batches):
        rows, ws = len(b.targets), head.room(len(b.targets), loss=False)
        logp, dlogp, row_stats = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV), torch.empty(rows, 2, device=DEV)
        margins.append(torch.empty((len(b.offsets) - 1) // 2, device=DEV))
        gs.gs_head_logp(b.x, w, bias, b.targets, logp, row_stats, d_workspace=ws)
        gs.gs_preference_loss(logp, b.ref_logp, b.weights, b.offsets, hp, margins[-1], dlogp, loss, head.workspace, accumulate=j > 0)
        gs.gs_head_logp_grad(b.x, w, bias, b.targets, row_stats, dlogp, None, dw, db, ws)
        for par, g in ((head.weight, dw), (head.bias, db)):
            gs.gs_accum_add(par.acc, g.view(-1), j == 0, 0, par.acc.numel())
    head.update(lr, max_norm)
    return loss, margins


class Tail(Head):
    """What lies behind a model's last block: dropout of the block's output onto the residual stream, layer norm, head."""

    def __init__(self, hidden: int, vocab: int, dropout: float = 0.1, seed: int = 0):
        super().__init__(hidden, vocab, seed)
        self.gamma = Parameter(torch.ones(hidden, dtype=torch.bfloat16, device=DEV))
        self.beta = Parameter(torch.zeros(hidden, dtype=torch.bfloat16, device=DEV))
        self.dropout, self.seed = dropout, seed
        self.count = torch.zeros(1, dtype=torch.int64, device=DEV)       # of steps, on the device: what the masks change by
        self.grads = [torch.empty_like(q.w) for q in self.parameters()]  # one micro-batch's

    def parameters(self):
        return [self.weight, self.bias, self.gamma, self.beta]


@dataclass
class Text:
    """One micro-batch: the last block's output and the residual stream it is added to (rows, hidden), the ids of the tokens that
    follow (-1: none), and the weight of each in the loss."""
    block: torch.Tensor
    residual: torch.Tensor
    targets: torch.Tensor
    weights: torch.Tensor


def text_gradients(tail: Tail, b: Text, loss, accumulate: bool, offset: int = 0):
    """Forward and backward of one micro-batch, whose elements are numbered from `offset` on: its loss is added up, the parameters' gradients are left in tail.grads; what
    the block and the residual stream get is returned."""
    rows, hidden = b.block.shape
    stream, y = torch.empty_like(b.block), torch.empty_like(b.block)
    stats, logp = torch.empty(rows, 2, device=DEV), torch.empty(rows, device=DEV)
    dw, db, dgamma, dbeta = tail.grads
    gs.gs_dropout(b.block, b.residual, stream, tail.dropout, tail.seed, offset, tail.count)
    gs.gs_layer_norm(stream, tail.gamma.w, tail.beta.w, y, stats)
    dy = torch.empty_like(y)
    gs.gs_head_cross_entropy(y, tail.weight.w, tail.bias.w, b.targets, b.weights, logp, dy, dw, db, loss, tail.room(rows), accumulate=accumulate)
    ws = torch.empty(gs.gs_layer_norm_workspace_bytes(rows, hidden), dtype=torch.uint8, device=DEV)
    gs.gs_layer_norm_grad(dy, stream, tail.gamma.w, stats, dy, dgamma, dbeta, ws)      # in dy's place: the residual stream's gradient
    dblock = torch.empty_like(dy)
    gs.gs_dropout(dy, None, dblock, tail.dropout, tail.seed, offset, tail.count)       # the same mask
    return dblock, dy


def supervised_step(tail: Tail, micro_batches: list[Text], lr: float, max_norm: float = 1.0):
    """One update; the loss over all tokens, on the device, and each micro-batch's gradients for what lies below."""
    loss, below, offset = torch.empty(1, device=DEV), [], 0
    for j, b in enumerate(micro_batches):
        below.append(text_gradients(tail, b, loss, j > 0, offset))
        offset += b.block.numel()
        for par, g in zip(tail.parameters(), tail.grads):
            gs.gs_accum_add(par.acc, g.view(-1), j == 0, 0, par.acc.numel())
    tail.update(lr, max_norm)
    tail.count += 1
    return loss, below


# ---- synthetic data, for the command and its test ---------------------------------------------------------------------

def text(tail: Tail, rows: int, k: int, seed: int = 0):
    """k micro-batches of hidden states, each with a token that depends on it; the first rows of each are a prompt."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    vocab, hidden = tail.weight.w.shape
    way = torch.randn(hidden, vocab, generator=g, device=DEV)
    out = []
    for _ in range(k):
        block, residual = (torch.randn(rows, hidden, generator=g, device=DEV).bfloat16() for _ in range(2))
        targets = ((block + residual).float() @ way).argmax(1)
        targets[:rows // 8] = -1
        out.append(Text(block, residual, targets, torch.full((rows,), 1.0 / (k * (rows - rows // 8)), device=DEV)))
    return out


def main():
    head = Head(256, 32_000, seed=1)
    pairs = ranked_pairs(head, pairs=8, length=64, k=4)
    for step in range(8):
        loss, margins = preference_step_without_logits(head, pairs, beta=0.1, lr=2e-3)
        print(f"preference  step {step}: loss {loss.item():.4f}  mean margin {torch.cat(margins).mean().item():+.3f}  norm {head.norm.item():.4f}")
    tail = Tail(256, 32_000, seed=2)
    batches = text(tail, rows=512, k=4)
    for step in range(8):
        loss, _ = supervised_step(tail, batches, lr=2e-3)
        print(f"supervised  step {step}: loss {loss.item():.4f}  norm {tail.norm.item():.4f}")


if __name__ == "__main__":
    main()
