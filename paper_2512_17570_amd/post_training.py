"""A small post-training program on the library's entry points: losses on logits, norm and clip of the gradients of several
tensors, and the optimizer step, as they are used together.

The model is a linear head: logits = x W^T + b over hidden states x that are given.  One step takes k micro-batches:
  * the loss leaves its gradient where the logits were (gs_policy_loss in place; for preferences gs_token_logp,
    gs_preference_loss and gs_token_logp_grad), its value is added up over the micro-batches on the device;
  * the parameters' bf16 gradients are added into an fp32 sum for each tensor (gs_accum_add);
  * gs_grads_sqnorm takes the norm of all sums together, gs_grads_clip scales them, gs_adamw_from_acc steps each tensor.
Nothing in a step waits for the GPU.  PyTorch supplies memory and the head's products.

    python -m paper_2512_17570_amd.post_training
"""
from __future__ import annotations

from dataclasses import dataclass, field

import torch

from . import gs

DEV = "cuda"


@dataclass
class Parameter:
    """One tensor: fp32 master weight and moments, bf16 working weight, fp32 gradient sum."""
    w: torch.Tensor                          # bf16, as the model uses it
    p: torch.Tensor = field(init=False)
    m: torch.Tensor = field(init=False)
    v: torch.Tensor = field(init=False)
    acc: torch.Tensor = field(init=False)

    def __post_init__(self):
        self.p = self.w.float().reshape(-1)
        self.m, self.v, self.acc = (torch.zeros_like(self.p) for _ in range(3))


class Head:
    def __init__(self, hidden: int, vocab: int, seed: int = 0):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.weight = Parameter((torch.randn(vocab, hidden, generator=g, device=DEV) * hidden ** -0.5).bfloat16())
        self.bias = Parameter(torch.zeros(vocab, dtype=torch.bfloat16, device=DEV))
        self.sq = torch.zeros(1, dtype=torch.float64, device=DEV)
        self.norm = torch.zeros(1, device=DEV)
        self.workspace = torch.empty(gs.gs_sqnorm_workspace_bytes(), dtype=torch.uint8, device=DEV)
        self.step = 0

    def logits(self, x):
        return torch.addmm(self.bias.w, x, self.weight.w.t())

    def add_gradients(self, x, dlogits, first: bool):
        for par, g in ((self.weight, dlogits.t() @ x), (self.bias, dlogits.sum(0))):
            gs.gs_accum_add(par.acc, g.reshape(-1), first, 0, par.acc.numel())

    def update(self, lr: float, max_norm: float):
        pars = [self.weight, self.bias]
        self.step += 1
        hp = gs.HParams(lr=lr, weight_decay=0.0, max_grad_norm=0.0, step=self.step)      # clipped before
        gs.gs_grads_sqnorm([q.acc for q in pars], self.sq, self.workspace)
        gs.gs_grads_clip([q.acc for q in pars], self.sq, max_norm, self.norm)
        for q in pars:
            gs.gs_adamw_from_acc(q.p, q.m, q.v, q.w.view(-1), q.acc, 0, q.acc.numel(), hp)


@dataclass
class Drawn:
    """One micro-batch of drawn tokens: hidden states and ids (-1: no token), what the policy that drew them and the reference
    gave them, their advantages, and the weight of each in the loss."""
    x: torch.Tensor
    targets: torch.Tensor
    old_logp: torch.Tensor
    ref_logp: torch.Tensor | None
    advantages: torch.Tensor
    weights: torch.Tensor


def score(head: Head, x, targets, row_stats=None):
    """Log-probabilities of the given tokens, and the logits they come from."""
    logits = head.logits(x)
    logp = torch.empty(len(targets), device=DEV)
    gs.gs_token_logp(logits, targets, logp, row_stats, d_workspace=head.workspace)
    return logp, logits


def policy_step(head: Head, micro_batches: list[Drawn], hp: gs.PolicyHParams, lr: float, max_norm: float = 1.0):
    """One update; the sums over all tokens of loss, policy term, KL term and clipped weight, on the device."""
    stats = torch.empty(4, device=DEV)
    for j, b in enumerate(micro_batches):
        logits = head.logits(b.x)
        logp = torch.empty(len(b.targets), device=DEV)
        gs.gs_policy_loss(logits, b.targets, b.old_logp, b.ref_logp, b.advantages, b.weights, hp, logp, logits, stats,
                          head.workspace, accumulate=j > 0)
        head.add_gradients(b.x, logits, j == 0)
    head.update(lr, max_norm)
    return stats


@dataclass
class Pairs:
    """One micro-batch of preference pairs: the tokens of the chosen sequences, then of the rejected ones; sequence s is
    [offsets[s], offsets[s + 1]).  weights: 1 for the tokens of an answer."""
    x: torch.Tensor
    targets: torch.Tensor
    ref_logp: torch.Tensor
    weights: torch.Tensor
    offsets: torch.Tensor


def preference_step(head: Head, micro_batches: list[Pairs], beta: float, lr: float, max_norm: float = 1.0):
    """One update; the mean loss over all pairs, and the margins of each micro-batch, on the device."""
    pairs = sum((len(b.offsets) - 1) // 2 for b in micro_batches)
    hp = gs.PreferenceHParams(beta=beta, scale=1.0 / pairs)
    loss, margins = torch.empty(1, device=DEV), []
    for j, b in enumerate(micro_batches):
        row_stats = torch.empty(len(b.targets), 2, device=DEV)
        logp, logits = score(head, b.x, b.targets, row_stats)
        dlogp = torch.empty_like(logp)
        margins.append(torch.empty((len(b.offsets) - 1) // 2, device=DEV))
        gs.gs_preference_loss(logp, b.ref_logp, b.weights, b.offsets, hp, margins[-1], dlogp, loss, head.workspace, accumulate=j > 0)
        gs.gs_token_logp_grad(logits, b.targets, row_stats, dlogp, logits)
        head.add_gradients(b.x, logits, j == 0)
    head.update(lr, max_norm)
    return loss, margins


# ---- synthetic data, for the command and its test ---------------------------------------------------------------------

def drawn_tokens(head: Head, rows: int, k: int, seed: int = 0):
    """k micro-batches whose tokens are drawn from the head itself; ids below half of the vocabulary are rewarded.  The first rows of each
    are a prompt."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    vocab, hidden = head.weight.w.shape
    out, tokens = [], 0
    for _ in range(k):
        x = torch.randn(rows, hidden, generator=g, device=DEV).bfloat16()
        targets = torch.multinomial(torch.softmax(head.logits(x).float(), 1), 1, generator=g)[:, 0]
        targets[:rows // 8] = -1
        logp, _ = score(head, x, targets)
        advantages = torch.where(targets < vocab // 2, 1.0, -1.0)
        out.append(Drawn(x, targets, logp, logp.clone(), advantages, torch.empty(rows, device=DEV)))
        tokens += rows - rows // 8
    for b in out:
        b.weights.fill_(1.0 / tokens)
    return out


def ranked_pairs(head: Head, pairs: int, length: int, k: int, seed: int = 0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    vocab, hidden = head.weight.w.shape
    out = []
    for _ in range(k):
        ends = torch.cumsum(torch.randint(1, length + 1, (2 * pairs,), generator=g, device=DEV), 0)
        offsets = torch.cat([ends.new_zeros(1), ends])
        tokens = int(offsets[-1])
        x = torch.randn(tokens, hidden, generator=g, device=DEV).bfloat16()
        targets = torch.randint(0, vocab, (tokens,), generator=g, device=DEV)
        logp, _ = score(head, x, targets)
        out.append(Pairs(x, targets, logp, torch.ones(tokens, device=DEV), offsets))
    return out


def main():
    head = Head(256, 32_000)
    batches = drawn_tokens(head, rows=512, k=4)
    hp = gs.PolicyHParams(clip_low=0.2, clip_high=0.28, kl_coef=0.02)
    for step in range(8):
        stats = policy_step(head, batches, hp, lr=2e-3)
        loss, policy, kl, clipped = stats.tolist()
        print(f"policy      step {step}: loss {loss:+.4f}  policy term {policy:+.4f}  kl {kl:.4f}  clipped {clipped:.1%}  norm {head.norm.item():.4f}")
    head = Head(256, 32_000, seed=1)
    pairs = ranked_pairs(head, pairs=8, length=64, k=4)
    for step in range(8):
        loss, margins = preference_step(head, pairs, beta=0.1, lr=2e-3)
        print(f"preference  step {step}: loss {loss.item():.4f}  mean margin {torch.cat(margins).mean().item():+.3f}  norm {head.norm.item():.4f}")


if __name__ == "__main__":
    main()
