"""GPU test of the post-training program: losses, norm, clip and step together, against the same steps in 64 bits."""
from __future__ import annotations

import math

import pytest
import torch

from gpu_util import DEV
from paper_2512_17570_amd import gs
from paper_2512_17570_amd import post_training as P

pytestmark = pytest.mark.gpu


def reference_gradients(head, batches, loss_of):
    """Gradients of the head in 64 bits, from autograd, with the working weights as they are."""
    w, b = (q.w.double().requires_grad_(True) for q in (head.weight, head.bias))
    total = 0.0
    for batch in batches:
        logits = torch.addmm(b, batch.x.double(), w.t())
        live = batch.targets >= 0
        logp = torch.log_softmax(logits, 1).gather(1, batch.targets.clamp(min=0)[:, None])[:, 0]
        total = total + loss_of(batch, torch.where(live, logp, 0.0), live)
    return float(total.detach()), torch.autograd.grad(total, (w, b))


def close(acc, want, k):
    """bf16 logits, bf16 logit gradients and bf16 parameter gradients, each k of them: 2^-8 of the size each, of which a product over rows
    averages most; against 3 x 2^-8 of the gradient's norm."""
    off = float((acc.double() - want.reshape(-1)).norm())
    assert off <= 3 * 2.0 ** -8 * float(want.norm()) * math.sqrt(k), off / float(want.norm())


def test_policy_steps():
    head = P.Head(64, 3001)
    batches = P.drawn_tokens(head, rows=200, k=3)
    hp = gs.PolicyHParams(clip_low=0.2, clip_high=0.28, kl_coef=0.02)
    torch.cuda.synchronize()

    def loss(b, logp, live):
        r = torch.exp(logp - b.old_logp)
        d = b.ref_logp - logp
        pg = -torch.minimum(r * b.advantages, r.clamp(0.8, 1.28) * b.advantages)
        return ((pg + 0.02 * (d.exp() - d - 1)) * b.weights)[live].sum()

    want, (dw, db) = reference_gradients(head, batches, loss)
    norm = math.sqrt(float(dw.square().sum() + db.square().sum()))
    stats = P.policy_step(head, batches, hp, lr=1e-3, max_norm=0.5 * norm)
    assert float(stats[0]) == pytest.approx(want, abs=0.02)
    assert head.norm.item() == pytest.approx(norm, rel=0.01)
    close(head.weight.acc, 0.5 * dw, 3)
    close(head.bias.acc, 0.5 * db, 3)
    first = float(stats[1])
    for _ in range(6):
        stats = P.policy_step(head, batches, hp, lr=1e-3)
    assert float(stats[1]) < first - 0.05 and torch.isfinite(stats).all()           # rewarded tokens got likelier
    assert torch.equal(head.weight.w.view(-1), head.weight.p.bfloat16())


def test_preference_steps():
    head = P.Head(64, 3001, seed=1)
    batches = P.ranked_pairs(head, pairs=4, length=30, k=2)

    def loss(b, logp, live):
        parts = [((logp - b.ref_logp) * b.weights)[a:c].sum() for a, c in zip(b.offsets[:-1].tolist(), b.offsets[1:].tolist())]
        h = 0.1 * (torch.stack(parts[:4]) - torch.stack(parts[4:]))
        return -torch.nn.functional.logsigmoid(h).sum() / 8

    want, (dw, db) = reference_gradients(head, batches, loss)
    value, margins = P.preference_step(head, batches, beta=0.1, lr=1e-3, max_norm=1e9)
    assert float(value) == pytest.approx(want, abs=0.02)
    close(head.weight.acc, dw, 2)
    close(head.bias.acc, db, 2)
    for _ in range(6):
        value, margins = P.preference_step(head, batches, beta=0.1, lr=1e-3)
    assert float(value) < math.log(2) - 0.02 and float(torch.cat(margins).mean()) > 0.05


def test_the_command_runs(capsys):
    P.main()
    lines = [l for l in capsys.readouterr().out.splitlines() if "step" in l]
    assert len(lines) == 16 and DEV
