"""Workspaces of a head's calls on the GPU: each call stays in the bytes that it asks for, and its results are those of a larger one's, bit for bit."""
from __future__ import annotations

import pytest
import torch

from paper_2512_17570_amd import gs
from tests.test_gpu_head import BF16, DEV, Case

pytestmark = pytest.mark.gpu
GUARD = 1 << 20


def room(size):
    """`size` bytes, and behind them some that hold a value."""
    whole = torch.full((size + GUARD,), 0xA5, dtype=torch.uint8, device=DEV)
    return whole[:size], whole[size:]


@pytest.mark.parametrize("rows, hidden, vocab, pad", [(1, 512, 3000, 0), (40, 512, 2000, 0), (40, 1000, 16_385, 3), (130, 640, 1500, 0), (300, 1024, 9001, 0), (300, 520, 700, 8), (70, 256, 900, 0)])
def test_gradient_from_logp_without_room_for_z(rows, hidden, vocab, pad):
    c = Case(rows, hidden, vocab, bias=True, prompt=rows > 4, w_stride=hidden + pad)
    dlogp = torch.randn(rows, device=DEV, generator=torch.Generator(device=DEV).manual_seed(2))
    small, large = gs.gs_head_logp_grad_workspace_bytes(rows, hidden, vocab), gs.gs_head_workspace_bytes(rows, hidden, vocab)
    assert (small < large) == (hidden > 448)
    got = []
    for size in (large, small):
        ws, behind = room(size)
        c.dx.fill_(7.0), c.dw.fill_(7.0), c.db.fill_(7.0)
        gs.gs_head_logp(c.x, c.w, c.bias, c.targets, c.logp, c.stats, d_workspace=ws)
        gs.gs_head_logp_grad(c.x, c.w, c.bias, c.targets, c.stats, dlogp, c.dx, c.dw, c.db, ws)
        assert bool((behind == 0xA5).all())
        got.append([t.clone() for t in (c.logp, c.stats, c.dx, c.dw, c.db)])
    for a, b in zip(*got):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)) if a.dtype != BF16 else torch.equal(a.view(torch.int16), b.view(torch.int16))
    with pytest.raises(gs.GsError):
        gs.gs_head_logp_grad(c.x, c.w, c.bias, c.targets, c.stats, dlogp, c.dx, c.dw, c.db, ws[:small - 1])


@pytest.mark.parametrize("rows, hidden, vocab, pad", [(1, 4096, 3000, 0), (40, 512, 2000, 0), (130, 640, 1500, 1), (300, 1024, 9001, 0), (300, 64, 700, 0)])
def test_losses_and_scores_stay_in_their_workspace(rows, hidden, vocab, pad):
    c = Case(rows, hidden, vocab, bias=True, prompt=rows > 4, w_stride=hidden + pad)
    ws, behind = room(gs.gs_head_workspace_bytes(rows, hidden, vocab))
    gs.gs_head_cross_entropy(c.x, c.w, c.bias, c.targets, c.weights, c.logp, c.dx, c.dw, c.db, c.loss, ws)
    assert bool((behind == 0xA5).all())
    ws, behind = room(gs.gs_head_workspace_bytes(rows, hidden, vocab, False))
    gs.gs_head_cross_entropy(c.x, c.w, c.bias, c.targets, c.weights, c.logp, None, None, None, c.loss, ws)
    gs.gs_head_logp(c.x, c.w, c.bias, c.targets, c.logp, c.stats, d_workspace=ws)
    assert bool((behind == 0xA5).all())


@pytest.mark.parametrize("rows, hidden, vocab", [(40, 1000, 200_000), (300, 5000, 30_000), (40, 1000, 8300)])
def test_a_loss_with_some_of_its_gradients(rows, hidden, vocab):
    """z is kept and the weights are packed: the gradients that are asked for are those of a call that is asked for all."""
    c = Case(rows, hidden, vocab, bias=True, prompt=True, w_stride=hidden + 3)
    want = {k: v.clone() for k, v in c.cross_entropy().items()} | {"loss": c.loss.clone()}
    for parts in ("dw db", "dw", "db", "dx"):
        for t in (c.logp, c.dx, c.dw, c.db, c.loss):
            t.fill_(7.0)
        gs.gs_head_cross_entropy(c.x, c.w, c.bias, c.targets, c.weights, c.logp, *[t if n in parts.split() else None for n, t in (("dx", c.dx), ("dw", c.dw), ("db", c.db))],
                                 c.loss, c.workspace())
        for n, t in {"logp": c.logp, "dx": c.dx, "dw": c.dw, "db": c.db, "loss": c.loss}.items():
            assert torch.equal(t, want[n]) if n in ("logp", "loss") or n in parts.split() else bool((t == 7.0).all()), (parts, n)
