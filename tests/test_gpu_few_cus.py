"""GPU tests of the losses and of norm and clip over many tensors on a stream that has few of the CUs: the bits of a stream that has all."""
from __future__ import annotations

import pytest
import torch

from gpu_util import DEV, gs

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(params=[16, 100])
def stream(request):
    s = gs.gs_cu_stream_create(request.param)
    yield torch.cuda.ExternalStream(s)
    torch.cuda.synchronize()
    gs.gs_cu_stream_destroy(s)


def workspace():
    return torch.full((gs.gs_sqnorm_workspace_bytes(),), 0xFF, dtype=torch.uint8, device=DEV)


def losses(rows, vocab, dtype, st):
    g = torch.Generator(device=DEV).manual_seed(rows)
    x = (torch.randn(rows, vocab, generator=g, device=DEV) * 3).to(dtype)
    t = torch.randint(-1, vocab, (rows,), generator=g, device=DEV)
    adv, old = torch.randn(rows, generator=g, device=DEV), torch.randn(rows, generator=g, device=DEV) - 9
    logp, rs, dlogp, plogp = (torch.full(s, float("nan"), device=DEV) for s in ((rows,), (rows, 2), (rows,), (rows,)))
    margins, loss, stats = (torch.full((n,), float("nan"), device=DEV) for n in (rows // 4, 1, 4))
    offsets = torch.arange(2 * (rows // 4) + 1, device=DEV) * 2
    grad, policy = torch.full_like(x, 7.0), torch.full_like(x, 7.0)
    ws = workspace()
    torch.cuda.synchronize()
    gs.gs_token_logp(x, t, logp, rs, d_workspace=ws, stream=st)
    gs.gs_preference_loss(logp, old, None, offsets, gs.PreferenceHParams(), margins, dlogp, loss, ws, stream=st)
    gs.gs_token_logp_grad(x, t, rs, dlogp, grad, stream=st)
    gs.gs_policy_loss(x, t, old, None, adv, None, gs.PolicyHParams(), plogp, policy, stats, ws, stream=st)
    torch.cuda.synchronize()
    return logp, rs, margins, dlogp, loss, grad, plogp, stats, policy


@pytest.mark.parametrize("rows,vocab,dtype", [(12, 60_000, F32), (100, 32_003, BF16), (700, 5000, BF16)])
def test_losses(stream, rows, vocab, dtype):
    for a, b in zip(losses(rows, vocab, dtype, torch.cuda.current_stream()), losses(rows, vocab, dtype, stream)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("sizes", [[5, 100, 3000], [4096] * 40, [3_000_001, 17]])
def test_norm_and_clip(stream, sizes):
    got = []
    for st in (torch.cuda.current_stream(), stream):
        g = torch.Generator(device=DEV).manual_seed(1)
        ts = [torch.randn(n, generator=g, device=DEV).to(BF16 if i % 2 else F32) for i, n in enumerate(sizes)]
        sq, norm, ws = torch.empty(1, dtype=torch.float64, device=DEV), torch.empty(1, device=DEV), workspace()
        torch.cuda.synchronize()
        gs.gs_grads_sqnorm(ts, sq, ws, stream=st)
        gs.gs_grads_clip(ts, sq, 1.0, norm, stream=st)
        torch.cuda.synchronize()
        got.append([sq, norm, *ts])
    for a, b in zip(*got):
        assert torch.equal(a, b)
