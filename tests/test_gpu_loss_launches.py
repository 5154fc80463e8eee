"""GPU tests of the losses and of the norm over many tensors where one call takes several launches of a kernel, or many rows in parts."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import loss_oracle as O
from gpu_util import DEV, gs
from test_gpu_losses import BF16, F32, Rows, logp_check, policy_check, within, workspace

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,vocab,dtype", [(128, 98_400, F32), (129, 98_400, F32), (300, 98_400, F32), (129, 200_000, BF16), (300, 98_307, F32)])
@pytest.mark.parametrize("kw", [{}, {"in_place": True, "accumulate": True}, {"gradient": False}, {"gradient": False, "accumulate": True}, {"offset": 1, "gap": 2}])
def test_policy_loss_of_many_rows_in_parts(rows, vocab, dtype, kw):
    """Rows too long to be held, more of them than meet in a launch: the sums are another launch's, of the log-probabilities that the
    gradient's, or the joining one, has left."""
    policy_check(Rows(rows, vocab, dtype, seed=rows, offset=1 if kw.get("in_place") else 0, gap=3 if kw.get("in_place") else 0), **kw)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows", [1, 16, 17, 32, 33, 64, 65, 128, 129])
@pytest.mark.parametrize("line", [30_000, 45_000, 55_000, 60_000, 100_000])
def test_few_rows_held_and_in_parts(line, rows, dtype):
    for vocab in (line, line + 1):
        if vocab > 98_000 and dtype == F32:
            continue
        x = Rows(rows, vocab, dtype, seed=rows, offset=rows % 3, prompt=0.2 if rows > 1 else 0.0)
        logp_check(x, stats=rows % 2 == 0)
        policy_check(x, in_place=True, accumulate=rows % 2 == 1)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,vocab,gap", [(5, 1000, 0), (7, 1003, 5), (3, 50_001, 0), (3, 98_400, 1), (140, 3000, 0)])
def test_gradients_beside_their_logits(rows, vocab, gap, dtype):
    """Rows of logits and of gradients in turn in one buffer: as into a buffer of their own, and the logits as they were."""
    g = torch.Generator(device=DEV).manual_seed(rows)
    both = torch.randn(rows, 2 * vocab + gap, generator=g, device=DEV).to(dtype)
    t = torch.randint(-1, vocab, (rows,), generator=g, device=DEV)
    adv, old = torch.randn(rows, generator=g, device=DEV), torch.randn(rows, generator=g, device=DEV) - 9
    for x, out in ((both[:, :vocab], both[:, vocab:2 * vocab]), (both[:, vocab + gap:], both[:, :vocab])):
        kept, want = x.clone(), torch.empty(rows, vocab, dtype=dtype, device=DEV)
        logp, rs, stats = torch.zeros(rows, device=DEV), torch.zeros(rows, 2, device=DEV), torch.zeros(4, device=DEV)
        gs.gs_token_logp(x, t, logp, rs, d_workspace=workspace())
        for call in (lambda o: gs.gs_token_logp_grad(x, t, rs, adv, o),
                     lambda o: gs.gs_policy_loss(x, t, old, None, adv, None, gs.PolicyHParams(), logp, o, stats, workspace())):
            call(want)
            call(out)
            assert torch.equal(x, kept)
            # rows cut in other places take their vectors' exponentials another way round
            off = 2.0 ** -7 if dtype == BF16 else 1e-5
            assert float((out.double() - want.double()).abs().max()) <= off * float(want.abs().max())


def long_batch(rows, vocab, dtype):
    g = torch.Generator(device=DEV).manual_seed(rows)
    z = torch.empty(rows, vocab, dtype=dtype, device=DEV)
    t = torch.randint(0, vocab, (rows,), generator=g, device=DEV)
    t[torch.rand(rows, generator=g, device=DEV) < 0.1] = -1
    logp = torch.zeros(rows, dtype=torch.float64, device=DEV)
    for a in range(0, rows, 128):
        z[a:a + 128] = torch.randn(min(128, rows - a), vocab, generator=g, device=DEV) * 2
        x = torch.log_softmax(z[a:a + 128].double(), 1)
        logp[a:a + 128] = torch.where(t[a:a + 128] >= 0, x.gather(1, t[a:a + 128].clamp(min=0)[:, None])[:, 0], 0.0)
    return g, z, t, logp


@pytest.mark.parametrize("rows,vocab,dtype", [(4100, 262_144, BF16), (3980, 524_300, BF16)])
def test_more_rows_in_parts_than_the_workspace_holds(rows, vocab, dtype):
    """A second run through the same partials: every log-probability, the sums, and the gradient of rows on both sides, in place."""
    g, z, t, logp = long_batch(rows, vocab, dtype)
    chunk = 262_144 // (2 * -(-vocab // (-(-(-(-vocab // 64)) // 8192) * 8192)))         # 16 bytes a part in a workspace of 2 MB
    look = [0, 1, chunk - 2, chunk - 1, chunk, chunk + 1, rows - 1]
    assert rows > chunk + 1
    live = (t >= 0).cpu().numpy()
    want = logp.cpu().numpy()
    bound = np.where(live, O.U * (8 * np.abs(want) + 8 * 20 + 64), 0.0)                    # ln S is less than 20
    got, rs = torch.full((rows,), 5.0, device=DEV), torch.full((rows, 2), 5.0, device=DEV)
    for stats in (None, rs):
        gs.gs_token_logp(z, t, got.fill_(5.0), stats, d_workspace=workspace())
        within(got, want, bound, "logp")
    old, adv = (logp - torch.randn(rows, generator=g, device=DEV).double() * 0.05).float(), torch.randn(rows, generator=g, device=DEV)
    w = torch.full((rows,), 1.0 / rows, device=DEV)
    n = lambda x: x.double().cpu().numpy()  # noqa: E731
    sums, off_sums, dlogp, off = O.policy(want, bound, live, n(old), n(old), n(adv), n(w), 0.2, 0.28, 0.1)
    rest, tt = n(z[look]), t[look].cpu().numpy()
    d, g_bound = O.dlogits(rest, tt, 1.0, dlogp[look], off[look], dtype == BF16)
    hp = gs.PolicyHParams(clip_high=0.28, kl_coef=0.1)
    for out in (None, z):
        stats = torch.full((4,), 9.0, device=DEV)
        gs.gs_policy_loss(z, t, old, old, adv, w, hp, got.fill_(5.0), out, stats, workspace())
        within(got, want, bound, "logp")
        within(stats, sums, off_sums, "stats")
    within(z[look], d, g_bound, "dlogits")


@pytest.mark.parametrize("dtype", [BF16])
def test_more_rows_than_a_launch_takes(dtype):
    """2^32 work items and more, of a wave a row: scored, with the policy loss in one pass, and the gradient of the log-probabilities."""
    rows, vocab = (1 << 26) + 1000, 2
    g = torch.Generator(device=DEV).manual_seed(2)
    z = torch.randn(rows, vocab, generator=g, device=DEV).to(dtype)
    t = torch.randint(-1, vocab, (rows,), generator=g, device=DEV)
    live = t >= 0
    x = torch.log_softmax(z.double(), 1)
    want = torch.where(live, x.gather(1, t.clamp(min=0)[:, None])[:, 0], 0.0)
    hot = torch.nn.functional.one_hot(t.clamp(min=0), vocab)
    grad = torch.where(live[:, None], hot - x.exp(), 0.0)
    del x, hot
    logp, rs = torch.full((rows,), 5.0, device=DEV), torch.full((rows, 2), 5.0, device=DEV)
    gs.gs_token_logp(z, t, logp, rs, d_workspace=workspace())
    assert float((logp - want).abs().max()) < 1e-5
    out = torch.full_like(z, 3.0)
    gs.gs_token_logp_grad(z, t, rs, torch.ones(rows, device=DEV), out)
    assert float((out - grad).abs().max()) < 2.0 ** -8 + 1e-5
    adv, stats = torch.ones(rows, device=DEV), torch.zeros(4, device=DEV)
    gs.gs_policy_loss(z, t, logp, None, adv, None, gs.PolicyHParams(), rs.view(-1)[:rows].fill_(5.0), out.fill_(3.0), stats, workspace())
    assert torch.equal(rs.view(-1)[:rows], logp)
    assert float((out + grad).abs().max()) < 2.0 ** -8 + 1e-5                              # ratios of 1
    n = int(live.sum())
    assert stats[0] == stats[1] == torch.tensor(-float(n)).float() and stats[2] == stats[3] == 0


def test_a_norm_of_more_tiles_than_partials():
    """300 tensors of 1024 tiles each over the same memory, in two tables: tiles twice as long."""
    n = 1 << 22
    flat = torch.randn(n + 3, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV)
    tensors = [flat[i % 4:i % 4 + n - i] for i in range(300)]
    sums = flat.double().square().cumsum(0)
    S = sum(float(sums[i % 4 + n - i - 1]) - (float(sums[i % 4 - 1]) if i % 4 else 0.0) for i in range(300))
    sq = torch.full((1,), 7.0, dtype=torch.float64, device=DEV)
    for accumulate in (False, True):
        gs.gs_grads_sqnorm(tensors, sq, workspace(), accumulate=accumulate)
        assert float(sq) == pytest.approx(S * (2 if accumulate else 1), rel=1e-11)          # the running sum's own error
