"""GPU tests of the losses' sums over tokens and pairs: what 64 bits hold and 32 do not, on both sides of the lines between the
launches that add them up."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import loss_oracle as O
from gpu_util import DEV, gs
from test_gpu_losses import BF16, F32, f32, within, workspace

pytestmark = pytest.mark.gpu


def certain_rows(rows, vocab, dtype):
    """Rows whose token has all of the probability: log-probabilities of exactly 0."""
    z = torch.full((rows, vocab), -float("inf"), dtype=dtype, device=DEV)
    t = torch.arange(rows, device=DEV) * 7 % vocab
    z[torch.arange(rows, device=DEV), t] = 0.0
    return z, t


@pytest.mark.parametrize("rows,vocab,dtype,gradient", [
    (2, 1, BF16, True), (100, 1, F32, True), (127, 5, BF16, False), (128, 1, BF16, True), (128, 300, F32, False), (129, 1, BF16, True), (5000, 3, F32, True),
    (2, 45_000, BF16, True), (16, 60_000, BF16, False), (50, 131_072, BF16, True), (50, 131_072, BF16, False), (128, 98_400, F32, True), (129, 98_400, F32, True)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_policy_terms_are_added_in_64_bits(rows, vocab, dtype, gradient, accumulate):
    """Two terms of a product of 48 bits each, of which all but the last bit cancels: in 64 bits nothing is rounded."""
    z, t = certain_rows(rows, vocab, dtype)
    w, adv = torch.ones(rows, device=DEV), torch.zeros(rows, device=DEV)
    w[0] = 1 + 2.0 ** -23
    adv[0] = 1 + 2.0 ** -23
    adv[rows - 1] = -(1 + 2.0 ** -22)
    logp, stats = torch.ones(rows, device=DEV), torch.zeros(4, device=DEV)
    gs.gs_policy_loss(z, t, torch.zeros(rows, device=DEV), None, adv, w, gs.PolicyHParams(), logp, z if gradient else None, stats, workspace(),
                      accumulate=accumulate)
    assert not logp.any()
    assert stats.tolist() == [-2.0 ** -46, -2.0 ** -46, 0.0, 0.0]


@pytest.mark.parametrize("pairs", [1, 100, 128, 129, 130, 1000, 70_000, 262_000, 262_144, 300_001])
@pytest.mark.parametrize("low,high", [(15.0, 25.0), (40.0, 60.0), (-1.0, 1.0)])
def test_preference_loss_of_well_separated_pairs(pairs, low, high):
    """ln(1 + exp(-h)) turns by h times what h turns by, relatively: from a margin in 64 bits, added in 64 and rounded once."""
    g = torch.Generator().manual_seed(pairs)
    h = torch.rand(pairs, generator=g).numpy() * (high - low) + low
    chosen = -torch.rand(pairs, generator=g).numpy()
    logp = np.concatenate([chosen, chosen - h]).astype(np.float32)
    offsets = np.arange(2 * pairs + 1, dtype=np.int64)
    x = logp.astype(float)
    h = x[:pairs] - x[pairs:]
    scale = float(np.float32(1.0 / pairs))
    want = scale * (np.maximum(-h, 0) + np.log1p(np.exp(-np.abs(h)))).sum()
    margins, dlogp, loss = (torch.zeros(n, dtype=F32, device=DEV) for n in (pairs, 2 * pairs, 1))
    gs.gs_preference_loss(f32(logp), None, None, torch.tensor(offsets, device=DEV), gs.PreferenceHParams(beta=1.0, scale=1.0 / pairs), margins, dlogp,
                          loss, workspace())
    within(margins, h, 2 * O.U * np.abs(h), "margins")
    within(loss, np.array([want]), 2 * O.U * want, "loss")
    up = scale / (1 + np.exp(h))
    within(dlogp, np.concatenate([-up, up]), np.tile(2 * O.U * up, 2) + O.TINY, "dlogp")


def test_preference_loss_of_more_pairs_than_partials():
    """Every output, sequences of any length, accumulating, the same bits every time."""
    pairs = 300_001
    g = torch.Generator().manual_seed(1)
    offsets = np.concatenate([[0], np.cumsum(torch.randint(0, 5, (2 * pairs,), generator=g).numpy())]).astype(np.int64)
    tokens = int(offsets[-1])
    logp = (-torch.rand(tokens, generator=g) * 6).numpy()
    ref = (logp + torch.randn(tokens, generator=g).numpy() * 0.3).astype(np.float32)
    w = (torch.rand(tokens, generator=g) < 0.8).float().numpy()
    w[offsets[5]:offsets[6]] = 0.0
    hp = gs.PreferenceHParams(beta=0.3, label_smoothing=0.1, scale=1.0 / pairs)
    e, beta, scale = (float(np.float32(v)) for v in (0.1, 0.3, 1.0 / pairs))
    r = np.concatenate([[0.0], np.cumsum(np.where(w != 0, w.astype(float) * (logp.astype(float) - ref), 0.0))])
    sums = r[offsets[1:]] - r[offsets[:-1]]
    h = beta * (sums[:pairs] - sums[pairs:])
    want = scale * ((1 - e) * np.log1p(np.exp(-h)) + e * np.log1p(np.exp(h))).sum()
    slope = scale * beta * (e / (1 + np.exp(-h)) - (1 - e) / (1 + np.exp(h)))
    d = np.repeat(np.concatenate([slope, -slope]), np.diff(offsets)) * w
    args = f32(logp), f32(ref), f32(w), torch.tensor(offsets, device=DEV), hp
    kept = None
    for first in (0.0, 3.0, 0.0):
        margins, dlogp, loss = torch.zeros(pairs, device=DEV), torch.full((tokens,), 9.0, device=DEV), torch.full((1,), first, device=DEV)
        gs.gs_preference_loss(*args, margins, dlogp, loss, workspace(), accumulate=first != 0)
        # running sums of a million terms of the oracle: 1e-9
        within(margins, h, 2 * O.U * np.abs(h) + 1e-9, "margins")
        within(loss, np.array([want + first]), 2 * O.U * (want + first) + 1e-9, "loss")
        within(dlogp, d, 4 * O.U * np.abs(d) + 1e-9 * scale, "dlogp")
        if first == 0.0:
            if kept is not None:
                assert all(torch.equal(a, b) for a, b in zip(kept, (margins, dlogp, loss)))
            kept = margins, dlogp, loss


@pytest.mark.parametrize("rows,vocab,dtype", [(8, 50, BF16), (8, 4000, F32), (150, 2000, BF16), (8, 70_000, BF16), (200, 100_000, F32)])
def test_ratios_beyond_32_bits(rows, vocab, dtype):
    """Tokens that the old policy gave next to nothing: a ratio over the largest 32-bit number times no advantage, or a tiny one, is what the
    formula has, and the other tokens' loss and gradient are theirs."""
    g = torch.Generator().manual_seed(rows)
    z = (torch.randn(rows, vocab, generator=g) * 2).to(dtype).to(DEV)
    t = torch.randint(0, vocab, (rows,), generator=g)
    zz = z.double().cpu().numpy()
    lp, bound, live = O.token_logp(zz, t.numpy(), 1.0)
    old = (lp - 0.05).astype(np.float32)
    adv = torch.randn(rows, generator=g).numpy()
    old[1], adv[1] = -300.0, 0.0
    old[2], adv[2] = -150.0, -0.0
    old[3], adv[3] = lp[3] - 89.5, -2e-38
    old[4], adv[4] = lp[4] - 95.0, -2e-38
    old[5], adv[5] = lp[5] - 200.0, 1.0                  # clipped
    old[6], adv[6] = -900.0, 0.0
    weights = np.full(rows, 1e-3, np.float32)
    rest = np.arange(rows) != 6                          # over the largest 64-bit number too, times 0
    held = old.copy()
    held[5] = lp[5] - 1.0                                # clipped as well: the same terms, with a bound of their size
    stats, off_stats, d, o = O.policy(lp[rest], bound[rest], live[rest], held[rest].astype(float), None, adv[rest].astype(float),
                                      weights[rest].astype(float), 0.2, 0.2, 0.0)
    dlogp, off = np.insert(d, 6, 0.0), np.insert(o, 6, 0.0)
    want, g_bound = O.dlogits(zz, t.numpy(), 1.0, dlogp, off, dtype == BF16)
    for gradient in (True, False):
        out = torch.full_like(z, 7.0) if gradient else None
        logp, got = torch.zeros(rows, device=DEV), torch.zeros(4, device=DEV)
        gs.gs_policy_loss(z, t.to(DEV), f32(old), None, f32(adv), f32(weights), gs.PolicyHParams(), logp, out, got, workspace())
        within(got, stats, off_stats, "stats")
        if gradient:
            within(out, want, g_bound, "dlogits")
