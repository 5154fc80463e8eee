"""GPU tests of the losses' sums over tokens: what 64 bits hold and 32 do not, on both sides of the lines between the
launches that add them up."""
from __future__ import annotations

import pytest
import torch

from gpu_util import DEV, gs
from test_gpu_losses import BF16, F32, workspace

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
