"""GPU tests of the losses on rows of logits: every entry point against its definition in 64 bits (loss_oracle.py, which
derives the bounds), at the lengths, alignments, masks and values where they can go wrong."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import loss_oracle as O
from gpu_util import DEV, gs

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
WS = 1 << 22


def workspace():
    return torch.full((WS,), 0xFF, dtype=torch.uint8, device=DEV)      # NaN: nothing of it may be read before it is written


def f32(x):
    return torch.tensor(np.asarray(x), dtype=F32, device=DEV)


def within(got, want, bound, what):
    got = got.detach().double().cpu().numpy()
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(got), nan), f"{what}: NaN in other places ({np.isnan(got).sum()} against {nan.sum()})"
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf]), f"{what}: infinities"
    ok = ~nan & ~inf
    bound = np.broadcast_to(bound, want.shape)
    over = np.abs(got - np.where(ok, want, got)) - bound
    worst = np.where(ok, over, -1).max() if want.size else -1
    assert worst <= 0, f"{what}: {(over[ok] > 0).sum()} of {want.size} too far off, by up to {worst}"


class Rows:
    """Rows of logits in a buffer of NaN: at `offset` elements from a 512-byte boundary, `gap` elements between them."""

    def __init__(self, rows, vocab, dtype, seed=0, offset=0, gap=0, prompt=0.2, spread=3.0, shift=0.0):
        g = torch.Generator().manual_seed(seed)
        self.rows, self.vocab, self.dtype, self.stride = rows, vocab, dtype, vocab + gap
        self.flat = torch.full((offset + rows * self.stride + 64,), float("nan"), dtype=dtype, device=DEV)
        self.logits = self.flat[offset:].as_strided((rows, vocab), (self.stride, 1))
        self.logits.copy_((torch.randn(rows, vocab, generator=g) * spread + shift).to(dtype))
        self.target = torch.randint(0, vocab, (rows,), generator=g)
        self.target[torch.rand(rows, generator=g) < prompt] = -1
        self.g = g

    def numpy(self):
        return self.logits.double().cpu().numpy(), self.target.numpy()

    def like(self, offset, gap, fill=7.0):
        flat = torch.full((offset + self.rows * (self.vocab + gap) + 64,), fill, dtype=self.dtype, device=DEV)
        return flat, flat[offset:].as_strided((self.rows, self.vocab), (self.vocab + gap, 1))

    def untouched(self, flat, offset, gap, fill=7.0):
        mask = torch.ones_like(flat, dtype=torch.bool)
        mask[offset:].as_strided((self.rows, self.vocab), (self.vocab + gap, 1)).fill_(False)
        assert bool((flat[mask] == fill).all()), "written outside the rows"


VOCABS = [1, 2, 3, 7, 8, 9, 63, 64, 65, 511, 1000, 2047, 2048, 2049, 4097, 8192, 16385, 32003, 50001, 65536, 100003, 131072, 140001, 262147]


def logp_check(x, temperature=1.0, stats=True):
    logp = torch.full((x.rows,), float("nan"), dtype=F32, device=DEV)
    rs = torch.full((x.rows, 2), float("nan"), dtype=F32, device=DEV) if stats else None
    gs.gs_token_logp(x.logits, x.target.to(DEV), logp, rs, temperature=temperature, d_workspace=workspace())
    z, t = x.numpy()
    want, bound, live = O.token_logp(z, t, temperature)
    within(logp, want, bound, "logp")
    if stats:
        _, s, m = O.soft_rows(z, 1.0 / temperature)
        assert np.array_equal(rs[:, 0].double().cpu().numpy(), np.where(live, m[:, 0], 0.0), equal_nan=True)
        within(rs[:, 1], np.where(live, s[:, 0], 1.0), np.where(live, 64 * O.U * s[:, 0], 0.0), "S")
    return logp, rs, want, bound, live


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("vocab", VOCABS)
def test_token_logp_at_every_vocabulary(vocab, dtype):
    for rows, offset, gap, temperature in ((1, 0, 0, 1.0), (5, 3, 0, 0.7), (3, 0, 5, 1.0)):
        logp_check(Rows(rows, vocab, dtype, seed=vocab, offset=offset, gap=gap), temperature)


@pytest.mark.parametrize("rows", [1, 2, 3, 4, 8, 15, 16, 31, 33, 64, 100, 127, 128, 129, 255, 256, 257, 300, 512, 600, 1025])
def test_token_logp_at_every_number_of_rows(rows):
    for vocab, dtype in ((9001, BF16), (40_003, BF16), (12_345, F32)):
        logp_check(Rows(rows, vocab, dtype, seed=rows), stats=rows % 2 == 0)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("temperature", [1e-4, 0.05, 3.0, 1e4])
def test_temperatures(dtype, temperature):
    logp_check(Rows(6, 5003, dtype, seed=3), temperature)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shift", [-30000.0, 300.0, 1e6])
def test_logits_far_from_zero(dtype, shift):
    x = Rows(6, 5003, dtype, seed=4, shift=shift)
    _, rs, *_ = logp_check(x)
    grad_check(x, rs, 1.0)


def grad_check(x, rs, temperature, offset=0, gap=0, in_place=False, seed=0, z=None):
    g = torch.Generator().manual_seed(seed)
    dlogp = torch.randn(x.rows, generator=g)
    dlogp[torch.rand(x.rows, generator=g) < 0.2] = 0.0
    z, t = x.numpy()
    if in_place:
        flat, out = x.flat, x.logits
    else:
        flat, out = x.like(offset, gap)
    gs.gs_token_logp_grad(x.logits, x.target.to(DEV), rs, f32(dlogp), out, temperature=temperature)
    want, bound = O.dlogits(z, t, temperature, dlogp.double().numpy(), np.zeros(x.rows), x.dtype == BF16)
    within(out, want, bound, "dlogits")
    if not in_place:
        x.untouched(flat, offset, gap)
    return want


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("vocab", VOCABS)
def test_gradient_at_every_vocabulary(vocab, dtype):
    for rows, offset, gap, o2, g2, temperature in ((4, 0, 0, 0, 0, 1.0), (5, 3, 0, 3, 0, 0.7), (5, 0, 3, 1, 0, 1.0)):
        x = Rows(rows, vocab, dtype, seed=vocab + 1, offset=offset, gap=gap)
        _, rs, *_ = logp_check(x, temperature)
        grad_check(x, rs, temperature, o2, g2)
        grad_check(x, rs, temperature, in_place=True)


def special(x):
    """Rows with what logits can hold besides numbers of ordinary size."""
    low = torch.finfo(x.dtype).min
    z = x.logits
    z[0, ::2] = -float("inf")                      # excluded tokens
    z[0, x.target[0]] = 1.0
    z[1, :] = -float("inf")                        # nothing left
    z[2, ::3] = low                                # masks of the type's lowest value
    z[2, x.target[2]] = 2.0
    z[3, :] = low                                  # nothing but them
    z[4, 17] = float("nan")
    z[5, 19] = float("inf")
    z[6, x.target[6]] = -float("inf")              # the token itself is excluded
    z[7, :] = -float("inf")
    z[7, x.target[7]] = -3.0                       # it is the only one left
    z[8, :] = torch.finfo(x.dtype).max
    z[9, 5::7] = low
    z[9, x.target[9]] = low
    z[10, :] = float("nan")
    x.target[10] = -100                            # no token: nothing of the row counts
    z[11, :] = float("nan")
    x.target[11] = x.vocab


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("vocab", [100, 5003, 40_001, 131_072, 200_000])
def test_masked_infinite_and_missing_logits(vocab, dtype):
    x = Rows(12, vocab, dtype, seed=8, prompt=0.0)
    special(x)
    z, t = x.numpy()
    with np.errstate(all="ignore"):
        logp, rs, *_ = logp_check(x, stats=False)
        rs = torch.zeros(12, 2, dtype=F32, device=DEV)
        gs.gs_token_logp(x.logits, t_dev(x), logp, rs, d_workspace=workspace())
        assert [bool(v) for v in torch.isnan(logp)] == [i in (1, 4, 5) for i in range(12)]
        grad_check(x, rs, 1.0)
        policy_check(x, plain_weights=True)


def t_dev(x):
    return x.target.to(DEV)


def policy_inputs(x, temperature, seed=0):
    g = torch.Generator().manual_seed(seed)
    z, t = x.numpy()
    with np.errstate(all="ignore"):
        logp, bound, live = O.token_logp(z, t, temperature)
    fine = np.where(np.abs(logp) < 1e4, logp, -1.0)        # else two log-probabilities would differ by their rounding
    delta = torch.randn(x.rows, generator=g).double().numpy() * 0.3
    for edge in (np.log(0.8), np.log(1.28)):       # 2^-24 units of logp decide there on which side a token is
        delta = np.where(np.abs(delta - edge) < 1e-3, delta + 5e-3, delta)
    old = (fine - delta).astype(np.float32)
    ref = (fine + torch.randn(x.rows, generator=g).double().numpy() * 0.3).astype(np.float32)
    adv = torch.randn(x.rows, generator=g).numpy()
    weights = torch.rand(x.rows, generator=g).numpy() + 0.1
    weights[torch.rand(x.rows, generator=g).numpy() < 0.15] = 0.0
    return logp, bound, live, old, ref, adv, weights


def policy_check(x, temperature=1.0, kl_coef=0.1, with_ref=True, plain_weights=False, offset=0, gap=0, in_place=False, accumulate=False, seed=0, gradient=True):
    logp, bound, live, old, ref, adv, weights = policy_inputs(x, temperature, seed)
    if plain_weights:
        weights = np.ones(x.rows, np.float32)
    z, t = x.numpy()
    with np.errstate(all="ignore"):
        stats, off_stats, dlogp, off = O.policy(logp, bound, live, *(v.astype(np.float64) for v in (old,)), ref.astype(np.float64) if with_ref else None,
                                                adv.astype(np.float64), weights.astype(np.float64), 0.2, 0.28, kl_coef)
        want, g_bound = O.dlogits(z, t, temperature, dlogp, off, x.dtype == BF16)
    dead = (weights == 0) | ~live
    for v in (old, ref, adv):
        v[dead] = np.nan                           # not looked at
    want[dead], g_bound[dead] = 0.0, 0.0
    flat, out = (x.flat, x.logits) if in_place else x.like(offset, gap)
    got_logp = torch.full((x.rows,), float("nan"), dtype=F32, device=DEV)
    got_stats = torch.full((4,), 2.5 if accumulate else float("nan"), dtype=F32, device=DEV)
    hp = gs.PolicyHParams(temperature=temperature, clip_low=0.2, clip_high=0.28, kl_coef=kl_coef)
    gs.gs_policy_loss(x.logits, t_dev(x), f32(old), f32(ref) if with_ref else None, f32(adv), None if plain_weights else f32(weights), hp,
                      got_logp, out if gradient else None, got_stats, workspace(), accumulate=accumulate)
    within(got_logp, np.where(dead, 0.0, logp), np.where(dead, 0.0, bound), "logp")
    if not np.isnan(stats).any():
        within(got_stats, stats + (2.5 if accumulate else 0.0), off_stats + 4 * O.U * 2.5, "stats")
    if gradient:
        within(out, want, g_bound, "dlogits")
        if not in_place:
            x.untouched(flat, offset, gap)
    return got_stats, got_logp, out


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("vocab", VOCABS)
def test_policy_loss_at_every_vocabulary(vocab, dtype):
    for rows, kw in ((5, {}), (1, {"temperature": 0.7}), (4, {"offset": 1}), (6, {"in_place": True}), (3, {"kl_coef": 0.0}), (3, {"with_ref": False})):
        policy_check(Rows(rows, vocab, dtype, seed=vocab + rows, prompt=0.2 if rows > 1 else 0.0), **kw)
    policy_check(Rows(7, vocab, dtype, seed=vocab, offset=5, gap=3), offset=2, gap=9)
    policy_check(Rows(7, vocab, dtype, seed=vocab, offset=1, gap=8), offset=1, gap=0)


@pytest.mark.parametrize("rows", [2, 100, 256, 1000, 1024, 1025, 5000, 40_000])
def test_policy_loss_at_every_number_of_rows(rows):
    policy_check(Rows(rows, 333, BF16, seed=rows), accumulate=rows % 2 == 0)
    policy_check(Rows(rows, 130, F32, seed=rows), gradient=False)


@pytest.mark.parametrize("vocab,dtype", [(40_003, BF16), (98_299, BF16), (98_310, BF16), (20_011, F32), (49_160, F32)])
@pytest.mark.parametrize("rows", [1, 15, 16, 17, 63, 64, 65, 130])
def test_policy_loss_of_few_long_rows(rows, vocab, dtype):
    """Both sides of the lines between rows in parts and rows held, with and without a gradient, and accumulating."""
    policy_check(Rows(rows, vocab, dtype, seed=rows), accumulate=rows % 2 == 1)
    policy_check(Rows(rows, vocab, dtype, seed=rows + 1, offset=1, gap=2), in_place=True, accumulate=rows % 2 == 0)
    policy_check(Rows(rows, vocab, dtype, seed=rows), gradient=False)


def test_no_rows():
    """An empty batch: sums of 0, or what was there; nothing else is touched."""
    z, t, none = torch.empty(0, 60_000, dtype=BF16, device=DEV), torch.empty(0, dtype=torch.int64, device=DEV), torch.empty(0, device=DEV)
    stats = torch.full((4,), 7.0, device=DEV)
    gs.gs_policy_loss(z, t, none, None, none, None, gs.PolicyHParams(), none, z, stats, workspace(), accumulate=True)
    assert stats.tolist() == [7.0] * 4
    gs.gs_policy_loss(z, t, none, None, none, None, gs.PolicyHParams(), none, z, stats, workspace())
    assert stats.tolist() == [0.0] * 4
    gs.gs_token_logp(z, t, none, d_workspace=workspace())
    gs.gs_token_logp_grad(z, t, none.view(0, 2), none, z)


def test_no_row_counts():
    """A batch of prompts, and one of weights of 0."""
    for rows in (1, 70, 300):
        x = Rows(rows, 9000, BF16, seed=rows, prompt=1.1)
        x.logits.fill_(float("nan"))
        _, out = x.like(0, 0)
        logp, stats = torch.full((rows,), 3.0, device=DEV), torch.full((4,), 3.0, device=DEV)
        nan = torch.full((rows,), float("nan"), device=DEV)
        gs.gs_policy_loss(x.logits, t_dev(x), nan, nan, nan, None, gs.PolicyHParams(kl_coef=0.1), logp, out, stats, workspace())
        assert not logp.any() and not out.any() and not stats.any()
        x.target.fill_(5)
        out.fill_(1.0)
        gs.gs_policy_loss(x.logits, t_dev(x), nan, nan, nan, torch.zeros(rows, device=DEV), gs.PolicyHParams(), logp.fill_(2.0), out, stats.fill_(2.0), workspace())
        assert not logp.any() and not out.any() and not stats.any()


# vectors of a row (8 or 4 elements) at which another kernel takes it, from both sides; with and without a first line to share
HELD_LINES = [256, 512, 1024, 2048, 3072, 4096, 6144, 8192, 12288, 16384, 20480, 24576]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("vecs", HELD_LINES)
def test_lines_between_kernels(vecs, dtype):
    per = 8 if dtype == BF16 else 4
    for vocab, offset, gap in ((vecs * per, 0, 0), (vecs * per + per, 0, 0), (vecs * per - 7 * per, 1, 1), (vecs * per - 7 * per + per - 1, per - 1, 1),
                               (vecs * per - 6 * per, 8 * per - 1, 1)):
        x = Rows(2, vocab, dtype, seed=vecs, offset=offset, gap=gap, prompt=0.0)
        x.logits[0, 0], x.logits[1, -1] = 9.0, 8.0          # the ends count
        x.target[0], x.target[1] = vocab - 1, 0
        logp_check(x)
        x = Rows(70 if vecs > 3000 else 3, vocab, dtype, seed=vecs, offset=offset, gap=gap)
        policy_check(x, in_place=True)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_policy_gradient_against_differences(dtype):
    """dlogits against central differences of the loss in 64 bits (step 1e-4: the loss is three times differentiable with
    derivatives of order one, so they are off by some 1e-8; the library's bound is added)."""
    x = Rows(4, 37, dtype, seed=2, prompt=0.0)
    logp, bound, live, old, ref, adv, weights = policy_inputs(x, 0.7)
    _, _, out = policy_check(x, temperature=0.7, seed=0)
    z, t = x.numpy()

    def loss(zz):
        lp, b, lv = O.token_logp(zz, t, 0.7)
        return O.policy(lp, b, lv, old.astype(float), ref.astype(float), adv.astype(float), weights.astype(float), 0.2, 0.28, 0.1)[0][0]

    step, want = 1e-4, np.zeros_like(z)
    for r in range(z.shape[0]):
        for i in range(z.shape[1]):
            up, down = z.copy(), z.copy()
            up[r, i] += step
            down[r, i] -= step
            want[r, i] = (loss(up) - loss(down)) / (2 * step)
    within(out, want, 1e-7 + np.abs(want) * (2.0 ** -8 if dtype == BF16 else 2e-5), "dlogits")


# sequences by their lengths: pairs of (chosen, rejected)
PAIRS = {
    "one token each": [(1, 1)],
    "empty ones": [(0, 3), (4, 0), (0, 0)],
    "uneven": [(5, 700), (512, 513), (64, 63), (1, 2000)],
    "long": [(30_001, 4)],
    "sixty-five": [(i % 7 + 1, i % 5) for i in range(65)],
    "two hundred and fifty-six": [(i % 3, 2) for i in range(256)],
    "many": [(i % 37, (i * 7) % 53) for i in range(1500)],
}


def pref_inputs(lengths, seed=0, before=0, behind=0):
    g = torch.Generator().manual_seed(seed)
    seqs = [c for c, _ in lengths] + [r for _, r in lengths]
    offsets = before + np.concatenate([[0], np.cumsum(seqs)])
    tokens = int(offsets[-1]) + behind
    logp = (-torch.rand(tokens, generator=g) * 6).numpy()
    ref = (logp + torch.randn(tokens, generator=g).numpy() * 0.3).astype(np.float32)
    weights = (torch.rand(tokens, generator=g) < 0.8).float().numpy()
    return tokens, offsets.astype(np.int64), logp, ref, weights


def pref_check(tokens, offsets, logp, ref, weights, pairs, hp, accumulate=False):
    w = np.ones(tokens, np.float32) if weights is None else weights
    beta, e, scale = (float(np.float32(v)) for v in (hp.beta, hp.label_smoothing, hp.scale))
    loss, h, d = O.preference(logp.astype(float), None if ref is None else ref.astype(float), w.astype(float), offsets, pairs, beta, e, scale)
    dead = w == 0
    logp, ref = logp.copy(), None if ref is None else ref.copy()
    logp[dead] = np.nan
    if ref is not None:
        ref[dead] = np.nan
    margins = torch.full((pairs,), float("nan"), dtype=F32, device=DEV)
    dlogp = torch.full((tokens,), float("nan"), dtype=F32, device=DEV)
    out = torch.full((1,), 1.5 if accumulate else float("nan"), dtype=F32, device=DEV)
    gs.gs_preference_loss(f32(logp), None if ref is None else f32(ref), None if weights is None else f32(weights),
                          torch.tensor(offsets, device=DEV), hp, margins, dlogp, out, workspace(), accumulate=accumulate)
    # all sums are in 64 bits: a margin is rounded once, the loss and the slopes are computed in 64 bits from it and rounded once
    within(margins, h, 2 * O.U * np.abs(h) + 1e-12, "margins")
    within(out, np.array([loss + (1.5 if accumulate else 0.0)]), 4 * O.U * (abs(loss) + 1.5) + 2 * O.U * beta * scale * np.abs(h).sum(), "loss")
    within(dlogp, d, 4 * O.U * np.abs(d) + O.TINY, "dlogp")
    return margins, dlogp, out


@pytest.mark.parametrize("name", PAIRS)
@pytest.mark.parametrize("smoothing", [0.0, 0.1])
def test_preference_loss(name, smoothing):
    lengths = PAIRS[name]
    for before, behind, use_ref, use_w in ((0, 0, True, True), (3, 5, True, False), (0, 1, False, True)):
        tokens, offsets, logp, ref, weights = pref_inputs(lengths, before=before, behind=behind)
        hp = gs.PreferenceHParams(beta=0.3, label_smoothing=smoothing, scale=1.0 / len(lengths))
        pref_check(tokens, offsets, logp, ref if use_ref else None, weights if use_w else None, len(lengths), hp, accumulate=before > 0)


def test_preference_loss_of_nothing():
    out = torch.full((1,), 9.0, dtype=F32, device=DEV)
    none = torch.empty(0, dtype=F32, device=DEV)
    d = torch.full((700,), 5.0, dtype=F32, device=DEV)
    gs.gs_preference_loss(d.clone(), None, None, torch.zeros(1, dtype=torch.int64, device=DEV), gs.PreferenceHParams(), none, d, out, workspace(), accumulate=True)
    assert float(out) == 9.0 and not d.any()
    gs.gs_preference_loss(none, None, None, torch.zeros(1, dtype=torch.int64, device=DEV), gs.PreferenceHParams(), none, none, out, workspace())
    assert float(out) == 0.0


def test_preference_offsets_outside_the_tokens_are_taken_inside():
    tokens, offsets, logp, ref, weights = pref_inputs([(50, 60), (70, 80)])
    wild = offsets.copy()
    wild[0], wild[-1] = -5_000_000_000, 1 << 40
    hp = gs.PreferenceHParams(beta=0.3, scale=0.5)
    a = pref_check(tokens, offsets, logp, ref, weights, 2, hp)
    b = pref_check(tokens, wild, logp, ref, weights, 2, hp)
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_preference_margins_far_out():
    """Margins of hundreds: sigmoids of 0 and 1, losses of |h| and of almost nothing."""
    tokens, offsets, logp, ref, weights = pref_inputs([(400, 400)] * 3, seed=5)
    ref = logp + np.repeat(np.array([-3, 0.001, 3, 3, 0.002, -3], np.float32), 400)
    pref_check(tokens, offsets, logp, ref, None, 3, gs.PreferenceHParams(beta=1.0))


def test_preference_gradient_against_differences():
    lengths = [(3, 4), (2, 6)]
    tokens, offsets, logp, ref, weights = pref_inputs(lengths, seed=3)
    hp = gs.PreferenceHParams(beta=0.5, label_smoothing=0.125, scale=0.5)
    _, dlogp, _ = pref_check(tokens, offsets, logp, ref, weights, 2, hp)
    f = lambda lp: O.preference(lp, ref.astype(float), weights.astype(float), offsets, 2, 0.5, 0.125, 0.5)[0]  # noqa: E731
    want = np.zeros(tokens)
    for i in range(tokens):
        up, down = logp.astype(float), logp.astype(float)
        up[i] += 1e-4
        down[i] -= 1e-4
        want[i] = (f(up) - f(down)) / 2e-4
    within(dlogp, want, 1e-7, "dlogp")


# ---- the calls together, streams, graphs, large offsets ----------------------------------------

def all_calls(x, seed=0):
    """Every entry point once, as a closure over its buffers, and the tensors it writes."""
    logp0, _, _, old, ref, adv, weights = policy_inputs(x, 1.0, seed)
    n, d = x.rows, {}
    d["logp"], d["rs"], d["plogp"], d["stats"] = (torch.zeros(s, dtype=F32, device=DEV) for s in (n, (n, 2), n, 4))
    d["dlogp"], d["margins"], d["loss"] = (torch.zeros(s, dtype=F32, device=DEV) for s in (n, 1, 1))
    d["g1"], d["g2"] = torch.zeros_like(x.logits), torch.zeros_like(x.logits)
    ws, t = workspace(), t_dev(x)
    old, ref, adv, weights = f32(old), f32(ref), f32(adv), f32(weights)
    offsets = torch.tensor([0, n // 3, n], device=DEV)

    def run(stream=None):
        gs.gs_token_logp(x.logits, t, d["logp"], d["rs"], d_workspace=ws, stream=stream)
        gs.gs_preference_loss(d["logp"], ref, weights, offsets, gs.PreferenceHParams(), d["margins"], d["dlogp"], d["loss"], ws, stream=stream)
        gs.gs_token_logp_grad(x.logits, t, d["rs"], d["dlogp"], d["g1"], stream=stream)
        gs.gs_policy_loss(x.logits, t, old, ref, adv, weights, gs.PolicyHParams(kl_coef=0.1), d["plogp"], d["g2"], d["stats"], ws, stream=stream)
    return run, d


@pytest.mark.parametrize("rows,vocab,dtype", [(3, 40_001, BF16), (300, 9000, BF16), (64, 50_001, F32), (2, 262_147, F32)])
def test_same_bits_every_time_on_every_stream_and_from_a_graph(rows, vocab, dtype):
    x = Rows(rows, vocab, dtype, seed=1, prompt=0.0)
    run, d = all_calls(x)
    run()
    torch.cuda.synchronize()
    want = {k: v.clone() for k, v in d.items()}

    def same():
        torch.cuda.synchronize()
        for k, v in d.items():
            assert torch.equal(v, want[k]), k
            v.fill_(3.0)
    same()
    run()
    same()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    run(side)
    same()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(4):
        graph.replay()
        same()
        torch.randn(1000, device=DEV).sum().item()


def test_small_launches_finish_alone():
    """Launches whose last workgroup finishes them, hundreds in a row with other inputs each, on two streams with a workspace each."""
    g = torch.Generator(device=DEV).manual_seed(3)
    z = torch.randn(40, 60_000, generator=g, device=DEV, dtype=F32)
    t = torch.randint(0, 4000, (40,), generator=g, device=DEV)
    adv, old = torch.randn(40, generator=g, device=DEV), torch.full((40,), -9.0, device=DEV)
    calls = [(1, 60_000), (7, 45_000), (40, 4000), (33, 5000), (3, 60_000)]
    want, got = {}, []
    streams, ws = [torch.cuda.Stream(), torch.cuda.Stream()], [workspace(), workspace()]
    torch.cuda.synchronize()
    for i in range(400):
        rows, vocab = calls[i % 5]
        first = (i * 7) % (41 - rows)
        logp, rs, plogp, stats = (torch.full(s, float("nan"), device=DEV) for s in ((rows,), (rows, 2), (rows,), (4,)))
        torch.cuda.current_stream().synchronize()
        x, tt, st = z[first:first + rows, :vocab], t[first:first + rows], streams[i % 2]
        gs.gs_token_logp(x, tt, logp, rs, d_workspace=ws[i % 2], stream=st)
        out = None if i % 3 else torch.empty_like(x)
        torch.cuda.current_stream().synchronize()
        gs.gs_policy_loss(x, tt, old[first:first + rows], None, adv[first:first + rows], None, gs.PolicyHParams(), plogp, out, stats, ws[i % 2], stream=st)
        got.append((rows, vocab, first, logp, rs, plogp, stats, out))
    torch.cuda.synchronize()
    for rows, vocab, first, logp, rs, plogp, stats, _ in got:
        key = rows, vocab, first
        if key not in want:
            x = z[first:first + rows, :vocab].double()
            tt = t[first:first + rows]
            w = torch.log_softmax(x, 1).gather(1, tt[:, None])[:, 0]
            r = (w - old[first:first + rows]).exp()
            a = adv[first:first + rows]
            pg = -torch.minimum(r * a, r.clamp(0.8, 1.2) * a)
            want[key] = w, pg.sum(), (pg.abs()).sum()
        w, pg, size = want[key]
        assert float((logp - w).abs().max()) < 2e-5 and float((plogp - w).abs().max()) < 2e-5
        assert float((stats[1] - pg).abs()) <= 3e-5 * float(size) and torch.equal(stats[0], stats[1])


def test_native_and_general_reading_agree(monkeypatch):
    x = Rows(9, 3001, BF16, seed=1, prompt=0.0)
    run, d = all_calls(x)
    taken = []

    class Counting:
        def __init__(self, call):
            self.call = call

        def __getattr__(self, name):
            return lambda *a: (taken.append(name), getattr(self.call, name)(*a))[1]

    with monkeypatch.context() as mp:
        mp.setattr(gs, "_call", Counting(gs._call))
        run()
    torch.cuda.synchronize()
    want = {k: v.clone() for k, v in d.items()}
    for v in d.values():
        v.fill_(3.0)

    class General:
        def __getattr__(self, name):
            return lambda *a: None

    with monkeypatch.context() as mp:
        mp.setattr(gs, "_call", General())
        run()
    torch.cuda.synchronize()
    assert set(taken) == {"token_logp", "preference_loss", "token_logp_grad", "policy_loss"}
    assert all(torch.equal(v, want[k]) for k, v in d.items())


def test_offsets_beyond_32_bits():
    """4.5 GB of logits: rows that start behind 2^31 and 2^32 elements' worth of bytes, in place."""
    rows, vocab = 33_200, 65_537
    z = torch.empty(rows, vocab, dtype=BF16, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(1)
    for a in range(0, rows, 2048):
        z[a:a + 2048] = torch.randn(min(2048, rows - a), vocab, generator=g, device=DEV)
    t = torch.randint(0, vocab, (rows,), generator=g, device=DEV)
    look = [0, 1, 16_000, 32_766, 32_768, 33_000, rows - 1]
    rest = z[look].double().cpu().numpy()
    logp, rs = torch.zeros(rows, dtype=F32, device=DEV), torch.zeros(rows, 2, dtype=F32, device=DEV)
    dlogp = torch.randn(rows, generator=g, device=DEV)
    gs.gs_token_logp(z, t, logp, rs, d_workspace=workspace())
    gs.gs_token_logp_grad(z, t, rs, dlogp, z)
    tt = t[look].cpu().numpy()
    want, bound, _ = O.token_logp(rest, tt, 1.0)
    within(logp[look], want, bound, "logp")
    want, bound = O.dlogits(rest, tt, 1.0, dlogp[look].double().cpu().numpy(), np.zeros(len(look)), True)
    within(z[look], want, bound, "dlogits")


def test_wrong_tensors_are_refused():
    x = Rows(4, 100, BF16)
    t, lp, ws = t_dev(x), torch.zeros(4, device=DEV), workspace()
    with pytest.raises(TypeError):
        gs.gs_token_logp(x.logits.half(), t, lp, d_workspace=ws)
    with pytest.raises(TypeError):
        gs.gs_token_logp(x.logits, t.int(), lp, d_workspace=ws)
    with pytest.raises(ValueError):
        gs.gs_token_logp(x.logits.cpu(), t, lp, d_workspace=ws)
    with pytest.raises(ValueError):
        gs.gs_token_logp(x.logits[0], t, lp, d_workspace=ws)
    with pytest.raises(ValueError):
        gs.gs_token_logp(x.logits.t(), t, lp, d_workspace=ws)
    with pytest.raises(ValueError):
        gs.gs_token_logp(x.logits, t[:3], lp, d_workspace=ws)
    with pytest.raises(ValueError):
        gs.gs_token_logp(x.logits, t.cpu(), lp, d_workspace=ws)
    with pytest.raises(gs.GsError):
        gs.gs_token_logp(x.logits, t, lp, d_workspace=ws[:100])
    with pytest.raises(gs.GsError):
        gs.gs_token_logp(x.logits, t, lp, temperature=0.0, d_workspace=ws)
    rs = torch.zeros(4, 2, device=DEV)
    with pytest.raises(ValueError):
        gs.gs_token_logp_grad(x.logits, t, rs, lp, torch.zeros(4, 99, dtype=BF16, device=DEV))
    with pytest.raises(ValueError):
        gs.gs_token_logp_grad(x.logits, t, rs, lp, torch.zeros(4, 100, device=DEV))
    with pytest.raises(gs.GsError):                # overlaps the logits without being them
        flat = torch.zeros(1000, dtype=BF16, device=DEV)
        gs.gs_token_logp_grad(flat[:400].view(4, 100), t, rs, lp, flat[100:500].view(4, 100))
    with pytest.raises(ValueError):
        gs.gs_preference_loss(lp, None, None, torch.zeros(2, dtype=torch.int64, device=DEV), gs.PreferenceHParams(),
                              torch.zeros(1, device=DEV), torch.zeros(4, device=DEV), torch.zeros(1, device=DEV), ws)


@pytest.mark.parametrize("bits", [0x7FF00001, 0x7FF00123, 0x7FF7FFFF, 0x7F800001, 0x7FC00000])
def test_what_a_call_leaves_in_the_workspace_is_no_tag(bits):
    """Upper halves of 64-bit words between 0x7ff00001 and 0x7ff7ffff mark what a launch has left for its last workgroup.  Rows in parts
    with NaN of such bits among the logits leave none."""
    z = torch.randn(4, 60_000, device=DEV, dtype=F32)
    z[:, 100] = torch.tensor(bits, dtype=torch.int32, device=DEV).view(F32)
    t, one, logp, stats = torch.zeros(4, dtype=torch.int64, device=DEV), torch.ones(4, device=DEV), torch.zeros(4, device=DEV), torch.zeros(4, device=DEV)
    for out in (None, torch.empty_like(z)):
        ws = torch.zeros(WS, dtype=torch.uint8, device=DEV)
        gs.gs_policy_loss(z, t, one, None, one, None, gs.PolicyHParams(), logp, out, stats, ws)
        gs.gs_token_logp(z, t, logp, None, d_workspace=ws)
        upper = ws.view(torch.int32)[1::2]
        assert not bool(((upper >= 0x7FF00001) & (upper <= 0x7FF7FFFF)).any())
        assert bool(logp.isnan().all()) and bool(stats[:2].isnan().all())
