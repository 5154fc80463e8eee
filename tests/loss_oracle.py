"""The losses on rows of logits in 64 bits, from their definitions, and how far the library may be from them.

u = 2^-24 is the rounding unit of the 32 bits in which the library holds maxima, sums and log-probabilities.
  S        each exponential is off by at most a few u times its exponent (the exponent's own rounding), and e^-a a is at most 0.37,
           so with the two roundings of a term and the depth of the sum S is off by less than 48 u S
  logp     that, the rounding of ln S and of the two products and differences: u (8 |it (z_t - M)| + 8 |ln S| + 64)
  dlogp    the ratio is off by as much as logp, relatively; each term is a product or two more: 16 u of each term
  dlogits  d ([i = t] - p) it with p off by u (4 |it (z - M)| + 64) p; rounded to bf16 by at most 2^-8 of itself, and a
           value under the smallest normal bf16 may be off by that much
"""
from __future__ import annotations

import numpy as np

U = 2.0 ** -24
TINY = 2.0 ** -126


def soft_rows(z, it):
    """(x = it (z - M), S, M) of rows z in 64 bits."""
    with np.errstate(invalid="ignore", over="ignore"):
        m = z.max(axis=1, keepdims=True)
        x = (z - m) * it
        return x, np.exp(x).sum(axis=1, keepdims=True), m


def token_logp(z, target, temperature):
    """(logp, its bound) with 0 in rows without a token."""
    it = 1.0 / temperature
    rows, vocab = z.shape
    live = (target >= 0) & (target < vocab)
    at = np.where(live, target, 0)
    x, s, _ = soft_rows(z, it)
    xt = x[np.arange(rows), at]
    with np.errstate(invalid="ignore"):
        ln = np.log(s[:, 0])
        logp = xt - ln
        bound = U * (8 * np.abs(xt) + 8 * np.abs(ln) + 64)
    return np.where(live, logp, 0.0), np.where(live, bound, 0.0), live


def policy(logp, bound, live, old, ref, adv, weights, low, high, kl_coef):
    """stats (4), their bounds, dlogp and its bound."""
    w = np.where(live, weights, 0.0)
    live = w != 0
    pick = lambda v: np.where(live, v, 0.0)  # noqa: E731  what is masked may hold anything
    old, adv, logp = pick(old), pick(adv), pick(logp)
    ratio = np.exp(logp - old)
    plain, held = ratio * adv, np.clip(ratio, 1 - low, 1 + high) * adv
    clipped = held < plain
    pg = -np.where(clipped, held, plain)
    off_ratio = bound + 16 * U * (1 + np.abs(logp) + np.abs(old))
    off_pg = np.abs(plain) * off_ratio
    slope, off = np.where(clipped, 0.0, -plain), np.where(clipped, 0.0, off_pg)
    kl = off_kl = np.zeros_like(logp)
    if ref is not None:
        ref = pick(ref)
        d = ref - logp
        kl = np.expm1(d) - d
        off_d = bound + 16 * U * (np.abs(logp) + np.abs(ref))
        off_kl = np.abs(np.expm1(d)) * off_d + 16 * U * (np.abs(np.expm1(d)) + np.abs(d)) + off_d ** 2
        slope = slope - kl_coef * np.expm1(d)
        off = off + kl_coef * (np.exp(d) * off_d + 16 * U * np.abs(np.expm1(d)))
    terms = [pg + kl_coef * kl, pg, kl, clipped.astype(float)]
    offs = [off_pg + 16 * U * np.abs(pg) + kl_coef * off_kl, off_pg + 16 * U * np.abs(pg), off_kl, np.zeros_like(logp)]
    stats = np.array([(w * t)[live].sum() for t in terms])
    off_stats = np.array([(np.abs(w) * o)[live].sum() for o in offs]) + 2 * U * np.abs(stats) + TINY
    return stats, off_stats, np.where(live, w * slope, 0.0), np.where(live, np.abs(w) * (off + 16 * U * np.abs(slope)), 0.0)


def dlogits(z, target, temperature, dlogp, off, bf16):
    """(gradient, bound) from dlogp and its bound; rows without one are 0."""
    it = 1.0 / temperature
    rows, vocab = z.shape
    x, s, _ = soft_rows(z, it)
    with np.errstate(invalid="ignore"):
        p = np.exp(x) / s
        hot = np.zeros_like(p)
        at = np.clip(target, 0, vocab - 1)
        hot[np.arange(rows), at] = 1.0
        d = dlogp[:, None] * it
        g = d * (hot - p)
        x = np.where(np.isfinite(x), x, 0.0)
        bound = (np.abs(d) * U * (p * (4 * np.abs(x) + 64) + 8 * hot) + (off[:, None] * it) * np.abs(hot - p) + 4 * U * np.abs(g) + TINY)
        if bf16:
            bound = bound + 2.0 ** -8 * np.abs(g)
    none = (dlogp == 0) | (target < 0) | (target >= vocab)
    g[none] = 0.0
    bound[none] = 0.0
    return g, bound


def preference(logp, ref, weights, offsets, pairs, beta, smoothing, scale):
    """(loss, margins, dlogp)"""
    tokens = len(logp)
    off = np.clip(offsets, 0, tokens)
    w = weights
    r = np.where(w != 0, w * (logp - (0.0 if ref is None else ref)), 0.0)
    sums = np.array([r[off[s]:off[s + 1]].sum() for s in range(2 * pairs)])
    h = beta * (sums[:pairs] - sums[pairs:])
    sig = lambda t: np.where(t > 0, 1 / (1 + np.exp(-np.abs(t))), np.exp(-np.abs(t)) / (1 + np.exp(-np.abs(t))))  # noqa: E731
    sp = lambda t: np.maximum(t, 0) + np.log1p(np.exp(-np.abs(t)))  # noqa: E731
    loss = scale * ((1 - smoothing) * sp(-h) + smoothing * sp(h)).sum()
    slope = scale * beta * (smoothing * sig(h) - (1 - smoothing) * sig(-h))
    d = np.zeros(tokens)
    for p in range(pairs):
        d[off[p]:off[p + 1]] = slope[p]
        d[off[pairs + p]:off[pairs + p + 1]] = -slope[p]
    return loss, h, np.where(w != 0, d * w, 0.0)
