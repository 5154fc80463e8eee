"""A linear head's log-probabilities, cross entropy and gradients from their definitions in 64 bits, and how far results in 32 bits and bf16 may be off.

    z = x W^T + b,  logp = it z_t - ln sum exp(it z),  dz = dlogp it ([t] - p),  dx = dz W,  dW = dz^T x,  db = sum dz

Rounding: u = 2^-24 in 32 bits (half a step), h = 2^-8 in bf16.  A sum of n products in 32 bits, in whatever order, is off by at most n u sum |products|
(Higham's gamma_n to first order; one more for each term that joins it).  So
    e_z    = (H + 2) u (sum_h |x_h W_ih| + |b_i|), the most of a row; z's difference from the maximum, its factor and the exponential add 2^-20 of a
             probability (an exponent up to 2^4 in 32 bits is off by 2^-20 of 1, the exponential and the sum by a few u); V u for a long sum
    e_logp = 2 it e_z + (|logp| + 16) 2^-22 + V u
    dz     is off by (h + 2 it e_z + 2^-18 + V u) |dz|, and for a target, whose 1 - p cancels, by as much of p + 1
    dx     by sum_i |W_i| e_dz + (V + 4) u sum_i |dz_i W_i| + h |dx|; dW by the same over rows, db too
Roundings to bf16 of many terms do not all go one way: as independent errors with a root mean square of at most h / sqrt(3) each, all elements
together are within h sqrt(sum (dz W)^2) in the 2-norm, which leaves a factor of sqrt(3).
"""
from __future__ import annotations

import torch

U, H8 = 2.0 ** -24, 2.0 ** -8
F64 = torch.float64


def oracle(x, w, bias, targets, dlogp, temperature=1.0, gradient=True):
    """Results in 64 bits for one dlogp a row (0: the row does not count), and a bound for each of their elements."""
    x, w = x.to(F64), w.to(F64)
    vocab, hidden = w.shape
    it = 1.0 / temperature
    live = (targets >= 0) & (targets < vocab)
    if dlogp is not None:
        live &= dlogp != 0
        dlogp = torch.where(live, dlogp.to(F64), 0.0)
    at = torch.where(live, targets, 0)[:, None]
    x = torch.where(live[:, None], x, 0.0)                # what other rows hold counts nowhere
    z = x @ w.t()
    size = x.abs() @ w.abs().t()
    if bias is not None:
        z = z + bias.to(F64)
        size = size + torch.where(bias.to(F64).isfinite(), bias.to(F64).abs(), 0.0)
    e_z = (hidden + 2) * U * size.amax(1)
    ls = torch.log_softmax(z * it, dim=1)
    out = {"logp": torch.where(live, ls.gather(1, at)[:, 0], 0.0)}
    bound = {"logp": torch.where(live, 2 * it * e_z + (out["logp"].abs() + 16) * 2.0 ** -22 + vocab * U, 0.0)}
    out["M"], bound["M"] = torch.where(live, z.amax(1), 0.0), torch.where(live, e_z + 2.0 ** -30, 0.0)
    out["S"] = torch.where(live, ((z - z.amax(1, keepdim=True)) * it).exp().sum(1), 1.0)
    bound["S"] = torch.where(live, out["S"] * (4 * it * e_z + 2.0 ** -18 + vocab * U), 0.0)
    if not gradient:
        return out, bound
    p = ls.exp()
    dz = -p * (dlogp * it)[:, None]
    dz.scatter_add_(1, at, (dlogp * it)[:, None])
    rel = (H8 + 2 * it * e_z + 2.0 ** -18 + vocab * U)[:, None]
    e_dz = rel * dz.abs()
    e_dz.scatter_add_(1, at, ((2 * it * e_z + 2.0 ** -18 + vocab * U) * (dlogp * it).abs())[:, None] * (1 + p.gather(1, at)))
    for name, terms, a, b in (("dx", vocab, dz, w), ("dw", len(x), dz.t(), x), ("db", len(x), dz.t(), torch.ones(len(x), 1, dtype=F64, device=x.device))):
        out[name] = a @ b
        err = {"dx": e_dz, "dw": e_dz.t(), "db": e_dz.t()}[name]
        bound[name] = err @ b.abs() + (terms + 4) * U * (a.abs() @ b.abs()) + H8 * out[name].abs() + 1e-38
        # in the 2-norm: of the roundings of dz, of the result, and of all that is not a rounding
        rest = (err - H8 * a.abs()).clamp(min=0) @ b.abs() + (terms + 4) * U * (a.abs() @ b.abs())
        bound[name + "_norm"] = H8 * ((a * a) @ (b * b)).sum().sqrt() + H8 * out[name].norm() + rest.norm()
    out["db"], bound["db"] = out["db"][:, 0], bound["db"][:, 0]
    return out, bound


def check(got, out, bound, names):
    for name in names:
        g, want, b = got[name].to(F64), out[name], bound[name]
        assert torch.equal(g.isnan(), want.isnan()), name
        ok = want.isnan() | (g == want) | ((g - want).abs() <= b)
        if not bool(ok.all()):
            i = int((~ok).flatten().nonzero()[0])
            raise AssertionError(f"{name}[{i}]: {g.flatten()[i].item()} for {want.flatten()[i].item()}, bound {b.flatten()[i].item()}, {int((~ok).sum())} of {ok.numel()}")
        if name + "_norm" in bound and bool(want.isfinite().all()):
            far = float((g - want).norm())
            assert far <= float(bound[name + "_norm"]), (name, far, float(bound[name + "_norm"]))
