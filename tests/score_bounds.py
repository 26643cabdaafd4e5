"""Bounds of the divergences' gradients that stay tight where logarithms of probabilities are large (beside tests/scoring.py, whose bounds let the factors be off by as
much as the weights).

gradient = g (p - q) + h p (ln p - ln q - KL(p||q)), over the draft's temperature.  A weight is off by 2 SUM (its normaliser and its exponential) and by 4 EPS |ln p| (two roundings of
its exponent, and of the scale); where |ln p| is above 88 the weight is below 2^-126 and may be missing.  The factor ln p - ln q - KL is a difference of numbers with a relative
error of a few EPS each (16 of them: scale, product, difference, factor, sum, and as many again for what is behind them), of the normalisers (2 SUM), and of the KL (its own bound).
"""
import torch

from tests import scoring as sc


def divergence_gradient(draft, target, g, h, Td, Tt):
    d = sc.divergences(draft, target, Td, Tt)
    lp, lq = d["lp"], d["lq"]
    p, q = torch.exp(lp), torch.exp(lq)
    lp0, lq0 = torch.where(lp > sc.NEG, lp, 0.0), torch.where(lq > sc.NEG, lq, 0.0)
    ep, eq = (2 * sc.SUM + 4 * sc.EPS * l.abs().clamp(max=90.0) for l in (lp0, lq0))
    grad, bound, lost = torch.zeros_like(lp), torch.zeros_like(lp), torch.zeros_like(lp)
    if g is not None:
        g = g.double()[..., None]
        grad = grad + g * (p - q)
        bound = bound + g.abs() * (p * ep + q * eq + 8 * sc.EPS * (p + q))
        lost = lost + g.abs() * (torch.where(p < 2.0 ** -125, p, 0.0) + torch.where(q < 2.0 ** -125, q, 0.0))
    if h is not None:
        rkl, tol = d["reverse_kl"]
        rkl, tol = rkl[..., None], tol[..., None]
        finite = torch.isfinite(rkl)
        h = torch.where(finite, h.double()[..., None], 0.0)
        rkl, tol = torch.where(finite, rkl, 0.0), torch.where(finite, tol, 0.0)
        factor = torch.where(p > 0, lp0 - lq0 - rkl, 0.0)
        grad = grad + h * p * factor
        sizes = torch.where(p > 0, lp0.abs() + lq0.abs() + rkl, 0.0)
        bound = bound + h.abs() * p * (ep * factor.abs() + 16 * sc.EPS * sizes + 2 * sc.SUM + tol)
        lost = lost + torch.where(p < 2.0 ** -125, 2 * h.abs() * p * (sizes + 1), 0.0)
    none = d["empty"][..., None]
    return torch.where(none, 0.0, grad / Td), torch.where(none, 0.0, (bound + 2 * lost) / Td)
