"""The scoring operators from their definitions, in 64 bits, and how far fp32 arithmetic may take a result from them.

Bounds (eps = 2^-24, half a step of fp32).  A weight 2^y is off by 2^-22 (the exponential) and by ln 2 |y| 2 eps (two roundings of y) relative to itself; sums
take at most 64 additions in a lane, 5 over a warp and 13 over the tiles: 82 eps.  Weighted by the weights themselves |y| is at most the entropy in bits
plus log2 Z, below 36 for 262,144 entries: a sum of weights is off by less than (4 + 36 * 1.4 + 82) eps < 9e-6, rounded up to 1e-5.
ln Z adds its own rounding (ln 2 eps |log2 Z|), a log-probability the two roundings of (v - m) / T.
"""
import numpy as np
import torch

SUM = 1e-5
EPS = 2.0 ** -24
NEG = float("-inf")


def clean(rows):
    """The rows in 64 bits with NaN and +inf as no entries."""
    z = rows.double()
    return torch.where(z < float("inf"), z, torch.full_like(z, NEG))


def log_softmax(rows, T):
    z = clean(rows)
    m = z.amax(-1, keepdim=True)
    none = m == NEG
    z = (z - torch.where(none, 0.0, m)) / T
    lp = z - torch.log(torch.exp(z).sum(-1, keepdim=True))
    return torch.where(none.expand_as(lp), NEG, lp)


def plogr(lp, lr):
    """p ln r with 0 where p is 0"""
    return torch.where(lp > NEG, torch.exp(lp) * torch.where(lp > NEG, lr, 0.0), 0.0)


def entropy(lp):
    return -plogr(lp, lp).sum(-1)


def top(rows, K):
    """(tokens, values): the K largest entries, equal values to the smaller token, -1 / -inf beyond the entries."""
    z = clean(rows)
    value, token = torch.sort(z + 0.0, dim=-1, descending=True, stable=True)
    value, token = value[..., :K], token[..., :K]
    pad = K - value.shape[-1]
    value, token = torch.nn.functional.pad(value, (0, pad), value=NEG), torch.nn.functional.pad(token, (0, pad), value=-1)
    return torch.where(value > NEG, token, -1).to(torch.int32), value


def close(got, want, tol, what):
    got, want = got.double(), want.double()
    beyond = want.abs() > torch.finfo(torch.float32).max        # (values beyond fp32's range are infinite there)
    want = torch.where(beyond, torch.sign(want) * float("inf"), want)
    tol = torch.as_tensor(tol, dtype=torch.float64, device=want.device).expand_as(want)
    fine = torch.isfinite(want)
    assert torch.equal(torch.isfinite(got), fine), what + ": not finite at other places"
    assert torch.equal(got[~fine], want[~fine]), what
    off = (got - want).abs()[fine] - tol[fine]
    assert off.numel() == 0 or float(off.max()) <= 0, "%s: off by %.3g, beyond the bound by %.3g" % (what, float((got - want).abs()[fine].max()), float(off.max()))


def check_scores(out, rows, token, K, T):
    """out of rsd_token_logprobs for these slots' rows [B, R, V] and token [B, R, T]"""
    lp = log_softmax(rows, T)
    H = entropy(lp)
    empty = lp.amax(-1) == NEG
    if token is not None:
        tok = token if token.dim() == 3 else token[..., None]
        there = (tok >= 0) & (tok < rows.shape[-1])
        want = torch.where(there, lp.gather(-1, torch.where(there, tok, 0).long()), 0.0)
        close(out["logprob"].reshape(want.shape), want, SUM + 4 * EPS * want.abs().nan_to_num(posinf=0.0), "logprob")
    if out.get("entropy") is not None:
        close(out["entropy"], H, 2 * SUM * (1 + H), "entropy")
    if K:
        want_token, value = top(rows, K)
        assert torch.equal(out["top_token"], want_token), "likeliest tokens"
        m = clean(rows).amax(-1, keepdim=True)
        at = torch.where(want_token >= 0, lp.gather(-1, want_token.clamp_min(0).long()), NEG)
        close(out["top_logprob"], at, SUM + 4 * EPS * at.abs().nan_to_num(posinf=0.0), "their log-probabilities")
    return lp, H, empty


def flushed(p, size, T):
    """A probability below 2^-126 is 0 in the exponential's result: its whole term, `size` / T (the factors of p included), may be missing."""
    return torch.where(p < 2.0 ** -125, 2 * size / T, 0.0)


def score_gradient(rows, token, g, h, T):
    """(gradient, bound of its fp32 evaluation before the rounding to the rows' dtype)"""
    lp = log_softmax(rows, T)
    p = torch.exp(lp)
    tok = token if token.dim() == 3 else token[..., None]
    g = g.reshape(tok.shape).double()
    there = (tok >= 0) & (tok < rows.shape[-1])
    g = torch.where(there, g, 0.0)
    G = g.sum(-1, keepdim=True)
    grad = -p * G
    H = entropy(lp)[..., None]
    lp0 = torch.where(lp > NEG, lp, 0.0)
    size = p * (G.abs() + g.abs().sum(-1, keepdim=True))
    if h is not None:
        h = h.double()[..., None]
        grad = grad - h * p * (lp0 + H)
        size = size + h.abs() * p * (lp0.abs() + H + 1)
    spike, spikes = torch.zeros_like(grad), torch.zeros_like(grad)
    for t in range(tok.shape[-1]):
        at = torch.where(there, tok, 0)[..., t:t + 1].long()
        spike.scatter_add_(-1, at, g[..., t:t + 1])
        spikes.scatter_add_(-1, at, g[..., t:t + 1].abs())
    empty = lp.amax(-1, keepdim=True) == NEG
    grad = torch.where(empty, 0.0, (grad + spike) / T)
    # p is off by SUM and by the rounding of its exponent, the factors by a few roundings, a sum of T weights by as many of the sum of their sizes
    bound = (size * (2 * SUM + 4 * EPS * lp0.abs()) + (8 + tok.shape[-1]) * EPS * (spikes + size) + 64 * EPS * size) / T
    return grad, bound + flushed(p, size, T)


def divergences(draft, target, Td, Tt):
    lp, lq = log_softmax(draft, Td), log_softmax(target, Tt)
    R = draft.shape[1]
    lq = lq[:, :R]
    empty = (lp.amax(-1) == NEG) | (lq.amax(-1) == NEG)

    def kl(la, lb):
        top_weight = la - la.amax(-1, keepdim=True)
        counts = (la > NEG) & (top_weight * 1.4426950408889634 >= -126)
        inf = (counts & (lb == NEG)).any(-1)
        both = (la > NEG) & (lb > NEG)
        term = torch.where(both, torch.exp(la) * (torch.where(both, la, 0.0) - torch.where(both, lb, 0.0)), 0.0)
        # what cancels: differences relative to the rows' largest entries
        da, db = la - la.amax(-1, keepdim=True), lb - lb.amax(-1, keepdim=True)
        size = torch.where(both, torch.exp(la) * (torch.where(both, da, 0.0) - torch.where(both, db, 0.0)).abs(), 0.0).sum(-1) + la.amax(-1).abs() + lb.amax(-1).abs()
        size = torch.where(empty, 0.0, size).nan_to_num()
        return torch.where(empty, 0.0, torch.where(inf, float("inf"), term.sum(-1))), SUM * (1 + size)

    overlap = torch.where(empty, 0.0, torch.exp(torch.minimum(lp, lq)).sum(-1).nan_to_num())
    return dict(kl=kl(lq, lp), reverse_kl=kl(lp, lq), overlap=(overlap, 2 * SUM + 0 * overlap), lp=lp, lq=lq, empty=empty)


def divergence_gradient(draft, target, g, h, Td, Tt):
    d = divergences(draft, target, Td, Tt)
    lp, lq = d["lp"], d["lq"]
    p, q = torch.exp(lp), torch.exp(lq)
    lp0, lq0 = torch.where(lp > NEG, lp, 0.0), torch.where(lq > NEG, lq, 0.0)
    each = 2 * SUM + 4 * EPS * (lp0.abs() + lq0.abs()) + 64 * EPS
    grad, bound = torch.zeros_like(lp), torch.zeros_like(lp)
    lost = torch.zeros_like(lp)
    if g is not None:
        g = g.double()[..., None]
        grad = grad + g * (p - q)
        bound = bound + g.abs() * (p + q) * each
        lost = lost + g.abs() * (torch.where(p < 2.0 ** -125, p, 0.0) + torch.where(q < 2.0 ** -125, q, 0.0))
    if h is not None:
        rkl, tol = d["reverse_kl"]
        rkl = rkl[..., None]
        finite = torch.isfinite(rkl)
        h = torch.where(finite, h.double()[..., None], 0.0)
        rkl = torch.where(finite, rkl, 0.0)
        grad = grad + h * torch.where(p > 0, p * (lp0 - lq0 - rkl), 0.0)
        size = h.abs() * p * (lp0.abs() + lq0.abs() + rkl + 1)
        bound = bound + size * each + h.abs() * p * tol[..., None].nan_to_num()
        lost = lost + flushed(p, size, 1.0)
    none = d["empty"][..., None]
    return torch.where(none, 0.0, grad / Td), torch.where(none, 0.0, (bound + 2 * lost) / Td)


def check_gradient(got, want, bound, what):
    half_step = torch.finfo(got.dtype).eps / 2
    tiny = 2.0 ** -126                                       # smaller weights may be flushed to 0
    close(got, want, bound + half_step * want.abs() * 1.01 + 4 * tiny * (1 + 0 * want), what)


def random_rows(shape, dtype, sigma, seed, offset=0):
    """Rows whose first entry lies `offset` entries behind a 256-byte boundary."""
    g = torch.Generator().manual_seed(seed)
    n = int(np.prod(shape))
    flat = torch.empty(n + offset, dtype=dtype, device="cuda")
    flat[offset:] = (torch.randn(n, generator=g) * sigma).to(dtype)
    return flat[offset:].view(shape)
