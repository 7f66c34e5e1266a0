"""Attention and its gradients in 64 bits, one head at a time, with the bound on what the kernels' roundings may add up to.

The kernels sum in fp32 and round where a comment beside a bound says so; a rounding to bf16 is off by at most 2^-8 of the value, one to
fp32 by 2^-24.  Every bound is a sum of those over the terms that they meet, so no element may exceed it."""
import math

import torch

B16, F32 = 2.0 ** -8, 2.0 ** -24


def visible(rows, keys, causal):
    see = torch.ones((rows, keys), dtype=torch.bool)
    return see.tril(keys - rows) if causal else see


def tree_visible(rows, keys, trees):
    """trees: bits of the rows that each row sees; the last `rows` keys are the rows' own."""
    first = keys - rows
    see = torch.zeros((rows, keys), dtype=torch.bool)
    for i in range(rows):
        for j in range(keys):
            d = j - first
            see[i, j] = d < 0 or (d < 64 and trees[i] >> d & 1)
    return see


def _scores(q, k, scale, see):
    """S, and how far the kernel's may be off: D products and as many additions, the scale's product."""
    s = (q @ k.t()) * scale
    err = (q.shape[1] + 4) * F32 * scale * (q.abs() @ k.abs().t())
    return s.masked_fill(~see, -math.inf), err


def attend(q, k, v, scale, see):
    """float64 q [r x d], k and v [n x d] -> o, lse, bound of o, bound of lse"""
    s, err = _scores(q, k, scale, see)
    r, n = s.shape
    if n == 0:
        return torch.zeros_like(q), torch.full((r,), -math.inf, dtype=torch.float64), torch.zeros_like(q), torch.zeros(r, dtype=torch.float64)
    lse = torch.logsumexp(s, 1)
    p = torch.where(see, torch.exp(s - lse.clamp_min(-1e300)[:, None]), torch.zeros_like(s))
    o = p @ v
    # a weight: the score's error, the exponential's argument and result, n additions behind its sum
    rel = torch.where(see, err + (s.abs() + lse.clamp_min(-1e300)[:, None].abs() + 8) * 4 * F32, torch.zeros_like(s)) + n * F32
    b_o = ((B16 * 1.01 + 2 * rel) * p) @ v.abs() + B16 * 1.01 * o.abs() + 1e-30         # weights rounded, then the output
    b_lse = (rel * see).amax(1) + n * F32 + 8 * F32 * (1 + torch.nan_to_num(lse, neginf=0.0).abs())
    return o, lse, b_o, b_lse


def gradients(q, k, v, o, do, lse, scale, see):
    """What a head's rows and keys get -> dq, dk, dv and their bounds (before the rounding of the outputs)"""
    s, err = _scores(q, k, scale, see)
    p = torch.where(see, torch.exp(s - lse[:, None]), torch.zeros_like(s))
    delta = (do * o).sum(1)
    dp = do @ v.t()
    ds = torch.where(see, p * (dp - delta[:, None]), torch.zeros_like(p))
    rel = torch.where(see, err + (s.abs() + lse[:, None].abs() + 8) * 4 * F32, torch.zeros_like(s))
    e_dp = (q.shape[1] + 4) * F32 * (do.abs() @ v.abs().t() + (do * o).abs().sum(1)[:, None])
    b_ds = ds.abs() * (B16 * 1.01 + rel) + p * e_dp                                      # rounded for its products
    b_p = p * (B16 * 1.01 + rel)
    n = max(s.shape)
    dq, dk, dv = scale * ds @ k, scale * ds.t() @ q, p.t() @ do
    # sums of fp32: as many additions as terms
    b_2 = ds.abs() * (2.0 ** -16 + rel) + p * e_dp                                       # in two parts for dQ: 8 bits cut off, the rest of them rounded
    b_dq = scale * (b_2 + 2 * n * F32 * ds.abs()) @ k.abs()
    b_dk = scale * (b_ds + n * F32 * ds.abs()).t() @ q.abs()
    b_dv = (b_p + n * F32 * p).t() @ do.abs()
    return dq, dk, dv, b_dq, b_dk, b_dv


def turn_back(x, cos, sin, pos):
    """Adjacent pairs of [rows x d] turned by minus the angle of position pos (taken to the nearest table row)"""
    at = pos.long().clamp(0, cos.shape[0] - 1)
    c, s = cos.double()[at], sin.double()[at]
    a, b = x[:, 0::2], x[:, 1::2]
    return torch.stack((a * c + b * s, b * c - a * s), 2).reshape(x.shape)


def turn_bound(b, cos, sin, pos):
    at = pos.long().clamp(0, cos.shape[0] - 1)
    c, s = cos.double()[at].abs(), sin.double()[at].abs()
    x, y = b[:, 0::2], b[:, 1::2]
    return torch.stack((x * c + y * s, y * c + x * s), 2).reshape(b.shape)


def rounded(value, bound):
    """The bound of an output that is rounded to bf16 at the end"""
    return bound * (1 + B16) + B16 * 1.01 * value.abs() + 1e-30


def head(x, h, d):
    return x[:, h * d: (h + 1) * d].double().cpu()


def check(got, want, bound, what):
    got, want = got.double().cpu(), want.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    off = (got - want).abs()
    bad = ~same & ~(off <= bound)
    assert not bad.any(), "%s: %d of %d elements beyond their bound, first at %s: %r for %r, bound %.3g" % (
        what, int(bad.sum()), bad.numel(), tuple(bad.nonzero()[0].tolist()), float(got[bad][0]), float(want[bad][0]), float(bound.expand_as(want)[bad][0]))
