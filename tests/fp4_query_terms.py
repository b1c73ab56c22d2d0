"""How the attention over the 4-bit cache holds a query for its scores with prefix keys, computed apart from the kernel: times the
soft-max scale and log2 e, then per group of 32 channels three E2M3 terms under scales 2^-4 apart."""
from __future__ import annotations

import math

import torch

import fp4_reference as R

# What three terms leave of a channel, of its group's largest magnitude.  The first scale s is such that the largest magnitude is in
# (3.75 s, 7.5 s] (7.5 is the largest E2M3 number).  E2M3 steps are 1/8 up to 2, 1/4 up to 4, 1/2 beyond: the first term leaves at
# most 1/4 s, which is 4 of the second's units s / 16; that leaves at most 1/8 of them, 2 of the third's units s / 256; that at most
# 1/16 of them, s / 4096, which is 2^-12 / 3.75 of the largest magnitude.
LEFT = 2.0 ** -12 / 3.75


def _e2m3(a):
    """The nearest E2M3 number (ties to the even fraction), float64."""
    size = a.abs()
    step = torch.where(size < 2, 0.125, torch.where(size < 4, 0.25, 0.5))
    return torch.sign(a) * (torch.round(size / step) * step).clamp(max=7.5)


def held(q, scale):
    """q bf16 [..., d] -> what the terms add up to, float64 [..., d], and q * scale * log2 e as the kernel makes it, in fp32."""
    c = torch.tensor(scale, dtype=torch.float32) * torch.tensor(1.4426950408889634, dtype=torch.float32)
    x = q.float() * c.to(q.device)
    g = x.double().unflatten(-1, (-1, 32))
    frac, exp = torch.frexp(g.abs().amax(-1, keepdim=True))           # m = frac * 2^exp, frac in [1/2, 1)
    unit = torch.exp2((exp - 1 - 2 + (frac > 1.875 / 2)).double())
    rest, total = g, torch.zeros_like(g)
    for t in range(3):
        term = _e2m3(rest / (unit * 2.0 ** (-4 * t))) * unit * 2.0 ** (-4 * t)
        total, rest = total + term, rest - term
    return torch.where(g == 0, 0.0, total).flatten(-2), x


def attention(q, kp, kt, vp, vt, seen, scale):
    """One head: q [R, d] bf16, prefix kp, vp [L, d] float64, tree kt, vt [n, d] bf16, seen [R, n]: outputs of the terms' scores, of the
    queries' own scores, the sum of weighted magnitudes, and what a score may be off by, in the order
    (of terms, of queries, magnitudes, terms against queries, fp32)."""
    terms, _ = held(q, scale)
    ln2 = math.log(2.0)
    k, v = torch.cat((kp, kt.double())), torch.cat((vp, vt.double()))
    own = torch.where(seen, q.double() @ kt.double().T * scale, -math.inf)
    outs = []
    for s in (torch.cat((terms @ kp.T * ln2, own), 1), torch.cat((q.double() @ kp.T * scale, own), 1)):
        w = torch.softmax(s, -1)
        outs.append(w @ v)
    gq, gk = q.double().abs().unflatten(-1, (-1, 32)).amax(-1), kp.abs().unflatten(-1, (-1, 32)).sum(-1)
    terms_off = (scale * LEFT * (gq @ gk.T)).amax(-1, keepdim=True)
    size = torch.where(torch.cat((torch.ones(len(q), len(kp), dtype=torch.bool, device=q.device), seen), 1), q.double().abs() @ k.abs().T * scale, 0.0)
    fp32_off = 160 * 2.0 ** -24 * (size + s.amax(-1, keepdim=True).abs()).amax(-1, keepdim=True)
    return outs[0], outs[1], w @ v.abs(), terms_off, fp32_off
