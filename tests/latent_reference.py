"""Plain 64-bit forms of the operators around a latent cache and between logits and verification, written from their definitions, and
the checks that their tests share."""
from __future__ import annotations

import math

import torch

from fp4_reference import tree_of, visible  # noqa: F401  (the tree is the same for every cache)


def attention(q, tree, past, seen, scale, d_latent):
    """One sequence: q [H][rows][d], tree [n][d], past [L][d], seen [rows][n] -> (out [H][rows][d_latent], limit of its error).

    Limit.  The output is rounded to bf16 (2^-8 of it), and so is every weight in the numerator (2^-8 of what the weights average
    of |x|, which `size` is).  A score is a sum of d products in fp32 and a product with the scale: off by d + 2 roundings of 2^-24 of
    scale * sum |q_c x_c| at most, `far`; the reference maximum, the difference and the exponential add 4 of them of the score and of 1.
    Weights are then off by that relative to them, in the numerator and in the denominator; sums over keys and the fold of parts
    add their own: together less than (far * (d + 6) + 200) * 2 * 2^-24 of `size`."""
    x = torch.cat((past, tree)).double()
    qd = q.double()
    d = qd.shape[-1]
    y = scale * (qd @ x.T)
    far = scale * (qd.abs() @ x.abs().T)
    L = past.shape[0]
    hide = torch.cat((torch.zeros(seen.shape[0], L, dtype=torch.bool, device=q.device), ~seen), 1)
    y = torch.where(hide, -math.inf, y)
    far = torch.where(hide, 0.0, far).amax(-1, keepdim=True)
    w = torch.exp(y - y.amax(-1, keepdim=True))
    total = w.sum(-1, keepdim=True)
    v = x[:, :d_latent]
    out = (w @ v) / total
    size = (w @ v.abs()) / total
    half = 2.0 ** -8
    return out, half * out.abs() + (half + (far * (d + 6) + 200) * 2.0 ** -23) * size


def latent_rows(kv, weight, eps, pos, freq, d_latent, rotary, interleaved):
    """kv [..., d], pos [...] -> (rows, the magnitudes they are made of), both [..., d]; weight None: no norm."""
    kv = kv.double()
    c, r = kv[..., :d_latent], kv[..., d_latent:]
    if weight is not None:
        c = c / torch.sqrt((c * c).mean(-1, keepdim=True) + eps) * weight.double()
    r, size = rotated(r, pos, freq, rotary, interleaved)
    return torch.cat((c, r), -1), torch.cat((c.abs(), size), -1)


def rotated(x, pos, freq, rotary, interleaved):
    x = x.double()
    out, size = x.clone(), x.abs()
    for i in range(rotary // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rotary // 2)
        angle = pos.double() * float(freq[i])
        co, si = torch.cos(angle), torch.sin(angle)
        out[..., a] = x[..., a] * co - x[..., b] * si
        out[..., b] = x[..., b] * co + x[..., a] * si
        size[..., a] = size[..., b] = x[..., a].abs() + x[..., b].abs()
    return out, size


def sample_row(x, T=1.0, top_k=0, top_p=1.0, min_p=0.0, us=(), distinct=False):
    """One row of logits (a CPU tensor) -> (probabilities float64 [V], tokens list)."""
    x = x.double()
    V = x.numel()
    if bool((~(x < math.inf)).any()) or not T >= 0 or math.isnan(top_p) or math.isnan(min_p):
        return torch.full((V,), math.nan, dtype=torch.float64), [-1] * len(us)
    y, order = torch.sort(x, dim=0, descending=True, stable=True)
    if y[0] == -math.inf:
        return torch.zeros(V, dtype=torch.float64), [-1] * len(us)
    n = int((y > -math.inf).sum())                       # candidates: the first n
    if T == 0:
        n = 1
    if top_k > 0:
        n = min(n, top_k)
    w = torch.exp((y[:n] - y[0]) / (T if T else 1.0))
    if top_p < 1:
        before = w.cumsum(0) - w
        n = max(1, int((before < top_p * w.sum()).sum()))
    if min_p > 0:
        n = min(n, int((w >= min(min_p, 1.0)).sum()))      # (above 1 it counts as 1)
    ids, _ = torch.sort(order[:n])
    z = x[ids]
    p = torch.zeros(V, dtype=torch.float64)
    w = torch.exp((z - z.max()) / (T if T else 1.0))
    p[ids] = w / w.sum()
    tokens = []
    for u in us:
        if ids.numel() == 0:
            tokens.append(-1)
            continue
        u = min(max(float(u), 0.0), 1 - 2.0 ** -24) if u == u else 0.0
        w = torch.exp((z - z.max()) / (T if T else 1.0))
        cum = w.cumsum(0)
        at = min(int((cum <= u * cum[-1]).sum()), ids.numel() - 1)
        tokens.append(int(ids[at]))
        if distinct:
            rest = torch.arange(ids.numel()) != at
            ids, z = ids[rest], z[rest]
    return p, tokens


def check_probs(got, want):
    """fp32 probabilities: 2^y of an exponent in two parts (1 step of the hardware's exponential, half of which is a rounding; the second
    part's factor, a fused product: 1), the reciprocal of the sum (2), two products (2): less than 8 roundings of 2^-24 of the value,
    and what is below the smallest normal number may be zero."""
    got = got.double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    g, w = torch.nan_to_num(got), torch.nan_to_num(want)
    assert bool((g[w == 0] == 0).all()), "a token that is not kept has a probability"
    err, lim = (g - w).abs(), 8 * 2.0 ** -24 * w + 2.0 ** -126
    assert bool((err <= lim).all()), f"{int((err > lim).sum())} probabilities off, worst {float(((err - lim) / w.clamp(min=1e-30)).max()):.2e} of the value"
