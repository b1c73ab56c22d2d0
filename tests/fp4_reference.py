"""Plain 64-bit forms of the operators around the 4-bit prefix cache, written from their definitions, on any device; and the
inputs and checks that their tests share."""
from __future__ import annotations

import math

import torch

VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def tree_of(branching):
    """(level, parent) of every node, nodes level by level."""
    level, parent, first, count = [], [], 0, 1
    for l, b in enumerate(branching):
        nodes = count * b
        level += [l + 1] * nodes
        parent += [-1 if l == 0 else first - count + i // b for i in range(nodes)]
        first, count = first + nodes, nodes
    return level, parent


def visible(branching, device="cpu"):
    parent = tree_of(branching)[1]
    seen = torch.zeros(len(parent), len(parent), dtype=torch.bool)
    for i in range(len(parent)):
        j = i
        while j >= 0:
            seen[i, j] = True
            j = parent[j]
    return seen.to(device)


def quantise(x):
    """[..., d] -> codes uint8 [..., d/2], scale bytes uint8 [..., d/32]."""
    g = x.double().reshape(*x.shape[:-1], -1, 32)
    m = g.abs().amax(-1)
    fine = torch.isfinite(g).all(-1)
    frac, exp = torch.frexp(torch.where(fine, m, 1.0))
    byte = (exp.long() - 1 + (frac >= 0.875) - 2 + 127).clamp(1, 254)
    byte = torch.where((m == 0) & fine, 1, byte)
    a = torch.where(fine[..., None], g.abs() / torch.exp2(byte[..., None].double() - 127), 0.0)
    table = torch.tensor(VALUES, dtype=torch.float64, device=x.device)
    far = (a[..., None] - table).abs()                      # to every element value; of two equally near the even code
    near = far.amin(-1, keepdim=True)
    code = torch.where(far == near, torch.tensor([0, 9, 2, 11, 4, 13, 6, 15], device=x.device), 99).amin(-1) % 8
    code = code + 8 * (torch.signbit(g) & fine[..., None])
    code = code.reshape(*x.shape[:-1], -1, 2).to(torch.uint8)
    return code[..., 0] | code[..., 1] << 4, torch.where(fine, byte, 255).to(torch.uint8)


def decode(codes, scales):
    """Numbers of the rows, float64 [..., d]."""
    table = torch.tensor(VALUES + tuple(-v for v in VALUES), dtype=torch.float64, device=codes.device)
    v = torch.stack((table[(codes & 15).long()], table[(codes >> 4).long()]), -1).reshape(*scales.shape, 32)
    unit = torch.where(scales == 255, math.nan, torch.exp2(scales.double() - 127))
    return (v * unit[..., None]).flatten(-2)


def attention_row_terms(q, k, v, seen, scale):
    """q [R, d], k and v [J, d], seen [R, J], float64: outputs [R, d] and what they may be off by, summed over the causes below.

    - the output is rounded to bf16: half a step, 2^-8 of it;
    - weights are rounded to bf16 for the product with the values: each by 2^-8 of itself, so 2^-8 of A = sum p |v| / sum p;
    - a score may be off by delta = scale * sum over groups of 32 channels of 2^-14 max |q| sum |k| (three 6-bit terms per group)
      and by the accumulation in fp32, at most 160 roundings of 2^-24 of scale * sum |q| |k| and of the reference maximum's
      size; a weight then changes by the factor e^(+-delta), numerator and denominator both: (e^(2 delta) - 1) A;
    - exponentials, fp32 sums of up to some thousands of weights and of the partial results: 2^-15 of A;
    - a weight below 2^-126 of the largest one has no fp32 number and may count as zero: 2^-126 of sum |v|."""
    s = (q @ k.T) * scale
    s = s.masked_fill(~seen, -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - top)
    w = p / p.sum(-1, keepdim=True)
    out = w @ v
    A = w @ v.abs()
    gq = q.abs().reshape(q.shape[0], -1, 32).amax(-1)
    gk = k.abs().reshape(k.shape[0], -1, 32).sum(-1)
    size = (q.abs() @ k.abs().T) * scale
    delta = scale * 2.0 ** -14 * (gq @ gk.T) + 160 * 2.0 ** -24 * (size + top.abs())
    delta = torch.where(seen, delta, 0.0).amax(-1, keepdim=True)
    return out, 2.0 ** -8 * out.abs() + (2.0 ** -8 + torch.expm1(2 * delta) + 2.0 ** -15) * A + 2.0 ** -126 * v.abs().sum(0)


def rotated(x, weight, eps, pos, inv_freq, rotary, interleaved):
    """x [..., d] float64, pos broadcastable to x's leading shape; y and the sum of magnitudes each output is made of."""
    y = x
    if weight is not None:
        y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * weight
    a = torch.arange(0, rotary, 2) if interleaved else torch.arange(rotary // 2)
    b = a + 1 if interleaved else a + rotary // 2
    t = pos.double()[..., None] * inv_freq.double()[: rotary // 2]
    out, size = y.clone(), y.abs()
    out[..., a] = y[..., a] * torch.cos(t) - y[..., b] * torch.sin(t)
    out[..., b] = y[..., b] * torch.cos(t) + y[..., a] * torch.sin(t)
    both = y[..., a].abs() + y[..., b].abs()
    size[..., a], size[..., b] = both, both
    return out, size


class Cache:
    """One layer's cache, [B][H][cap] rows with `gap` rows between heads that belong to nobody, sequences in reverse order."""

    def __init__(self, binding, B, H, cap, d, gap=0, fill=0xA5):
        self.B, self.H, self.cap, self.d = B, H, cap, d
        rows = B * H * (cap + gap)
        mk = lambda w: torch.full((rows, w), fill, dtype=torch.uint8, device="cuda")
        self.arrays = (mk(d // 2), mk(d // 32), mk(d // 2), mk(d // 32))
        self.head_stride = (cap + gap) * d
        self.base = torch.arange(B - 1, -1, -1, dtype=torch.int64, device="cuda") * (H * self.head_stride)
        self.handle = binding.make_fp4_cache(*self.arrays)

    def view(self, i):
        """Array i as [B][H][cap][..], sequences in order."""
        a = self.arrays[i].reshape(self.B, self.H, -1, self.arrays[i].shape[-1])
        return a.flip(0)[:, :, :self.cap]
