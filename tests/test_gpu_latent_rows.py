"""Norm and rotation of latent rows and of the queries that meet them, against the plain 64-bit form.

Tolerance: the output's rounding to bf16 (2^-8 of it), and fp32 on the way: the sum of squares (8 fused steps and 6 additions, half
of its relative error in the root), root, division and two products: 11 roundings of 2^-24; an angle of up to pi rounded to fp32
and the functions' own error: pi + 4 of them; product and sum of the rotation: 3; together less than 32 x 2^-24 of the magnitudes
that an output is made of."""
import numpy as np
import pytest
import torch

import latent_reference as R

pytestmark = pytest.mark.gpu
CODE = {torch.float32: 0, torch.bfloat16: 1}


@pytest.fixture(scope="module")
def binding():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2409_10644_amd import binding as b
    return b


def _close(got, want, size):
    lim = 2.0 ** -8 * want.abs() + 32 * 2.0 ** -24 * size
    err = (got.double() - want).abs()
    assert bool((err <= lim).all()), f"worst {float((err - lim).max()):.3e} over the limit, {int((~(err <= lim)).sum())} of {err.numel()}"


def _freq(dr, base):
    return (base ** (-torch.arange(0, dr, 2, dtype=torch.float64) / dr)).float().cuda()


EPS = float(np.float32(1e-5))


@pytest.mark.parametrize("dtype", CODE)
@pytest.mark.parametrize("dl,dr,rotary,interleaved,norm", [(512, 64, 64, True, True), (512, 64, 64, False, True), (512, 64, 32, False, True), (512, 64, 48, True, False),
                                                           (256, 32, 32, True, True), (256, 32, 32, False, True), (256, 32, 16, False, False), (256, 32, 0, False, True)])
@pytest.mark.parametrize("H,branching,newest", [(1, (1,), False), (5, (4, 2, 2, 1), False), (128, (16, 1, 1), True)])
def test_tree_rows(binding, dtype, dl, dr, rotary, interleaved, norm, H, branching, newest):
    d, B = dl + dr, 3
    gen = torch.Generator("cuda").manual_seed(d + rotary + H)
    level, _ = R.tree_of(branching)
    n = len(level)
    row0 = level.index(level[-1]) if newest else 0
    T, ns = n - row0, n + 3
    view = binding.slice_mask(binding.build_mask(branching + (2,)), len(branching))
    q = torch.randn(B, T, H, dr + 24, generator=gen, device="cuda").to(dtype)                 # (the rotated channels behind 16 others, a gap behind them)
    kv = torch.randn(B, T + 1, d + 16, generator=gen, device="cuda").to(dtype)
    lens = torch.tensor([0, 1000, 99999], dtype=torch.int32, device="cuda")
    weight = 1 + 0.2 * torch.randn(dl, generator=gen, device="cuda") if norm else None
    freq = _freq(dr, 10000.0)
    rope = binding.make_rope(rotary, freq, None, weight, 1e-5, interleaved)
    qo = torch.full((B, H, ns, d), 5.0, dtype=torch.bfloat16, device="cuda")
    out = torch.full((B, ns, d), 5.0, dtype=torch.bfloat16, device="cuda")
    binding.tree_latent_norm_rope(view, CODE[dtype], B, H, dl, dr, row0, q[..., 16:], kv, T * H * (dr + 24), H * (dr + 24), dr + 24, (T + 1) * (d + 16), d + 16, rope, lens, 5000,
                                  qo, out, ns)
    torch.cuda.synchronize()
    pos = lens.clamp(0, 5000).long()[:, None] + torch.tensor(level[row0:], device="cuda") - 1           # (the third length is clamped)
    want, size = R.latent_rows(kv[:, :T, :d], weight, EPS, pos, freq, dl, rotary, interleaved)
    _close(out[:, row0:n], want, size)
    want, size = R.rotated(q[..., 16:16 + dr], pos[:, :, None], freq, rotary, interleaved)
    _close(qo[:, :, row0:n, dl:], want.transpose(1, 2), size.transpose(1, 2))
    qo[:, :, row0:n, dl:] = 5                                # all else is as it was
    assert bool((qo == 5).all()) and bool((out[:, :row0] == 5).all()) and bool((out[:, n:] == 5).all())


@pytest.mark.parametrize("dtype", CODE)
@pytest.mark.parametrize("dl,dr,rotary,interleaved,norm", [(512, 64, 64, False, True), (512, 64, 64, True, False), (256, 32, 32, False, True), (256, 32, 16, True, True)])
@pytest.mark.parametrize("T", [1, 5, 300])
def test_prompt_rows(binding, dtype, dl, dr, rotary, interleaved, norm, T):
    d, B, cap = dl + dr, 6, 700
    gen = torch.Generator("cuda").manual_seed(d + T)
    first = torch.tensor([0, 17, 690, -3, 100, 650], dtype=torch.int32, device="cuda")               # (rows before the cache and behind it are skipped)
    counts = torch.tensor([T, T // 2, T, T + 9, 0, -4], dtype=torch.int32, device="cuda")
    kv = torch.randn(B, T, d, generator=gen, device="cuda").to(dtype)
    weight = 1 + 0.2 * torch.randn(dl, generator=gen, device="cuda") if norm else None
    freq = _freq(dr, 500000.0)
    rope = binding.make_rope(rotary, freq, None, weight, 1e-5, interleaved)
    cache = torch.full((B, cap, d), 5.0, dtype=torch.bfloat16, device="cuda")
    base = torch.arange(B, device="cuda", dtype=torch.int64).flip(0) * cap * d
    binding.store_latent(CODE[dtype], B, dl, dr, T, kv, T * d, d, rope, first, counts, cache, base, cap)
    torch.cuda.synchronize()
    for b in range(B):
        f, c = int(first[b]), min(max(int(counts[b]), 0), T)
        rows = cache[B - 1 - b].clone()
        at = torch.arange(f, f + c, device="cuda")
        inside = (at >= 0) & (at < cap)
        if c:
            want, size = R.latent_rows(kv[b, :c], weight, EPS, at, freq, dl, rotary, interleaved)
            _close(rows[at[inside]], want[inside], size[inside])
        rows[at[inside]] = 5
        assert bool((rows == 5).all()), f"sequence {b}: other rows were written"


def test_far_positions(binding):
    """Angles of positions around 10^6 are those of 64 bits; the largest and smallest vectors have their norm."""
    dl, dr, T = 512, 64, 40
    d = dl + dr
    gen = torch.Generator("cuda").manual_seed(9)
    kv = torch.randn(1, T, d, generator=gen, device="cuda")
    for t, s in enumerate((1e38, 3e37, 1e25, 1e-25, 1e-36, 1e-30)):
        kv[0, t, :dl] = kv[0, t, :dl].clamp(-3, 3) * s
    kv[0, 6, :dl] = torch.finfo(torch.float32).max
    kv[0, 7, :dl] = 0
    freq = _freq(dr, 10000.0)
    weight = torch.ones(dl, device="cuda")
    first, cap = 1_000_000, 1_000_000 + T
    cache = torch.zeros(cap * d, dtype=torch.bfloat16, device="cuda")
    args = (torch.tensor([first], dtype=torch.int32, device="cuda"), torch.tensor([T], dtype=torch.int32, device="cuda"), cache, torch.zeros(1, dtype=torch.int64, device="cuda"), cap)
    binding.store_latent(0, 1, dl, dr, T, kv, T * d, d, binding.make_rope(dr, freq, None, weight, 0.0, False), *args)
    torch.cuda.synchronize()
    keep = torch.arange(T, device="cuda") != 7               # (nothing has no direction: NaN without an eps)
    want, size = R.latent_rows(kv[0], weight, 0.0, torch.arange(first, cap, device="cuda"), freq, dl, dr, False)
    got = cache.view(cap, d)[first:]
    _close(got[keep], want[keep], size[keep])
    binding.store_latent(0, 1, dl, dr, T, kv, T * d, d, binding.make_rope(dr, freq, None, weight, 1e-6, False), *args)
    torch.cuda.synchronize()
    assert bool((got[7, :dl] == 0).all())


def test_no_rows(binding):
    z = torch.zeros(8, device="cuda")
    i = torch.zeros(1, dtype=torch.int32, device="cuda")
    binding.store_latent(0, 1, 512, 64, 0, z, 0, 0, binding.make_rope(0, None), i, i, torch.zeros(576, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda"), 1)
    torch.cuda.synchronize()
