"""Norm and rotation of queries and keys against the plain 64-bit form.

Tolerance: the output's rounding, half a step of its type relative to it, and fp32 on the way: the sum of squares (16 fused steps
and 3 additions, half of its relative error in the root), root, division and two products: 14 roundings of 2^-24; an angle of up
to pi rounded to fp32 and the functions' own error: pi + 4 of them; product and sum of the rotation: 3; together less than 32 x
2^-24 of the magnitudes that an output is made of."""
import numpy as np
import pytest
import torch

import fp4_reference as R

pytestmark = pytest.mark.gpu
CODE = {torch.float32: 0, torch.bfloat16: 1}


@pytest.fixture(scope="module")
def binding():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2409_10644_amd import binding as b
    return b


def _close(got, want, size, dtype):
    lim = torch.finfo(dtype).eps / 2 * want.abs() + 32 * 2.0 ** -24 * size
    err = (got.double() - want).abs()
    assert bool((err <= lim).all()), f"worst {float((err - lim).max()):.3e} over the limit, {int((err > lim).sum())} of {err.numel()}"


def _inv_freq(rotary, base):
    return (base ** (-torch.arange(0, rotary, 2, dtype=torch.float64) / max(rotary, 1))).float().cuda()


def _weights(gen, d, norm):
    return (1 + 0.2 * torch.randn(2, d, generator=gen, device="cuda")).unbind(0) if norm else (None, None)


@pytest.mark.parametrize("dtype", CODE)
@pytest.mark.parametrize("d,rotary,interleaved,norm", [(128, 128, False, True), (128, 128, True, True), (64, 64, False, False), (64, 32, True, True), (128, 32, False, True),
                                                       (128, 48, True, False), (64, 16, False, True), (128, 0, False, True), (128, 112, False, False)])
@pytest.mark.parametrize("B,Hq,Hkv,branching,newest", [(1, 1, 1, (1,), False), (3, 8, 2, (4, 2, 2, 1), False), (2, 5, 5, (16, 1, 1), True)])
def test_tree_rows(binding, dtype, d, rotary, interleaved, norm, B, Hq, Hkv, branching, newest):
    gen = torch.Generator("cuda").manual_seed(d + rotary + B)
    level, _ = R.tree_of(branching)
    n = len(level)
    row0 = level.index(level[-1]) if newest else 0
    T, ns = n - row0, n + 3
    view = binding.slice_mask(binding.build_mask(branching + (2,)), len(branching))         # (a slice of a larger tree)
    qkv = torch.randn(B, T, (Hq + 2 * Hkv) * d, generator=gen, device="cuda").to(dtype)
    q, k, v = qkv.split([Hq * d, Hkv * d, Hkv * d], -1)
    lens = torch.tensor([0, 1000, 99999][:B] if B > 1 else [777], dtype=torch.int32, device="cuda")
    wq, wk = _weights(gen, d, norm)
    freq = _inv_freq(rotary, 10000.0)
    rope = binding.make_rope(rotary, freq, wq, wk, 1e-5, interleaved)
    qo, ko, vo = (torch.full((B, h, ns, d), 5.0, dtype=dtype, device="cuda") for h in (Hq, Hkv, Hkv))
    w = qkv.shape[-1]
    binding.tree_qk_norm_rope(view, CODE[dtype], B, Hq, Hkv, d, row0, q, k, v, T * w, w, T * w, w, rope, lens, 5000, qo, ko, vo, ns)
    torch.cuda.synchronize()
    pos = lens.clamp(0, 5000).long()[:, None] + torch.tensor(level[row0:], device="cuda") - 1           # (the third length is clamped)
    for x, o, wt, h in ((q, qo, wq, Hq), (k, ko, wk, Hkv)):
        want, size = R.rotated(x.double().unflatten(-1, (h, d)), None if wt is None else wt.double(), float(np.float32(1e-5)), pos[..., None], freq, rotary, interleaved)
        _close(o[:, :, row0:n], want.transpose(1, 2), size.transpose(1, 2), dtype)
    assert torch.equal(vo[:, :, row0:n], v.unflatten(-1, (Hkv, d)).transpose(1, 2))
    for o in (qo, ko, vo):
        assert bool((o[:, :, :row0] == 5).all()) and bool((o[:, :, n:] == 5).all())


@pytest.mark.parametrize("dtype", CODE)
@pytest.mark.parametrize("d,rotary,interleaved,norm", [(128, 128, False, True), (64, 64, True, True), (128, 64, False, False)])
@pytest.mark.parametrize("B,Hq,Hkv,T", [(1, 1, 1, 1), (1, 7, 1, 5), (3, 4, 2, 37), (5, 3, 3, 500)])
def test_prompt_rows(binding, dtype, d, rotary, interleaved, norm, B, Hq, Hkv, T):
    gen = torch.Generator("cuda").manual_seed(d + rotary + T)
    first = torch.tensor([0, 2 ** 20, 131072, -3, 17][:B], dtype=torch.int32, device="cuda")
    counts = [T, T // 2, 0, T + 9, 1][:B]
    q = torch.randn(B, T, Hq * d + 8, generator=gen, device="cuda").to(dtype)                # (rows with a gap; keys and values apart)
    kv = torch.randn(2, B, T + 1, Hkv * d, generator=gen, device="cuda").to(dtype)
    wq, wk = _weights(gen, d, norm)
    freq = _inv_freq(rotary, 500000.0)
    rope = binding.make_rope(rotary, freq, wq, wk, 0.0, interleaved)
    out_rows = T + 2
    qo, ko, vo = (torch.full((B, h, out_rows, d), 5.0, dtype=dtype, device="cuda") for h in (Hq, Hkv, Hkv))
    n_rows = torch.tensor(counts, dtype=torch.int32, device="cuda")
    for values in (True, False):
        binding.prompt_qk_norm_rope(CODE[dtype], B, Hq, Hkv, d, T, q, kv[0], kv[1] if values else None, T * (Hq * d + 8), Hq * d + 8, (T + 1) * Hkv * d,
                                    Hkv * d, rope, first, n_rows, qo, ko, vo if values else None, out_rows)
    torch.cuda.synchronize()
    for b in range(B):
        n = min(max(counts[b], 0), T)
        pos = int(first[b]) + torch.arange(n, device="cuda")
        for x, o, wt, h in ((q[b, :n, :Hq * d], qo, wq, Hq), (kv[0, b, :n], ko, wk, Hkv)):
            want, size = R.rotated(x.double().unflatten(-1, (h, d)), None if wt is None else wt.double(), 0.0, pos[:, None], freq, rotary, interleaved)
            _close(o[b, :, :n], want.transpose(0, 1), size.transpose(0, 1), dtype)
        assert torch.equal(vo[b, :, :n], kv[1, b, :n].unflatten(-1, (Hkv, d)).transpose(0, 1))
        for o in (qo, ko, vo):
            assert bool((o[b, :, n:] == 5).all())


def test_one_norm_without_the_other_and_rows_of_no_length(binding):
    """A row of zeros: divided by the root of eps it stays zero; non-finite values stay in their own vector."""
    d, T = 128, 6
    gen = torch.Generator("cuda").manual_seed(1)
    x = torch.randn(1, T, 3 * d, generator=gen, device="cuda")
    x[0, 0, :d] = 0
    x[0, 1, d + 3] = float("nan")
    x[0, 2, 5] = float("inf")
    q, k, v = x.split(d, -1)
    wq = torch.ones(d, device="cuda")
    rope = binding.make_rope(d, _inv_freq(d, 1e4), wq, None, 1e-6)
    outs = [torch.zeros(1, 1, T, d, device="cuda") for _ in range(3)]
    i32 = lambda a: torch.tensor([a], dtype=torch.int32, device="cuda")
    binding.prompt_qk_norm_rope(0, 1, 1, 1, d, T, q, k, v, T * 3 * d, 3 * d, T * 3 * d, 3 * d, rope, i32(40), i32(T), *outs, T)
    torch.cuda.synchronize()
    freq = _inv_freq(d, 1e4)
    pos = 40 + torch.arange(T, device="cuda")
    for o, src, w, skip in ((outs[0], q, wq.double(), 2), (outs[1], k, None, 1)):
        want, size = R.rotated(src[0].double(), w, float(np.float32(1e-6)), pos, freq, d, False)
        keep = [t for t in range(T) if t != skip]
        _close(o[0, 0, keep], want[keep], size[keep], torch.float32)
    assert not outs[0][0, 0, 0].any()
    assert not torch.isfinite(outs[0][0, 0, 2]).all() and int(torch.isnan(outs[1][0, 0, 1]).sum()) == 2


def test_another_stream(binding):
    d, T, B = 64, 9, 2
    x = torch.randn(B, T, 3 * d, device="cuda")
    rope = binding.make_rope(d, _inv_freq(d, 1e4))
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")
    first, n = i32(3, 4), i32(T, 5)
    side = torch.cuda.Stream()
    res = []
    for stream in (None, side):
        outs = [torch.zeros(B, 1, T, d, device="cuda") for _ in range(3)]
        torch.cuda.synchronize()
        binding.prompt_qk_norm_rope(0, B, 1, 1, d, T, x, x[..., d:], x[..., 2 * d:], T * 3 * d, 3 * d, T * 3 * d, 3 * d, rope, first, n, *outs, T, stream)
        torch.cuda.synchronize()
        res.append(outs)
    assert all(torch.equal(a, b) for a, b in zip(*res))
