"""Pins of the plain forms that the tests of the 4-bit cache compare with, and the refusals of its entry points (no GPU needed:
a call that is refused launches nothing)."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import fp4_reference as R
from paper_2409_10644_amd import binding as b


def test_values_of_codes_and_scales():
    codes = torch.tensor([[0x10, 0x32, 0x54, 0x76, 0x98, 0xBA, 0xDC, 0xFE] + [0] * 8], dtype=torch.uint8)
    got = R.decode(codes, torch.tensor([[128]], dtype=torch.uint8))[0, :16]
    assert got.tolist() == [0, 1, 2, 3, 4, 6, 8, 12, 0, -1, -2, -3, -4, -6, -8, -12]
    assert R.decode(codes, torch.tensor([[0]], dtype=torch.uint8))[0, 1] == 0.5 * 2.0 ** -127
    assert torch.isnan(R.decode(codes, torch.tensor([[255]], dtype=torch.uint8))).all()


def test_quantised_numbers():
    x = torch.zeros(1, 32, dtype=torch.float64)
    x[0, :12] = torch.tensor([6, 0.25, 0.26, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -5.1, -0.2, 0.74])
    codes, scale = R.quantise(x)
    assert scale.tolist() == [[127]]
    assert R.decode(codes, scale)[0, :12].tolist() == [6, 0, 0.5, 1, 1, 2, 2, 4, 4, -6, 0, 0.5]
    for top, byte in ((6.99, 127), (7.0, 128), (8, 128), (13.9, 128), (14, 129), (3.99, 127), (3.49, 126), (1.0, 125), (0.0, 1), (1e-39, 1), (2.9e38, 252), (3e38, 253), (math.nan, 255), (-math.inf, 255)):
        x = torch.full((1, 32), 1e-45, dtype=torch.float64)
        x[0, 7] = top
        codes, scale = R.quantise(x)
        assert scale.tolist() == [[byte]], top
        if byte == 255:
            assert not codes.any()


@pytest.mark.parametrize("power", range(-120, 120, 17))
def test_no_number_is_off_by_more_than_half_a_step(power):
    x = torch.randn(400, 128, generator=torch.Generator().manual_seed(power + 200), dtype=torch.float64) * 2.0 ** power
    codes, scales = R.quantise(x)
    y = R.decode(codes, scales)
    unit = torch.exp2(scales.double() - 127).repeat_interleave(32, -1)
    step = unit * torch.where(x.abs() < 2 * unit, 0.5, torch.where(x.abs() < 4 * unit, 1.0, 2.0))
    assert ((y - x).abs() <= step / 2).all()
    again = R.quantise(y)                                  # what is in the format already stays as it is
    assert torch.equal(R.decode(*again), y)


ONE = C.c_void_p(256)                                      # never dereferenced: validation fails first
CACHE = b.Fp4Cache(256, 256, 256, 256)


def _view(branching=(4, 2, 2, 1)):
    m = b.build_mask(branching)
    v = b.slice_mask(m, len(branching))
    v._mask = m
    if v.device < 0:
        v.bits_dev = 256                                   # as if it had been uploaded
    return v


def _attention(view=None, B=1, Hq=4, Hkv=2, d=128, row=0, q=ONE, kt=ONE, vt=ONE, ns=44, cache=CACHE, base=ONE, lens=ONE, hs=128 * 128, mp=100,
               scale=0.1, out=ONE, ws=None, ws_bytes=0):
    view = _view() if view is None else view
    return b.lib.mcsd_tree_attention_fp4kv(C.byref(view), B, Hq, Hkv, d, row, q, kt, vt, ns, None if cache is None else C.byref(cache), base, lens,
                                           hs, mp, scale, out, ws, ws_bytes, None)


@pytest.mark.parametrize("wrong,status", [
    (dict(B=0), b.MCSD_EINVAL), (dict(B=65536), b.MCSD_EINVAL), (dict(Hq=3), b.MCSD_EINVAL), (dict(Hkv=0), b.MCSD_EINVAL), (dict(Hq=0), b.MCSD_EINVAL),
    (dict(row=44), b.MCSD_EINVAL), (dict(row=-1), b.MCSD_EINVAL), (dict(q=None), b.MCSD_EINVAL), (dict(kt=None), b.MCSD_EINVAL),
    (dict(vt=None), b.MCSD_EINVAL), (dict(out=None), b.MCSD_EINVAL), (dict(base=None), b.MCSD_EINVAL), (dict(lens=None), b.MCSD_EINVAL),
    (dict(cache=None), b.MCSD_EINVAL), (dict(cache=b.Fp4Cache(256, 0, 256, 256)), b.MCSD_EINVAL), (dict(cache=b.Fp4Cache(256, 256, 264, 256)), b.MCSD_EINVAL),
    (dict(cache=b.Fp4Cache(256, 258, 256, 256)), b.MCSD_EINVAL), (dict(ns=43), b.MCSD_EINVAL), (dict(hs=-128), b.MCSD_EINVAL), (dict(hs=64), b.MCSD_EINVAL),
    (dict(mp=-1), b.MCSD_EINVAL), (dict(scale=0.0), b.MCSD_EINVAL), (dict(scale=math.inf), b.MCSD_EINVAL), (dict(scale=math.nan), b.MCSD_EINVAL),
    (dict(scale=-1.0), b.MCSD_EINVAL), (dict(d=96), b.MCSD_EUNSUPPORTED), (dict(q=C.c_void_p(264)), b.MCSD_EINVAL)])
def test_attention_refuses(wrong, status):
    assert _attention(**wrong) == status


def test_attention_refuses_trees_beyond_the_limit_and_masks_of_no_device():
    assert _attention(view=_view((64, 2, 1)), ns=400) == b.MCSD_EUNSUPPORTED
    host = _view()
    host.bits_dev = None
    assert _attention(view=host) == b.MCSD_EINVAL
    other = _view()
    other.device = 63
    assert _attention(view=other) == b.MCSD_EINVAL


def test_attention_workspace_of_bad_shapes_is_zero():
    good = (1, 32, 8, 128, 44, 0, 1000)
    for i, bad in ((0, 0), (1, 31), (2, 0), (3, 96), (4, 0), (4, 129), (5, 44), (5, -1), (6, -1)):
        args = list(good)
        args[i] = bad
        assert b.tree_attention_fp4kv_workspace(*args) == 0, args


def test_attention_workspace_serves_smaller_calls():
    rng = np.random.default_rng(5)
    for _ in range(400):
        B, Hkv, g, d = (int(rng.choice(x)) for x in ((1, 2, 5, 16, 64, 200), (1, 2, 8, 32), (1, 3, 4, 8), (64, 128)))
        n, prefix = int(rng.integers(1, 129)), int(rng.choice((0, 1, 64, 65, 500, 4096, 100000)))
        row = int(rng.integers(0, n))
        size = b.tree_attention_fp4kv_workspace(B, Hkv * g, Hkv, d, n, row, prefix)
        fewer = int(rng.integers(1, n + 1))
        rows, shorter = int(rng.integers(1, min(fewer, n - row) + 1)), int(rng.integers(0, prefix + 1))
        assert b.tree_attention_fp4kv_workspace(B, Hkv * g, Hkv, d, fewer, fewer - rows, shorter) <= size


def _store(dtype=1, B=2, H=4, d=128, rows=5, k=ONE, v=ONE, bs=4096, hs=128, rs=512, first=ONE, n=ONE, cache=CACHE, base=ONE, dst=128 * 128, cap=128):
    return b.lib.mcsd_store_fp4kv(dtype, B, H, d, rows, k, v, bs, hs, rs, first, n, None if cache is None else C.byref(cache), base, dst, cap, None)


def _load(dtype=1, B=2, H=4, d=128, layers=1, rows=5, k=256, v=256, bs=4096, hs=128, rs=512, first=ONE, n=ONE, cache=CACHE, base=ONE, dst=128 * 128, cap=128):
    arr = (b.Fp4Cache * 70)(*[cache] * 70)
    ks, vs = (C.c_void_p * 70)(*[k] * 70), (C.c_void_p * 70)(*[v] * 70)
    return b.lib.mcsd_load_fp4kv(dtype, B, H, d, layers, rows, arr, base, dst, cap, first, n, ks, vs, bs, hs, rs, None)


SHARED = [(dict(B=0), b.MCSD_EINVAL), (dict(B=65536), b.MCSD_EINVAL), (dict(H=0), b.MCSD_EINVAL), (dict(dtype=2), b.MCSD_EINVAL), (dict(rows=-1), b.MCSD_EINVAL),
          (dict(bs=-8), b.MCSD_EINVAL), (dict(hs=4), b.MCSD_EINVAL), (dict(rs=12), b.MCSD_EINVAL), (dict(first=None), b.MCSD_EINVAL), (dict(n=None), b.MCSD_EINVAL),
          (dict(base=None), b.MCSD_EINVAL), (dict(dst=64), b.MCSD_EINVAL), (dict(cap=-1), b.MCSD_EINVAL), (dict(d=32), b.MCSD_EUNSUPPORTED),
          (dict(rows=2 ** 31 - 1, H=2), b.MCSD_EUNSUPPORTED), (dict(cache=b.Fp4Cache(256, 256, 256, 0)), b.MCSD_EINVAL),
          (dict(cache=b.Fp4Cache(260, 256, 256, 256)), b.MCSD_EINVAL)]


@pytest.mark.parametrize("wrong,status", SHARED)
def test_store_and_load_refuse(wrong, status):
    assert _store(**wrong) == status
    assert _load(**wrong) == status


def test_store_and_load_refuse_their_own():
    assert _store(k=None) == b.MCSD_EINVAL and _store(v=C.c_void_p(8)) == b.MCSD_EINVAL and _store(cache=None) == b.MCSD_EINVAL
    assert _load(k=None) == b.MCSD_EINVAL and _load(v=8) == b.MCSD_EINVAL and _load(layers=0) == b.MCSD_EINVAL
    assert _load(layers=65) == b.MCSD_EUNSUPPORTED
    assert _store(rows=0) == b.MCSD_OK and _load(rows=0) == b.MCSD_OK            # nothing to do, nothing launched


def _commit(B=2, H=4, d=128, layers=2, kt=256, vt=256, ns=44, cache=CACHE, base=ONE, hs=128 * 128, mp=100, cap=104, path=ONE, alen=ONE, tokens=ONE,
            new=ONE, n_new=1, n_append=1, lens=ONE, ids=ONE, n_ids=ONE):
    view = _view()
    arr = (b.Fp4Cache * 70)(*[cache] * 70)
    kts, vts = (C.c_void_p * 70)(*[kt] * 70), (C.c_void_p * 70)(*[vt] * 70)
    return b.lib.mcsd_commit_path_fp4kv(C.byref(view), B, H, d, layers, kts, vts, ns, arr, base, hs, mp, cap, path, alen, tokens, new, n_new, n_append,
                                        lens, ids, n_ids, None)


@pytest.mark.parametrize("wrong,status", [
    (dict(B=0), b.MCSD_EINVAL), (dict(H=0), b.MCSD_EINVAL), (dict(layers=0), b.MCSD_EINVAL), (dict(layers=65), b.MCSD_EUNSUPPORTED), (dict(d=96), b.MCSD_EUNSUPPORTED),
    (dict(ns=43), b.MCSD_EINVAL), (dict(hs=-128), b.MCSD_EINVAL), (dict(hs=192), b.MCSD_EINVAL), (dict(cap=103), b.MCSD_EINVAL), (dict(mp=-1), b.MCSD_EINVAL),
    (dict(n_append=2), b.MCSD_EINVAL), (dict(new=None), b.MCSD_EINVAL), (dict(n_new=-1), b.MCSD_EINVAL), (dict(kt=None), b.MCSD_EINVAL), (dict(vt=8), b.MCSD_EINVAL),
    (dict(path=None), b.MCSD_EINVAL), (dict(alen=None), b.MCSD_EINVAL), (dict(tokens=None), b.MCSD_EINVAL), (dict(lens=None), b.MCSD_EINVAL), (dict(ids=None), b.MCSD_EINVAL),
    (dict(n_ids=None), b.MCSD_EINVAL), (dict(base=None), b.MCSD_EINVAL), (dict(cache=b.Fp4Cache(0, 256, 256, 256)), b.MCSD_EINVAL)])
def test_commit_refuses(wrong, status):
    assert _commit(**wrong) == status


def _qk(tree, dtype=1, B=2, Hq=4, Hkv=2, d=128, row=0, q=ONE, k=ONE, v=ONE, qb=8 * 1024, qr=1024, kvb=8 * 1024, kvr=1024, rope=None, first=ONE, mp=100, qo=ONE, ko=ONE,
        vo=ONE, out=44, rows=44, n=ONE):
    rope = b.Rope(128, 0, 1e-6, 256, 256, 256) if rope is None else rope
    if tree:
        return b.lib.mcsd_tree_qk_norm_rope(C.byref(_view()), dtype, B, Hq, Hkv, d, row, q, k, v, qb, qr, kvb, kvr, C.byref(rope), first, mp, qo, ko, vo, out, None)
    return b.lib.mcsd_prompt_qk_norm_rope(dtype, B, Hq, Hkv, d, rows, q, k, v, qb, qr, kvb, kvr, C.byref(rope), first, n, qo, ko, vo, out, None)


@pytest.mark.parametrize("tree", [True, False])
@pytest.mark.parametrize("wrong,status", [
    (dict(dtype=3), b.MCSD_EINVAL), (dict(B=0), b.MCSD_EINVAL), (dict(Hq=0), b.MCSD_EINVAL), (dict(Hkv=0), b.MCSD_EINVAL), (dict(d=192), b.MCSD_EUNSUPPORTED),
    (dict(q=None), b.MCSD_EINVAL), (dict(k=None), b.MCSD_EINVAL), (dict(v=None), b.MCSD_EINVAL), (dict(vo=None), b.MCSD_EINVAL), (dict(qo=None), b.MCSD_EINVAL),
    (dict(ko=None), b.MCSD_EINVAL), (dict(first=None), b.MCSD_EINVAL), (dict(qb=4), b.MCSD_EINVAL), (dict(qr=-8), b.MCSD_EINVAL), (dict(kvb=9), b.MCSD_EINVAL),
    (dict(kvr=-1024), b.MCSD_EINVAL), (dict(out=43), b.MCSD_EINVAL), (dict(q=C.c_void_p(8)), b.MCSD_EINVAL), (dict(vo=C.c_void_p(8)), b.MCSD_EINVAL),
    (dict(rope=b.Rope(136, 0, 1e-6, 256, None, None)), b.MCSD_EINVAL), (dict(rope=b.Rope(24, 0, 1e-6, 256, None, None)), b.MCSD_EINVAL),
    (dict(rope=b.Rope(-16, 0, 1e-6, 256, None, None)), b.MCSD_EINVAL), (dict(rope=b.Rope(64, 0, -1.0, 256, None, None)), b.MCSD_EINVAL),
    (dict(rope=b.Rope(64, 0, math.nan, 256, None, None)), b.MCSD_EINVAL), (dict(rope=b.Rope(64, 0, math.inf, 256, None, None)), b.MCSD_EINVAL),
    (dict(rope=b.Rope(64, 0, 1e-6, None, None, None)), b.MCSD_EINVAL), (dict(Hq=65000, Hkv=1000), b.MCSD_EUNSUPPORTED)])
def test_qk_refuses(tree, wrong, status):
    assert _qk(tree, **wrong) == status


def test_qk_refuses_what_one_of_the_two_has():
    assert _qk(True, row=44) == b.MCSD_EINVAL and _qk(True, row=-1) == b.MCSD_EINVAL and _qk(True, mp=-1) == b.MCSD_EINVAL
    assert _qk(False, n=None) == b.MCSD_EINVAL and _qk(False, rows=-1) == b.MCSD_EINVAL
    assert _qk(False, rows=0) == b.MCSD_OK


def test_structures_are_checked_by_class():
    t, view, codes = torch.zeros(8), _view(), torch.zeros(64, dtype=torch.uint8)
    cache, rope = b.make_fp4_cache(codes, codes, codes, codes), b.make_rope(16, t)
    for wrong in (rope, b.Mlp(), bytearray(64), None, 7):
        with pytest.raises((C.ArgumentError, TypeError)):
            b.tree_attention_fp4kv(view, 1, 4, 4, 64, 0, t, t, t, 44, wrong, t, t, 128, 8, 0.1, t, t)
        with pytest.raises((C.ArgumentError, TypeError)):
            b.store_fp4kv(0, 1, 1, 64, 1, t, t, 0, 0, 0, t, t, wrong, t, 128, 8)
        with pytest.raises((C.ArgumentError, TypeError)):
            b.load_fp4kv(0, 1, 1, 64, 1, [wrong], t, 128, 8, t, t, [t], [t], 0, 0, 0)
        with pytest.raises((C.ArgumentError, TypeError)):
            b.commit_path_fp4kv(view, 1, 1, 64, [t], [t], 44, [wrong], t, 128, 8, 16, t, t, t, t, 1, 1, t, t, t)
    for wrong in (cache, b.Mlp(), bytearray(64), None, 7):
        with pytest.raises((C.ArgumentError, TypeError)):
            b.tree_qk_norm_rope(view, 0, 1, 1, 1, 64, 0, t, t, t, 0, 0, 0, 0, wrong, t, 8, t, t, t, 44)
        with pytest.raises((C.ArgumentError, TypeError)):
            b.prompt_qk_norm_rope(0, 1, 1, 1, 64, 1, t, t, t, 0, 0, 0, 0, wrong, t, t, t, t, t, 44)
    with pytest.raises((C.ArgumentError, TypeError)):
        b.tree_attention_fp4kv(cache, 1, 4, 4, 64, 0, t, t, t, 44, cache, t, t, 128, 8, 0.1, t, t)


class NoStream:
    cuda_stream = 0


def test_lists_of_other_lengths_are_refused():
    t, view, codes = torch.zeros(8), _view(), torch.zeros(64, dtype=torch.uint8)
    cache = b.make_fp4_cache(codes, codes, codes, codes)
    with pytest.raises(AssertionError):
        b.load_fp4kv(0, 1, 1, 64, 1, [cache, cache], t, 128, 8, t, t, [t], [t], 0, 0, 0, NoStream)
    with pytest.raises(AssertionError):
        b.commit_path_fp4kv(view, 1, 1, 64, [t, t], [t, t], 44, [cache], t, 128, 8, 16, t, t, t, t, 1, 1, t, t, t, NoStream)


def test_structures_are_made_of_the_right_tensors():
    codes = torch.zeros(64, dtype=torch.uint8)
    with pytest.raises(b.McsdError):
        b.make_fp4_cache(codes, codes, codes, torch.zeros(64))
    with pytest.raises(b.McsdError):
        b.make_rope(16, torch.zeros(8, dtype=torch.float64))
    with pytest.raises(b.McsdError):
        b.make_rope(32, torch.zeros(8))
    with pytest.raises(b.McsdError):
        b.make_rope(16, torch.zeros(8), torch.zeros(128, dtype=torch.bfloat16))
