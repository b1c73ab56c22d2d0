"""Rows into and out of the 4-bit prefix cache: what is stored is the definition's codes and scales bit for bit, what is read back
the numbers they stand for, and nothing else is touched."""
import math

import numpy as np
import pytest
import torch

import fp4_reference as R
from fp4_reference import Cache

pytestmark = pytest.mark.gpu
DTYPES = {torch.float32: 0, torch.bfloat16: 1}


@pytest.fixture(scope="module")
def binding():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2409_10644_amd import binding as b
    return b


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _numbers(gen, shape, dtype):
    x = torch.randn(shape, generator=gen, device="cuda") * torch.exp(2.0 * torch.randn(shape[:-1] + (1,), generator=gen, device="cuda"))
    return x.to(dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,H,T", [(1, 1, 1), (3, 5, 1), (2, 3, 17), (4, 8, 33), (2, 32, 130)])
def test_rows_are_stored_as_defined_and_read_back(binding, dtype, d, B, H, T):
    gen = torch.Generator("cuda").manual_seed(B * 1000 + H * 10 + T + d)
    first = [(7 * b) % 5 for b in range(B)]
    n = [T if b == 0 else (T * (b + 1)) // (B + 1) for b in range(B)]
    cap = T + 6 + (T % 2)
    cache = Cache(binding, B, H, cap, d, gap=4 if (cap + 4) * d % 128 == 0 else 5)
    assert cache.head_stride % 128 == 0
    k, v = _numbers(gen, (B, T, H, d), dtype), _numbers(gen, (B, T, H, d), dtype)
    before = [a.clone() for a in cache.arrays]
    binding.store_fp4kv(DTYPES[dtype], B, H, d, T, k, v, T * H * d, d, H * d, _i32(first), _i32(n), cache.handle, cache.base,
                        cache.head_stride, cap)
    ko, vo = (torch.full((B, H, T + 2, d), 9.0, dtype=dtype, device="cuda") for _ in range(2))
    binding.load_fp4kv(DTYPES[dtype], B, H, d, T, [cache.handle], cache.base, cache.head_stride, cap, _i32(first), _i32(n), [ko], [vo],
                       H * (T + 2) * d, (T + 2) * d, d)
    torch.cuda.synchronize()
    want = [a.clone() for a in before]
    whole = Cache(binding, B, H, cap, d, gap=cache.head_stride // d - cap)
    for a, w in zip(whole.arrays, want):
        a.copy_(w)
    for i, x in ((0, k), (2, v)):
        codes, scales = R.quantise(x.transpose(1, 2))
        for b in range(B):
            at = B - 1 - b
            for j, new in ((i, codes), (i + 1, scales)):
                a = whole.arrays[j].reshape(B, H, -1, whole.arrays[j].shape[-1])
                a[at, :, first[b]:first[b] + n[b]] = new[b, :, :n[b]]
    for a, w in zip(cache.arrays, whole.arrays):
        assert torch.equal(a, w)
    for out, i in ((ko, 0), (vo, 2)):
        num = R.decode(cache.view(i), cache.view(i + 1))
        want = torch.full_like(out, 9.0)
        for b in range(B):
            want[b, :, :n[b]] = num[b, :, first[b]:first[b] + n[b]].to(dtype)
        assert torch.equal(out, want)


@pytest.mark.parametrize("dtype", DTYPES)
def test_numbers_at_the_ends_of_the_range(binding, dtype):
    """Ties, the largest magnitude near the next power of two, subnormals, zeros of both signs, infinities, NaN."""
    tiny = 2.0 ** -126
    rows = [[6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -5.0, -0.25, -2.5, -0.0], [7.0, 1.75, 1], [6.96875, 1.75, 1], [3.4e38, -1e38, 1e36], [2.9e38], [tiny, tiny / 2, -tiny / 4],
            [tiny / 2, tiny / 4 * 3, -tiny / 8], [6 * tiny, 0.75 * tiny, 0.25 * tiny, 0.125 * tiny], [0.0, -0.0], [math.inf, 1.0], [math.nan, 2.0], [-math.inf, math.nan, 5.0], [448.0, 1.0, 37.0, -40.0]]
    x = torch.zeros(1, len(rows), 1, 64, dtype=torch.float64)
    for i, r in enumerate(rows):
        x[0, i, 0, 13:13 + len(r)] = torch.tensor(r, dtype=torch.float64)
        x[0, i, 0, 40] = float(i)
    x = x.to(dtype).cuda()
    T = len(rows)
    cache = Cache(binding, 1, 1, T + 1, 64)
    binding.store_fp4kv(DTYPES[dtype], 1, 1, 64, T, x, -x, T * 64, 64, 64, _i32([0]), _i32([T]), cache.handle, cache.base, 0, T)
    torch.cuda.synchronize()
    for i, y in ((0, x), (2, -x)):
        codes, scales = R.quantise(y.transpose(1, 2))
        assert torch.equal(cache.view(i + 1)[:, :, :T], scales), (cache.view(i + 1)[0, 0, :T], scales)
        assert torch.equal(cache.view(i)[:, :, :T], codes), torch.nonzero(cache.view(i)[:, :, :T] != codes)
    # every code under every scale byte
    all_bytes = Cache(binding, 1, 1, 256, 128)
    all_bytes.arrays[0].copy_(torch.arange(64, device="cuda", dtype=torch.uint8) * 4 + (torch.arange(256, device="cuda", dtype=torch.uint8) % 4)[:, None])
    all_bytes.arrays[1].copy_(torch.arange(256, device="cuda", dtype=torch.uint8)[:, None].expand(256, 4))
    all_bytes.arrays[2].copy_(all_bytes.arrays[0].flip(0))
    all_bytes.arrays[3].copy_(all_bytes.arrays[1])
    ko, vo = (torch.zeros(1, 1, 256, 128, dtype=dtype, device="cuda") for _ in range(2))
    binding.load_fp4kv(DTYPES[dtype], 1, 1, 128, 256, [all_bytes.handle], all_bytes.base, 256 * 128, 256, _i32([0]), _i32([256]), [ko], [vo],
                       256 * 128, 256 * 128, 128)
    torch.cuda.synchronize()
    for out, i in ((ko, 0), (vo, 2)):
        num = R.decode(all_bytes.view(i), all_bytes.view(i + 1))
        want = num.float().to(dtype) if dtype == torch.bfloat16 else num.float()
        # (beyond the largest finite number: infinite; below the smallest of bf16's subnormals nothing is asked: byte 0 and 1 stay above them)
        assert torch.equal(torch.isnan(out), torch.isnan(want))
        assert torch.equal(out[~torch.isnan(want)], want[~torch.isnan(want)])


def test_rows_outside_the_cache_are_skipped(binding):
    B, H, T, d, cap = 4, 2, 8, 128, 10
    cache = Cache(binding, B, H, cap, d, gap=6)
    k = torch.ones(B, H, T, d, dtype=torch.bfloat16, device="cuda")
    before = [a.clone() for a in cache.arrays]
    first, n = _i32([-3, 6, 2 ** 31 - 1, -2 ** 31]), _i32([99, 8, 8, 8])
    binding.store_fp4kv(1, B, H, d, T, k, k, H * T * d, T * d, d, first, n, cache.handle, cache.base, cache.head_stride, cap)
    torch.cuda.synchronize()
    live = torch.zeros(B, cap, dtype=torch.bool)
    live[0, 0:5] = live[1, 6:10] = True                    # (rows -3 .. 4 of a count clamped to 8; rows 6 .. 13 of a cache of 10)
    codes, scales = R.quantise(torch.ones(1, d))
    for i, want in ((0, codes), (1, scales), (2, codes), (3, scales)):
        whole, old = (a.reshape(B, H, cap + 6, -1).flip(0) for a in (cache.arrays[i], before[i]))
        for b in range(B):
            for r in range(cap + 6):
                is_new = r < cap and bool(live[b, r])
                assert torch.equal(whole[b, :, r], want.cuda().expand(H, -1) if is_new else old[b, :, r]), (i, b, r)
    out = torch.full((B, H, T, d), -7.0, dtype=torch.bfloat16, device="cuda")
    binding.load_fp4kv(1, B, H, d, T, [cache.handle], cache.base, cache.head_stride, cap, first, n, [out], [out.clone()], H * T * d, T * d, d)
    torch.cuda.synchronize()
    want = torch.full_like(out, -7.0)
    want[0, :, 3:8], want[1, :, :4] = 1.0, 1.0
    assert torch.equal(out, want)


def test_negative_counts_are_none(binding):
    cache = Cache(binding, 1, 1, 4, 64)
    before = [a.clone() for a in cache.arrays]
    x = torch.ones(1, 4, 64, device="cuda")
    binding.store_fp4kv(0, 1, 1, 64, 4, x, x, 256, 64, 64, _i32([0]), _i32([-5]), cache.handle, cache.base, 0, 4)
    torch.cuda.synchronize()
    assert all(torch.equal(a, w) for a, w in zip(cache.arrays, before))


@pytest.mark.parametrize("H,d,layers,B,branching,n_append", [(1, 64, 1, 1, (1,), 0), (5, 128, 3, 5, (2, 2, 1), 1), (32, 128, 2, 3, (4, 2, 2, 1), 2), (3, 64, 64, 4, (1,) * 32, 40),
                                                              (33, 128, 2, 4, (16, 1, 1, 1, 1), 0)])
def test_the_accepted_path_is_appended_to_every_layer(binding, H, d, layers, B, branching, n_append):
    rng = np.random.default_rng(H * d + B)
    gen = torch.Generator("cuda").manual_seed(H)
    G, view = len(branching), binding.slice_mask(binding.build_mask(branching), len(branching))
    n, max_prefix = view.n_nodes, 12
    cap = max_prefix + G + (max_prefix + G) % 2
    path = rng.integers(0, n, (B, G)).astype(np.int32)
    alen = np.resize(np.array([G, 0, max(G - 1, 1), G + 9, -1], np.int32), B)            # the last two clamped
    lens = np.resize(np.array([12, 0, 5, 99, -4], np.int32), B)
    if B > 2:
        path[0, 0], path[2, G - 1] = -1, n                                                # skipped
    tokens, new = (rng.integers(0, 1000, s).astype(np.int32) for s in ((B, n), (B, n_append + 2)))
    kt, vt = (torch.randn((layers, B, H, n + 1, d), generator=gen, device="cuda").bfloat16() for _ in range(2))
    caches = [Cache(binding, B, H, cap, d) for _ in range(layers)]
    want = [[a.clone() for a in c.arrays] for c in caches]
    want_ids, want_n, want_lens = np.full((B, G + n_append), -1, np.int32), np.zeros(B, np.int32), lens.copy()
    quantised = [[y for x in (kt, vt) for y in R.quantise(x[l])] for l in range(layers)]
    for b in range(B):
        a, L = min(max(alen[b], 0), G), min(max(lens[b], 0), max_prefix)
        for j in range(a):
            node = int(path[b, j])
            if 0 <= node < n:
                want_ids[b, j] = tokens[b, node]
                for l in range(layers):
                    for w, q in zip(want[l], quantised[l]):
                        w.reshape(B, H, cap, -1)[B - 1 - b, :, L + j] = q[b, :, node]
        want_ids[b, a:a + n_append] = new[b, :n_append]
        want_n[b], want_lens[b] = a + n_append, L + a
    dev = lambda x: torch.from_numpy(x).cuda()
    d_lens, ids, n_ids = dev(lens), torch.full((B, G + n_append), -9, dtype=torch.int32, device="cuda"), dev(np.zeros(B, np.int32))
    binding.commit_path_fp4kv(view, B, H, d, list(kt), list(vt), n + 1, [c.handle for c in caches], caches[0].base, caches[0].head_stride, max_prefix,
                              cap, dev(path), dev(alen), dev(tokens), dev(new), n_append + 2, n_append, d_lens, ids, n_ids)
    torch.cuda.synchronize()
    for c, w in zip(caches, want):
        for a, x in zip(c.arrays, w):
            assert torch.equal(a, x)
    assert np.array_equal(d_lens.cpu().numpy(), want_lens) and np.array_equal(n_ids.cpu().numpy(), want_n)
    assert np.array_equal(ids.cpu().numpy(), want_ids)


def test_several_layers_are_read_at_once(binding):
    B, H, d, cap, layers = 2, 3, 128, 8, 64
    gen = torch.Generator("cuda").manual_seed(3)
    caches = [Cache(binding, B, H, cap, d) for _ in range(layers)]
    for c in caches:
        for i, a in enumerate(c.arrays):
            a.copy_(torch.randint(0, 256 if i % 2 == 0 else 200, a.shape, generator=gen, device="cuda", dtype=torch.uint8))
    ko, vo = (torch.zeros(layers, H, B, cap, d, device="cuda") for _ in range(2))          # heads outermost: any strides
    binding.load_fp4kv(0, B, H, d, cap, [c.handle for c in caches], caches[0].base, caches[0].head_stride, cap, _i32([0, 2]), _i32([8, 5]),
                       list(ko), list(vo), cap * d, B * cap * d, d)
    torch.cuda.synchronize()
    for l, c in enumerate(caches):
        for out, i in ((ko[l], 0), (vo[l], 2)):
            num = R.decode(c.view(i), c.view(i + 1)).float()
            assert torch.equal(out[:, 0], num[0]) and torch.equal(out[:, 1, :5], num[1, :, 2:7]) and not out[:, 1, 5:].any()
