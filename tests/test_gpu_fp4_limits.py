"""The largest bounds that the entry points around the 4-bit cache document, with few rows that exist: the launch is as large as it
gets, and all but a few of its workgroups find nothing to do."""
import math

import pytest
import torch

import fp4_reference as R
from fp4_reference import Cache
from test_gpu_fp4_attention import Call

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def binding():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2409_10644_amd import binding as b
    return b


def _i32(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("d,H,most", [(128, 1, 2 ** 28 - 16), (64, 3, (2 ** 29 - 32) // 3)])
def test_rows_up_to_a_launch(binding, d, H, most):
    gen = torch.Generator("cuda").manual_seed(d)
    n, cap = 21, 32
    cache = Cache(binding, 1, H, cap, d, fill=0)
    k, v = (torch.randn(H, n, d, generator=gen, device="cuda").bfloat16() for _ in range(2))
    ko, vo = (torch.full((H, n + 1, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    binding.store_fp4kv(1, 1, H, d, most, k, v, 0, n * d, d, _i32(5), _i32(n), cache.handle, cache.base, cache.head_stride, cap)
    binding.load_fp4kv(1, 1, H, d, most, [cache.handle], cache.base, cache.head_stride, cap, _i32(5), _i32(n), [ko], [vo], 0, (n + 1) * d, d)
    torch.cuda.synchronize()
    for x, out, i in ((k, ko, 0), (v, vo, 2)):
        codes, scales = R.quantise(x)
        assert torch.equal(cache.view(i)[0, :, 5:5 + n], codes) and torch.equal(cache.view(i + 1)[0, :, 5:5 + n], scales)
        assert torch.equal(out[:, :n].double(), R.decode(codes, scales)) and bool((out[:, n:] == 7).all())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("most", [2 ** 24 - 1, 2 ** 24, 2 ** 26 - 4])
def test_prompt_rows_up_to_a_launch(binding, d, most):
    """One row per workgroup, and four where a launch does not hold so many."""
    n = 7
    gen = torch.Generator("cuda").manual_seed(d)
    q, k = (torch.randn(n, d, generator=gen, device="cuda") for _ in range(2))
    inv = (10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)).float().cuda()
    qo, ko = (torch.full((n + 1, d), 7.0, device="cuda") for _ in range(2))
    binding.prompt_qk_norm_rope(0, 1, 1, 1, d, most, q, k, None, 0, d, 0, d, binding.make_rope(d, inv), _i32(40), _i32(n), qo, ko, None, most)
    torch.cuda.synchronize()
    for x, out in ((q, qo), (k, ko)):
        want, size = R.rotated(x.double(), None, 0.0, 40 + torch.arange(n, device="cuda"), inv, d, False)
        # fp32: half a step of the output, and fewer than 32 roundings on the way (angle, sine, products)
        assert bool(((out[:n].double() - want).abs() <= 2.0 ** -24 * want.abs() + 32 * 2.0 ** -24 * size).all())
        assert bool((out[n:] == 7).all())


@pytest.mark.parametrize("branching", [(2,), (4, 2, 2, 1), (8, 2, 2, 1, 1)])
@pytest.mark.parametrize("L,tail", [(2 ** 31 - 1, 63), (2 ** 31 - 63, 1)])
def test_the_longest_prefix(binding, branching, L, tail):
    """As many keys of one head as a length can say, and so many that the last tile of 64 holds one; 68 GiB of codes and scales that
    keys and values share.  All numbers are 1 but those of the last rows, which are 6 and draw much of the weight: an output that
    misses them, or counts one for each row of the tile, is far off."""
    d, g = 64, len(branching)
    codes = torch.full((2 ** 31, d // 2), 0x22, dtype=torch.uint8, device="cuda")
    codes[L - tail:] = 0x77
    scales = torch.full((2 ** 31, d // 32), 127, dtype=torch.uint8, device="cuda")
    view = binding.slice_mask(binding.build_mask(branching), g)
    n, scale = view.n_nodes, 0.125
    q = torch.full((1, 1, n, d), 0.5, dtype=torch.bfloat16, device="cuda")
    kt, vt, out = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(q)
    size = binding.tree_attention_fp4kv_workspace(1, 1, 1, d, n, 0, L)
    binding.tree_attention_fp4kv(view, 1, 1, 1, d, 0, q, kt, vt, n, binding.make_fp4_cache(codes, scales, codes, scales), torch.zeros(1, dtype=torch.int64, device="cuda"),
                                 _i32(L), 0, L, scale, out, binding.new_workspace(size))
    torch.cuda.synchronize()
    got = out.double()
    del codes, scales
    torch.cuda.empty_cache()
    # scores 4 and 24, of the tree's own keys 0 (their values are 0; a node sees at most g of them)
    ones, sixes = (L - tail) * math.exp(4.0 - 24.0), float(tail)
    want = (ones + 6 * sixes) / (ones + sixes)
    # output and weights rounded to bf16 (2^-8 each); a score off by scale * 2^-12 / 3.75 * max|q| * sum|k| (two groups of 32) and by
    # 160 roundings of fp32 of its size; the sums: parts of 2^26 equal weights at most, added 16 at a time and so exact up to 2^28,
    # and 32 parts of 2^-24; the tree's weights
    delta = scale * 2.0 ** -12 / 3.75 * 0.5 * d * 6 + 160 * 2.0 ** -24 * 24
    lim = want * (2 * 2.0 ** -8 + math.expm1(2 * delta) + 64 * 2.0 ** -24 + g * math.exp(-4.0) / L)
    assert abs(want - 1) > 10 * lim and abs(want - 6) > lim and bool(((got - want).abs() <= lim).all()), (want, lim, got.min().item(), got.max().item())


@pytest.mark.parametrize("B,H,hi", [(256, 80, 100), (1000, 1, 900), (700, 3, 40)])
def test_many_sequences_and_heads(binding, B, H, hi):
    """More than 32 whole pairs to a workgroup; and more sequences than a workgroup keeps the lengths of."""
    gen = torch.Generator().manual_seed(B)
    lens = torch.randint(0, hi + 1, (B,), generator=gen).tolist()
    lens[0], lens[-1] = hi, 0
    c = Call(binding, (2,), B, H, H, 64, lens, seed=B)
    pairs = {(int(b), int(h)) for b, h in zip(torch.randint(0, B, (60,), generator=gen), torch.randint(0, H, (60,), generator=gen))}
    out = c.check(pairs | {(0, 0), (B - 1, H - 1), (B // 2, 0), (256 % B, 0), (255, H - 1)})
    assert not bool((out[:, :, :c.n] == 31).all(-1).any())                       # every pair is written
    c.out.fill_(31)
    assert torch.equal(c.run(), out)
