"""Infinities and NaN in the attention over the 4-bit cache, in every variant of the kernel: they reach the rows that see them and no
others, in the first and in later pieces of a pair, and what stands behind a length or beside a tree is never looked at."""
import math

import pytest
import torch

import fp4_reference as R
from test_gpu_fp4_attention import Call, binding  # noqa: F401  (binding: the fixture)

pytestmark = pytest.mark.gpu
TREES = {"nine": (3, 2), "44": (4, 2, 2, 1), "120": (8, 2, 2, 1, 1)}              # one, two and four blocks of 32 rows
LENGTHS = (300, 3001)                                                             # no multiples of a tile; the longer in several pieces


def _close(c, out, b, h, rows, cols=slice(None)):
    want, lim = c.wanted(b, h)
    err = (out[b, h].double() - want).abs()
    assert bool((err[rows][:, cols] <= lim[rows][:, cols]).all()), (b, h, float((err - lim)[rows][:, cols].max()))


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("tree", TREES)
@pytest.mark.parametrize("L", LENGTHS)
@pytest.mark.parametrize("Hq", [2, 4])
def test_nan_scales_of_prefix_rows(binding, d, tree, L, Hq):  # noqa: F811
    c = Call(binding, TREES[tree], 3, Hq, 2, d, (L,) * 3, seed=L + d)
    k, v = (c.cache.arrays[i].reshape(3, 2, -1, d // 32) for i in (1, 3))         # (sequences in reverse order)
    k[1, 0, L // 2, d // 32 - 1] = 255                     # sequence 1, first key head: a key
    v[0, 1, L - 1, 0] = 255                                # sequence 2, second key head: 32 channels of the last value
    k[2, :, L:] = 255                                      # sequence 0: rows behind its length
    v[2, :, L:] = 255
    out = c.run()[:, :, :c.n]
    every, g = slice(None), Hq // 2
    for b in range(3):
        for h in range(Hq):
            if b == 1 and h < g:
                assert bool(torch.isnan(out[b, h]).all())
            elif b == 2 and h >= g:
                assert bool(torch.isnan(out[b, h, :, :32]).all())
                _close(c, out, b, h, every, slice(32, None))
            else:
                _close(c, out, b, h, every)


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("tree", TREES)
@pytest.mark.parametrize("L", (0,) + LENGTHS)
@pytest.mark.parametrize("Hq", [3, 6])
def test_tree_rows_and_queries(binding, d, tree, L, Hq):  # noqa: F811
    """In the first node, the last of the first level, one in the middle and the last: a NaN key, infinite and NaN values, an infinite
    query; rows that see none of them are bit for bit what they are without."""
    c = Call(binding, TREES[tree], 1, Hq, 3, d, (L,), seed=L + d, max_prefix=max(L, 1))
    g, n = Hq // 3, c.n
    first, mid, last = TREES[tree][0] - 1, n // 2, n - 1
    c.q[0, :g, :, d - 1] = c.q[0, :g, :, d - 1].abs() + 0.125                     # (an infinite key's score is infinite, not its negative)
    clean = c.check()[:, :, :n]
    c.kt[0, 0, mid, 3] = math.nan
    c.kt[0, 0, first, d - 1] = math.inf
    c.vt[0, 1, mid, 9], c.vt[0, 1, first, d - 2], c.vt[0, 1, last, 40] = math.inf, -math.inf, math.nan
    c.q[0, 2 * g, last, 7] = math.inf
    c.kt[:, :, n:], c.vt[:, :, n:], c.q[:, :, n:] = math.nan, math.nan, math.nan
    out = c.run()[:, :, :n]
    sees = lambda node: c.seen[:, node]
    for h in range(g):
        hit = sees(mid) | sees(first)
        assert not bool(torch.isfinite(out[0, h][hit]).any()) and torch.equal(out[0, h][~hit], clean[0, h][~hit])
    for h in range(g, 2 * g):
        hit = torch.zeros(n, d, dtype=torch.bool, device="cuda")
        for node, col, kind in ((mid, 9, math.inf), (first, d - 2, -math.inf), (last, 40, math.nan)):
            hit[sees(node), col] = True
            got = out[0, h][sees(node), col]
            assert bool((torch.isnan(got) if math.isnan(kind) else got == kind).all()), (h, node)
        assert torch.equal(out[0, h][~hit], clean[0, h][~hit])
    for h in range(2 * g, Hq):
        rows = torch.ones(n, dtype=torch.bool, device="cuda")
        if h == 2 * g:
            rows[last] = False
            assert bool(torch.isnan(out[0, h, last]).all())
        assert torch.equal(out[0, h][rows], clean[0, h][rows])


def test_a_call_in_several_pieces_needs_a_workspace(binding):  # noqa: F811
    """Of the size asked for: without one, with a shorter or a misaligned one it is refused, and the output stays as it was."""
    c = Call(binding, TREES["44"], 1, 4, 4, 128, (3000,), seed=17)
    size = binding.tree_attention_fp4kv_workspace(1, 4, 4, 128, 44, 0, 3000)
    assert size > 0 and c.ws is not None
    c.check()
    c.out.fill_(31)
    for bad in (None, c.ws[:size - 1], torch.zeros(size + 512, dtype=torch.uint8, device="cuda")[8:]):
        keep, c.ws = c.ws, bad
        with pytest.raises(binding.McsdError) as e:
            c.call()
        assert e.value.status == binding.MCSD_EWORKSPACE
        c.ws = keep
    torch.cuda.synchronize()
    assert bool((c.out == 31).all())
    c.check()
