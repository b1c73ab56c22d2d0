"""Queries with one channel far above the others of its group, as models have them, in every variant of the attention over the 4-bit
cache: within the documented bound of the scores, and, far closer, what three 6-bit terms of each query give."""
import math

import pytest
import torch

import fp4_query_terms as T
import fp4_reference as R
from test_gpu_fp4_attention import Call, binding  # noqa: F401  (binding: the fixture)

pytestmark = pytest.mark.gpu
TREES = {"one block": (3, 2), "two": (4, 2, 2, 1), "four": (8, 2, 2, 1, 1)}       # blocks of 32 rows in a workgroup: 9, 44, 120 rows


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("tree", TREES)
@pytest.mark.parametrize("above", [30.0, 100.0, 1000.0])
@pytest.mark.parametrize("code", ["zero", "small"])
def test_scores_beside_a_large_channel(binding, d, tree, above, code):  # noqa: F811
    """`above` times the others' deviation, in another channel for each row of a group of 32 channels; the keys' codes there are zero
    or half a step of their group."""
    L, H = 777, 2
    c = Call(binding, TREES[tree], 1, H, H, d, (L,), seed=int(above) + d)
    at = torch.tensor([5, d - 3], device="cuda")           # one channel in the first group, one in the last
    c.q[:, :, :, at] = above
    c.kt[:, :, :, at] = 0
    byte = c.cache.arrays[0][:, at // 2]
    nibble = torch.tensor([4 * int(x % 2) for x in at.tolist()], device="cuda", dtype=torch.uint8)
    byte = byte & ~(15 << nibble) | ((1 if code == "small" else 0) << nibble)
    c.cache.arrays[0][:, at // 2] = byte.to(torch.uint8)
    out = c.run()
    for h in range(H):
        kp, vp = (R.decode(c.cache.view(i)[0, h, :L], c.cache.view(i + 1)[0, h, :L]) for i in (0, 2))
        if code == "zero":
            assert not kp[:, at].any()
        of_terms, of_queries, A, terms_off, fp32_off = T.attention(c.q[0, h, :c.n], kp, c.kt[0, h, :c.n], vp, c.vt[0, h, :c.n], c.seen, c.scale)
        got = out[0, h, :c.n].double()
        # output and weights rounded to bf16, 2^-8 each; exponentials and sums in fp32, 2^-15; scores by the causes given, each in
        # numerator and denominator
        for want, off in ((of_terms, fp32_off), (of_queries, fp32_off + terms_off)):
            lim = 2.0 ** -8 * want.abs() + (2.0 ** -8 + torch.expm1(2 * off) + 2.0 ** -15) * A
            err = (got - want).abs()
            assert bool((err <= lim).all()), f"head {h}: worst {float((err - lim).max()):.3e} over, {int((err > lim).sum())} of {err.numel()}"
