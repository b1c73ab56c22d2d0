"""NaN and infinities in tree rows of the attention over a latent cache, in every variant of the kernel: they reach the output rows that see
the node and no others."""
import math

import pytest
import torch

from test_gpu_latent_attention import SIZES, Call, binding  # noqa: F401

pytestmark = pytest.mark.gpu

# heads, prefix lengths: one chunk of rows or several, keys of a sequence in one piece or cut
SHAPES = [((2, 2), 4, (20, 300)), ((4, 2, 2, 1), 16, (20, 0, 7)), ((3, 2, 2), 2, (2500,)), ((8, 2, 2, 1, 1), 5, (1000, 90))]


@pytest.mark.parametrize("branching,H,lens", SHAPES)
@pytest.mark.parametrize("dl,dr", SIZES)
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_tree_rows_that_are_not_finite(binding, branching, H, lens, dl, dr, value):  # noqa: F811
    c = Call(binding, branching, H, dl, dr, lens)
    want = c.check().clone()
    clean = c.tree.clone()
    for node, channel in ((0, 5), (c.n // 2, dl - 1), (c.n - 1, dl // 2), (c.n - 1, dl + dr - 1)):
        c.tree.copy_(clean)
        c.tree[0, node, channel] = value
        c.out.fill_(9)
        c.call()
        torch.cuda.synchronize()
        sees = c.seen[:, node]
        assert torch.equal(c.out[1:], want[1:])
        assert bool(torch.isnan(c.out[0, :, :c.n][:, sees].float()).all()), (node, channel)
        # (a node that is not seen has no part in a row: the same bits)
        assert torch.equal(c.out[0, :, :c.n][:, ~sees], want[0, :, :c.n][:, ~sees]), (node, channel)
        assert torch.equal(c.out[0, :, c.n:], want[0, :, c.n:])


@pytest.mark.parametrize("dl,dr", SIZES)
def test_all_nodes_but_one_branch(binding, dl, dr):  # noqa: F811
    """Every row that the last node does not see is NaN in all channels: its own output, and its ancestors', stay."""
    c = Call(binding, (8, 2, 2, 1, 1), 16, dl, dr, (333,))
    want = c.check().clone()
    kept = c.seen[c.n - 1]
    c.tree[0, :c.n][~kept] = math.nan
    c.out.fill_(9)
    c.call()
    torch.cuda.synchronize()
    assert torch.equal(c.out[0, :, :c.n][:, kept], want[0, :, :c.n][:, kept])
    assert bool(torch.isnan(c.out[0, :, :c.n][:, ~kept].float()).all())


@pytest.mark.parametrize("branching,H,lens", [((2, 2), 2, (20, 300)), ((2, 1), 4, (2500,)), ((1, 1, 1), 5, (700, 0))])
@pytest.mark.parametrize("dl,dr", SIZES)
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_no_more_than_16_rows(binding, branching, H, lens, dl, dr, value):  # noqa: F811
    test_tree_rows_that_are_not_finite(binding, branching, H, lens, dl, dr, value)
