"""What three 6-bit terms per 32 channels leave of a query, and of its scores (no GPU needed)."""
import math

import pytest
import torch

import fp4_query_terms as T
import fp4_reference as R


def _queries(kind, seed):
    gen = torch.Generator().manual_seed(seed)
    q = torch.randn(2000, 64, generator=gen, dtype=torch.float64)
    if kind == "uniform":
        q = 0.66 * torch.rand(2000, 64, generator=gen, dtype=torch.float64)       # (the largest, times c, a little above 3.75 / 32)
    elif kind != "normal":
        q[:, 5] = float(kind)
    return q.bfloat16()


@pytest.mark.parametrize("kind", ["normal", "uniform", "30", "100", "1000"])
def test_what_the_terms_leave(kind):
    q = _queries(kind, 1)
    got, x = T.held(q, 0.125)
    m = x.double().unflatten(-1, (-1, 32)).abs().amax(-1, keepdim=True)
    left = (got - x.double()).unflatten(-1, (-1, 32)).abs() / m
    assert bool((left <= T.LEFT).all())
    if kind == "uniform":
        assert float(left.max()) > 2.0 ** -14              # (2^-14 is less than it can be)


def test_scores_with_a_channel_far_above_the_others():
    """Where the key is zero in that channel all of the score comes from the others: off by more than 2^-13 of |q| |k|, within
    sqrt(32) * LEFT of it, and within LEFT * max |q| * sum |k| per group."""
    q = _queries("84.5", 2)                                # (times c a little above 3.75 * 4)
    got, x = T.held(q, 0.125)
    off = got - x.double()
    k = torch.sign(off)                                    # the worst key of ones; a code of 0 where the large channel is
    k[:, 5] = 0
    err, size = (off * k).sum(-1).abs(), x.double().norm(dim=-1) * k.norm(dim=-1)
    bound = T.LEFT * (x.double().abs().unflatten(-1, (-1, 32)).amax(-1) * k.abs().unflatten(-1, (-1, 32)).sum(-1)).sum(-1)
    assert bool((err <= bound).all()) and bool((bound <= math.sqrt(32) * T.LEFT * size * (1 + 1e-12)).all())
    assert float((err / size).max()) > 2.0 ** -13


def test_a_channel_within_a_thirtieth_of_the_largest_keeps_the_bits_of_bf16():
    """bf16 rounds by 2^-9 of a number at the least; the terms by LEFT of the largest: coarser below 1/30 of it."""
    assert 1 / 31 < T.LEFT / 2.0 ** -9 < 1 / 29
