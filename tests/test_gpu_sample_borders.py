"""Borders and draws that fall among tokens of 2^-45 of the largest weight, in rows whose weights' sum has more than 53 bits."""
import math

import pytest
import torch

import latent_reference as R
from test_gpu_sample_rows import CODE, _settings, binding  # noqa: F401

pytestmark = pytest.mark.gpu

LARGE, SMALL = 0.0, -45 * math.log(2)      # (in bf16 a weight of 0.94 .. 1.06 times 2^-45; what is asked for depends on no more than that they are alike)


@pytest.mark.parametrize("dtype", CODE)
@pytest.mark.parametrize("N,s", [(2000, 1005), (31000, 2001), (260000, 2001)])
@pytest.mark.parametrize("u", [0.25, 0.5, 0.75])
@pytest.mark.parametrize("scheme", [0, 1])
@pytest.mark.parametrize("copies", [1, 300])
def test_draws(binding, dtype, N, s, u, scheme, copies):  # noqa: F811
    """u N large weights L, s small ones, the other large ones: the sum first exceeds u (N L + s) at small token number floor(u s), counted
    from 0.  (u s is no whole number.)"""
    V, first = N + s, int(N * u)
    assert first == N * u and u * s != int(u * s)
    x = torch.full((V,), LARGE, device="cuda")
    x[first:first + s] = SMALL
    tokens = torch.empty(copies, dtype=torch.int32, device="cuda")
    binding.sample_rows(CODE[dtype], 1, copies, V, x.to(dtype), 0, 0, binding.make_sampler(), None, 0, scheme, 1, torch.full((copies,), u, device="cuda"), tokens, copies)
    assert tokens.tolist() == [first + int(u * s)] * copies


@pytest.mark.parametrize("dtype", CODE)
@pytest.mark.parametrize("N,s,top_k", [(510, 1, 511), (31000, 31, 0), (31000, 31, 31031), (262042, 101, 0)])
@pytest.mark.parametrize("n", [0, 1])
@pytest.mark.parametrize("copies", [1, 300])
def test_top_p(binding, dtype, N, s, top_k, n, copies):  # noqa: F811
    """Half of N large weights and s small ones is more than N / 2 large ones: the next is kept too."""
    V, kept = N + s + 1, N // 2 + 1
    x = torch.full((V,), LARGE, device="cuda")
    x[N:] = SMALL
    x[V - 1] = -1e4
    arrays, _ = _settings([(1.0, top_k, 0.5, 0.0)])
    probs = torch.empty(copies, V, device="cuda")
    tokens = torch.empty(copies, dtype=torch.int32, device="cuda")
    u = torch.full((copies,), 1 - 2.0 ** -24, device="cuda")
    binding.sample_rows(CODE[dtype], 1, copies, V, x.to(dtype), 0, 0, binding.make_sampler(*arrays), probs, copies * V, 0, n, u if n else None, tokens if n else None, copies * n)
    torch.cuda.synchronize()
    want = torch.zeros(V, dtype=torch.float64)
    want[:kept] = 1 / kept
    R.check_probs(probs[0], want)
    assert torch.equal(probs, probs[:1].expand_as(probs))
    if n:
        assert tokens.tolist() == [kept - 1] * copies
