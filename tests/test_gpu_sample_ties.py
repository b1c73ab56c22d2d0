"""Ties at the cut of a row, wherever among eight neighbouring tokens its last kept one is: of zeros of both signs, of the lowest finite
number, and of a number with larger ones above it."""
import pytest
import torch

from test_gpu_sample_rows import CODE, binding, run  # noqa: F401

pytestmark = pytest.mark.gpu

KEPT = (*range(2, 20), 40, 41, 42, 43, 44, 45, 46, 47, 600, 601, 602, 603, 604, 605, 606, 607, 608, 1202)


@pytest.mark.parametrize("dtype", CODE)
@pytest.mark.parametrize("kind", ["zeros", "lowest", "above"])
def test_last_kept_token_of_a_tie(binding, dtype, kind):  # noqa: F811
    V = 1203
    x = torch.zeros(V, device="cuda")
    if kind == "zeros":
        x[::3] = -0.0
        x[::7] = -1e-30
    elif kind == "lowest":
        x[:] = torch.finfo(dtype).min
        x[::5] = -float("inf")
    else:
        x[100::50] = 2.0
        x[1::2] = -1.0
    gen = torch.Generator("cuda").manual_seed(11)
    settings = [(1.0, k, 1.0, 0.0) for k in KEPT] + [(1.0, 0, k / 97, 0.0) for k in range(1, 17)]
    us = torch.rand(len(settings), 1, 3, generator=gen, device="cuda")
    for distinct in (False, True):
        run(binding, x.to(dtype).expand(len(settings), 1, V).contiguous(), settings, us, distinct)
