"""Equal logits at the border of top-k where top-p keeps all that top-k kept: what top-k left out stays out, whichever way the cut is
found, in small batches and in ones of more rows than compute units."""
import pytest
import torch

import latent_reference as R
from test_gpu_sample_rows import CODE, _settings, binding, run  # noqa: F401

pytestmark = pytest.mark.gpu

# (tokens, (temperature, top-k, top-p, min-p))
EQUAL = [(3000, (1.0, 50, 0.99, 0.0)), (2000, (1.0, 600, 0.9995, 0.0)), (32000, (1.0, 50, 0.99, 0.0)), (32000, (1.0, 300, 0.999, 0.0)), (32000, (1.0, 3000, 0.99999, 0.0)),
         (32000, (0.6, 3000, 0.99999, 0.9)), (32000, (1.0, 12345, 0.99999, 0.0))]
DRAWN = [(top_k, top_p, min_p) for top_k in (300, 600, 3000) for top_p in (0.999, 0.99999) for min_p in (0.0, 1e-30)]


def _rows(x, settings, n):
    """x [V] -> rows of it for every setting, and numbers to draw by, the last of them up to the end of what is kept."""
    us = torch.rand(len(settings), 1, n, generator=torch.Generator("cuda").manual_seed(3), device="cuda") if n else None
    if n:
        us[..., 0] = 1 - 2.0 ** -24
    return x.expand(len(settings), 1, x.numel()).contiguous(), us


def _check(binding, x, settings, n, distinct):
    """Against the definition, one row for each setting, then the same rows in a batch of more rows than compute units."""
    x, us = _rows(x, settings, n)
    B, V = len(settings), x.shape[-1]
    run(binding, x, settings, us, distinct)
    copies = torch.cuda.get_device_properties(0).multi_processor_count // B + 1
    arrays, numbers = _settings(settings)
    many = torch.empty(B, copies, V, device="cuda")
    tokens = torch.empty(B, copies, max(n, 1), dtype=torch.int32, device="cuda")
    binding.sample_rows(CODE[x.dtype], B, copies, V, x.repeat(1, copies, 1), copies * V, V, binding.make_sampler(*arrays), many, copies * V,
                        binding.MCSD_WITHOUT_REPLACEMENT if distinct else binding.MCSD_WITH_REPLACEMENT, n, us.repeat(1, copies, 1) if n else None,
                        tokens if n else None, copies * n)
    torch.cuda.synchronize()
    assert torch.equal(many, many[:, :1].expand_as(many)) and (not n or torch.equal(tokens, tokens[:, :1].expand_as(tokens)))
    for b in range(B):
        want, want_tokens = R.sample_row(x[b, 0].cpu(), *numbers[b], us=us[b, 0].tolist() if n else [], distinct=distinct)
        R.check_probs(many[b, 0], want)
        assert int((many[b, 0] > 0).sum()) <= settings[b][1]
        # (each probability is off by at most 8 roundings of 2^-24 of it: so is their sum)
        assert abs(float(many[b, 0].double().sum()) - 1) <= 8 * 2.0 ** -24
        if n:
            assert tokens[b, 0].tolist() == want_tokens, settings[b]


@pytest.mark.parametrize("dtype", CODE)
@pytest.mark.parametrize("n,distinct", [(0, False), (4, False), (4, True)])
@pytest.mark.parametrize("V,settings", EQUAL)
def test_rows_of_equal_logits(binding, dtype, n, distinct, V, settings):  # noqa: F811
    _check(binding, torch.full((V,), -0.75, device="cuda", dtype=dtype), [settings], n, distinct)


@pytest.mark.parametrize("dtype", CODE)
@pytest.mark.parametrize("n,distinct", [(0, False), (4, False), (4, True)])
@pytest.mark.parametrize("T", [1.0, 1.3])
def test_rows_of_drawn_logits(binding, dtype, n, distinct, T):  # noqa: F811
    """Logits of 8 bits, so that the border of every top-k here is a tie."""
    V = 32000
    x = (3 * torch.randn(V, generator=torch.Generator("cuda").manual_seed(21), device="cuda")).bfloat16()
    sorted_x = torch.sort(x.float(), descending=True).values
    assert all(bool(sorted_x[k - 1] == sorted_x[k]) for k, _, _ in DRAWN)
    _check(binding, x.to(dtype), [(T, *s) for s in DRAWN], n, distinct)


@pytest.mark.parametrize("dtype", CODE)
@pytest.mark.parametrize("n,distinct", [(0, False), (4, False), (4, True)])
def test_a_tie_larger_than_the_list(binding, dtype, n, distinct):  # noqa: F811
    """A few larger logits above 20000 equal ones, through which every top-k goes."""
    gen = torch.Generator("cuda").manual_seed(4)
    x = torch.full((30000,), -4.0, device="cuda")
    x[torch.randperm(30000, generator=gen, device="cuda")[:20000]] = -1.0
    x[torch.randperm(30000, generator=gen, device="cuda")[:25]] = 2.0
    _check(binding, x.to(dtype), [(1.0, *s) for s in DRAWN] + [(1.0, 50, 0.999, 0.0), (1.0, 26, 0.999, 0.0), (1.0, 15000, 0.999999, 0.0)], n, distinct)
