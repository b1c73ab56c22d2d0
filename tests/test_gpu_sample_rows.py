"""From logits to probability rows and tokens, against the plain 64-bit form: probabilities within the limit that is derived there, kept
tokens and drawn tokens exactly."""
import math

import pytest
import torch

import latent_reference as R

pytestmark = pytest.mark.gpu
CODE = {torch.float32: 0, torch.bfloat16: 1}
NEAREST_1 = 1 - 2.0 ** -24


@pytest.fixture(scope="module")
def binding():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2409_10644_amd import binding as b
    return b


def _settings(rows):
    """Per sequence (temperature, top_k, top_p, min_p) -> the device arrays, and the numbers as fp32 holds them."""
    t, k, p, m = zip(*rows)
    f = [torch.tensor(x, dtype=torch.float32) for x in (t, p, m)]
    numbers = list(zip(f[0].tolist(), k, f[1].tolist(), f[2].tolist()))
    return (f[0].cuda(), torch.tensor(k, dtype=torch.int32, device="cuda"), f[1].cuda(), f[2].cuda()), numbers


def run(binding, x, settings, us=None, distinct=False, probs=True, skew=0, pad=0):
    """x [B][W][V] (device); rows are laid `pad` elements apart and begin `skew` elements behind an aligned place."""
    B, W, V = x.shape
    arrays, numbers = _settings(settings)
    store = torch.full((skew + B * W * (V + pad) + 8,), math.nan, dtype=x.dtype, device="cuda")
    laid = store[skew:skew + B * W * (V + pad)].view(B, W, V + pad)
    laid[..., :V] = x
    n = 0 if us is None else us.shape[-1]
    out = torch.full((B * W * V + 3 + 8,), 7.0, device="cuda") if probs else None
    tokens = torch.full((B, W * n + 5), -9, dtype=torch.int32, device="cuda") if n else None
    binding.sample_rows(CODE[x.dtype], B, W, V, laid, W * (V + pad), V + pad, binding.make_sampler(*arrays), out[3:] if probs else None, W * V,
                        binding.MCSD_WITHOUT_REPLACEMENT if distinct else binding.MCSD_WITH_REPLACEMENT, n, us, tokens, W * n + 5)
    torch.cuda.synchronize()
    if probs:
        assert bool((out[:3] == 7).all()) and bool((out[3 + B * W * V:] == 7).all())
    if n:
        assert bool((tokens[:, W * n:] == -9).all())
    for b in range(B):
        for r in range(W):
            want, want_tokens = R.sample_row(x[b, r].cpu(), *numbers[b], us=[] if us is None else us[b, r].tolist(), distinct=distinct)
            if probs:
                R.check_probs(out[3:][(b * W + r) * V:(b * W + r + 1) * V], want)
            if n:
                assert tokens[b, r * n:(r + 1) * n].tolist() == want_tokens, (b, r, numbers[b])
    return None if not probs else out[3:3 + B * W * V], tokens


ALL = [(1.0, 0, 1.0, 0.0), (0.7, 50, 0.9, 0.02), (1.3, 0, 0.95, 0.0), (0.3, 7, 1.0, 0.0), (0.0, 5, 0.5, 0.5), (2.0, 0, 1.0, 0.2), (0.9, 1, 1.0, 0.0), (1.0, 10 ** 9, 0.3, 0.001)]


@pytest.mark.parametrize("dtype", CODE)
@pytest.mark.parametrize("V", [1, 9, 511, 4095, 4096, 4097, 33003, 262144])
@pytest.mark.parametrize("distinct", [None, False, True])
def test_more_rows_than_compute_units(binding, dtype, V, distinct):
    """Rows of a large batch go two to a compute unit; every row is what it is in a small one."""
    gen = torch.Generator("cuda").manual_seed(V + 1)
    B, W, n = len(ALL), 2, 0 if distinct is None else 5
    x, us = _logits(gen, B, W, V, dtype), torch.rand(B, W, n, generator=gen, device="cuda") if n else None
    p, tokens = run(binding, x, ALL, us, distinct)
    copies = torch.cuda.get_device_properties(0).multi_processor_count // (B * W) + 1
    arrays, _ = _settings(ALL)
    many = torch.empty(B * copies * W * V, device="cuda")
    many_tokens = torch.empty(B, copies * W * n, dtype=torch.int32, device="cuda") if n else None
    binding.sample_rows(CODE[dtype], B, copies * W, V, x.repeat(1, copies, 1), copies * W * V, V, binding.make_sampler(*arrays), many, copies * W * V,
                        binding.MCSD_WITHOUT_REPLACEMENT if distinct else binding.MCSD_WITH_REPLACEMENT, n, us.repeat(1, copies, 1) if n else None, many_tokens, copies * W * n)
    torch.cuda.synchronize()
    many = many.view(B, copies, W * V)
    # the copies alike, and off from the small call's by a step of 1 / sum (2^-23) and half a step of each product
    assert torch.equal(many, many[:, :1].expand_as(many))
    p = p.view(B, W * V)
    assert bool(((many[:, 0] - p).abs() <= 4 * 2.0 ** -24 * p + 2.0 ** -149).all()), (many[:, 0] - p).abs().max()
    if n:
        assert torch.equal(many_tokens.view(B, copies, W * n), tokens[:, :W * n].reshape(B, 1, W * n).expand(B, copies, W * n))


def _logits(gen, B, W, V, dtype, spread=3.0):
    x = spread * torch.randn(B, W, V, generator=gen, device="cuda")
    if V > 20:
        x[..., gen.initial_seed() % V] += 6
    return x.to(dtype)


@pytest.mark.parametrize("dtype", CODE)
@pytest.mark.parametrize("V", [1, 2, 7, 8, 511, 512, 513, 1000, 8191, 8192, 8193, 32000, 32769, 50257, 65537])
@pytest.mark.parametrize("distinct", [False, True])
def test_against_the_definition(binding, dtype, V, distinct):
    gen = torch.Generator("cuda").manual_seed(V)
    B, W, n = len(ALL), 2, 5
    us = torch.rand(B, W, n, generator=gen, device="cuda")
    us[0, 0, 0], us[0, 1, 0], us[1, 0, 1] = 0, NEAREST_1, NEAREST_1
    run(binding, _logits(gen, B, W, V, dtype), ALL, us, distinct, skew=V % 3, pad=V % 2)


@pytest.mark.parametrize("dtype", CODE)
@pytest.mark.parametrize("V", [131077, 262144])
def test_large_vocabularies(binding, dtype, V):
    gen = torch.Generator("cuda").manual_seed(V)
    us = torch.rand(len(ALL), 1, 4, generator=gen, device="cuda")
    run(binding, _logits(gen, len(ALL), 1, V, dtype), ALL, us, True, skew=1)


@pytest.mark.parametrize("dtype", CODE)
@pytest.mark.parametrize("kinds", ["one", "two", "few", "ties at the cut"])
def test_equal_logits(binding, dtype, kinds):
    """Many tokens with the same logit: the lowest indices are kept, however many more there are."""
    gen = torch.Generator("cuda").manual_seed(5)
    V = 20000
    x = {"one": torch.full((V,), 1.5, device="cuda"), "two": torch.randint(0, 2, (V,), generator=gen, device="cuda").float() - 0.5,
         "few": torch.randint(-4, 5, (V,), generator=gen, device="cuda") / 4, "ties at the cut": torch.where(torch.arange(V, device="cuda") % 3 == 0, 2.0, -3.0)}[kinds]
    x[17] = x[19] = x[400] = 0.0
    x[18] = -0.0                                              # (the same number as 0)
    settings = [(1.0, 3000, 1.0, 0.0), (1.0, 0, 0.37, 0.0), (0.5, 9999, 0.8, 0.0), (1.0, 1, 1.0, 0.0), (0.0, 0, 1.0, 0.0), (1.0, 0, 1.0, 1.0), (1.0, 0, 0.0, 0.0), (1.0, 0, 1.0, 2.0)]
    B = len(settings)
    us = torch.rand(B, 1, 6, generator=gen, device="cuda")
    for distinct in (False, True):
        run(binding, x.to(dtype).expand(B, 1, V).contiguous(), settings, us, distinct)


@pytest.mark.parametrize("dtype", CODE)
def test_masked_logits(binding, dtype):
    """Tokens masked with minus infinity or the type's lowest number; rows of one candidate, and of none."""
    gen = torch.Generator("cuda").manual_seed(6)
    V, B = 5000, len(ALL)
    low = torch.finfo(dtype).min
    for mask in (-math.inf, low):
        x = _logits(gen, B, 4, V, dtype)
        x[:, 0, 100:] = mask
        x[:, 1, :4999] = mask
        x[:, 2, torch.randperm(V, generator=gen, device="cuda")[:4000]] = mask
        x[:, 3] = mask
        run(binding, x, ALL, torch.rand(B, 4, 4, generator=gen, device="cuda"), True)
        run(binding, x, ALL, torch.rand(B, 4, 4, generator=gen, device="cuda"), False)


def test_the_largest_numbers(binding):
    """Logits that span fp32, the coldest and hottest temperatures."""
    V = 600
    big = torch.finfo(torch.float32).max
    x = torch.linspace(-1, 1, V, device="cuda").mul(big).repeat(8, 1, 1)
    x[4:] = torch.linspace(-1, 1, V, device="cuda")
    settings = [(1.0, 0, 0.9, 0.0), (1e38, 0, 0.9, 0.0), (math.inf, 0, 0.9, 0.0), (1e38, 5, 1.0, 0.1), (1e-40, 0, 0.9, 0.0), (1e-3, 0, 0.9, 0.0), (math.inf, 20, 1.0, 0.0), (1e-45, 30, 1.0, 0.0)]
    us = torch.rand(8, 1, 3, generator=torch.Generator("cuda").manual_seed(1), device="cuda")
    for distinct in (False, True):
        run(binding, x, settings, us, distinct)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_rows_that_are_no_distribution(binding, bad):
    gen = torch.Generator("cuda").manual_seed(8)
    x = _logits(gen, 3, 3, 3000, torch.float32)
    x[0, 1, 2999] = bad
    x[2, 0, 0] = bad
    run(binding, x, [(1.0, 0, 1.0, 0.0), (0.5, 50, 0.9, 0.0), (0.0, 0, 1.0, 0.0)], torch.rand(3, 3, 2, generator=gen, device="cuda"))


@pytest.mark.parametrize("settings", [(math.nan, 0, 1.0, 0.0), (-1.0, 0, 1.0, 0.0), (1.0, 0, math.nan, 0.0), (1.0, 0, 1.0, math.nan)])
def test_settings_that_are_no_numbers(binding, settings):
    x = _logits(torch.Generator("cuda").manual_seed(8), 2, 1, 100, torch.float32)
    run(binding, x, [settings, (1.0, 5, 0.9, 0.0)], torch.rand(2, 1, 3, device="cuda"))


def test_uniform_numbers_are_kept_within_the_interval(binding):
    x = _logits(torch.Generator("cuda").manual_seed(8), 1, 1, 1000, torch.float32)
    run(binding, x, [(1.0, 0, 1.0, 0.0)], torch.tensor([[[0.0, -1.0, math.nan, 1.0, 2.0, NEAREST_1, 1e-45, 2.0 ** -30]]], device="cuda"))


def test_distinct_draws_use_up_a_row(binding):
    """As many draws as a call takes, from rows of fewer kept tokens, and of tokens that weigh very differently."""
    gen = torch.Generator("cuda").manual_seed(11)
    x = torch.randn(4, 2, 900, generator=gen, device="cuda") * 5
    x[1] = -100 * torch.arange(900, device="cuda")            # each e^100 times less than the one before
    run(binding, x, [(1.0, 40, 1.0, 0.0), (1.0, 64, 1.0, 0.0), (0.2, 0, 0.9, 0.0), (1.0, 0, 1.0, 0.0)], torch.rand(4, 2, 64, generator=gen, device="cuda"), True)


@pytest.mark.parametrize("n", [1, 16, 17, 64])
def test_many_independent_draws(binding, n):
    gen = torch.Generator("cuda").manual_seed(n)
    x = _logits(gen, 2, 2, 32000, torch.bfloat16)
    run(binding, x, [(1.0, 0, 1.0, 0.0), (0.8, 0, 0.9, 0.0)], torch.rand(2, 2, n, generator=gen, device="cuda"), probs=False)


def test_shares_of_the_draws(binding):
    """A uniform number per place of a fine grid: every token is drawn for its share of the grid, to within two places."""
    x = torch.tensor([0.0, 1.0, -1.0, 2.0, -math.inf, 0.5], device="cuda").view(1, 1, 6)
    grid = torch.arange(64 * 100, device="cuda").add(0.5).div(6400).view(100, 1, 64)
    tokens = torch.zeros(100, 64, dtype=torch.int32, device="cuda")
    binding.sample_rows(0, 100, 1, 6, x, 0, 6, binding.make_sampler(), None, 0, 0, 64, grid, tokens, 64)          # (one row for all: a stride of zero is read)
    p = torch.softmax(x.double().flatten(), 0).cpu()
    counts = torch.bincount(tokens.flatten().cpu(), minlength=6)
    assert bool(((counts - 6400 * p).abs() <= 2).all())


def test_streams_and_graphs(binding):
    gen = torch.Generator("cuda").manual_seed(4)
    B, W, V, n = 3, 4, 32000, 4
    x = _logits(gen, B, W, V, torch.bfloat16)
    u = torch.rand(B, W, n, generator=gen, device="cuda")
    arrays, _ = _settings([(0.7, 50, 0.9, 0.0), (1.0, 0, 0.95, 0.0), (0.0, 0, 1.0, 0.0)])
    sampler = binding.make_sampler(*arrays)
    probs, tokens = torch.zeros(B, W, V, device="cuda"), torch.zeros(B, W, n, dtype=torch.int32, device="cuda")

    def call(stream=None):
        binding.sample_rows(1, B, W, V, x, W * V, V, sampler, probs, W * V, 1, n, u, tokens, W * n, stream)

    def result():
        torch.cuda.synchronize()
        r = probs.clone(), tokens.clone()
        probs.fill_(-1)
        tokens.fill_(-7)
        return r

    call()
    want = result()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call(side)
    assert all(torch.equal(a, b) for a, b in zip(result(), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    keep = x.clone()
    for i in range(3):
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(result(), want))
        x.copy_(keep.roll(i + 1, -1))                          # other logits between the replays
        call()
        eager = result()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(result(), eager))
        x.copy_(keep)
