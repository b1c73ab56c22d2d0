"""The largest bounds that the entry points around the 4-bit cache document, with few rows that exist: the launch is as large as it
gets, and all but a few of its workgroups find nothing to do."""
import pytest
import torch

import fp4_reference as R
from fp4_reference import Cache

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
