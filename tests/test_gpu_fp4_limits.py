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
