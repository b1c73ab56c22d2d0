"""Norm and rotation of vectors whose squares fp32 does not hold, in the largest and the smallest numbers of either type; tolerance as in
test_gpu_qk_rope: fewer than 32 roundings of fp32 and the output's."""
import numpy as np
import pytest
import torch

import fp4_reference as R

pytestmark = pytest.mark.gpu
CODE = {torch.float32: 0, torch.bfloat16: 1}


@pytest.fixture(scope="module")
def binding():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2409_10644_amd import binding as b
    return b


@pytest.mark.parametrize("dtype", CODE)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("eps", [0.0, 1e-6, 1e-36])
@pytest.mark.parametrize("rows", [12, 3000])
def test_vectors_of_any_size(binding, dtype, d, eps, rows):
    """Rows of different sizes side by side, so that neighbouring lanes take different ways; enough rows for four to a workgroup."""
    gen = torch.Generator("cuda").manual_seed(d)
    size = torch.tensor([2.0 ** e for e in (0, 60, 64, 100, 124, -20, -50, -60, -64, -70, -100, -112)], device="cuda").repeat(rows // 12)
    x = torch.randn(1, rows, 2 * d, generator=gen, device="cuda") * size[None, :, None]
    x[0, 1::12, 5::d] *= 2.0 ** 60                         # one number far above the others, one far below
    x[0, 2::12, 7::d] *= 2.0 ** -100
    x[0, 8::12, 9::d] *= 2.0 ** -40
    x = x.to(dtype)
    assert bool(torch.isfinite(x).all())
    q, k = x.split(d, -1)
    wq, wk = (1 + 0.2 * torch.randn(2, d, generator=gen, device="cuda")).unbind(0)
    inv = (10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)).float().cuda()
    rope = binding.make_rope(d, inv, wq, wk, eps)
    qo, ko = (torch.zeros(1, 1, rows, d, dtype=dtype, device="cuda") for _ in range(2))
    i32 = lambda a: torch.tensor([a], dtype=torch.int32, device="cuda")
    binding.prompt_qk_norm_rope(CODE[dtype], 1, 1, 1, d, rows, q, k, None, 0, 2 * d, 0, 2 * d, rope, i32(7), i32(rows), qo, ko, None, rows)
    torch.cuda.synchronize()
    pos = 7 + torch.arange(rows, device="cuda")
    for src, w, out in ((q, wq, qo), (k, wk, ko)):
        want, parts = R.rotated(src[0].double(), w.double(), float(np.float32(eps)), pos, inv, d, False)
        got = out[0, 0].double()
        # (and below fp32's normal numbers, of which 2^-149 is the step, what the products round to)
        lim = torch.finfo(dtype).eps / 2 * want.abs() + 32 * 2.0 ** -24 * parts + 4 * 2.0 ** -149 + (2.0 ** -134 if dtype == torch.bfloat16 else 0)
        err = (got - want).abs()
        assert bool((err <= lim).all()), [(float(size[t]), float((err - lim)[t].max())) for t in range(12) if not bool((err <= lim)[t].all())]
