"""One workspace, prepared once, for the attention over a 4-bit cache and over the same numbers in bf16, in turn on one stream and in one
graph: both leave it as they found it, and give the bits they give with workspaces of their own."""
import pytest
import torch

import fp4_reference as R
from test_gpu_fp4_attention import Call, binding  # noqa: F401  (binding: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("branching,Hq,Hkv,lens", [((4, 2, 2, 1), 8, 8, (1200, 333)), ((1,), 8, 2, (4000, 5, 1000, 2)), ((8, 2, 2, 1, 1), 4, 4, (2500,)), ((3, 2), 2, 1, (6000,))])
def test_two_formats_share_a_workspace(binding, branching, Hq, Hkv, lens):  # noqa: F811
    d, B = 128, len(lens)
    c = Call(binding, branching, B, Hq, Hkv, d, lens, seed=len(branching))
    kp, vp = (R.decode(c.cache.arrays[i], c.cache.arrays[i + 1]).bfloat16() for i in (0, 2))       # (offsets are in channels in both)
    assert torch.equal(kp.double(), R.decode(c.cache.arrays[0], c.cache.arrays[1]))
    other = torch.zeros_like(c.out)
    size = binding.tree_attention_gqa_workspace(B, Hq, Hkv, d, c.n, 0, c.max_prefix)
    assert size > 0 and c.ws is not None                   # (both cut their keys)

    def plain(ws):
        binding.tree_attention_gqa(c.view, 1, B, Hq, Hkv, d, 0, c.q, c.kt, c.vt, c.ns, kp, vp, c.cache.base, c.lens_dev, c.cache.head_stride, c.max_prefix, c.scale, other, ws)

    want = c.check()
    plain(binding.new_workspace(size))
    torch.cuda.synchronize()
    want_other = other.clone()
    assert not bool(torch.isnan(want_other[:, :, :c.n]).any())
    shared = c.ws = binding.new_workspace(max(size, c.ws.numel()))

    def both():
        c.call()
        plain(shared)
        c.call()

    def checked():
        torch.cuda.synchronize()
        assert torch.equal(c.out, want) and torch.equal(other, want_other)
        c.out.fill_(31)
        other.zero_()

    for _ in range(3):
        both()
        checked()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    checked()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(3):
        graph.replay()
        checked()
        both()                                             # eager work between the replays
        checked()
