"""Tree attention over a latent cache against the plain 64-bit form."""
import math

import pytest
import torch

import latent_reference as R

pytestmark = pytest.mark.gpu
SIZES = [(512, 64), (256, 32)]


@pytest.fixture(scope="module")
def binding():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2409_10644_amd import binding as b
    return b


class Call:
    """Inputs of one call; cache rows behind a sequence's end, input rows behind the tree and below the first row are NaN."""

    def __init__(self, binding, branching, H, dl, dr, lens, newest=False, max_prefix=None, extra=2, gap=0, seed=0, levels=None, gain=1.0):
        self.binding, d, B = binding, dl + dr, len(lens)
        self.sizes = (B, H, dl, dr)
        gen = torch.Generator("cuda").manual_seed(seed + 7 * H + dl)
        level, _ = R.tree_of(branching)
        n = self.n = len(level)
        self.row0 = level.index(level[-1]) if newest else 0
        self.ns = n + extra
        self.view = binding.slice_mask(binding.build_mask(tuple(branching) + ((2,) if levels is None else ())), len(branching))
        self.L = [min(max(x, 0), max_prefix if max_prefix is not None else 1 << 30) for x in lens]
        self.max_prefix = max(self.L) if max_prefix is None else max_prefix
        cap = max(self.L) + 3
        self.q = torch.randn(B, H, self.ns, d, generator=gen, device="cuda").mul(gain).bfloat16()
        self.q[:, :, n:] = self.q[:, :, :self.row0] = math.nan
        self.tree = torch.randn(B, self.ns, d, generator=gen, device="cuda").bfloat16()
        self.tree[:, n:] = math.nan
        self.cache = torch.randn(B * (cap * d + gap), generator=gen, device="cuda").bfloat16()
        self.base = torch.arange(B, device="cuda", dtype=torch.int64).flip(0) * (cap * d + gap)      # (the last sequence first)
        self.past = [self.cache[int(s):int(s) + l * d].view(l, d) for s, l in zip(self.base.tolist(), self.L)]
        for s, l in zip(self.base.tolist(), self.L):
            self.cache[s + l * d:s + cap * d + gap] = math.nan
        self.lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.scale = 1 / math.sqrt(d)
        self.seen = R.visible(branching, "cuda")
        self.out = torch.full((B, H, self.ns, dl), 9.0, dtype=torch.bfloat16, device="cuda")
        size = binding.tree_attention_latent_workspace(B, H, dl, dr, n, self.row0, self.max_prefix)
        self.ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda") if size else None      # (it needs no preparation)

    def call(self, stream=None):
        self.binding.tree_attention_latent(self.view, *self.sizes, self.row0, self.q, self.tree, self.ns, self.cache, self.base, self.lens, self.max_prefix,
                                           self.scale, self.out, self.ws, stream)

    def compare(self):
        B, H, dl, _ = self.sizes
        n, row0 = self.n, self.row0
        assert bool((self.out[:, :, :row0] == 9).all()) and bool((self.out[:, :, n:] == 9).all()), "rows that are not the call's were written"
        for b in range(B):
            want, lim = R.attention(self.q[b, :, row0:n], self.tree[b, :n], self.past[b], self.seen[row0:], self.scale, dl)
            err = (self.out[b, :, row0:n].double() - want).abs()
            assert bool((err <= lim).all()), f"sequence {b}: worst {float((err / lim).max()):.2f} of the limit, {int((~(err <= lim)).sum())} of {err.numel()}"

    def check(self):
        self.call()
        torch.cuda.synchronize()
        self.compare()
        return self.out.clone()


@pytest.mark.parametrize("dl,dr", SIZES)
@pytest.mark.parametrize("branching,H,newest", [((1,), 1, False), ((1,), 16, False), ((2, 2, 2), 5, False), ((16, 1, 1), 12, True), ((4, 2, 2, 1), 16, False), ((8, 2, 2, 1, 1), 3, False),
                                                ((64, 1), 2, False), ((64, 1), 3, True), ((5, 13), 7, False)])
@pytest.mark.parametrize("lens", [(0,), (1,), (63, 64, 65), (128, 0, 1000, 7)])
def test_against_the_definition(binding, dl, dr, branching, H, newest, lens):
    Call(binding, branching, H, dl, dr, lens, newest).check()


@pytest.mark.parametrize("dl,dr", SIZES)
@pytest.mark.parametrize("branching,H,lens", [((1,), 4, (20000,)),                                     # one chunk, cut into many pieces
                                              ((4, 2, 2, 2), 16, tuple(range(100, 1700, 100))),         # pieces that cross chunks and sequences
                                              ((4, 2, 2, 1), 128, (1024,)),                             # several pieces of each chunk
                                              ((1,), 16, tuple((37 * i) % 700 for i in range(130))),    # more than 64 sequences
                                              ((2,), 3, tuple((11 * i) % 90 for i in range(300))),      # more sequences than workgroups
                                              ((8, 2, 2, 1, 1), 64, (700, 3, 65))])
def test_shared_work(binding, dl, dr, branching, H, lens):
    first = (c := Call(binding, branching, H, dl, dr, lens)).check()
    for _ in range(2):                                       # and the same bits again
        c.out.fill_(9)
        c.call()
        torch.cuda.synchronize()
        assert torch.equal(c.out, first)


def test_all_heads_of_a_large_model(binding):
    Call(binding, (3, 2), 128, 512, 64, (777, 2000, 31)).check()


@pytest.mark.parametrize("dl,dr", SIZES)
def test_lengths_are_clamped(binding, dl, dr):
    Call(binding, (2, 2), 4, dl, dr, (50, -3, 500, 200), max_prefix=130).check()


@pytest.mark.parametrize("dl,dr", SIZES)
def test_sequences_anywhere_in_the_cache(binding, dl, dr):
    Call(binding, (2, 2), 4, dl, dr, (50, 300, 200), gap=8 * 37, extra=5).check()


@pytest.mark.parametrize("dl,dr", SIZES)
def test_references_that_are_outgrown(binding, dl, dr):
    """Scores grow along the keys, so that the running maximum is passed again and again, in one wavefront's keys or another's."""
    c = Call(binding, (2, 2), 16, dl, dr, (1500, 100), gain=4.0)
    for b, past in enumerate(c.past):
        past.mul_((torch.arange(past.shape[0], device="cuda") / past.shape[0] * 2 + 0.01)[:, None])
    c.check()


def test_no_prefix_and_no_cache(binding):
    c = Call(binding, (4, 2, 2, 1), 16, 512, 64, (0, 0))
    c.cache = None
    assert c.ws is None
    c.check()


def test_offsets_beyond_32_bits(binding):
    """The last sequence begins behind 2^31 elements of the cache, and one row of queries behind 2^31 bytes."""
    c = Call(binding, (2, 1), 16, 512, 64, (100, 900))
    d = 576
    far = torch.empty(2 ** 31 + 2000 * d, dtype=torch.bfloat16, device="cuda")
    start = (2 ** 31 // 8 + 5) * 8
    for b, at in ((0, 8), (1, start)):
        far[at:at + c.L[b] * d] = c.past[b].flatten()
        far[at + c.L[b] * d:at + (c.L[b] + 64) * d] = math.nan
    c.cache, c.base = far, torch.tensor([8, start], device="cuda")
    c.check()
    wide = Call(binding, (1,), 2, 512, 64, (70, 5), extra=2 ** 21)         # (rows far apart: 2.4 GB between two heads)
    wide.check()


@pytest.mark.parametrize("where", ["prefix", "tree"])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_values_that_are_not_finite(binding, where, value):
    """A key that a row sees makes that row's output NaN or infinite; other sequences keep theirs.  (A row of the tree that a node does not
    see has weight zero, and zero times infinity is NaN: trees hold finite rows.)"""
    c = Call(binding, (3, 2), 16, 512, 64, (130, 100))
    want = c.check()
    (c.past[0] if where == "prefix" else c.tree[0])[-1 if where == "prefix" else 0, 5] = value
    c.out.fill_(9)
    c.call()
    torch.cuda.synchronize()
    assert torch.equal(c.out[1], want[1])
    assert not bool(torch.isfinite(c.out[0, :, :c.n, 5].float()).any()) if where == "prefix" else not bool(torch.isfinite(c.out[0, :, 0, 5].float()).any())


def test_streams_graphs_and_a_shared_workspace(binding):
    a, b = Call(binding, (4, 2, 2, 1), 16, 512, 64, (1200, 333), seed=1), Call(binding, (1,), 16, 512, 64, (4000, 5, 1000, 2), seed=2)
    want_a, want_b = a.check(), b.check()
    a.ws = b.ws = max(a.ws, b.ws, key=lambda t: t.numel())

    def both():
        a.call()
        b.call()

    def checked():
        torch.cuda.synchronize()
        assert torch.equal(a.out, want_a) and torch.equal(b.out, want_b)
        a.out.fill_(9)
        b.out.fill_(9)

    both()
    checked()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a.call(side)
    b.call(side)
    checked()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g, f in zip(graphs, (both, b.call)):
        with torch.cuda.graph(g):
            f()
    a.out.fill_(9)
    b.out.fill_(9)
    for _ in range(3):
        graphs[0].replay()
        checked()
        a.call()
        graphs[1].replay()
        checked()


def test_a_workspace_of_another_attention_call(binding):
    """The head of a prepared workspace stays as it is: calls of both kinds take turns on one."""
    c = Call(binding, (1,), 16, 512, 64, (4000, 5))
    want = c.check()
    H, d, L, n = 8, 128, 2000, c.n
    gen = torch.Generator("cuda").manual_seed(3)
    q, kt, vt = (torch.randn(1, H, n, d, generator=gen, device="cuda").bfloat16() for _ in range(3))
    kp, vp = (torch.randn(1, H, L, d, generator=gen, device="cuda").bfloat16() for _ in range(2))
    base, lens, out = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.tensor([L], dtype=torch.int32, device="cuda"), torch.zeros_like(q)
    size = binding.tree_attention_workspace(1, H, d, n, L)
    assert size > 0
    c.ws = ws = binding.new_workspace(max(size, c.ws.numel()))
    outs = []
    for _ in range(3):
        binding.tree_attention(c.view, 1, 1, H, d, q, kt, vt, n, kp, vp, base, lens, L * d, L, 0.1, out, ws)
        c.out.fill_(9)
        c.call()
        torch.cuda.synchronize()
        outs.append(out.clone())
        assert torch.equal(c.out, want)
    assert not bool(torch.isnan(outs[0]).any()) and all(torch.equal(o, outs[0]) for o in outs)


def test_a_workspace_serves_smaller_calls(binding):
    big = Call(binding, (4, 2, 2, 1), 16, 512, 64, (1500, 900, 30))
    for branching, lens, newest in (((1,), (1500, 3, 9), False), ((4, 2, 2, 1), (1000, 1000, 1000), True), ((2, 2), (1499, 64, 0), False)):
        c = Call(binding, branching, 16, 512, 64, lens, newest)
        assert c.ws is None or c.ws.numel() <= big.ws.numel()
        c.ws = big.ws
        c.check()
