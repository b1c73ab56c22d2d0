"""Tree attention over a prefix cache in 4 bits against the plain 64-bit form on the numbers that the cache stands for; tolerances
as fp4_reference.attention_row_terms derives them."""
import math

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


class Call:
    """One call's tensors: random queries and tree rows, a cache filled with quantised normals (or `fill`'s codes and scales)."""

    def __init__(self, binding, branching, B, Hq, Hkv, d, lens, seed=0, levels=None, newest=False, gap=8, extra_nodes=2, mult=1.0, cap=None, max_prefix=None):
        self.b, self.B, self.Hq, self.Hkv, self.d = binding, B, Hq, Hkv, d
        gen = self.gen = torch.Generator("cuda").manual_seed(seed)
        levels = len(branching) if levels is None else levels
        self.view = binding.slice_mask(binding.build_mask(branching), levels)
        level, _ = R.tree_of(branching[:levels])
        self.n = len(level)
        self.row0 = level.index(levels) if newest else 0
        self.seen = R.visible(branching[:levels], "cuda")
        self.ns = self.n + extra_nodes
        rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda")
        self.q = (rnd(B, Hq, self.ns, d) * mult).bfloat16()
        self.kt, self.vt = rnd(B, Hkv, self.ns, d).bfloat16(), rnd(B, Hkv, self.ns, d).bfloat16()
        self.lens = list(lens)
        self.max_prefix = max(max(lens), 0) if max_prefix is None else max_prefix
        cap = max(self.max_prefix, 1) if cap is None else cap
        cap += cap % 2
        self.cache = Cache(binding, B, Hkv, cap, d, gap=gap, fill=0)
        for i in (0, 2):
            codes, scales = R.quantise(rnd(self.cache.arrays[i].shape[0], d) * torch.exp(0.5 * rnd(1, d)))
            self.cache.arrays[i].copy_(codes)
            self.cache.arrays[i + 1].copy_(scales)
        self.scale = 1.0 / math.sqrt(d)
        self.out = torch.full((B, Hq, self.ns, d), 31.0, dtype=torch.bfloat16, device="cuda")
        self.workspace()

    def workspace(self):
        size = self.b.tree_attention_fp4kv_workspace(self.B, self.Hq, self.Hkv, self.d, self.n, self.row0, self.max_prefix)
        self.ws = self.b.new_workspace(size) if size else None

    def run(self, stream=None):
        self.lens_dev = torch.tensor(self.lens, dtype=torch.int32, device="cuda")
        self.call(stream)
        torch.cuda.synchronize()
        return self.out

    def call(self, stream=None):
        self.b.tree_attention_fp4kv(self.view, self.B, self.Hq, self.Hkv, self.d, self.row0, self.q, self.kt, self.vt, self.ns, self.cache.handle,
                                    self.cache.base, self.lens_dev, self.cache.head_stride, self.max_prefix, self.scale, self.out, self.ws, stream)

    def wanted(self, b, h):
        L = min(max(self.lens[b], 0), self.max_prefix)
        g = h // (self.Hq // self.Hkv)
        k, v = (torch.cat((R.decode(self.cache.view(i)[b, g, :L], self.cache.view(i + 1)[b, g, :L]), t[b, g, :self.n].double())) for i, t in ((0, self.kt), (2, self.vt)))
        seen = torch.cat((torch.ones(self.n, L, dtype=torch.bool, device="cuda"), self.seen), 1)[self.row0:]
        return R.attention_row_terms(self.q[b, h, self.row0:self.n].double(), k, v, seen, self.scale)

    def check(self, pairs=None):
        out = self.run()
        for b in range(self.B):
            for h in range(self.Hq):
                if pairs is not None and (b, h) not in pairs:
                    continue
                want, lim = self.wanted(b, h)
                got = out[b, h, self.row0:self.n].double()
                assert bool(torch.isfinite(got).all()), (b, h)
                err = (got - want).abs()
                assert bool((err <= lim).all()), f"sequence {b} head {h} length {self.lens[b]}: worst {float((err - lim).max()):.3e} over, {int((err > lim).sum())} of {err.numel()}"
        assert bool((out[:, :, :self.row0] == 31).all()) and bool((out[:, :, self.n:] == 31).all())
        return out.clone()


TREES = {"one": (1,), "pair": (2,), "nine": (3, 2), "chain": (1,) * 5, "44": (4, 2, 2, 1), "120": (8, 2, 2, 1, 1), "128": (64, 1)}


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("tree", TREES)
@pytest.mark.parametrize("L", [0, 1, 31, 32, 33, 63, 64, 65, 127, 128, 129, 192, 300, 1000, 2049])
def test_prefix_lengths_around_tiles(binding, d, tree, L):
    Call(binding, TREES[tree], 1, 2, 2, d, (L,), seed=L).check()


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (8, 2), (6, 2), (5, 1), (32, 1), (7, 7)])
@pytest.mark.parametrize("tree,newest", [("one", False), ("nine", True), ("44", False), ("44", True), ("120", False), ("128", True)])
def test_heads_that_share_keys(binding, d, Hq, Hkv, tree, newest):
    Call(binding, TREES[tree], 2, Hq, Hkv, d, (150, 37), seed=Hq, newest=newest).check()


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("B,Hq,Hkv,tree,lo,hi", [(16, 8, 8, "44", 0, 900), (5, 4, 4, "120", 1, 700), (64, 4, 1, "one", 0, 1500), (33, 16, 16, "nine", 0, 300), (3, 32, 8, "44", 1000, 4000),
                                                 (70, 2, 2, "one", 0, 3000), (130, 1, 1, "pair", 0, 64)])
def test_ragged_batches(binding, d, B, Hq, Hkv, tree, lo, hi):
    gen = torch.Generator().manual_seed(B + d)
    lens = torch.randint(lo, hi + 1, (B,), generator=gen).tolist()
    lens[0], lens[-1] = lo, hi
    c = Call(binding, TREES[tree], B, Hq, Hkv, d, lens, seed=B)
    pairs = None if B * Hq <= 130 else {(b, h) for b in range(B) for h in ((b * 7) % Hq, (b * 3 + 1) % Hq)}
    first = c.check(pairs)
    c.out.fill_(31)
    assert torch.equal(c.run(), first)                     # the same call gives the same bits


@pytest.mark.parametrize("B,Hq,Hkv,d,tree,lo,hi", [(64, 32, 32, 64, "one", 0, 700), (20, 32, 32, 128, "44", 0, 900), (48, 24, 12, 128, "120", 1, 400), (61, 40, 40, 64, "nine", 0, 200),
                                                     (64, 9, 9, 128, "one", 7, 7), (40, 26, 13, 64, "120", 0, 1500),
                                                     (100, 16, 8, 128, "one", 0, 1200), (256, 6, 6, 64, "nine", 0, 150), (300, 8, 2, 64, "one", 0, 500), (257, 1, 1, 128, "44", 100, 130)])
def test_more_pairs_than_workgroups(binding, B, Hq, Hkv, d, tree, lo, hi):
    """Several whole pairs to a workgroup, or pieces that cross them: every pair is written, a sample of them compared."""
    gen = torch.Generator().manual_seed(B * d)
    lens = torch.randint(lo, hi + 1, (B,), generator=gen).tolist()
    lens[1], lens[-1] = lo, hi
    c = Call(binding, TREES[tree], B, Hq, Hkv, d, lens, seed=B)
    pairs = {(int(b), int(h)) for b, h in zip(torch.randint(0, B, (40,), generator=gen), torch.randint(0, Hq, (40,), generator=gen))}
    out = c.check(pairs | {(0, 0), (1, Hq - 1), (B - 1, 0), (B - 1, Hq - 1)})
    assert bool(torch.isfinite(out[:, :, :c.n].float()).all()) and not bool((out[:, :, :c.n] == 31).all(-1).any())
    again = c.run()
    assert torch.equal(out, again)


def test_a_serving_batch_of_conversations(binding):
    lens = [512 + (3584 * i) // 15 for i in range(16)][::-1]
    Call(binding, (4, 2, 2, 2), 16, 32, 8, 128, lens, seed=4).check({(b, h) for b in range(16) for h in (b, 31 - b)})


def test_long_documents_under_the_widest_tree(binding):
    Call(binding, TREES["120"], 2, 4, 4, 128, (16384, 16001), seed=5).check()


@pytest.mark.parametrize("tree", ["one", "44", "120"])
def test_a_very_long_prefix(binding, tree):
    Call(binding, TREES[tree], 1, 2, 1, 128, (131072 + 77,), seed=6).check()


def test_lengths_beyond_the_bound_and_below_zero_are_clamped(binding):
    Call(binding, TREES["44"], 4, 2, 2, 128, (5000, -3, 400, 401), seed=7, cap=500, max_prefix=400).check()


def test_a_slice_of_a_larger_mask_and_a_larger_workspace(binding):
    c = Call(binding, (4, 2, 2, 1), 2, 4, 4, 128, (700, 90), seed=8, levels=2)
    c.ws = binding.new_workspace(max(binding.tree_attention_fp4kv_workspace(2, 4, 4, 128, 44, 0, 5000), 1))
    first = c.check()
    c.out.fill_(31)
    c.ws = binding.new_workspace(64 * 1024 * 1024)
    assert torch.equal(c.run(), first)


def test_masks_of_more_words_than_the_slice_needs(binding):
    Call(binding, (4, 8, 8), 1, 2, 2, 64, (100,), seed=9, levels=2).check()                 # 292 nodes in the full mask, 36 in use


@pytest.mark.parametrize("mult", [8.0, 60.0, 1e-3])
def test_sharp_and_flat_distributions(binding, mult):
    Call(binding, TREES["44"], 2, 2, 2, 128, (777, 64), seed=10, mult=mult).check()


def test_scores_that_grow_along_the_prefix(binding):
    """Every tile brings a larger maximum than the one before: the running reference moves all the time."""
    c = Call(binding, TREES["44"], 1, 2, 2, 128, (1500,), seed=11)
    c.q[:] = c.q.abs() + 1
    k = torch.linspace(0.01, 4.0, c.cache.cap, device="cuda")[:, None].expand(-1, 128)
    codes, scales = R.quantise(k)
    for a, new in ((c.cache.arrays[0], codes), (c.cache.arrays[1], scales)):
        a.reshape(1, 2, -1, a.shape[-1])[:, :, :c.cache.cap] = new
    c.check()
    c.cache.arrays[0].copy_(c.cache.arrays[0].reshape(2, -1, 64).flip(1).reshape(c.cache.arrays[0].shape))
    c.cache.arrays[1].copy_(c.cache.arrays[1].reshape(2, -1, 4).flip(1).reshape(c.cache.arrays[1].shape))
    c.check()


def test_every_code_and_many_scales(binding):
    c = Call(binding, TREES["44"], 1, 2, 2, 128, (600,), seed=12)
    gen = torch.Generator("cuda").manual_seed(5)
    for i in (0, 2):
        c.cache.arrays[i].copy_(torch.randint(0, 256, c.cache.arrays[i].shape, generator=gen, device="cuda", dtype=torch.uint8))
        c.cache.arrays[i + 1].copy_(torch.randint(118, 127, c.cache.arrays[i + 1].shape, generator=gen, device="cuda", dtype=torch.uint8))
    c.check()


def test_scale_bytes_at_the_ends(binding):
    """Byte 0 is 2^-127, nothing beside the others; byte 254 in a value makes its channels large but finite in bf16 where codes allow."""
    c = Call(binding, TREES["nine"], 1, 1, 1, 128, (200,), seed=13)
    c.cache.arrays[1].reshape(-1, 4)[5:60, 1] = 0
    c.cache.arrays[3].reshape(-1, 4)[50:90, 2] = 0
    c.cache.arrays[3].reshape(-1, 4)[:, 3] = 230
    c.check()


@pytest.mark.parametrize("d", [128, 64])
def test_nan_in_the_cache_reaches_the_rows_that_see_it(binding, d):
    c = Call(binding, TREES["44"], 3, 2, 2, d, (300, 300, 300), seed=14)
    scales = [c.cache.arrays[i].reshape(3, 2, -1, d // 32) for i in (1, 3)]                 # (sequences in reverse order)
    scales[0][1, 0, 77, 1] = 255                           # sequence 1, head 0: a key that every row sees
    scales[1][0, 1, 200, 0] = 255                          # sequence 2, head 1: the first 32 channels of a value
    scales[0][2, :, 300:] = 255                            # sequence 0: rows behind its length
    scales[1][2, :, 300:] = 255
    out = c.run()[:, :, :c.n]
    assert bool(torch.isnan(out[1, 0]).all())
    assert bool(torch.isnan(out[2, 1, :, :32]).all())
    for b, h, cols in ((0, 0, slice(None)), (0, 1, slice(None)), (1, 1, slice(None)), (2, 0, slice(None)), (2, 1, slice(32, None))):
        want, lim = c.wanted(b, h)
        err = (out[b, h].double() - want).abs()[:, cols]
        assert bool((err <= lim[:, cols]).all()), (b, h)


def test_nan_and_infinity_in_tree_rows_stay_where_they_are_seen(binding):
    c = Call(binding, TREES["44"], 1, 2, 2, 128, (130,), seed=15)
    level, parent = R.tree_of((4, 2, 2, 1))
    node = 17
    c.kt[0, 0, node, 3] = float("nan")
    c.vt[0, 1, node, 9] = float("inf")
    c.q[0, 0, 40, 7] = float("inf")
    c.kt[:, :, c.n:], c.vt[:, :, c.n:], c.q[:, :, c.n:] = float("nan"), float("nan"), float("nan")
    out = c.run()[:, :, :c.n]
    below = c.seen[:, node].clone()
    hit = below.clone()
    hit[40] = True
    assert bool(torch.isnan(out[0, 0][hit]).all()) and bool(torch.isfinite(out[0, 0][~hit]).all())
    assert bool(torch.isinf(out[0, 1][below][:, 9]).all()) and bool(torch.isfinite(out[0, 1][:, :9]).all()) and bool(torch.isfinite(out[0, 1][~below]).all())
    # (the rows that do not see the node are what they are without it)
    c.kt[0, 0, node, 3], c.vt[0, 1, node, 9], c.q[0, 0, 40, 7] = 0.5, 0.5, 0.5
    clean = c.run()[:, :, :c.n]
    assert torch.equal(out[0, 0][~hit], clean[0, 0][~hit]) and torch.equal(out[0, 1][~below], clean[0, 1][~below])


def test_offsets_beyond_32_bits(binding):
    """The second sequence starts 2^33 channels into the cache: code bytes beyond 2^32."""
    c = Call(binding, TREES["nine"], 2, 1, 1, 128, (500, 333), seed=16)
    far = 2 ** 33
    old = [a.clone() for a in c.cache.arrays]
    big = [torch.empty((far // 128 + 600, a.shape[-1]), dtype=torch.uint8, device="cuda") for a in old]
    rows = c.cache.head_stride // 128
    for a, o in zip(big, old):
        a[:rows], a[far // 128:far // 128 + rows] = o[rows:], o[:rows]           # (sequences were in reverse order)
    c.cache.base = torch.tensor([0, far], dtype=torch.int64, device="cuda")
    c.cache.handle = binding.make_fp4_cache(*big)
    c.check()


def test_workspaces(binding):
    """A workspace that is missing, short or misaligned is refused; one that was never prepared fills the rows with NaN or is not
    needed; one prepared once serves calls of other shapes in turn."""
    c = Call(binding, TREES["44"], 1, 4, 4, 128, (3000,), seed=17)
    first = c.check()
    size = binding.tree_attention_fp4kv_workspace(1, 4, 4, 128, 44, 0, 3000)
    if size:
        for bad in (None, c.ws[:size - 1], torch.zeros(size + 512, dtype=torch.uint8, device="cuda")[8:]):
            keep, c.ws = c.ws, bad
            with pytest.raises(binding.McsdError) as e:
                c.call()
            assert e.value.status == binding.MCSD_EWORKSPACE
            c.ws = keep
        c.ws = torch.zeros_like(c.ws)
        assert bool(torch.isnan(c.run()[:, :, :c.n]).all())
    shared = binding.new_workspace(64 * 1024 * 1024)
    other = Call(binding, TREES["one"], 8, 4, 1, 64, tuple(range(0, 4000, 500)), seed=18)
    for x in (c, other, c, other):
        x.ws = shared
        x.check()
    assert torch.equal(c.out[:, :, :c.n], first[:, :, :c.n])


def test_two_streams_with_a_workspace_each(binding):
    cs = [Call(binding, TREES["44"], 4, 8, 8, 128, (2000, 100, 900, 1500), seed=20 + i) for i in range(2)]
    want = [c.check() for c in cs]
    streams = [torch.cuda.Stream() for _ in cs]
    for c in cs:
        c.out.fill_(31)
    torch.cuda.synchronize()
    for _ in range(10):
        for c, s in zip(cs, streams):
            c.call(s)
    torch.cuda.synchronize()
    for c, w in zip(cs, want):
        assert torch.equal(c.out, w)


def test_calls_of_a_graph_share_a_workspace(binding):
    cs = [Call(binding, TREES["44"], 2, 8, 8, 128, (1200, 333), seed=30), Call(binding, TREES["one"], 4, 8, 2, 128, (4000, 5, 1000, 2), seed=31)]
    shared = binding.new_workspace(64 * 1024 * 1024)
    for c in cs:
        c.ws = shared
    want = [c.check() for c in cs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for c in cs:
            c.call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for c in cs:
            c.call()
    for _ in range(4):
        for c in cs:
            c.out.fill_(31)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for c, w in zip(cs, want):
            assert torch.equal(c.out, w)
        cs[0].out.fill_(31)
        cs[0].call()                                       # eager work between the replays
        torch.cuda.synchronize()
        assert torch.equal(cs[0].out, want[0])
