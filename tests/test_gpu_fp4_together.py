"""The operators around the 4-bit prefix cache as a decoding turn runs them: a prompt's queries and keys normalised, rotated and
stored; then turn by turn the tree's rows prepared, attended, verified, the accepted path appended to every layer's cache and read
back.  Every step against its plain form on the state the step before left, and a captured turn against eager ones."""
import math

import numpy as np
import pytest
import torch

import fp4_reference as R
from fp4_reference import Cache
from workloads import DRAFT_INIT, WORKLOADS, scaled, verify_inputs

pytestmark = pytest.mark.gpu

BF16 = 1


@pytest.fixture(scope="module")
def binding():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2409_10644_amd import binding as b
    return b


class Model:
    """Projections of a few layers drawn at random, prompts, and the tensors that a turn works on."""

    def __init__(self, binding, branching, B, Hq, Hkv, d, prompts, cap, layers=2, seed=0):
        self.b, self.B, self.Hq, self.Hkv, self.d, self.layers, self.cap, self.branching = binding, B, Hq, Hkv, d, layers, cap, branching
        self.gen = torch.Generator("cuda").manual_seed(seed)
        self.view = binding.slice_mask(binding.build_mask(branching), len(branching))
        self.n, self.G = self.view.n_nodes, len(branching)
        self.width = (Hq + 2 * Hkv) * d
        self.w = [(torch.rand(d, generator=self.gen, device="cuda") + 0.5) for _ in range(2)]
        self.inv = 10000.0 ** (-2.0 * torch.arange(d // 2, device="cuda") / d)
        self.rope = binding.make_rope(d, self.inv, *self.w)
        self.T = max(prompts)
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
        self.prompts, self.zero, self.lens = i32(prompts), i32([0] * B), i32(prompts)
        self.max_prefix = cap - self.G
        self.caches = [Cache(binding, B, Hkv, cap, d, gap=4, fill=0) for _ in range(layers)]
        w = scaled(WORKLOADS["fork"], B=B, H=Hq, branching=branching, cfg_id=96)
        self.V = w.V
        vi = verify_inputs(w, seed=seed, mode=DRAFT_INIT, replacement=False)
        self.verify = [torch.from_numpy(vi[k]).cuda() for k in ("tokens", "p_target", "q_draft", "u_accept", "u_sample")]
        self.x = torch.randn(layers, B, self.n, self.width, generator=self.gen, device="cuda").bfloat16()     # the tree's projections
        mk = lambda h, t: torch.zeros(layers, B, h, t, d, dtype=torch.bfloat16, device="cuda")
        self.q, self.k, self.v, self.out = mk(Hq, self.n), mk(Hkv, self.n), mk(Hkv, self.n), mk(Hq, self.n)
        self.k_back, self.v_back = mk(Hkv, self.G), mk(Hkv, self.G)
        self.path, self.alen, self.new = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((B, self.G), (B,), (B, 1)))
        self.ids, self.n_ids, self.before = torch.zeros(B, self.G + 1, dtype=torch.int32, device="cuda"), i32([0] * B), self.lens.clone()
        self.ws = binding.new_workspace(max(binding.tree_attention_fp4kv_workspace(B, Hq, Hkv, d, self.n, 0, self.max_prefix), 256))
        self.scale = 1.0 / math.sqrt(d)

    def parts(self, x):
        return x, x[..., self.Hq * self.d:], x[..., (self.Hq + self.Hkv) * self.d:]

    def store_rows(self, layer, x, counts, first):
        """Rows x [B][T][width] of consecutive tokens through norm and rotation into a layer's cache."""
        B, T, d, W, c = self.B, x.shape[1], self.d, self.width, self.caches[layer]
        q, k, v = (torch.zeros(B, h, T, d, dtype=torch.bfloat16, device="cuda") for h in (self.Hq, self.Hkv, self.Hkv))
        self.b.prompt_qk_norm_rope(BF16, B, self.Hq, self.Hkv, d, T, *self.parts(x), T * W, W, T * W, W, self.rope, first, counts, q, k, v, T)
        self.b.store_fp4kv(BF16, B, self.Hkv, d, T, k, v, self.Hkv * T * d, T * d, d, first, counts, c.handle, c.base, c.head_stride, self.cap)
        return q, k, v

    def turn(self):
        b, B, Hq, Hkv, d, n, W = self.b, self.B, self.Hq, self.Hkv, self.d, self.n, self.width
        self.before.copy_(self.lens)
        for l, c in enumerate(self.caches):
            b.tree_qk_norm_rope(self.view, BF16, B, Hq, Hkv, d, 0, *self.parts(self.x[l]), n * W, W, n * W, W, self.rope, self.lens, self.max_prefix,
                                self.q[l], self.k[l], self.v[l], n)
            b.tree_attention_fp4kv(self.view, B, Hq, Hkv, d, 0, self.q[l], self.k[l], self.v[l], n, c.handle, c.base, self.lens, c.head_stride,
                                   self.max_prefix, self.scale, self.out[l], self.ws)
        tokens, p, qd, ua, us = self.verify
        b.verify_tree(self.view, DRAFT_INIT, B, self.V, tokens, p, qd, p.shape[1] * self.V, qd.shape[1] * self.V, ua, us, 1, self.path, self.alen, self.new, None)
        c = self.caches[0]
        handles = [x.handle for x in self.caches]
        b.commit_path_fp4kv(self.view, B, Hkv, d, list(self.k), list(self.v), n, handles, c.base, c.head_stride, self.max_prefix, self.cap, self.path,
                            self.alen, tokens, self.new, 1, 1, self.lens, self.ids, self.n_ids)
        b.load_fp4kv(BF16, B, Hkv, d, self.G, handles, c.base, c.head_stride, self.cap, self.before, self.alen, list(self.k_back), list(self.v_back),
                     Hkv * self.G * d, self.G * d, d)

    def fresh_tree(self):
        self.x.copy_(torch.randn(self.x.shape, generator=self.gen, device="cuda"))
        self.verify[3].copy_(torch.rand(self.verify[3].shape, generator=self.gen, device="cuda"))

    def state(self):
        return [a for c in self.caches for a in c.arrays] + [self.lens, self.ids, self.n_ids, self.out, self.k_back, self.v_back, self.alen, self.path]


BRANCHING = (4, 2, 2, 1)


@pytest.mark.parametrize("B,Hq,Hkv,d,prompts", [(3, 8, 2, 128, (150, 1, 77)), (2, 5, 5, 64, (40, 300))])
def test_turns_of_decoding(binding, B, Hq, Hkv, d, prompts):
    m = Model(binding, BRANCHING, B, Hq, Hkv, d, prompts, cap=400)
    level, seen = torch.tensor(R.tree_of(BRANCHING)[0], device="cuda"), R.visible(BRANCHING, "cuda")
    prompt = torch.randn(m.layers, B, m.T, m.width, generator=m.gen, device="cuda").bfloat16()
    for l in range(m.layers):
        _, k, v = m.store_rows(l, prompt[l], m.prompts, m.zero)
        for i, x in ((0, k), (2, v)):                       # what the cache holds is what the definition quantises these rows to
            codes, scales = R.quantise(x)
            for b, T in enumerate(prompts):
                assert torch.equal(m.caches[l].view(i)[b, :, :T], codes[b, :, :T]) and torch.equal(m.caches[l].view(i + 1)[b, :, :T], scales[b, :, :T])
    accepted = 0
    for _ in range(4):
        m.fresh_tree()
        m.turn()
        torch.cuda.synchronize()
        before, alen = m.before.tolist(), m.alen.tolist()
        accepted += sum(alen)
        assert m.lens.tolist() == [x + a for x, a in zip(before, alen)] and m.n_ids.tolist() == [a + 1 for a in alen]
        for l, c in enumerate(m.caches):
            for b, L in enumerate(before):
                pos = L + level - 1
                for x, w, got, H in ((m.x[l, b, :, :Hq * d], m.w[0], m.q, Hq), (m.x[l, b, :, Hq * d:(Hq + Hkv) * d], m.w[1], m.k, Hkv)):
                    want, size = R.rotated(x.unflatten(-1, (H, d)).double().cpu(), w.double().cpu(), 1e-6, pos[:, None].cpu(), m.inv.cpu(), d, False)
                    err = (got[l, b].transpose(0, 1).double().cpu() - want).abs()
                    # rounded to bf16; norm, angle, sine and products in fp32: fewer than 32 roundings
                    assert bool((err <= 2.0 ** -8 * want.abs() + 32 * 2.0 ** -24 * size).all())
                assert torch.equal(m.v[l, b], m.x[l, b, :, (Hq + Hkv) * d:].unflatten(-1, (Hkv, d)).transpose(0, 1))
                for h in range(Hq):
                    g = h // (Hq // Hkv)
                    kd, vd = (torch.cat((R.decode(c.view(i)[b, g, :L], c.view(i + 1)[b, g, :L]), t[l, b, g].double())) for i, t in ((0, m.k), (2, m.v)))
                    all_seen = torch.cat((torch.ones(m.n, L, dtype=torch.bool, device="cuda"), seen), 1)
                    want, lim = R.attention_row_terms(m.q[l, b, h].double(), kd, vd, all_seen, m.scale)
                    assert bool(((m.out[l, b, h].double() - want).abs() <= lim).all()), (l, b, h)
                if alen[b] == 0:
                    continue
                nodes = m.path[b, :alen[b]].long()
                for i, t, back in ((0, m.k, m.k_back), (2, m.v, m.v_back)):
                    codes, scales = R.quantise(t[l, b][:, nodes])
                    at = slice(L, L + alen[b])
                    assert torch.equal(c.view(i)[b, :, at], codes) and torch.equal(c.view(i + 1)[b, :, at], scales)
                    assert torch.equal(back[l, b, :, :alen[b]].double(), R.decode(codes, scales))
    assert accepted > 0


def test_accepted_nodes_leave_what_a_longer_prompt_would(binding):
    """A chain of nodes committed and the same tokens as part of the prompt: the same bytes in the cache."""
    B, Hq, Hkv, d, T = 2, 4, 2, 128, 50
    m, longer = (Model(binding, (1, 1, 1), B, Hq, Hkv, d, (T, T), cap=64, seed=5) for _ in range(2))
    x = torch.randn(m.layers, B, T + 3, m.width, generator=m.gen, device="cuda").bfloat16()
    counts = longer.prompts + 3
    for l in range(m.layers):
        m.store_rows(l, x[l, :, :T].contiguous(), m.prompts, m.zero)
        longer.store_rows(l, x[l], counts, longer.zero)
    m.x.copy_(x[:, :, T:])
    m.turn()
    torch.cuda.synchronize()
    m.path.copy_(torch.arange(3, device="cuda").expand(B, 3))
    m.alen.fill_(3)
    m.lens.fill_(T)
    c = m.caches[0]
    m.b.commit_path_fp4kv(m.view, B, Hkv, d, list(m.k), list(m.v), m.n, [x.handle for x in m.caches], c.base, c.head_stride, m.max_prefix, m.cap, m.path,
                          m.alen, m.verify[0], m.new, 1, 1, m.lens, m.ids, m.n_ids)
    torch.cuda.synchronize()
    for a, b in zip(m.caches, longer.caches):
        for i in range(4):
            assert torch.equal(a.view(i)[:, :, :T + 3], b.view(i)[:, :, :T + 3])


def test_a_captured_turn_is_the_eager_one(binding):
    args = (binding, BRANCHING, 3, 8, 2, 128, (333, 1, 77))
    eager, graphed = (Model(*args, cap=500, seed=9) for _ in range(2))
    for m in (eager, graphed):
        for l in range(m.layers):
            m.store_rows(l, torch.randn(m.B, m.T, m.width, generator=m.gen, device="cuda").bfloat16(), m.prompts, m.zero)
    kept = [t.clone() for t in graphed.state()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graphed.turn()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        graphed.turn()
    for t, w in zip(graphed.state(), kept):
        t.copy_(w)
    for _ in range(5):
        for m in (eager, graphed):
            m.fresh_tree()
        eager.turn()                                       # eager work of another model between the replays
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager.state(), graphed.state()):
            assert torch.equal(a, b)
