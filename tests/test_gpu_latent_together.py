"""Speculative decoding on a latent cache as its turns run: prompts stored; then turn by turn the draft's rows and children drawn level by
level, the tree's latent rows and queries prepared in two layers, attended, the target's rows made of logits that depend on the
attention's output, verified, and the accepted path appended to both layers' caches.  Every step against its plain form on the state
the step before left, and a captured turn against eager ones."""
import numpy as np
import pytest
import torch

import latent_reference as R

pytestmark = pytest.mark.gpu
F32, BF16 = 0, 1
DRAFT_INIT, TARGET_INIT = 0, 1
BRANCHING = (4, 2, 2, 1)
EPS = float(np.float32(1e-6))


@pytest.fixture(scope="module")
def binding():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2409_10644_amd import binding as b
    return b


class Model:
    def __init__(self, binding, mode, distinct, B, H, dl, dr, prompts, V, cap=500, layers=2, seed=0):
        self.b, self.mode, self.distinct, self.B, self.H, self.dl, self.dr, self.d, self.V, self.cap, self.layers = binding, mode, distinct, B, H, dl, dr, dl + dr, V, cap, layers
        self.gen = torch.Generator("cuda").manual_seed(seed)
        self.view = binding.slice_mask(binding.build_mask(BRANCHING), len(BRANCHING))
        self.n, self.G = self.view.n_nodes, len(BRANCHING)
        self.widths = [int(np.prod(BRANCHING[:g])) for g in range(self.G + 1)]       # 1, 4, 8, ..: nodes of a level, the first is the context before the tree
        self.contexts = sum(self.widths[:self.G])                                    # rows of the draft
        self.T = max(prompts)
        self.max_prefix = cap - self.G
        self.scale = (dl + dr) ** -0.5
        mk = lambda *shape, dtype=torch.bfloat16: torch.zeros(*shape, dtype=dtype, device="cuda")
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
        self.weight = torch.rand(dl, generator=self.gen, device="cuda") + 0.5
        self.freq = (10000.0 ** (-torch.arange(0, dr, 2, dtype=torch.float64) / dr)).float().cuda()
        self.rope = binding.make_rope(dr, self.freq, None, self.weight, EPS, True)
        self.prompts, self.zero, self.lens = i32(prompts), i32([0] * B), i32(prompts)
        self.base = torch.arange(B, dtype=torch.int64, device="cuda") * cap * self.d
        self.caches = [mk(B, cap, self.d) for _ in range(layers)]
        self.q_in, self.kv_in = mk(layers, B, self.n, H, dr), mk(layers, B, self.n, self.d)       # projections of the tree's tokens
        self.q_latent = mk(layers, B, H, self.n, dl)
        self.q, self.tree, self.out = mk(layers, B, H, self.n, self.d), mk(layers, B, self.n, self.d), mk(layers, B, H, self.n, dl)
        self.draft_logits = mk(B, self.contexts, V, dtype=torch.float32)
        self.noise = mk(B, self.n + 1, V, dtype=torch.float32)
        self.logits = mk(B, self.n + 1, V)
        self.p_target, self.q_draft = mk(B, self.n + 1, V, dtype=torch.float32), mk(B, self.contexts, V, dtype=torch.float32)
        self.tokens, self.u = mk(B, self.n, dtype=torch.int32), mk(B, self.n, dtype=torch.float32)
        self.u_accept, self.n_new = mk(B, self.n, dtype=torch.float32), BRANCHING[0] if mode == TARGET_INIT else 1
        self.n_append = 0 if mode == TARGET_INIT else 1
        self.u_new = mk(B, self.n_new, dtype=torch.float32)
        self.path, self.alen, self.new = mk(B, self.G, dtype=torch.int32), mk(B, dtype=torch.int32), torch.randint(0, V, (B, self.n_new), generator=self.gen, device="cuda").int()
        self.ids, self.n_ids, self.before = mk(B, self.G + self.n_append, dtype=torch.int32), mk(B, dtype=torch.int32), self.lens.clone()
        self.settings = (torch.tensor([1.0, 0.7, 1.2][:B], device="cuda"), i32([0, 40, 500][:B]), torch.tensor([1.0, 0.95, 0.9][:B], device="cuda"), torch.tensor([0.0, 0.0, 0.01][:B], device="cuda"))
        self.sampler = binding.make_sampler(*self.settings)
        self.ws = torch.empty(max(binding.tree_attention_latent_workspace(B, H, dl, dr, self.n, 0, self.max_prefix), 256), dtype=torch.uint8, device="cuda")
        vb = binding.verify_tree_workspace(self.view, mode, B, self.n_new)
        self.verify_ws = torch.empty(vb, dtype=torch.uint8, device="cuda") if vb else None

    def store(self, layer, kv, counts):
        T = kv.shape[1]
        self.b.store_latent(BF16, self.B, self.dl, self.dr, T, kv, T * self.d, self.d, self.rope, self.zero, counts, self.caches[layer], self.base, self.cap)

    def turn(self):
        b, B, H, dl, dr, d, n, V, G = self.b, self.B, self.H, self.dl, self.dr, self.d, self.n, self.V, self.G
        scheme = b.MCSD_WITHOUT_REPLACEMENT if self.distinct else b.MCSD_WITH_REPLACEMENT
        self.before.copy_(self.lens)
        if self.mode == TARGET_INIT:                     # the first level comes from the target, the turn before
            self.tokens[:, :self.widths[1]].copy_(self.new)
        row, first = 0, 0                                # contexts from `row` on have their children from node `first` on
        for g in range(G):
            draws = BRANCHING[g] if g or self.mode == DRAFT_INIT else 0
            per = self.widths[g] * draws
            u = self.u[:, first:first + per].contiguous() if draws else None
            b.sample_rows(F32, B, self.widths[g], V, self.draft_logits[:, row:], self.contexts * V, V, self.sampler, self.q_draft[:, row:], self.contexts * V, scheme, draws,
                          u, self.tokens[:, first:] if draws else None, n)
            row += self.widths[g]
            first += self.widths[g + 1]
        for l, cache in enumerate(self.caches):
            self.q[l][..., :dl].copy_(self.q_latent[l])
            b.tree_latent_norm_rope(self.view, BF16, B, H, dl, dr, 0, self.q_in[l], self.kv_in[l], n * H * dr, H * dr, dr, n * d, d, self.rope, self.lens, self.max_prefix,
                                    self.q[l], self.tree[l], n)
            b.tree_attention_latent(self.view, B, H, dl, dr, 0, self.q[l], self.tree[l], n, cache, self.base, self.lens, self.max_prefix, self.scale, self.out[l], self.ws)
        hidden = (self.out[0].float() + self.out[1].float()).transpose(1, 2).reshape(B, n, H * dl)[..., :V]
        self.logits.copy_(self.noise)
        self.logits[:, 1:] += (0.3 * hidden).bfloat16()
        b.sample_rows(BF16, B, n + 1, V, self.logits, (n + 1) * V, V, self.sampler, self.p_target, (n + 1) * V, scheme, 0, None, None, 0)
        b.verify_tree_sampling(self.view, self.mode, scheme, B, V, self.tokens, self.p_target, self.q_draft, (n + 1) * V, self.contexts * V, self.u_accept, self.u_new, self.n_new,
                               self.path, self.alen, self.new, self.verify_ws)
        tree, caches = list(self.tree), self.caches
        b.commit_path(self.view, BF16, B, 1, d, tree, tree, n, caches, caches, self.base, 0, self.max_prefix, self.cap, self.path, self.alen, self.tokens, self.new, self.n_new,
                      self.n_append, self.lens, self.ids, self.n_ids)

    def fresh(self):
        """Other projections, logits (the target's near the draft's) and uniform numbers."""
        for t in (self.q_in, self.kv_in, self.q_latent):
            t.copy_(torch.randn(t.shape, generator=self.gen, device="cuda"))
        self.draft_logits.copy_(2 * torch.randn(self.draft_logits.shape, generator=self.gen, device="cuda"))
        self.noise.copy_(0.5 * torch.randn(self.noise.shape, generator=self.gen, device="cuda"))
        self.noise[:, :self.contexts] += self.draft_logits
        for t in (self.u, self.u_accept, self.u_new):
            t.copy_(torch.rand(t.shape, generator=self.gen, device="cuda"))

    def state(self):
        return self.caches + [self.lens, self.ids, self.n_ids, self.tokens, self.new, self.path, self.alen, self.out, self.p_target, self.q_draft]


def _rounded(got, want, size):
    # rounded to bf16; norm, angle, sine and products in fp32: fewer than 32 roundings
    err = (got.double() - want).abs()
    assert bool((err <= 2.0 ** -8 * want.abs() + 32 * 2.0 ** -24 * size).all()), float(err.max())


@pytest.mark.parametrize("mode,distinct", [(DRAFT_INIT, False), (DRAFT_INIT, True), (TARGET_INIT, False), (TARGET_INIT, True)])
@pytest.mark.parametrize("B,H,dl,dr,prompts,V", [(3, 8, 512, 64, (150, 1, 377), 1000), (2, 5, 256, 32, (64, 33), 997)])
def test_turns_of_decoding(binding, oracle, mode, distinct, B, H, dl, dr, prompts, V):
    m = Model(binding, mode, distinct, B, H, dl, dr, prompts, V)
    level, seen = torch.tensor(R.tree_of(BRANCHING)[0], device="cuda"), R.visible(BRANCHING, "cuda")
    prompt = torch.randn(m.layers, B, m.T, m.d, generator=m.gen, device="cuda").bfloat16()
    for l in range(m.layers):
        m.store(l, prompt[l], m.prompts)
        for b, T in enumerate(prompts):
            want, size = R.latent_rows(prompt[l, b, :T], m.weight, EPS, torch.arange(T, device="cuda"), m.freq, dl, dr, True)
            _rounded(m.caches[l][b, :T], want, size)
            assert bool((m.caches[l][b, T:] == 0).all())
    numbers = list(zip(*(t.tolist() for t in m.settings)))
    accepted = 0
    for _ in range(3):
        kept, new_before = [c.clone() for c in m.caches], m.new.clone()
        m.fresh()
        m.turn()
        torch.cuda.synchronize()
        before, alen = m.before.tolist(), m.alen.tolist()
        accepted += sum(alen)
        assert m.lens.tolist() == [x + a for x, a in zip(before, alen)] and m.n_ids.tolist() == [a + m.n_append for a in alen]
        for b in range(B):
            row, first = 0, 0
            for g in range(m.G):
                draws = BRANCHING[g]
                for r in range(m.widths[g]):
                    at = slice(first + r * draws, first + (r + 1) * draws)
                    drawn = g or mode == DRAFT_INIT
                    want, tokens = R.sample_row(m.draft_logits[b, row + r].cpu(), *numbers[b], us=m.u[b, at].tolist() if drawn else [], distinct=distinct)
                    R.check_probs(m.q_draft[b, row + r], want)
                    assert m.tokens[b, at].tolist() == (tokens if drawn else new_before[b].tolist())
                row += m.widths[g]
                first += m.widths[g + 1]
            for r in range(m.n + 1):
                R.check_probs(m.p_target[b, r], R.sample_row(m.logits[b, r].cpu(), *numbers[b])[0])
        want = oracle.verify_tree(mode, BRANCHING, m.tokens.cpu().numpy(), m.p_target.cpu().numpy(), m.q_draft.cpu().numpy(), m.u_accept.cpu().numpy(), m.u_new.cpu().numpy(),
                                  replacement=not distinct)
        for got, w in zip((m.path, m.alen, m.new), want):
            assert np.array_equal(got.cpu().numpy(), w)
        for l, cache in enumerate(m.caches):
            for b, L in enumerate(before):
                pos = L + level - 1
                want, size = R.latent_rows(m.kv_in[l, b], m.weight, EPS, pos, m.freq, dl, dr, True)
                _rounded(m.tree[l, b], want, size)
                want, size = R.rotated(m.q_in[l, b], pos[:, None], m.freq, dr, True)
                _rounded(m.q[l, b, :, :, dl:].transpose(0, 1), want, size)
                assert torch.equal(m.q[l, b, :, :, :dl], m.q_latent[l, b])
                want, lim = R.attention(m.q[l, b], m.tree[l, b], kept[l][b, :L], seen, m.scale, dl)
                assert bool(((m.out[l, b].double() - want).abs() <= lim).all()), (l, b)
                kept[l][b, L:L + alen[b]] = m.tree[l, b, m.path[b, :alen[b]].long()]
            assert torch.equal(cache, kept[l])           # the accepted rows, and nothing else
    assert accepted > 0


@pytest.mark.parametrize("mode,distinct", [(DRAFT_INIT, True), (TARGET_INIT, False)])
def test_a_captured_turn_is_the_eager_one(binding, mode, distinct):
    args = (binding, mode, distinct, 3, 8, 512, 64, (333, 1, 77), 1000)
    eager, graphed = (Model(*args, seed=9) for _ in range(2))
    for m in (eager, graphed):
        for l in range(m.layers):
            m.store(l, torch.randn(m.B, m.T, m.d, generator=m.gen, device="cuda").bfloat16(), m.prompts)
        m.fresh()
    torch.cuda.synchronize()
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
            m.fresh()
        eager.turn()                                       # eager work of another model between the replays
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager.state(), graphed.state()):
            assert torch.equal(a, b)
