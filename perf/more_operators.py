"""The operators of a decoding turn around a latent cache and between logits and verification, over the sizes they are called at,
each in its plain form (elementary torch operations, in 32 bits; 64 where a border or a far angle asks for it) and through the binding.

  attention   one layer's tree attention over a prefix cache of one latent vector per token, which all heads share: keys are its
              d_latent + d_rope channels, values the first d_latent of them
  rows        what feeds it: norm of the latents, rotation by position of their last d_rope channels and of the queries', for tree
              nodes, or a prompt's rows on their way into the cache
  sample      logits through temperature, top-k, top-p and min-p to the probability rows that the verification takes, and tokens
              drawn from them with given uniforms, independent or distinct

Queries and latents ~ N(0, 1), logits ~ N(0, 3^2) with a few tokens that stand out; rotation base 10000 or 500000.
"""
from __future__ import annotations

import math

import torch

own = False

F32, BF16 = 0, 1
TREES = ("4,2,2,1", "3,2,2,1,1,1,1,1", "4,2,2,2", "8,2,2,1,1", "16,1,1,1,1", "2,4,3,1,1", "2,2,2", "1,1,1,1", "1")
MAX_KEYS, MAX_FLOPS = 4.0e5, 5.2e11                  # what a drawn attention call may cost
MAX_ROW_BYTES, MAX_LOGITS = 2.0e8, 9.0e7             # what the others may move, or look at


def _branching(tree):
    return [int(x) for x in tree.split(",")]


def _levels(tree):
    """Level (1-based) and parent of every node, nodes level by level."""
    level, parent, first, count = [], [], 0, 1
    for l, b in enumerate(_branching(tree)):
        nodes = count * b
        level += [l + 1] * nodes
        parent += [-1 if l == 0 else first - count + i // b for i in range(nodes)]
        first += nodes
        count = nodes
    return level, parent


def _nodes(tree):
    return len(_levels(tree)[0])


def _first_row(case):
    level = _levels(case["tree"])[0]
    return level.index(level[-1]) if case.get("newest") else 0


# ---------------------------------------------------------------------------------------------------- cases
def _attention(name, B, H, d_latent, d_rope, lo, hi, tree, newest=False):
    return {"name": name, "kind": "attention", "B": B, "H": H, "d_latent": d_latent, "d_rope": d_rope, "prefix_min": lo, "prefix_max": hi,
            "tree": tree, "newest": newest}


def _sample(name, dtype, B, W, V, temperature, top_k, top_p, min_p, probs, scheme, n_draw, mixed=False):
    return {"name": name, "kind": "sample", "dtype": dtype, "B": B, "W": W, "V": V, "temperature": temperature, "top_k": top_k,
            "top_p": top_p, "min_p": min_p, "probs": probs, "scheme": scheme, "n_draw": n_draw, "mixed": mixed}


def listed():
    return [
        # the smallest call: a short prompt under a small tree; latency counts
        _attention("latent_small", 1, 16, 512, 64, 128, 128, "2,2,2"),
        # plain decoding of a serving batch, one token each, long and short conversations
        _attention("latent_decode", 32, 16, 512, 64, 777, 8191, "1"),
        # one chat on a model of 128 heads: 1024 cached tokens under the (4,2,2,1) tree
        _attention("latent_single", 1, 128, 512, 64, 1024, 1024, "4,2,2,1"),
        # a serving batch of conversations of very different lengths under a tree
        _attention("latent_ragged", 16, 16, 512, 64, 512, 4096, "4,2,2,2"),
        # a draft model's newest tree level, smaller latents, odd lengths
        _attention("latent_newest", 8, 12, 256, 32, 1333, 2001, "16,1,1,1,1", newest=True),
        # the largest call: long documents under the widest tree
        _attention("latent_long_wide", 2, 64, 512, 64, 16384, 16384, "8,2,2,1,1"),
        # one chat's tree nodes on their way to the attention
        {"name": "rows_tree", "kind": "rows", "dtype": "bf16", "B": 1, "H": 128, "d_latent": 512, "d_rope": 64, "interleaved": True,
         "base": 10000, "prefix": 1024, "tree": "4,2,2,1", "newest": False, "rows_min": 0, "rows_max": 0},
        # ragged prompts of a batch on their way into the cache, far into a long context
        {"name": "rows_prompts", "kind": "rows", "dtype": "bf16", "B": 8, "H": 0, "d_latent": 512, "d_rope": 64, "interleaved": False,
         "base": 500000, "prefix": 20000, "tree": "", "newest": False, "rows_min": 500, "rows_max": 4000},
        # the target's rows of one chat's tree: every filter at work
        _sample("sample_tree", "bf16", 1, 45, 32000, 0.7, 50, 0.9, 0.02, True, "independent", 0),
        # a draft model's level: rows for the verification and four distinct children of each node
        _sample("sample_level", "f32", 16, 4, 32000, 0.9, 0, 0.95, 0.0, True, "distinct", 4),
        # plain decoding of a serving batch over a large vocabulary of odd size, each conversation with its own settings, tokens alone
        _sample("sample_decode", "bf16", 32, 1, 131077, 0.8, 200, 0.95, 0.0, False, "independent", 1, mixed=True),
        # the target's rows of a large serving batch, temperature alone
        _sample("sample_batch", "bf16", 64, 44, 32000, 1.0, 0, 1.0, 0.0, True, "independent", 0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("attention", "attention", "attention", "rows", "sample", "sample", "sample"))
    if kind == "attention":
        while True:
            lo, hi = sorted((_log_int(rng, 1, 16384), _log_int(rng, 64, 16384)))
            d_latent, d_rope = rng.choice(((512, 64), (512, 64), (256, 32)))
            c = {"kind": kind, "B": _log_int(rng, 1, 64), "H": rng.choice((1, 4, 5, 8, 12, 16, 16, 32, 64, 128)), "d_latent": d_latent,
                 "d_rope": d_rope, "prefix_min": lo, "prefix_max": hi, "tree": rng.choice(TREES), "newest": rng.random() < 0.25}
            if c["B"] * hi <= MAX_KEYS and work(c)["flops"] <= MAX_FLOPS:
                return c
    if kind == "rows":
        while True:
            tree = rng.choice(TREES + ("",) * 6)
            lo, hi = sorted((_log_int(rng, 1, 4000), _log_int(rng, 1, 4000)))
            d_latent, d_rope = rng.choice(((512, 64), (512, 64), (256, 32)))
            c = {"kind": kind, "dtype": rng.choice(("bf16", "bf16", "f32")), "B": _log_int(rng, 1, 64),
                 "H": rng.choice((1, 4, 5, 12, 16, 64, 128)) if tree else 0, "d_latent": d_latent, "d_rope": d_rope,
                 "interleaved": rng.random() < 0.5, "base": rng.choice((10000, 500000)), "prefix": _log_int(rng, 1, 30000), "tree": tree,
                 "newest": bool(tree) and rng.random() < 0.4, "rows_min": 0 if tree else lo, "rows_max": 0 if tree else hi}
            if work(c)["bytes"] <= MAX_ROW_BYTES and c["B"] * (c["prefix"] if not tree else 0) <= 1000000:
                return c
    while True:
        c = {"kind": kind, "dtype": rng.choice(("bf16", "bf16", "f32")), "B": _log_int(rng, 1, 64), "W": _log_int(rng, 1, 60),
             "V": rng.choice((32000, 32000, 1000, 50257, 65536, _log_int(rng, 100, 262144))), "temperature": rng.choice((0.3, 0.6, 0.8, 1.0, 1.3)),
             "top_k": rng.choice((0, 0, 1, 20, 50, 500)), "top_p": rng.choice((1.0, 1.0, 0.3, 0.8, 0.95)),
             "min_p": rng.choice((0.0, 0.0, 0.01, 0.1)), "probs": rng.random() < 0.75, "scheme": rng.choice(("independent", "distinct")),
             "n_draw": rng.choice((0, 1, 2, 4, 8, 16)), "mixed": rng.random() < 0.3}
        if not c["probs"]:
            c["n_draw"] = max(c["n_draw"], 1)
        if c["B"] * c["W"] * c["V"] <= MAX_LOGITS:
            return c


# ---------------------------------------------------------------------------------------------------- what a pass cannot do without
def _spread(lo, hi, count):
    """Lengths from lo to hi, evenly spread; which sequence has which goes by the seed."""
    return [hi if count == 1 else lo + (hi - lo) * i // (count - 1) for i in range(count)]


def work(case):
    if case["kind"] == "sample":
        e = 2 if case["dtype"] == "bf16" else 4
        rows, V = case["B"] * case["W"], case["V"]
        return {"bytes": rows * V * (e + (4 if case["probs"] else 0)) + rows * case["n_draw"] * 8, "flops": rows * V * 4}
    dl, d = case["d_latent"], case["d_latent"] + case["d_rope"]
    if case["kind"] == "attention":
        level = _levels(case["tree"])[0]
        n, rows = len(level), len(level) - _first_row(case)
        keys = sum(_spread(case["prefix_min"], case["prefix_max"], case["B"]))
        seen = sum(level[_first_row(case):])
        return {"bytes": keys * d * 2 + case["B"] * 2 * (case["H"] * rows * (d + dl) + n * d),
                "flops": 2 * (d + dl) * case["H"] * (rows * keys + case["B"] * seen)}
    e = 2 if case["dtype"] == "bf16" else 4
    if case["tree"]:
        rows = case["B"] * (_nodes(case["tree"]) - _first_row(case))
    else:
        rows = sum(_spread(case["rows_min"], case["rows_max"], case["B"]))
    return {"bytes": rows * (case["H"] * case["d_rope"] + d) * (e + 2), "flops": rows * (case["H"] * case["d_rope"] * 3 + d * 4)}


# ---------------------------------------------------------------------------------------------------- inputs
def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)


def _shuffled(values, seed):
    order = torch.randperm(len(values), generator=torch.Generator().manual_seed(seed))
    return torch.tensor(values)[order].to(device="cuda", dtype=torch.int32)


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _prepare_attention(case, seed, gen):
    B, H, dl, dr = case["B"], case["H"], case["d_latent"], case["d_rope"]
    d = dl + dr
    level, parent = _levels(case["tree"])
    n, L = len(level), case["prefix_max"]
    cap = L + len(_branching(case["tree"]))
    s = {"case": case, "n": n, "row0": _first_row(case), "max_prefix": L, "cap": cap, "scale": 1.0 / math.sqrt(d)}
    s["q"] = _randn(gen, B, H, n, d).bfloat16()
    s["tree"] = _randn(gen, B, n, d).bfloat16()
    s["cache"] = _randn(gen, B, cap, d).bfloat16()
    s["lens"] = _shuffled(_spread(case["prefix_min"], L, B), seed)
    s["lens_host"] = s["lens"].tolist()                  # (products of plain operations need the lengths as numbers)
    s["base"] = torch.arange(B, device="cuda", dtype=torch.int64) * (cap * d)
    seen = torch.zeros(n, n, dtype=torch.bool)
    for i in range(n):
        j = i
        while j >= 0:
            seen[i, j] = True
            j = parent[j]
    s["seen"] = seen.cuda()
    s["out"] = torch.zeros(B, H, n, dl, dtype=torch.bfloat16, device="cuda")
    if own:
        from paper_2409_10644_amd import binding
        s["mask"] = binding.build_mask(_branching(case["tree"]))
        s["view"] = binding.slice_mask(s["mask"], len(_branching(case["tree"])))
        s["ws"] = binding.new_workspace(binding.tree_attention_latent_workspace(B, H, dl, dr, n, s["row0"], L))
    return s


def _prepare_rows(case, seed, gen):
    B, H, dl, dr, t = case["B"], case["H"], case["d_latent"], case["d_rope"], _type(case)
    d = dl + dr
    s = {"case": case, "eps": 1e-6, "weight": 1 + 0.2 * _randn(gen, dl)}
    s["freq"] = (case["base"] ** (-torch.arange(0, dr, 2, dtype=torch.float64) / dr)).float().cuda()
    if case["tree"]:
        level = _levels(case["tree"])[0]
        s["n"], s["row0"] = len(level), _first_row(case)
        T = s["n"] - s["row0"]
        s["level"] = torch.tensor(level[s["row0"]:], device="cuda")
        s["max_prefix"] = case["prefix"]
        s["lens"] = _shuffled(_spread(max(case["prefix"] // 2, 1), case["prefix"], B), seed)
        s["q"] = _randn(gen, B, T, H, 2 * dr).to(t)          # (the rotated channels stand behind others, as a projection leaves them)
        s["q_out"] = torch.zeros(B, H, s["n"], d, dtype=torch.bfloat16, device="cuda")
        s["out"] = torch.zeros(B, s["n"], d, dtype=torch.bfloat16, device="cuda")
    else:
        T = case["rows_max"]
        s["first"] = torch.full((B,), case["prefix"], dtype=torch.int32, device="cuda")
        s["n_rows"] = _shuffled(_spread(case["rows_min"], T, B), seed)
        s["cap"] = case["prefix"] + T
        s["base"] = torch.arange(B, device="cuda", dtype=torch.int64) * (s["cap"] * d)
        s["cache"] = torch.zeros(B, s["cap"], d, dtype=torch.bfloat16, device="cuda")
    s["kv"] = _randn(gen, B, T, d).to(t)
    if own:
        from paper_2409_10644_amd import binding
        s["rope"] = binding.make_rope(dr, s["freq"], None, s["weight"], s["eps"], case["interleaved"])
        if case["tree"]:
            s["mask"] = binding.build_mask(_branching(case["tree"]))
            s["view"] = binding.slice_mask(s["mask"], len(_branching(case["tree"])))
    return s


def _settings(case):
    """Temperature, top-k, top-p and min-p of every sequence."""
    B, out = case["B"], []
    for b in range(B):
        t, k, p, m = case["temperature"], case["top_k"], case["top_p"], case["min_p"]
        if case["mixed"]:
            t, k, p, m = ((t, k, p, m), (0.0, 0, 1.0, 0.0), (t + 0.25, 0, 0.9, m), (t, 40, 1.0, 0.05), (t, 0, 1.0, 0.0))[b % 5]
        out.append((t, k, p, m))
    return out


def _prepare_sample(case, seed, gen):
    B, W, V, n = case["B"], case["W"], case["V"], case["n_draw"]
    x = torch.empty(B, W, V, dtype=_type(case), device="cuda")
    for b in range(B):
        y = 3.0 * _randn(gen, W, V)
        best = torch.randint(0, V, (W, 6), generator=gen, device="cuda")
        x[b] = y.scatter_add_(1, best, 7.0 + 2.0 * _randn(gen, W, 6)).to(x.dtype)
    t, k, p, m = zip(*_settings(case))
    s = {"case": case, "x": x, "temperature": torch.tensor(t, dtype=torch.float32, device="cuda"),
         "top_k": torch.tensor(k, dtype=torch.int32, device="cuda"), "top_p": torch.tensor(p, dtype=torch.float32, device="cuda"),
         "min_p": torch.tensor(m, dtype=torch.float32, device="cuda")}
    s["u"] = torch.rand(B, W, max(n, 1), generator=gen, device="cuda", dtype=torch.float32)
    s["tokens"] = torch.zeros(B, W, n, dtype=torch.int32, device="cuda") if n else None
    s["probs"] = torch.zeros(B, W, V, dtype=torch.float32, device="cuda") if case["probs"] else None
    if own:
        from paper_2409_10644_amd import binding
        s["sampler"] = binding.make_sampler(s["temperature"], s["top_k"], s["top_p"], s["min_p"])
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return {"attention": _prepare_attention, "rows": _prepare_rows, "sample": _prepare_sample}[case["kind"]](case, seed, gen)


# ---------------------------------------------------------------------------------------------------- plain forms
def _plain_attention(s):
    case, n, row0, dl = s["case"], s["n"], s["row0"], s["case"]["d_latent"]
    H, rows = case["H"], n - row0
    for b, L in enumerate(s["lens_host"]):
        x = torch.cat((s["cache"][b, :L], s["tree"][b])).float()
        q = s["q"][b, :, row0:].float().reshape(H * rows, -1)
        y = (q @ x.t().contiguous()) * s["scale"]
        hide = torch.cat((torch.zeros(rows, L, dtype=torch.bool, device="cuda"), ~s["seen"][row0:]), 1)
        y = torch.where(hide.repeat(H, 1), -math.inf, y)
        w = torch.exp(y - y.amax(1, keepdim=True))
        o = (w @ x[:, :dl].contiguous()) / w.sum(1, keepdim=True)
        s["out"][b, :, row0:] = o.reshape(H, rows, dl).bfloat16()
    return s["out"]


def _turned(x, cos, sin, interleaved):
    if interleaved:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    a, b = x.chunk(2, -1)
    return torch.cat((a * cos - b * sin, b * cos + a * sin), -1)


def _latents(s, pos):
    """The rows of the latents at these positions [B, T], and cosines and sines [B, T, d_rope / 2]."""
    dl = s["case"]["d_latent"]
    angle = pos.double()[..., None] * s["freq"].double()
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    x = s["kv"].float()
    c = x[..., :dl]
    c = c / torch.sqrt((c * c).mean(-1, keepdim=True) + s["eps"]) * s["weight"]
    return torch.cat((c, _turned(x[..., dl:], cos, sin, s["case"]["interleaved"])), -1).bfloat16(), cos, sin


def _plain_rows(s):
    case, dl, dr = s["case"], s["case"]["d_latent"], s["case"]["d_rope"]
    if case["tree"]:
        rows, cos, sin = _latents(s, s["lens"].clamp(0, s["max_prefix"])[:, None] + s["level"] - 1)
        s["out"][:, s["row0"]:] = rows
        q = _turned(s["q"][..., dr:].float(), cos[:, :, None], sin[:, :, None], case["interleaved"])
        s["q_out"][:, :, s["row0"]:, dl:] = q.transpose(1, 2).bfloat16()
        return s["q_out"][..., dl:], s["out"]
    T, first = case["rows_max"], case["prefix"]
    t = torch.arange(T, device="cuda")
    rows = _latents(s, s["first"][:, None] + t)[0]
    there = s["cache"][:, first:first + T]
    there.copy_(torch.where((t < s["n_rows"][:, None])[..., None], rows, there))
    return there


def _plain_sample(s):
    case = s["case"]
    B, W, V, n = case["B"], case["W"], case["V"], case["n_draw"]
    per = max(1, int(6.0e7) // (W * V))
    for b in range(0, B, per):
        e = min(b + per, B)
        x = s["x"][b:e].double()
        t, p, m = (s[k][b:e].double()[:, None, None] for k in ("temperature", "top_p", "min_p"))
        k = s["top_k"][b:e][:, None, None]
        greedy = t == 0
        y, order = torch.sort(x, dim=-1, descending=True, stable=True)       # (ties: the lowest index first)
        place = torch.arange(V, device="cuda")
        w = torch.exp((y - y[..., :1]) / torch.where(greedy, 1.0, t))
        keep = (place < torch.where(k > 0, k, V)) & (place < torch.where(greedy, 1, V))
        w = torch.where(keep, w, 0.0)
        cum = w.cumsum(-1)
        keep = keep & ((cum - w < p * cum[..., -1:]) | (p >= 1) | (place == 0)) & (w >= m)
        w = torch.where(keep, w, 0.0)
        kept = torch.zeros_like(keep).scatter_(-1, order, keep)
        w = torch.zeros_like(w).scatter_(-1, order, w)
        if case["probs"]:
            s["probs"][b:e] = (w / w.sum(-1, keepdim=True)).float()
        if n:
            z = torch.where(kept, x, -math.inf)
            for i in range(n):
                if case["scheme"] == "distinct" and i:                   # (the weights anew, around the largest that is left)
                    z.scatter_(-1, token.clamp(min=0), -math.inf)
                    top = z.amax(-1, keepdim=True)
                    w = torch.where(top == -math.inf, 0.0, torch.exp((z - top) / torch.where(greedy, 1.0, t)))
                cum = w.cumsum(-1)
                total = cum[..., -1:]
                token = (cum <= s["u"][b:e, :, i:i + 1].double() * total).sum(-1, keepdim=True).clamp(max=V - 1)
                token = torch.where(total > 0, token, -1)
                s["tokens"][b:e, :, i] = token[..., 0].int()
    return [x for x in (s["probs"], s["tokens"]) if x is not None]


def run(state):
    s = state
    kind = s["case"]["kind"]
    if not own:
        return {"attention": _plain_attention, "rows": _plain_rows, "sample": _plain_sample}[kind](s)
    from paper_2409_10644_amd import binding
    case = s["case"]
    if kind == "sample":
        W, V, n = case["W"], case["V"], case["n_draw"]
        binding.sample_rows(BF16 if case["dtype"] == "bf16" else F32, case["B"], W, V, s["x"], W * V, V, s["sampler"], s["probs"], W * V,
                            binding.MCSD_WITHOUT_REPLACEMENT if case["scheme"] == "distinct" else binding.MCSD_WITH_REPLACEMENT, n,
                            s["u"] if n else None, s["tokens"], W * n)
        return [x for x in (s["probs"], s["tokens"]) if x is not None]
    B, H, dl, dr = case["B"], case["H"], case["d_latent"], case["d_rope"]
    if kind == "attention":
        binding.tree_attention_latent(s["view"], B, H, dl, dr, s["row0"], s["q"], s["tree"], s["n"], s["cache"], s["base"], s["lens"],
                                      s["max_prefix"], s["scale"], s["out"], s["ws"])
        return s["out"]
    dtype, d = BF16 if case["dtype"] == "bf16" else F32, dl + dr
    T = s["kv"].shape[1]
    if case["tree"]:
        binding.tree_latent_norm_rope(s["view"], dtype, B, H, dl, dr, s["row0"], s["q"][..., dr:], s["kv"], T * H * 2 * dr, H * 2 * dr, 2 * dr,
                                      T * d, d, s["rope"], s["lens"], s["max_prefix"], s["q_out"], s["out"], s["n"])
        return s["q_out"][..., dl:], s["out"]
    binding.store_latent(dtype, B, dl, dr, T, s["kv"], T * d, d, s["rope"], s["first"], s["n_rows"], s["cache"], s["base"], s["cap"])
    return s["cache"][:, case["prefix"]:case["prefix"] + T]


# ---------------------------------------------------------------------------------------------------- definitions in 64 bits
def _exact_attention(s):
    """Row by row of the definition: a prefix key counts as exp(s <q, x>), a tree key where it is the node or one of its ancestors."""
    case, dl, row0 = s["case"], s["case"]["d_latent"], s["row0"]
    parent = _levels(case["tree"])[1]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    for b, L in enumerate(s["lens"].tolist()):
        past, nodes = s["cache"][b, :L].double(), s["tree"][b].double()
        values = past[:, :dl].contiguous()
        for i in range(row0, s["n"]):
            chain, j = [], i
            while j >= 0:
                chain.append(j)
                j = parent[j]
            q = s["q"][b, :, i].double()
            far, near = s["scale"] * (q @ past.T), s["scale"] * (q @ nodes[chain].T)
            top = torch.maximum(near.max(1).values, far.max(1).values if L else near.max(1).values)[:, None]
            far, near = (far - top).exp(), (near - top).exp()
            out[b, :, i] = (far @ values + near @ nodes[chain][:, :dl]) / (far.sum(1) + near.sum(1))[:, None]
    return out


def _exact_rows(s):
    case, dl, dr = s["case"], s["case"]["d_latent"], s["case"]["d_rope"]
    half = dr // 2
    pair = [(2 * i, 2 * i + 1) if case["interleaved"] else (i, i + half) for i in range(half)]
    first, second = (torch.tensor(list(c), device="cuda") for c in zip(*pair))

    def turn(v, pos):                                  # v [..., dr], pos [...]: pairs as complex numbers
        z = torch.complex(v[..., first], v[..., second]) * torch.exp(1j * pos.double()[..., None] * s["freq"].double())
        y = torch.empty_like(v)
        y[..., first], y[..., second] = z.real, z.imag
        return y

    kv = s["kv"].double()
    rms = (kv[..., :dl].square().sum(-1, keepdim=True) / dl + s["eps"]).rsqrt()
    latent = kv[..., :dl] * rms * s["weight"].double()
    if case["tree"]:
        pos = s["lens"].long()[:, None] + s["level"] - 1
        out, q_out = s["out"].double() * 0, s["q_out"][..., dl:].double() * 0
        out[:, s["row0"]:] = torch.cat((latent, turn(kv[..., dl:], pos)), -1)
        q = s["q"][..., dr:].double()
        q_out[:, :, s["row0"]:] = turn(q, pos[:, :, None].expand(q.shape[:-1])).permute(0, 2, 1, 3)
        return q_out, out
    pos = case["prefix"] + torch.arange(kv.shape[1], device="cuda").expand(kv.shape[:2])
    rows = torch.cat((latent, turn(kv[..., dl:], pos)), -1)
    for b, count in enumerate(s["n_rows"].tolist()):
        rows[b, count:] = 0
    return rows


def _exact_sample(s):
    """One row at a time, over its distinct logits: each stands for as many tokens as have it."""
    case = s["case"]
    B, W, V, n = case["B"], case["W"], case["V"], case["n_draw"]
    if B * W > 4000:
        return None
    probs = torch.zeros(B, W, V, dtype=torch.float64, device="cuda") if case["probs"] else None
    tokens = torch.full((B, W, n), -1, dtype=torch.int32, device="cuda") if n else None
    settings = [[float(v) for v in z] for z in zip(*(s[k].tolist() for k in ("temperature", "top_k", "top_p", "min_p")))]
    for b in range(B):
        t, k, p, m = settings[b]
        for r in range(W):
            x = s["x"][b, r].double()
            if t == 0:
                kept = torch.zeros(V, dtype=torch.bool, device="cuda")
                kept[torch.nonzero(x == x.max())[0]] = True
            else:
                value, where, count = torch.unique(-x, return_inverse=True, return_counts=True)       # ascending: the largest logit first
                weight = torch.exp((value[0] - value) / t)
                if m > 0:
                    weight = weight.clone()
                before = count.cumsum(0) - count                                # tokens above
                allowed = (k - before).clamp(min=0).minimum(count) if k > 0 else count
                mass = weight * allowed
                if p < 1:
                    need = p * mass.sum() - (mass.cumsum(0) - mass)               # of this value's tokens
                    most = torch.where(weight > 0, torch.ceil(need / weight.clamp(min=1e-300)).clamp(min=0), 0.0)
                    allowed = most.minimum(allowed.double()).long()
                    allowed[0] = allowed[0].clamp(min=1)
                allowed = torch.where(weight >= m, allowed, 0)
                kept = (allowed == count)[where]
                for g in torch.nonzero((allowed > 0) & (allowed < count)).flatten().tolist():
                    kept[torch.nonzero(where == g).flatten()[:int(allowed[g])]] = True
            ids = torch.nonzero(kept).flatten()
            z = x[ids]
            w = torch.exp((z - z.max()) / (t if t else 1.0))
            if probs is not None:
                probs[b, r, ids] = w / w.sum()
            for i in range(n):
                if ids.numel() == 0:
                    break
                w = torch.exp((z - z.max()) / (t if t else 1.0))
                at = torch.searchsorted(w.cumsum(0), float(s["u"][b, r, i]) * w.sum(), right=True).clamp(max=ids.numel() - 1)
                tokens[b, r, i] = ids[at]
                if case["scheme"] == "distinct":
                    rest = torch.arange(ids.numel(), device="cuda") != at
                    ids, z = ids[rest], z[rest]
    return [v for v in (probs, tokens) if v is not None]


def exact(case, seed):
    if case["kind"] == "attention" and work(case)["flops"] > 1.0e12:
        return None
    return {"attention": _exact_attention, "rows": _exact_rows, "sample": _exact_sample}[case["kind"]](prepare(case, seed))
