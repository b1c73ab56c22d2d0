"""The operators around a 4-bit prefix cache, over the sizes they are called at, each in its plain form (elementary torch
operations in 32 bits) and through the binding.

  attention   one layer's tree attention over a prefix cache in MXFP4: E2M1 elements, one power-of-two scale per 32 channels
  store       a prompt's (or single tokens') rows quantised into the cache, and read back as the numbers they stand for
  commit      the accepted path of every sequence appended to the cache of every layer, and those rows read back
  qk          norm of queries and keys per head and rotation by position, from the projections' layout to the attention's:
              tree nodes at prefix length + level - 1, or the consecutive tokens of a prompt

q, k, v ~ N(0, 1), cached channels with a gain of their own (log-normal); norm weights around 1; rotation base 10000 or 500000.
"""
from __future__ import annotations

import math

import torch

own = False

F32, BF16 = 0, 1
TREES = ("4,2,2,1", "3,2,2,1,1,1,1,1", "4,2,2,2", "8,2,2,1,1", "16,1,1,1,1", "2,4,3,1,1", "2,2,2", "1,1,1,1", "1")
MAX_KEY_HEADS, MAX_FLOPS = 4.3e6, 2.6e11             # what a drawn attention call may cost
MAX_ROW_BYTES = 2.0e8                                # what the others may move


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
def _attention(name, B, H_q, H_kv, d, lo, hi, tree, newest=False):
    return {"name": name, "kind": "attention", "B": B, "H_q": H_q, "H_kv": H_kv, "d": d, "prefix_min": lo, "prefix_max": hi,
            "tree": tree, "newest": newest}


def listed():
    return [
        # the smallest call: a few heads of a small draft model, a short prompt; latency counts
        _attention("attn_small", 1, 4, 4, 64, 128, 128, "2,2,2"),
        # one chat on a 7B model: 1024 cached tokens under the (4,2,2,1) tree
        _attention("attn_single", 1, 32, 32, 128, 1024, 1024, "4,2,2,1"),
        # plain decoding of a serving batch, one token each, long and short conversations, grouped-query heads
        _attention("attn_decode", 32, 32, 8, 128, 777, 8191, "1"),
        # a serving batch of conversations of very different lengths under a tree, grouped-query heads
        _attention("attn_ragged_gqa", 16, 32, 8, 128, 512, 4096, "4,2,2,2"),
        # the largest call: long documents under the widest tree
        _attention("attn_long_wide", 8, 32, 32, 128, 16384, 16384, "8,2,2,1,1"),
        # one new token for each of 16 sequences, grouped-query heads: latency counts
        {"name": "store_tokens", "kind": "store", "dtype": "bf16", "B": 16, "H": 8, "d": 128, "rows_min": 1, "rows_max": 1, "first": 1000},
        # ragged prompts of a batch, as the projections leave them
        {"name": "store_prompts", "kind": "store", "dtype": "bf16", "B": 4, "H": 32, "d": 128, "rows_min": 300, "rows_max": 2000, "first": 0},
        # one chat's accepted path in 32 layers
        {"name": "commit_single", "kind": "commit", "layers": 32, "B": 1, "H": 32, "d": 128, "prefix": 1024, "tree": "4,2,2,1", "n_append": 1},
        # the accepted paths of a serving batch in 32 layers
        {"name": "commit_batch", "kind": "commit", "layers": 32, "B": 64, "H": 8, "d": 128, "prefix": 600, "tree": "4,2,2,2", "n_append": 1},
        # one chat's tree nodes on their way to the attention
        {"name": "qk_tree_single", "kind": "qk", "dtype": "bf16", "B": 1, "H_q": 32, "H_kv": 32, "d": 128, "rotary": 128, "norm": True,
         "interleaved": False, "base": 10000, "prefix": 1024, "tree": "4,2,2,1", "newest": False, "rows_min": 0, "rows_max": 0},
        # ragged prompts of a batch, far into a long context
        {"name": "qk_prompts", "kind": "qk", "dtype": "bf16", "B": 4, "H_q": 32, "H_kv": 8, "d": 128, "rotary": 128, "norm": True,
         "interleaved": False, "base": 500000, "prefix": 100000, "tree": "", "newest": False, "rows_min": 500, "rows_max": 2000},
        # a draft model's newest tree level in fp32, rotation of half the channels in neighbouring pairs, no norm
        {"name": "qk_newest_f32", "kind": "qk", "dtype": "f32", "B": 8, "H_q": 12, "H_kv": 12, "d": 64, "rotary": 32, "norm": False,
         "interleaved": True, "base": 10000, "prefix": 2000, "tree": "16,1,1,1,1", "newest": True, "rows_min": 0, "rows_max": 0},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng):
    H_kv = rng.choice((1, 2, 4, 5, 8, 12, 16, 32))
    return H_kv * rng.choice([g for g in (1, 1, 2, 3, 4, 8) if g * H_kv <= 64]), H_kv


def draw(rng):
    kind = rng.choice(("attention", "attention", "store", "commit", "qk"))
    if kind == "attention":
        while True:
            H_q, H_kv = _heads(rng)
            lo, hi = sorted((_log_int(rng, 1, 16384), _log_int(rng, 64, 16384)))
            c = {"kind": kind, "B": _log_int(rng, 1, 64), "H_q": H_q, "H_kv": H_kv, "d": rng.choice((64, 128, 128)), "prefix_min": lo,
                 "prefix_max": hi, "tree": rng.choice(TREES), "newest": rng.random() < 0.25}
            if c["B"] * H_kv * hi <= MAX_KEY_HEADS and work(c)["flops"] <= MAX_FLOPS:
                return c
    if kind == "store":
        while True:
            lo, hi = sorted((_log_int(rng, 1, 4000), _log_int(rng, 1, 4000)))
            c = {"kind": kind, "dtype": rng.choice(("bf16", "bf16", "f32")), "B": _log_int(rng, 1, 32), "H": rng.choice((1, 2, 5, 8, 12, 32)),
                 "d": rng.choice((64, 128, 128)), "rows_min": lo, "rows_max": hi, "first": rng.choice((0, _log_int(rng, 1, 4000)))}
            if work(c)["bytes"] <= MAX_ROW_BYTES:
                return c
    if kind == "commit":
        while True:
            c = {"kind": kind, "layers": rng.choice((1, 2, 12, 32, 40, 64)), "B": _log_int(rng, 1, 64), "H": rng.choice((1, 4, 8, 12, 32)),
                 "d": rng.choice((64, 128, 128)), "prefix": _log_int(rng, 1, 1000), "tree": rng.choice(TREES), "n_append": rng.choice((0, 1))}
            if c["layers"] * c["B"] * c["H"] * c["prefix"] * c["d"] <= 2e9 and c["layers"] * c["B"] * c["H"] * _nodes(c["tree"]) * c["d"] <= 5e8:
                return c
    while True:
        H_q, H_kv = _heads(rng)
        d, tree = rng.choice((64, 128, 128)), rng.choice(TREES + ("",) * 4)
        lo, hi = sorted((_log_int(rng, 1, 4000), _log_int(rng, 1, 4000)))
        c = {"kind": kind, "dtype": rng.choice(("bf16", "bf16", "f32")), "B": _log_int(rng, 1, 64), "H_q": H_q, "H_kv": H_kv, "d": d,
             "rotary": rng.choice((d, d, d // 2)), "norm": rng.random() < 0.7, "interleaved": rng.random() < 0.3,
             "base": rng.choice((10000, 500000)), "prefix": _log_int(rng, 1, 200000), "tree": tree,
             "newest": bool(tree) and rng.random() < 0.4, "rows_min": 0 if tree else lo, "rows_max": 0 if tree else hi}
        if work(c)["bytes"] <= MAX_ROW_BYTES:
            return c


# ---------------------------------------------------------------------------------------------------- what a pass cannot do without
def _spread(lo, hi, count):
    """Lengths from lo to hi, evenly spread; which sequence has which goes by the seed."""
    return [hi if count == 1 else lo + (hi - lo) * i // (count - 1) for i in range(count)]


def _accepted(case):
    """Accepted lengths of a batch: every number of levels, nothing accepted among them."""
    G = len(_branching(case["tree"]))
    return [(i + G) % (G + 1) for i in range(case["B"])]


def work(case):
    d = case["d"]
    row4 = 2 * (d // 2 + d // 32)                     # a key and a value of one head in the cache
    if case["kind"] == "attention":
        level = _levels(case["tree"])[0]
        n, rows = len(level), len(level) - _first_row(case)
        keys = sum(_spread(case["prefix_min"], case["prefix_max"], case["B"]))
        seen = sum(level[_first_row(case):])
        return {"bytes": keys * case["H_kv"] * row4 + case["B"] * d * 2 * (2 * case["H_q"] * rows + 2 * case["H_kv"] * n),
                "flops": 4 * d * case["H_q"] * (rows * keys + case["B"] * seen)}
    if case["kind"] == "store":                       # quantised, then read back
        rows = sum(_spread(case["rows_min"], case["rows_max"], case["B"])) * case["H"]
        e = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": rows * (2 * (2 * d * e) + 2 * row4), "flops": rows * 2 * d * 4}
    if case["kind"] == "commit":
        rows = sum(_accepted(case)) * case["H"] * case["layers"]
        return {"bytes": rows * (2 * (2 * d * 2) + 2 * row4) + case["B"] * 64, "flops": rows * 2 * d * 4}
    if case["tree"]:
        rows = case["B"] * (_nodes(case["tree"]) - _first_row(case))
    else:
        rows = sum(_spread(case["rows_min"], case["rows_max"], case["B"]))
    e = 2 if case["dtype"] == "bf16" else 4
    return {"bytes": rows * (case["H_q"] + 2 * case["H_kv"]) * d * e * 2, "flops": rows * (case["H_q"] + case["H_kv"]) * d * 8}


# ---------------------------------------------------------------------------------------------------- the 4-bit format
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0)


def _quantise(x):
    """fp32 [..., d] -> codes uint8 [..., d/2] (even channel in the low half), scale bytes uint8 [..., d/32]."""
    g = x.reshape(*x.shape[:-1], -1, 32)
    m = g.abs().amax(-1)
    fine = torch.isfinite(m)
    e = (((m.contiguous().view(torch.int32) + 0x200000) >> 23) - 2).clamp(1, 254)      # exponent of the maximum rounded to one fraction bit
    e = torch.where(fine, e, 255)
    a = (g * torch.where(fine, torch.exp2((127 - e).float()), 0.0)[..., None]).abs()
    a = torch.where(fine[..., None], a, 0.0)
    code = (a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)      # ties to the even code
    code = torch.where(torch.signbit(g) & fine[..., None], code + 8, code).to(torch.uint8).reshape(*x.shape[:-1], -1, 2)
    return code[..., 0] | (code[..., 1] << 4), e.to(torch.uint8)


def _decode(codes, scales):
    """The numbers that a cache's rows stand for, fp32 [..., d]."""
    table = torch.tensor(E2M1, dtype=torch.float32, device=codes.device)
    v = torch.stack((table[(codes & 15).int()], table[(codes >> 4).int()]), -1).reshape(*scales.shape, 32)
    s = torch.exp2(scales.float() - 127.0)
    return (v * torch.where(scales == 255, math.nan, s)[..., None]).reshape(*scales.shape[:-1], -1)


# ---------------------------------------------------------------------------------------------------- inputs
def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)


def _cache(gen, B, H, cap, d, empty=False):
    """Codes and scales of keys and of values, [B][H][cap][..]."""
    def half():
        codes = torch.zeros(B, H, cap, d // 2, dtype=torch.uint8, device="cuda")
        scales = torch.full((B, H, cap, d // 32), 127, dtype=torch.uint8, device="cuda")
        if not empty:
            gain = torch.exp(0.3 * _randn(gen, H, 1, d))
            for b in range(B):
                codes[b], scales[b] = _quantise(_randn(gen, H, cap, d) * gain)
        return codes, scales
    return half() + half()


def _shuffled(values, seed, **kw):
    order = torch.randperm(len(values), generator=torch.Generator().manual_seed(seed))
    return torch.tensor(values)[order].to(device="cuda", dtype=torch.int32, **kw)


def _i32(*shape):
    return torch.zeros(*shape, dtype=torch.int32, device="cuda")


def _prepare_attention(case, seed, gen):
    B, H_q, H_kv, d = case["B"], case["H_q"], case["H_kv"], case["d"]
    level, parent = _levels(case["tree"])
    n, L = len(level), case["prefix_max"]
    cap = (L + len(_branching(case["tree"])) + 7) // 8 * 8
    s = {"case": case, "n": n, "row0": _first_row(case), "max_prefix": L, "cap": cap, "scale": 1.0 / math.sqrt(d)}
    s["q"] = _randn(gen, B, H_q, n, d).bfloat16()
    s["kt"], s["vt"] = (_randn(gen, B, H_kv, n, d).bfloat16() for _ in range(2))
    s["cache"] = _cache(gen, B, H_kv, cap, d)
    s["lens"] = _shuffled(_spread(case["prefix_min"], L, B), seed)
    s["base"] = torch.arange(B, device="cuda", dtype=torch.int64) * (H_kv * cap * d)
    seen = torch.zeros(n, n, dtype=torch.bool)
    for i in range(n):
        j = i
        while j >= 0:
            seen[i, j] = True
            j = parent[j]
    s["seen"] = seen.cuda()
    s["out"] = torch.zeros_like(s["q"])
    if own:
        from paper_2409_10644_amd import binding
        s["mask"] = binding.build_mask(_branching(case["tree"]))
        s["view"] = binding.slice_mask(s["mask"], len(_branching(case["tree"])))
        s["handle"] = binding.make_fp4_cache(*s["cache"])
        s["ws"] = binding.new_workspace(binding.tree_attention_fp4kv_workspace(B, H_q, H_kv, d, n, s["row0"], L))
    return s


def _prepare_store(case, seed, gen):
    B, H, d, T = case["B"], case["H"], case["d"], case["rows_max"]
    t = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    cap = (case["first"] + T + 7) // 8 * 8
    gain = torch.exp(0.3 * _randn(gen, H, d))
    s = {"case": case, "cap": cap, "k": (_randn(gen, B, T, H, d) * gain).to(t), "v": _randn(gen, B, T, H, d).to(t)}
    s["n_rows"] = _shuffled(_spread(case["rows_min"], T, B), seed)
    s["first"] = torch.full((B,), case["first"], dtype=torch.int32, device="cuda")
    s["cache"] = _cache(gen, B, H, cap, d, empty=True)
    s["base"] = torch.arange(B, device="cuda", dtype=torch.int64) * (H * cap * d)
    s["k_out"], s["v_out"] = (torch.zeros(B, H, T, d, dtype=t, device="cuda") for _ in range(2))
    if own:
        from paper_2409_10644_amd import binding
        s["handle"] = binding.make_fp4_cache(*s["cache"])
    return s


def _prepare_commit(case, seed, gen):
    N, B, H, d, L = case["layers"], case["B"], case["H"], case["d"], case["prefix"]
    level, parent = _levels(case["tree"])
    n, G = len(level), len(_branching(case["tree"]))
    cap = (L + G + 7) // 8 * 8
    s = {"case": case, "n": n, "G": G, "cap": cap, "max_prefix": L}
    s["kt"], s["vt"] = (_randn(gen, N, B, H, n, d).bfloat16() for _ in range(2))
    s["cache"] = tuple(torch.stack(x) for x in zip(*(_cache(gen, B, H, cap, d, empty=True) for _ in range(N))))
    # (every sequence is as long as the bound: a pass finds the lengths of the pass before clamped to where it began)
    s["lens"] = torch.full((B,), L, dtype=torch.int32, device="cuda")
    s["first"] = s["lens"].clone()
    s["alen"] = _shuffled(_accepted(case), seed)
    leaf = torch.randint(level.index(G), n, (B,), generator=torch.Generator().manual_seed(seed)).tolist()
    path = []
    for b in range(B):
        up = [leaf[b]]
        while parent[up[-1]] >= 0:
            up.append(parent[up[-1]])
        path.append(up[::-1])
    path = torch.tensor(path, dtype=torch.int32, device="cuda").reshape(B, G)
    s["path"] = torch.where(torch.arange(G, device="cuda") < s["alen"][:, None], path, -1)
    s["tokens"] = torch.randint(0, 32000, (B, n), generator=gen, device="cuda", dtype=torch.int32)
    s["new"] = torch.randint(0, 32000, (B, 1), generator=gen, device="cuda", dtype=torch.int32)
    s["base"] = torch.arange(B, device="cuda", dtype=torch.int64) * (H * cap * d)
    s["ids"], s["n_ids"] = _i32(B, G + case["n_append"]), _i32(B)
    s["k_out"], s["v_out"] = (torch.zeros(N, B, H, G, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    if own:
        from paper_2409_10644_amd import binding
        s["mask"] = binding.build_mask(_branching(case["tree"]))
        s["view"] = binding.slice_mask(s["mask"], G)
        s["handles"] = [binding.make_fp4_cache(*(x[l] for x in s["cache"])) for l in range(N)]
        s["layers"] = [list(s[k].unbind(0)) for k in ("kt", "vt", "k_out", "v_out")]
    return s


def _prepare_qk(case, seed, gen):
    B, H_q, H_kv, d = case["B"], case["H_q"], case["H_kv"], case["d"]
    t = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    s = {"case": case, "row0": 0, "eps": 1e-6}
    if case["tree"]:
        level = _levels(case["tree"])[0]
        s["row0"] = _first_row(case)
        s["out_rows"] = n = len(level)
        s["rows"] = T = n - s["row0"]
        s["level"] = torch.tensor(level, device="cuda")
        s["n_rows"] = torch.full((B,), T, dtype=torch.int32, device="cuda")
    else:
        s["out_rows"] = s["rows"] = T = case["rows_max"]
        s["n_rows"] = _shuffled(_spread(case["rows_min"], T, B), seed)
    qkv = _randn(gen, B, T, (H_q + 2 * H_kv) * d).to(t)               # one projection's output
    s["q"], s["k"], s["v"] = qkv[..., :H_q * d], qkv[..., H_q * d:(H_q + H_kv) * d], qkv[..., (H_q + H_kv) * d:]
    s["first"] = torch.randint(0, case["prefix"] + 1, (B,), generator=gen, device="cuda", dtype=torch.int32)
    s["wq"], s["wk"] = (1.0 + 0.1 * _randn(gen, 2, d)).unbind(0) if case["norm"] else (None, None)
    i = torch.arange(0, case["rotary"], 2, dtype=torch.float64, device="cuda")
    s["inv_freq"] = torch.pow(float(case["base"]), -i / case["rotary"]).float()
    s["q_out"] = torch.zeros(B, H_q, s["out_rows"], d, dtype=t, device="cuda")
    s["k_out"], s["v_out"] = (torch.zeros(B, H_kv, s["out_rows"], d, dtype=t, device="cuda") for _ in range(2))
    if own:
        from paper_2409_10644_amd import binding
        s["rope"] = binding.make_rope(case["rotary"], s["inv_freq"], s["wq"], s["wk"], s["eps"], case["interleaved"])
        if case["tree"]:
            s["mask"] = binding.build_mask(_branching(case["tree"]))
            s["view"] = binding.slice_mask(s["mask"], len(_branching(case["tree"])))
    return s


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    return {"attention": _prepare_attention, "store": _prepare_store, "commit": _prepare_commit, "qk": _prepare_qk}[case["kind"]](case, seed, gen)


# ---------------------------------------------------------------------------------------------------- plain forms
def _attention_plain(s):
    c = s["case"]
    B, H_q, H_kv, d, n, row0 = c["B"], c["H_q"], c["H_kv"], c["d"], s["n"], s["row0"]
    R = n - row0
    kc, ks, vc, vs = s["cache"]
    q = s["q"][:, :, row0:].float().reshape(B, H_kv, -1, d)
    pre = torch.matmul(q, _decode(kc, ks).transpose(2, 3)) * s["scale"]
    pre = pre.masked_fill(torch.arange(s["cap"], device="cuda") >= s["lens"][:, None, None, None], -math.inf)
    own_keys = torch.matmul(q, s["kt"].float().transpose(2, 3)) * s["scale"]
    own_keys = own_keys.masked_fill(~s["seen"][row0:].repeat(H_q // H_kv, 1), -math.inf)
    top = torch.maximum(pre.amax(-1, keepdim=True), own_keys.amax(-1, keepdim=True))
    pre, own_keys = torch.exp(pre - top), torch.exp(own_keys - top)
    total = pre.sum(-1, keepdim=True) + own_keys.sum(-1, keepdim=True)
    out = torch.matmul(pre, _decode(vc, vs)) + torch.matmul(own_keys, s["vt"].float())
    return (out / total).reshape(B, H_q, R, d).bfloat16()


def _put(cache, src, first, count):
    """Rows src [.., B, H, T, d], the first count[b] of them, into the cache [.., B, H, cap, ..] from row first[b] on."""
    T, cap = src.shape[-2], cache[0].shape[-2]
    row = torch.arange(T, device="cuda")
    at = (first.long()[:, None] + row).clamp(max=cap - 1)
    live = (row < count[:, None])[:, None, :, None]
    for store, new in zip(cache, _quantise(src.float())):
        index = at[:, None, :, None].expand(new.shape)
        store.scatter_(-2, index, torch.where(live, new, store.gather(-2, index)))


def _get(cache, first, count, T, t):
    codes, scales = cache
    row = torch.arange(T, device="cuda")
    at = (first.long()[:, None] + row).clamp(max=codes.shape[-2] - 1)[:, None, :, None]
    lead = codes.shape[:-2] + (T,)
    v = _decode(codes.gather(-2, at.expand(lead + codes.shape[-1:])), scales.gather(-2, at.expand(lead + scales.shape[-1:])))
    return torch.where((row < count[:, None])[:, None, :, None], v, 0.0).to(t)


def _store_plain(s):
    T = s["case"]["rows_max"]
    _put(s["cache"][:2], s["k"].transpose(1, 2), s["first"], s["n_rows"])
    _put(s["cache"][2:], s["v"].transpose(1, 2), s["first"], s["n_rows"])
    return tuple(_get(s["cache"][i:i + 2], s["first"], s["n_rows"], T, s["k"].dtype) for i in (0, 2))


def _commit_plain(s):
    c, G = s["case"], s["G"]
    row = torch.arange(G, device="cuda")
    live = row < s["alen"][:, None]
    node = torch.where(live, s["path"], 0).long()
    first = s["lens"].clamp(0, s["max_prefix"])
    index = node[:, None, :, None].expand(s["k_out"].shape)
    _put(s["cache"][:2], s["kt"].gather(-2, index), first, s["alen"])
    _put(s["cache"][2:], s["vt"].gather(-2, index), first, s["alen"])
    ids = torch.full_like(s["ids"], -1)
    ids[:, :G] = torch.where(live, s["tokens"].gather(1, node), -1)
    if c["n_append"]:
        ids.scatter_(1, s["alen"].long()[:, None], s["new"])
    k, v = (_get(s["cache"][i:i + 2], s["first"], s["alen"], G, torch.bfloat16) for i in (0, 2))
    return k, v, first + s["alen"], ids, s["alen"] + c["n_append"]


def _turned(x, cos, sin, rotary, interleaved):
    r = x[..., :rotary]
    a, b = (r[..., 0::2], r[..., 1::2]) if interleaved else (r[..., :rotary // 2], r[..., rotary // 2:])
    u, v = a * cos - b * sin, b * cos + a * sin
    r = torch.stack((u, v), -1).flatten(-2) if interleaved else torch.cat((u, v), -1)
    return torch.cat((r, x[..., rotary:]), -1)


def _qk_plain(s):
    c, T = s["case"], s["rows"]
    t, d = s["q"].dtype, c["d"]
    where = s["first"][:, None] + (s["level"][s["row0"]:] - 1 if c["tree"] else torch.arange(T, device="cuda"))
    angle = where.double()[..., None] * s["inv_freq"].double()
    cos, sin = (f(angle).float()[:, :, None] for f in (torch.cos, torch.sin))
    live = (torch.arange(T, device="cuda") < s["n_rows"][:, None])[:, None, :, None]
    got = []
    for x, w in ((s["q"], s["wq"]), (s["k"], s["wk"]), (s["v"], None)):
        y = x.unflatten(-1, (-1, d)).float()
        if w is not None:
            y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + s["eps"]) * w
        if x is not s["v"]:
            y = _turned(y, cos, sin, c["rotary"], c["interleaved"])
        y = torch.where(live, y.transpose(1, 2), 0.0).to(t)
        got.append(torch.cat((torch.zeros_like(y[:, :, :1]).expand(-1, -1, s["row0"], -1), y), 2))
    return tuple(got)


# ---------------------------------------------------------------------------------------------------- a pass
def _run_own(s):
    from paper_2409_10644_amd import binding
    c = s["case"]
    kind, B, d = c["kind"], c["B"], c["d"]
    if kind == "attention":
        binding.tree_attention_fp4kv(s["view"], B, c["H_q"], c["H_kv"], d, s["row0"], s["q"], s["kt"], s["vt"], s["n"], s["handle"],
                                     s["base"], s["lens"], s["cap"] * d, s["max_prefix"], s["scale"], s["out"], s["ws"])
        return s["out"][:, :, s["row0"]:]
    if kind == "store":
        H, T, dtype = c["H"], c["rows_max"], BF16 if c["dtype"] == "bf16" else F32
        binding.store_fp4kv(dtype, B, H, d, T, s["k"], s["v"], T * H * d, d, H * d, s["first"], s["n_rows"], s["handle"], s["base"],
                            s["cap"] * d, s["cap"])
        binding.load_fp4kv(dtype, B, H, d, T, [s["handle"]], s["base"], s["cap"] * d, s["cap"], s["first"], s["n_rows"], [s["k_out"]],
                           [s["v_out"]], H * T * d, T * d, d)
        return s["k_out"], s["v_out"]
    if kind == "commit":
        H, G = c["H"], s["G"]
        kt, vt, k_out, v_out = s["layers"]
        binding.commit_path_fp4kv(s["view"], B, H, d, kt, vt, s["n"], s["handles"], s["base"], s["cap"] * d, s["max_prefix"], s["cap"],
                                  s["path"], s["alen"], s["tokens"], s["new"], 1, c["n_append"], s["lens"], s["ids"], s["n_ids"])
        binding.load_fp4kv(BF16, B, H, d, G, s["handles"], s["base"], s["cap"] * d, s["cap"], s["first"], s["alen"], k_out, v_out,
                           H * G * d, G * d, d)
        return s["k_out"], s["v_out"], s["lens"], s["ids"], s["n_ids"]
    dtype, width, T = BF16 if c["dtype"] == "bf16" else F32, (c["H_q"] + 2 * c["H_kv"]) * d, s["rows"]
    if c["tree"]:
        binding.tree_qk_norm_rope(s["view"], dtype, B, c["H_q"], c["H_kv"], d, s["row0"], s["q"], s["k"], s["v"], T * width, width, T * width,
                                  width, s["rope"], s["first"], c["prefix"], s["q_out"], s["k_out"], s["v_out"], s["out_rows"])
    else:
        binding.prompt_qk_norm_rope(dtype, B, c["H_q"], c["H_kv"], d, T, s["q"], s["k"], s["v"], T * width, width, T * width, width, s["rope"],
                                    s["first"], s["n_rows"], s["q_out"], s["k_out"], s["v_out"], s["out_rows"])
    return s["q_out"], s["k_out"], s["v_out"]


def run(state):
    if own:
        return _run_own(state)
    kind = state["case"]["kind"]
    if kind == "attention":
        return _attention_plain(state)
    if kind == "store":
        return _store_plain(state)
    return _commit_plain(state) if kind == "commit" else _qk_plain(state)


# ---------------------------------------------------------------------------------------------------- from the definitions, in 64 bits
def _number(codes, scales):
    """Each element by its parts: sign, two exponent bits of bias 1, one fraction bit, times its group's power of two."""
    c = torch.stack((codes % 16, codes // 16), -1).flatten(-2).double()
    sign, e, f = 1.0 - 2.0 * (c >= 8), (c % 8) // 2, c % 2
    mag = torch.where(e == 0, f / 2, (1 + f / 2) * torch.exp2(e - 1))
    power = torch.exp2(scales.double() - 127)
    power[scales == 255] = math.nan
    return sign * mag * power.repeat_interleave(32, -1)


def _held(x):
    """What a row of numbers becomes in the cache: the nearest of the elements' values at the group's scale."""
    g = x.double().unflatten(-1, (-1, 32))
    m = g.abs().amax(-1, keepdim=True)
    frac, exp = torch.frexp(m)                                         # m = frac * 2^exp, frac in [1/2, 1)
    unit = torch.exp2((exp.double() - 1 + (frac >= 0.875) - 2).clamp(min=-126.0))
    grid = torch.tensor((0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0), dtype=torch.float64, device=x.device)
    a = g.abs() / unit
    up = torch.bucketize(a, grid).clamp(max=7)                         # grid[up - 1] < a <= grid[up]
    low = (up - 1).clamp(min=0)
    below, above = a - grid[low], grid[up] - a
    code = torch.where((below < above) | ((below == above) & (low % 2 == 0)), low, up)
    return (torch.sign(g) * grid[code] * unit).flatten(-2)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "attention":
        B, d, row0, n = case["B"], case["d"], s["row0"], s["n"]
        share = case["H_q"] // case["H_kv"]
        out = torch.empty(B, case["H_q"], n - row0, d, dtype=torch.float64, device="cuda")
        for b in range(B):
            L = int(s["lens"][b])
            k, v = (torch.cat((_number(s["cache"][i][b, :, :L], s["cache"][i + 1][b, :, :L]), t[b].double()), 1) for i, t in ((0, s["kt"]), (2, s["vt"])))
            seen = torch.cat((torch.ones(n, L, dtype=torch.bool, device="cuda"), s["seen"]), 1)[row0:]
            for h in range(case["H_q"]):
                z = s["q"][b, h, row0:].double() @ k[h // share].T / math.sqrt(d)
                z[~seen] = -math.inf
                out[b, h] = torch.softmax(z, -1) @ v[h // share]
        return out
    if kind == "store":
        live = torch.arange(case["rows_max"], device="cuda") < s["n_rows"][:, None]
        return tuple((_held(x) * live[..., None, None]).permute(0, 2, 1, 3) for x in (s["k"], s["v"]))
    if kind == "commit":
        got = []
        for x in (s["kt"], s["vt"]):
            y = torch.zeros(s["k_out"].shape, dtype=torch.float64, device="cuda")
            for b, a in enumerate(s["alen"].tolist()):
                y[:, b, :, :a] = _held(x[:, b][:, :, s["path"][b, :a].long()])
            got.append(y)
        return got[0], got[1], None, None, None
    T, d, R, row0 = s["rows"], case["d"], case["rotary"], s["row0"]
    place = (s["level"][row0:] - 1 if case["tree"] else torch.arange(T, device="cuda"))[None] + s["first"][:, None]
    z = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), place[..., None].double() * s["inv_freq"].double())[:, :, None]
    got = []
    for name, w in (("q", s["wq"]), ("k", s["wk"]), ("v", None)):
        x = s[name].double().unflatten(-1, (-1, d))
        if w is not None:
            x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / d + s["eps"]) * w.double()
        if name != "v":
            x = x.clone()
            i = torch.arange(R // 2, device="cuda")
            first, second = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + R // 2)
            turned = torch.complex(x[..., first], x[..., second]) * z
            x[..., first], x[..., second] = turned.real, turned.imag
        y = torch.zeros(case["B"], x.shape[2], s["out_rows"], d, dtype=torch.float64, device="cuda")
        y[:, :, row0:] = torch.where((torch.arange(T, device="cuda") < s["n_rows"][:, None])[..., None, None], x, 0.0).permute(0, 2, 1, 3)
        got.append(y)
    return tuple(got)
