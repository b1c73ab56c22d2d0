"""The plain forms of the latent cache's and the sampling operators against values known otherwise, and what the entry points refuse
(no GPU needed: a call that is refused launches nothing)."""
import ctypes as C
import math

import pytest
import torch

import latent_reference as R
from paper_2409_10644_amd import binding as b

ONE = C.c_void_p(256)                                      # never dereferenced: the call is refused first


# ------------------------------------------------------------------------------------------------ plain forms
def test_attention_is_that_of_expanded_heads():
    """Scores and outputs with each head's keys and values made from the latents are those of the absorbed form."""
    g = torch.Generator().manual_seed(0)
    dl, dr, dn, H, L, branching = 12, 4, 6, 3, 9, (2, 2)
    seen = R.visible(branching)
    n = seen.shape[0]
    wk, wv = torch.randn(H, dn, dl, generator=g, dtype=torch.float64), torch.randn(H, 5, dl, generator=g, dtype=torch.float64)
    past, tree = torch.randn(L, dl + dr, generator=g, dtype=torch.float64), torch.randn(n, dl + dr, generator=g, dtype=torch.float64)
    qn, qr = torch.randn(H, n, dn, generator=g, dtype=torch.float64), torch.randn(H, n, dr, generator=g, dtype=torch.float64)
    out, _ = R.attention(torch.cat((qn @ wk, qr), -1), tree, past, seen, 0.3, dl)
    x = torch.cat((past, tree))
    for h in range(H):
        keys, values = torch.cat((x[:, :dl] @ wk[h].T, x[:, dl:]), -1), x[:, :dl] @ wv[h].T
        for i in range(n):
            see = list(range(L)) + [L + j for j in range(n) if seen[i, j]]
            w = torch.softmax(0.3 * keys[see] @ torch.cat((qn[h, i], qr[h, i])), 0)
            assert torch.allclose(w @ values[see], out[h, i] @ wv[h].T, atol=1e-12)


def test_rotation_keeps_lengths_and_differences():
    g = torch.Generator().manual_seed(1)
    freq = torch.tensor([1.0, 0.1, 0.01, 0.001])
    for interleaved in (False, True):
        x, y = (torch.randn(1, 8, generator=g, dtype=torch.float64) for _ in range(2))
        turn = lambda v, p: R.rotated(v, torch.tensor([p]), freq, 8, interleaved)[0]
        assert torch.allclose(turn(x, 1000).norm(), x.norm())
        assert torch.allclose((turn(x, 1007) * turn(y, 1000)).sum(), (turn(x, 7) * y).sum())
        assert torch.equal(turn(x, 0), x)


def test_sample_row_by_hand():
    x = torch.tensor([1.0, 3.0, 2.0, 3.0, 0.0]).log()                      # weights 1, 3, 2, 3 and none
    p, t = R.sample_row(x, us=[0.0, 0.111, 0.112, 0.5, 0.7, NEAR_1])
    assert torch.allclose(p, torch.tensor([1.0, 3, 2, 3, 0]).double() / 9) and t == [0, 0, 1, 2, 3, 3]
    assert R.sample_row(x, top_k=1)[0].tolist() == [0, 1, 0, 0, 0]           # of equal logits the first
    assert R.sample_row(x, T=0.0, us=[0.9])[1] == [1]
    assert (R.sample_row(x, top_p=0.5)[0] > 0).tolist() == [False, True, False, True, False]        # 3 of 9 is less than half, 6 is not
    assert (R.sample_row(x, min_p=0.5)[0] > 0).tolist() == [False, True, True, True, False]
    assert (R.sample_row(x, top_k=3, top_p=0.7)[0] > 0).tolist() == [False, True, False, True, False]   # 6 of the 8 that are left
    p, t = R.sample_row(x, us=[0.4, 0.4, 0.4, 0.4, 0.4], distinct=True)
    assert t == [1, 2, 3, 0, -1]                                            # of 9: 3.6 -> 1; of 1 2 3: 2.4 -> 2; of 1 3: 1.6 -> 3
    assert R.sample_row(torch.full((3,), -math.inf), us=[0.5]) [1] == [-1]


NEAR_1 = 1 - 2.0 ** -24


# ------------------------------------------------------------------------------------------------ refusals
def _view(branching=(4, 2, 2, 1), device=None):
    m = b.build_mask(branching)
    v = b.slice_mask(m, len(branching))
    copy = b.MaskView()
    C.memmove(C.byref(copy), C.byref(v), C.sizeof(v))
    copy._owner = m
    if not copy.bits_dev:
        copy.bits_dev = 256                                # so that a machine without a GPU gets to the other checks
    if device is not None:
        copy.device = device
    return copy


def _attn(view=None, **kw):
    a = dict(B=1, H=16, dl=512, dr=64, row=0, q=ONE, tree=ONE, ns=44, prefix=ONE, base=ONE, lens=ONE, mp=1000, scale=0.1, out=ONE, ws=None, bytes=0)
    a.update(kw)
    v = _view() if view is None else view
    return b.lib.mcsd_tree_attention_latent(C.byref(v) if v else None, a["B"], a["H"], a["dl"], a["dr"], a["row"], a["q"], a["tree"], a["ns"], a["prefix"], a["base"], a["lens"],
                                            a["mp"], a["scale"], a["out"], a["ws"], a["bytes"], None)


@pytest.mark.parametrize("wrong", [dict(q=None), dict(tree=None), dict(out=None), dict(base=None), dict(lens=None), dict(prefix=None), dict(B=0), dict(B=65536), dict(H=0), dict(H=65536),
                                   dict(ns=43), dict(row=-1), dict(row=44), dict(mp=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf), dict(scale=math.nan),
                                   dict(q=C.c_void_p(264)), dict(tree=C.c_void_p(258)), dict(prefix=C.c_void_p(264)), dict(out=C.c_void_p(260))])
def test_attention_refuses(wrong):
    assert _attn(**wrong) == b.MCSD_EINVAL


def test_attention_refuses_sizes():
    for dl, dr in ((512, 32), (256, 64), (128, 64), (576, 64), (0, 0), (512, 0)):
        assert _attn(dl=dl, dr=dr) == b.MCSD_EUNSUPPORTED
        assert b.tree_attention_latent_workspace(1, 16, dl, dr, 44, 0, 1000) == 0
    assert _attn(view=_view((64, 2)), ns=200) == b.MCSD_EUNSUPPORTED          # 192 nodes
    assert _attn(view=_view(device=99)) == b.MCSD_EINVAL                      # (or no device here)
    assert b.lib.mcsd_tree_attention_latent(None, 1, 16, 512, 64, 0, ONE, ONE, 44, ONE, ONE, ONE, 1000, 0.1, ONE, None, 0, None) == b.MCSD_EINVAL
    for wrong in ((0, 16, 512, 64, 44, 0, 1000), (1, 0, 512, 64, 44, 0, 1000), (1, 16, 512, 64, 0, 0, 1000), (1, 16, 512, 64, 129, 0, 1000), (1, 16, 512, 64, 44, 44, 1000),
                  (1, 16, 512, 64, 44, -1, 1000), (1, 16, 512, 64, 44, 0, -1)):
        assert b.tree_attention_latent_workspace(*wrong) == 0


def test_workspace_of_smaller_calls():
    """The size for a call serves calls with fewer nodes, rows or prefix keys."""
    for B, H in ((1, 1), (1, 128), (7, 16), (64, 16), (300, 4)):
        for dl, dr in ((512, 64), (256, 32)):
            most = b.tree_attention_latent_workspace(B, H, dl, dr, 60, 0, 5000)
            for n, row, L in ((60, 30, 5000), (60, 59, 5000), (1, 0, 5000), (44, 0, 5000), (60, 0, 100), (60, 0, 0), (13, 3, 2500)):
                assert b.tree_attention_latent_workspace(B, H, dl, dr, n, row, L) <= most


def _rope(**kw):
    r = b.Rope(64, 0, 1e-6, 256, None, 256)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def _rows(tree, view=None, rope=None, **kw):
    a = dict(dtype=1, B=1, H=16, dl=512, dr=64, row=0, rows=10, q=ONE, kv=ONE, qb=4096, qr=1024, qh=64, kvb=8192, kvr=576, first=ONE, n=ONE, mp=1000, qo=ONE, out=ONE, ns=44, base=ONE, cap=100)
    a.update(kw)
    r = _rope() if rope is None else rope
    if tree:
        v = _view() if view is None else view
        return b.lib.mcsd_tree_latent_norm_rope(C.byref(v), a["dtype"], a["B"], a["H"], a["dl"], a["dr"], a["row"], a["q"], a["kv"], a["qb"], a["qr"], a["qh"], a["kvb"], a["kvr"],
                                                C.byref(r), a["first"], a["mp"], a["qo"], a["out"], a["ns"], None)
    return b.lib.mcsd_store_latent(a["dtype"], a["B"], a["dl"], a["dr"], a["rows"], a["kv"], a["kvb"], a["kvr"], C.byref(r), a["first"], a["n"], a["out"], a["base"], a["cap"], None)


@pytest.mark.parametrize("tree", [True, False])
@pytest.mark.parametrize("wrong", [dict(dtype=2), dict(B=0), dict(B=65536), dict(kv=None), dict(out=None), dict(first=None), dict(kvb=-8), dict(kvr=4), dict(kv=C.c_void_p(264)), dict(out=C.c_void_p(258)),
                                   dict(rope=_rope(eps=-1.0)), dict(rope=_rope(eps=math.nan)), dict(rope=_rope(eps=math.inf)), dict(rope=_rope(rotary_dim=8)), dict(rope=_rope(rotary_dim=80)),
                                   dict(rope=_rope(rotary_dim=-16)), dict(rope=_rope(inv_freq=None)), dict(rope=_rope(q_weight=256)), dict(rope=_rope(k_weight=260))])
def test_rows_refuse(tree, wrong):
    assert _rows(tree, **wrong) == b.MCSD_EINVAL


@pytest.mark.parametrize("wrong", [dict(q=None), dict(qo=None), dict(H=0), dict(H=65536), dict(row=44), dict(row=-1), dict(ns=43), dict(mp=-1), dict(qb=-8), dict(qr=12), dict(qh=4), dict(q=C.c_void_p(8)),
                                   dict(qo=C.c_void_p(8))])
def test_tree_rows_refuse(wrong):
    assert _rows(True, **wrong) == b.MCSD_EINVAL


@pytest.mark.parametrize("wrong", [dict(n=None), dict(base=None), dict(rows=-1), dict(cap=-1)])
def test_prompt_rows_refuse(wrong):
    assert _rows(False, **wrong) == b.MCSD_EINVAL


def test_rows_refuse_sizes():
    for tree in (True, False):
        for dl, dr in ((512, 32), (256, 64), (128, 64)):
            assert _rows(tree, dl=dl, dr=dr, rope=_rope(rotary_dim=32)) == b.MCSD_EUNSUPPORTED
        assert _rows(tree, dl=256, dr=32) == b.MCSD_EINVAL                     # 64 rotated channels of 32
    assert _rows(False, rows=2 ** 24) == b.MCSD_EUNSUPPORTED
    t = torch.zeros(8)
    for call in (lambda r: b.tree_latent_norm_rope(_view(), 0, 1, 1, 512, 64, 0, t, t, 0, 0, 0, 0, 0, r, t, 8, t, t, 44, NoStream),
                 lambda r: b.store_latent(0, 1, 512, 64, 1, t, 0, 0, r, t, t, t, t, 8, NoStream)):
        with pytest.raises(b.McsdError) as e:
            call(b.make_rope(0, None, None, torch.ones(256)))                  # a weight per channel: 256 do not serve 512
        assert e.value.status == b.MCSD_EINVAL


class NoStream:
    cuda_stream = 0


SAMPLER = b.Sampler()


def _sample(sampler=SAMPLER, **kw):
    a = dict(dtype=1, B=2, W=3, V=1000, x=ONE, bs=3000, rs=1000, probs=ONE, pbs=3000, scheme=0, n=2, u=ONE, tokens=ONE, tbs=6)
    a.update(kw)
    return b.lib.mcsd_sample_rows(a["dtype"], a["B"], a["W"], a["V"], a["x"], a["bs"], a["rs"], C.byref(sampler) if sampler else None, a["probs"], a["pbs"], a["scheme"], a["n"], a["u"], a["tokens"],
                                  a["tbs"], None)


@pytest.mark.parametrize("wrong", [dict(sampler=None), dict(dtype=2), dict(B=0), dict(B=65536), dict(W=0), dict(V=0), dict(x=None), dict(probs=None, n=0), dict(bs=-1), dict(rs=-1), dict(pbs=2999),
                                   dict(scheme=2), dict(n=-1), dict(u=None), dict(tokens=None), dict(tbs=5), dict(x=C.c_void_p(257)), dict(x=C.c_void_p(258), dtype=0), dict(probs=C.c_void_p(258)),
                                   dict(u=C.c_void_p(258)), dict(tokens=C.c_void_p(258))])
def test_sample_refuses(wrong):
    assert _sample(**wrong) == b.MCSD_EINVAL


def test_sample_refuses_sizes():
    assert _sample(V=262145, pbs=3 * 262145) == b.MCSD_EUNSUPPORTED
    assert _sample(n=65, tbs=195) == b.MCSD_EUNSUPPORTED
    assert _sample(W=2 ** 22, pbs=2 ** 40, tbs=2 ** 30) == b.MCSD_EUNSUPPORTED


def test_samplers():
    with pytest.raises(b.McsdError):
        b.make_sampler(torch.ones(4, dtype=torch.float64))
    with pytest.raises(b.McsdError):
        b.make_sampler(top_k=torch.ones(4))
    with pytest.raises(b.McsdError):
        b.make_sampler(torch.ones(8)[::2])
    t = torch.zeros(8)
    with pytest.raises(b.McsdError) as e:                    # settings of three sequences for four
        b.sample_rows(0, 4, 1, 2, t, 2, 2, b.make_sampler(torch.ones(3)), t, 2, 0, 0, None, None, 0, NoStream)
    assert e.value.status == b.MCSD_EINVAL
    with pytest.raises((C.ArgumentError, TypeError)):
        b.sample_rows(0, 1, 1, 2, t, 2, 2, b.Mlp(), t, 2, 0, 0, None, None, 0, NoStream)
