"""The largest calls that the entry points around the 4-bit cache document, and the refusal of the next larger ones (no GPU needed:
a call that is refused launches nothing)."""
import pytest
import torch

from paper_2409_10644_amd import binding as b
from test_fp4_reference import NoStream, _load, _qk, _store, _view

LANES = 2 ** 32                                            # of a launch, in one direction: fewer than that


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H", [1, 3, 128])
def test_rows_beyond_a_launch_are_refused(d, H):
    """Eight channels per lane, whole workgroups of 256 lanes."""
    per_wg = 256 // (d // 8)
    most = (LANES // 256 - 1) * per_wg // H
    for rows in (most + 1, (2 ** 31 - 1) // H):
        assert _store(d=d, H=H, rows=rows) == b.MCSD_EUNSUPPORTED, rows
        assert _load(d=d, H=H, rows=rows) == b.MCSD_EUNSUPPORTED, rows


@pytest.mark.parametrize("wrong", [dict(bs=0), dict(hs=0), dict(rs=0), dict(rs=120), dict(hs=64), dict(bs=8)])
def test_rows_are_not_read_into_one_place(wrong):
    """An expanded tensor can be stored from, not loaded into; with one of a kind its stride says nothing."""
    assert _load(**wrong) == b.MCSD_EINVAL
    assert _load(B=1, H=1, rows=1, bs=0, hs=0, rs=0, layers=65) == b.MCSD_EUNSUPPORTED           # (refused for the layers alone)
    assert _store(bs=0, hs=0, rs=0, d=32) == b.MCSD_EUNSUPPORTED                                 # (for d alone)


@pytest.mark.parametrize("Hq,Hkv", [(4, 2), (32, 8), (1, 1)])
def test_prompts_beyond_a_launch_are_refused(Hq, Hkv):
    """Four rows per workgroup where one would be too many workgroups."""
    most = 4 * (LANES // 256 - 1)
    for rows in (most + 1, 2 ** 31 - 1):
        assert _qk(False, Hq=Hq, Hkv=Hkv, rows=rows, out=rows) == b.MCSD_EUNSUPPORTED, rows


@pytest.mark.parametrize("short", ["q", "k", "both"])
def test_norm_weights_shorter_than_a_head_are_refused(short):
    """The kernel reads a weight per channel: 64 of them do not serve heads of 128."""
    t, weight = torch.zeros(128), torch.ones(64)
    rope = b.make_rope(64, torch.zeros(32), t if short == "k" else weight, t if short == "q" else weight)
    view = _view()
    for call in (lambda: b.tree_qk_norm_rope(view, 0, 1, 1, 1, 128, 0, t, t, None, 0, 0, 0, 0, rope, t, 8, t, t, None, 44, NoStream),
                 lambda: b.prompt_qk_norm_rope(0, 1, 1, 1, 128, 1, t, t, None, 0, 0, 0, 0, rope, t, t, t, t, None, 44, NoStream)):
        with pytest.raises(b.McsdError) as e:
            call()
        assert e.value.status == b.MCSD_EINVAL
