"""The largest calls that the entry points around the 4-bit cache document, and the refusal of the next larger ones (no GPU needed:
a call that is refused launches nothing)."""
import pytest

from paper_2409_10644_amd import binding as b
from test_fp4_reference import _load, _qk, _store

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


@pytest.mark.parametrize("Hq,Hkv", [(4, 2), (32, 8), (1, 1)])
def test_prompts_beyond_a_launch_are_refused(Hq, Hkv):
    """Four rows per workgroup where one would be too many workgroups."""
    most = 4 * (LANES // 256 - 1)
    for rows in (most + 1, 2 ** 31 - 1):
        assert _qk(False, Hq=Hq, Hkv=Hkv, rows=rows, out=rows) == b.MCSD_EUNSUPPORTED, rows
