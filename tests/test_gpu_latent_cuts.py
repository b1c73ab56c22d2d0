"""Attention over a latent cache around the longest units that stay whole, and where all of a batch's units are whole, some are cut or all
are planned: the outputs are the definition's, and sequences shorter than the longest are theirs whatever the others are."""
import pytest
import torch

from test_gpu_latent_attention import SIZES, Call, binding  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dl,dr", SIZES)
@pytest.mark.parametrize("branching,H,lens", [
    ((1,), 16, (480, 1, 0, 33)), ((1,), 16, (481, 1, 0, 33)), ((1,), 16, (320, 319)), ((4, 2, 2, 1), 16, (448, 449, 3, 0, 100, 200, 31, 32)),
    ((2, 2, 2), 128, (448, 20)), ((2, 2, 2), 128, (449, 480)), ((8, 2, 2, 1, 1), 8, tuple(range(0, 480, 32))), ((4, 2, 2, 1), 128, (95, 96, 97)),
    ((2, 2), 64, tuple(range(3, 303, 6)))])
def test_around_the_cut(binding, dl, dr, branching, H, lens):  # noqa: F811
    c = Call(binding, branching, H, dl, dr, lens)
    want = c.check()
    for _ in range(2):
        c.out.fill_(9)
        c.call()
        torch.cuda.synchronize()
        assert torch.equal(c.out, want)


def test_more_sequences_than_lanes_stay_whole(binding):  # noqa: F811
    """A workgroup for every unit, the sequences' lengths read 64 at a time."""
    Call(binding, (2, 2), 16, 256, 32, tuple((37 * i) % 130 for i in range(130))).check()


@pytest.mark.parametrize("dl,dr", SIZES)
@pytest.mark.parametrize("branching,H", [((1,), 16), ((1,), 17), ((2, 2), 2), ((2, 2), 3), ((3, 1), 1), ((4, 2, 2), 1), ((8,), 2), ((17,), 1)])
@pytest.mark.parametrize("lens,gain", [((0, 33, 700), 1.0), ((3000, 1), 8.0), ((95, 96, 97, 31), 30.0)])
def test_around_16_rows(binding, dl, dr, branching, H, lens, gain):  # noqa: F811
    """The variant for 16 rows and the other; large scores move the references."""
    Call(binding, branching, H, dl, dr, lens, gain=gain).check()
