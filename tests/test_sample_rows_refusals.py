"""What mcsd_sample_rows refuses, with logits and probabilities at places of their own (no GPU needed: a call that is refused launches
nothing)."""
import ctypes as C

import pytest

from paper_2409_10644_amd import binding as b
from test_latent_reference import _sample

X, PROBS, U, TOKENS = (C.c_void_p(at) for at in (4096, 8192, 12288, 16384))      # never dereferenced


def _apart(**kw):
    return _sample(**{**dict(x=X, probs=PROBS, u=U, tokens=TOKENS), **kw})


@pytest.mark.parametrize("wrong", [dict(sampler=None), dict(dtype=2), dict(B=0), dict(B=65536), dict(W=0), dict(V=0), dict(x=None), dict(probs=None, n=0), dict(bs=-1), dict(rs=-1), dict(pbs=2999),
                                   dict(scheme=2), dict(n=-1), dict(u=None), dict(tokens=None), dict(tbs=5), dict(x=C.c_void_p(257)), dict(x=C.c_void_p(258), dtype=0), dict(probs=C.c_void_p(258)),
                                   dict(u=C.c_void_p(258)), dict(tokens=C.c_void_p(258))])
def test_refuses(wrong):
    assert _apart(**wrong) == b.MCSD_EINVAL


def test_refuses_sizes():
    assert _apart(V=262145, pbs=3 * 262145) == b.MCSD_EUNSUPPORTED
    assert _apart(n=65, tbs=195) == b.MCSD_EUNSUPPORTED
    assert _apart(W=2 ** 22, pbs=2 ** 40, tbs=2 ** 30) == b.MCSD_EUNSUPPORTED


@pytest.mark.parametrize("dtype", [0, 1])
def test_refuses_probabilities_in_the_place_of_the_logits(dtype):
    assert _apart(dtype=dtype, probs=X) == b.MCSD_EINVAL
