"""What the GPU tests of updates' accuracy can tell (CPU): the model of the stated
roundings is as accurate as the header says, and without the diagonals, or with
fewer bits in the rests, it leaves what those tests allow."""
import numpy as np
import pytest

from tests import muon_ref as R
from tests import muon_rounded_ref as M

OF_DIAGONALS = ["noise 128 x 2048", "noise 2100 x 300", "orthogonal 64 x 64", "orthogonal 100 x 260",
                "orthogonal 300 x 2100", "rank 1 of one large element, 64 x 4100"]
OF_RESTS = ["rank 1, 100 x 300", "rank 1, 300 x 2100", "rank 1 in noise, 257 x 129",
            "rank 1 of one large element, 64 x 4100", "rank 4, 128 x 128"]


@pytest.mark.parametrize("kind", list(M.KINDS))
def test_stated_accuracy(kind):
    most, ds = M.KINDS[kind]
    assert max(M.off(M.rounded(d), R.orthogonalized(d)) for d in ds) <= most


@pytest.mark.parametrize("name,d", M.MATRICES, ids=[n for n, _ in M.MATRICES])
def test_mistakes_are_seen(name, d):
    want = M.exact(name, d)
    most = M.allowed(d, want)
    assert M.beyond_rounding(M.rounded(d), want) <= most
    assert name in OF_DIAGONALS + OF_RESTS
    if name in OF_DIAGONALS:
        assert M.beyond_rounding(M.rounded(d, diagonals=False), want) > most
    if name in OF_RESTS:
        for bits in (0, 4):
            assert M.beyond_rounding(M.rounded(d, bits=bits), want) > most


def test_matrices_reach_both_ways_of_the_first_steps():
    ways = {M.two_as_one(min(d.shape), max(d.shape)) for n, d in M.MATRICES if n in OF_DIAGONALS}
    assert ways == {False, True}


def test_rests_hold_eight_bits():
    rng = np.random.default_rng(33)
    v = (rng.standard_normal(100000) * np.exp2(rng.integers(-13, 12, 100000))).astype(np.float32)
    v = v[np.abs(v) >= 2.0 ** -14]
    h = M.f16(v)
    # half a step of 2^-8 of fp16's 2^-10; next to the middle of two fp16 numbers a whole one
    assert (np.abs(h + M.rest8(v, h) - v) <= np.abs(v) * 2.0 ** -18).all()
    assert np.median(np.abs(h + M.rest8(v, h) - v) / np.abs(v)) <= 2.0 ** -20
