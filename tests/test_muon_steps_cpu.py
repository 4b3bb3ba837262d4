"""Which steps an orthogonalised update may take: polynomials that the kernels'
roundings do not carry away (CPU)."""
import numpy as np
import pytest

from paper_2509_03047_amd import flashrestore as F

INVAL = -1
# Fast steps made for singular values up to 1 and no further: a value of 1 + 2^-10 leaves them behind.
TIGHT = [(8.2872, -23.5959, 17.3004), (4.1071, -2.9478, 0.5448), (3.9487, -2.9089, 0.5518), (3.3184, -2.4885, 0.5100),
         (2.3007, -1.6689, 0.4188)]
MARGIN = [(a / 1.01, b / 1.01 ** 3, c / 1.01 ** 5) for a, b, c in TIGHT]  # the same with room for 1 %


def accepted(coeffs):
    t, r, ab, gb, ub = F.fr_muon_state_table([(20, 30)])
    try:
        F.fr_muon_query(t, 4096, ab, r, 1, gb, ub, coeffs)
        return True
    except F.FlashRestoreError as e:
        assert e.status == INVAL
        return False


def largest(coeffs, top):
    """The largest value on the way of those that start in [0, top]."""
    s, most = np.linspace(0, top, 4097), 0.0
    with np.errstate(over="ignore", invalid="ignore"):
        for a, b, c in coeffs:
            s = a * s + b * s ** 3 + c * s ** 5
            most = max(most, float(np.abs(s).max()))
    return most


def growth(coeffs):
    """How much a small change of a singular value in [0, 1] can come to, after the steps that follow it."""
    s = np.linspace(0, 1, 1 << 16)
    g = worst = np.ones_like(s)
    for a, b, c in coeffs:
        g = np.maximum(g * np.abs(a + 3 * b * s ** 2 + 5 * c * s ** 4), 1.0)
        s = a * s + b * s ** 3 + c * s ** 5
        worst = np.maximum(worst, g)
    return float(worst.max())


@pytest.mark.parametrize("coeffs", [TIGHT, [(2.0, -7.5, 6.5)] * 5, TIGHT[:3]])
def test_steps_that_only_exact_values_keep_to_are_refused(coeffs):
    """In [0, 1] they stay within 4, and with what fp16 rounds by on the way they do not."""
    assert largest(coeffs, 1.0) <= 4 and largest(coeffs, 1 + 2.0 ** -9) > 4
    assert not accepted(coeffs)


def test_steps_that_pass_roundings_on_without_end_are_refused():
    """Inside [-1, 1] all the way, but each step tears neighbours apart."""
    coeffs = [(2.9, -3.8, 0.0)] * 16
    assert largest(coeffs, 1 + 2.0 ** -9) <= 1.01 and growth(coeffs) > 2.0 ** 14
    assert not accepted(coeffs)


@pytest.mark.parametrize("coeffs", [
    None, MARGIN, MARGIN[:4] + TIGHT[4:], [(3.4445, -4.775, 2.0315)] * 5, [(3.4445, -4.775, 2.0315)] * 16,
    [(1.875, -1.25, 0.375)] * 16, [(4.0, 0.0, 0.0)], [(0.0, 0.0, 0.0)], [(8.5, -34.0, 27.2), (8.8235, -12.2125, 3.3806)]])
def test_steps_with_room_are_taken(coeffs):
    assert accepted(coeffs)
