"""Optimizers and states that look right by their sizes alone and are not (CPU)."""
import numpy as np
import pytest

from paper_2509_03047_amd import flashrestore as F

INVAL, RANGE = -1, -3


def _status(t, r, ab, gb, C=4096):
    try:
        F.fr_adamw_query(t, C, ab, r, 1, gb)
        return 0
    except F.FlashRestoreError as e:
        return e.status


@pytest.mark.parametrize("bits", [32, 8])
def test_a_parameter_is_derived_from_its_own_master(bits):
    """A restore derives a parameter from the master that the table names; a step that wrote it from another one
    would leave a state that its restored copy differs from."""
    t, r, ab, gb = F.fr_adamw_state_table([300, 300], bits)
    assert _status(t, r, ab, gb) == 0
    swapped = r.copy()
    swapped["param"] = r["param"][::-1]
    assert _status(t, swapped, ab, gb) == INVAL
    swapped = r.copy()
    swapped["master"] = r["master"][::-1]
    assert _status(t, swapped, ab, gb) == INVAL
    one = r[:1].copy()
    one["param"] = r["param"][1]  # the other tensor, which no step writes
    assert _status(t, one, ab, gb) == INVAL
    one["param"] = -1  # an image that the caller brings up to date
    assert _status(t, one, ab, gb) == 0
    plain = t.copy()
    plain["derive_from"] = -1  # images that are sent, not derived: any master's
    assert _status(plain, r, ab, gb) == 0
    swapped = r.copy()
    swapped["param"] = r["param"][::-1]
    assert _status(plain, swapped, ab, gb) == 0


def test_a_moment_in_the_masters_place():
    """The master's index names a moment's entry of the same size and the moment's the master's."""
    for numel in (300, 0):  # (an empty parameter has nothing to differ in)
        t, r, ab, gb = F.fr_adamw_state_table([numel], 32)
        r["master"], r["m"] = int(r["m"][0]), int(r["master"][0])
        assert _status(t, r, ab, gb) == (INVAL if numel else 0)


def test_states_whose_sizes_pass_64_bits():
    """5,000 tensors of 2^48 elements are 2e19 bytes of state: refused, where the sum wrapped around 2^64 before."""
    with pytest.raises(F.FlashRestoreError) as ei:
        F.fr_adamw_state_table([1 << 48] * 5000)
    assert ei.value.status == RANGE
    for bits in (32, 8):
        n = 1 << 10  # 2^58 elements in all are the most
        t, r, ab, gb = F.fr_adamw_state_table([1 << 48] * n, bits, F.FR_F32)
        size = (2 + 4 + 4 + 4) << 48 if bits == 32 else (2 + 4 + 1 + 1) * (1 << 48) + 2 * ((1 << 48) // 256 * 4)
        assert ab == n * size and gb == n * (4 << 48)
        assert int(t[-1]["src_offset"]) < ab and int(r[-1]["grad_offset"]) == (n - 1) * (4 << 48)
        with pytest.raises(F.FlashRestoreError) as ei:
            F.fr_adamw_state_table([1 << 48] * n + [1], bits, F.FR_F32)
        assert ei.value.status == RANGE
    with pytest.raises(F.FlashRestoreError) as ei:
        F.fr_adamw_state_table([(1 << 48) + 1])
    assert ei.value.status == RANGE


def test_hyperparameters_of_no_step():
    """Steps count from 1: the corrections of step 0 would be 0, and a step would divide by them."""
    for step in (0, -1, np.int64(0)):
        with pytest.raises(ValueError, match="step"):
            F.adamw_hyper([dict(lr=1e-3)], step)
    h = F.adamw_hyper([dict(lr=1e-3)], 1)
    assert h[0]["bias1"] == np.float32(1 - 0.9) and h[0]["bias2"] == np.float32(1 - 0.999)
