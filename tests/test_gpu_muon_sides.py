"""Which tiles the products take, told by the optimizer's device memory: large
ones where matrices fill them, and never for lists of small or narrow ones."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2509_03047_amd import flashrestore as F  # noqa: E402

from tests.test_gpu_muon import LARGE  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def scratch(shapes, side):
    """Bytes of X twice, its rest, three squares and their diagonals, sides rounded up."""
    total = 0
    for a, b in shapes:
        if a and b:
            m, n = (-(-x // side) * side for x in sorted((a, b)))
            total += 5 * m * n + 6 * m * m + 12 * m
    return total


def lists(shapes):
    """At most so many bytes of lists lie beside the scratch: for each tile of 64 x 64 208 in four of them and some 150 of
    places, parts of sums and folds for 4,096 elements; for each matrix 192 + 96 that describe it and as much again."""
    return 1024 * sum(-(-a // 64) * -(-b // 64) for a, b in shapes) + 512 * len(shapes) + (1 << 16)


def device_bytes(shapes):
    t, r, ab, gb, ub = F.fr_muon_state_table(shapes)
    opt = F.Muon(F.Plan(t, 1 << 16, ab, ab), r, 1, gb, ub)
    used = opt.info["device_bytes"]
    opt.destroy()
    return used


@pytest.mark.parametrize("shapes", [
    [(8, 8)] * 300, [(64, 64)] * 300, [(16, 4096)] * 20, [(4096, 16)] * 64, [(128, 4096)] * 64, [(320, 320)] * 80,
    [(512, 512)] + [(64, 64)] * 400, [(2048, 2048)] * 4 + [(64, 64)] * 1500, [(1, 3000)] * 300])
def test_small_and_narrow_matrices_take_small_tiles(shapes):
    """(Tiles of 256 x 256 need 1.5 to 64 times the multiplications.)"""
    assert device_bytes(shapes) <= scratch(shapes, 64) + lists(shapes) < scratch(shapes, 256)


@pytest.mark.parametrize("shapes", [
    LARGE, [(512, 4096), (128, 4096), (128, 4096), (4096, 512), (1792, 4096), (4096, 1792)] * 4, [(1100, 2100)] * 8,
    [(1100, 1100)] * 14, [(1500, 1500)] * 8 + [(2, 4000)] * 8])
def test_matrices_that_fill_them_take_large_tiles(shapes):
    assert device_bytes(shapes) >= scratch(shapes, 256) > scratch(shapes, 64) + lists(shapes)
