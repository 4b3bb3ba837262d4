"""How far updates are off: no further than the roundings that the library
states make them (tests/muon_rounded_ref.py), on matrices that need the
diagonals' and the rests' bits, also of low rank."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2509_03047_amd import flashrestore as F  # noqa: E402

from tests import muon_ref as R  # noqa: E402
from tests import muon_rounded_ref as M  # noqa: E402
from tests.gpu_util import log  # noqa: E402
from tests.test_gpu_muon import Dev  # noqa: E402
from tests.test_muon_steps_cpu import MARGIN  # noqa: E402

MIXED = [(3.4445, -4.775, 2.0315), (2.0, -1.5, 0.5)] * 4


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def updates(matrices, coeffs=None):
    s = R.Matrices([d.shape for _, d in matrices], F.FR_F32, seed=41)
    for k, (_, d) in enumerate(matrices):
        s.set_grad(k, d)
    u = Dev(s, coeffs=coeffs).orthogonalized()
    return [s.update(k, u) for k in range(len(matrices))]


@pytest.mark.parametrize("coeffs", [None, MIXED], ids=["five", "mixed"])
def test_errors_are_those_of_the_stated_roundings(coeffs):
    steps = R.STEPS if coeffs is None else coeffs
    worst = []
    for (name, d), u in zip(M.MATRICES, updates(M.MATRICES, coeffs)):
        want = M.exact(name, d, steps)
        have, most = M.beyond_rounding(u, want), M.allowed(d, want, steps)
        log(name, f"off {M.off(u, want):.2e}, beyond bf16 {have:.2e} of {most:.2e}")
        if not have <= most:
            worst.append((name, have, most))
    assert not worst


@pytest.mark.parametrize("kind", list(M.KINDS))
def test_stated_accuracy(kind):
    most, ds = M.KINDS[kind]
    offs = [M.off(u, R.orthogonalized(d)) for d, u in zip(ds, updates([(kind, d) for d in ds]))]
    log(kind, f"{min(offs):.2e} to {max(offs):.2e}")
    assert max(offs) <= most, [d.shape for d, e in zip(ds, offs) if e > most]


def test_steps_with_little_room_near_rank_one():
    """Steps that start with a slope of 8 and are accepted."""
    low = [(n, d) for n, d in M.MATRICES if n.startswith("rank 1")]
    for (name, d), u in zip(low, updates(low, MARGIN)):
        want = M.exact(name, d, MARGIN)
        log(name, f"{M.off(u, want):.2e}")
        # the top value's own rounding, which varies with the order of sums, is passed on by slopes of up to 12: to 0.12
        # were it half a step of fp16 each time; a mean over 64 elements or more leaves an eighth of that at most
        assert M.off(u, want) <= 0.12 / 8, name


def test_whole_matrices_of_a_layer():
    """Not a rank's shares: matrices of 4,096 x 14,336 either way up, and square."""
    shapes = [(4096, 14336), (14336, 4096), (4096, 4096)]
    t, rows, ab, gb, ub = F.fr_muon_state_table(shapes)
    opt = F.Muon(F.Plan(t, 1 << 20, ab, ab), rows, 1, gb, ub)
    gen = torch.Generator(device="cuda").manual_seed(42)
    grads = (torch.randn(gb // 2, generator=gen, device="cuda") * 1e-3).to(torch.bfloat16)
    u = opt.empty_updates()
    opt.orthogonalize(grads.view(torch.uint8), torch.from_numpy(F.muon_hyper([dict(lr=0.0)]).view(np.uint8)).cuda(), u)
    for k, (a, b) in enumerate(shapes):
        x = grads[int(rows[k]["grad_offset"]) // 2:][: a * b].view(a, b).double()
        got = u[int(rows[k]["update_offset"]):][: 2 * a * b].view(torch.bfloat16).view(a, b)
        x = x.t().contiguous() if a > b else x
        got = (got.t().contiguous() if a > b else got).double()
        x = x / (torch.linalg.norm(x) + 1e-7)
        for ca, cb, cc in np.asarray(R.STEPS, np.float32).astype(np.float64).tolist():
            m = x @ x.t().contiguous()
            x = ca * x + (cb * m + cc * (m @ m)) @ x
        e = float(torch.linalg.norm(got - x) / torch.linalg.norm(x))
        log((a, b), f"{e:.2e}")
        assert e <= M.KINDS["spread"][0], (a, b)
