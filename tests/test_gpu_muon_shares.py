"""Ranks that share the orthogonalisation: each has an optimizer of some of the
matrices and one of all for the step; the updates are what they exchange.  One
optimizer of all gives the same state, bit for bit."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2509_03047_amd import flashrestore as F  # noqa: E402

from tests import muon_ref as R  # noqa: E402
from tests.gpu_util import sums_host, to_dev, to_host  # noqa: E402
from tests.test_gpu_muon import Dev, hyper_dev  # noqa: E402

SHAPES = [(200, 300), (64, 64), (1, 77), (300, 200), (0, 3), (128, 2048), (513, 130)]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("dtype", [F.FR_BF16, F.FR_F32])
@pytest.mark.parametrize("ranks", [2, 3])
def test_ranks_share_the_products(dtype, ranks):
    s = R.Matrices(SHAPES, dtype, seed=51, shuffle=True)
    h = hyper_dev(F.muon_hyper([dict(lr=3e-3, weight_decay=0.1)]))
    one = Dev(s)
    whole = one.plan.empty_sums().fill_(-1)
    one.opt.direction(one.state, one.grads, h, one.updates, None, whole)
    one.opt.apply(one.state, one.updates, h, None, whole)
    torch.cuda.synchronize()

    share = [np.arange(len(SHAPES)) % ranks == r for r in range(ranks)]
    plans = [F.Plan(s.table, 4096, s.arena_bytes, s.arena_bytes) for _ in range(ranks)]
    states, updates, sums, opts = [], [], [], []  # (optimizers live until their work is done)
    for plan, mine in zip(plans, share):
        opt = F.Muon(plan, s.rows[mine], 1, s.grad_bytes, s.update_bytes)  # (updates keep their places)
        opts.append(opt)
        states.append(to_dev(s.arena))
        updates.append(opt.empty_updates().zero_())
        sums.append(plan.empty_sums().fill_(-1))
        opt.direction(states[-1], to_dev(s.grads), h, updates[-1], None, sums[-1])
    torch.cuda.synchronize()
    both = torch.stack(updates).sum(0, dtype=torch.uint8)  # an all-gather: each byte has one writer
    assert np.array_equal(to_host(both)[: s.update_bytes], np.where(outside(s), 0, to_host(one.updates)[: s.update_bytes]))
    for plan, mine, state, out in zip(plans, share, states, sums):
        every = F.Muon(plan, s.rows, 1, s.grad_bytes, s.update_bytes)
        every.apply(state, both, h, None, out)
        torch.cuda.synchronize()
        got = to_host(state)
        for k in range(len(SHAPES)):
            for name in ("param", "master") + (("m",) if mine[k] else ()):
                assert np.array_equal(s.raw(k, name, got), s.raw(k, name, to_host(one.state))), (k, name)
            if not mine[k]:  # its momentum is another rank's
                assert np.array_equal(s.raw(k, "m", got), s.raw(k, "m"))
        # sums of what this rank wrote are those of the whole step
        a, b = (sums_host(x, plan.n_chunks).reshape(-1, 2) for x in (out, whole))
        _, _, base = F.fr_layout_query(s.table, 4096, s.arena_bytes, s.arena_bytes)
        for k in range(len(SHAPES)):
            for name in ("param", "master", "m"):
                at = slice(int(base[int(s.rows[k][name])]), int(base[int(s.rows[k][name]) + 1]))
                if name != "m" or mine[k]:
                    assert np.array_equal(a[at], b[at]), (k, name)
                else:
                    assert (a[at] == np.uint64((1 << 64) - 1)).all()


def outside(s):
    """The bytes of an update arena that belong to no matrix."""
    left = np.ones(s.update_bytes, bool)
    for k, (a, b) in enumerate(s.shapes):
        o = int(s.rows[k]["update_offset"])
        left[o:o + 2 * a * b] = False
    return left
