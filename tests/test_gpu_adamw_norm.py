"""The gradient norm on the GPU where its form changes or a number leaves its
range."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2509_03047_amd import flashrestore as F  # noqa: E402

from tests import adamw_ref as R  # noqa: E402
from tests.test_gpu_adamw import Dev, _gpu, hyper_dev, same_floats, two_groups  # noqa: E402, F401


def stats_of(d):
    """(sum_sq, norm, scale, nonfinite)"""
    f = d.stats.view(torch.float32).cpu().numpy()
    return float(d.stats[0]), f[2], f[3], int(d.stats.view(torch.int64)[2])


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("max_norm", [1.0, 0.25, 3e38, np.inf])
def test_a_norm_past_32_bits_of_finite_gradients(bits, max_norm):
    """Four gradients of 3e38: their norm, 6e38, is past fp32's range and reads infinity; the scale brings them to
    max_norm all the same (and is 1 where nothing is to be clipped), and a step takes it.  A scale is one quotient
    in 64 bits rounded to fp32, so the model gives its bits."""
    s = R.State([1000, 77], bits, F.FR_F32, groups=2, seed=13)
    g = s.grad(0)
    g[[3, 300, 301, 999]] = np.array([3e38, -3e38, 3e38, -3e38], np.float32)
    s.set_grad(0, g)
    d, h = Dev(s), two_groups()
    root = 2 * float(np.float32(3e38))  # the other gradients are below 2^-53 of it
    want = np.float32(float(np.float32(max_norm)) / root) if max_norm < np.inf else np.float32(1)
    assert max_norm == np.inf or want > 0
    d.opt.grad_norm(d.grads, max_norm, d.stats)
    sq, norm, scale, bad = stats_of(d)
    assert abs(sq - root * root) <= 1e-12 * sq and norm == np.inf and bad == 0
    assert scale == want
    d.opt.grad_scale(max_norm, d.stats)
    assert stats_of(d) == (sq, norm, scale, bad)
    if max_norm < np.inf:
        d.opt.step(d.state, d.grads, hyper_dev(h), d.stats)
        assert same_floats(s, d.host(), s.stepped(h, scale))
