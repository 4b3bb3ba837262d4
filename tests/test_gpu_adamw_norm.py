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


F32_TILE, BF16_TILE = 4096, 8192  # gradients of the 16 KiB that a workgroup of the norm takes
LAUNCHES = {  # name: element counts in tiles of the type; up to 1,024 tiles are one launch, more are two
    "1,024 whole tiles": lambda t: [1024 * t],
    "1,024 tiles, the last one element": lambda t: [1023 * t + 1],
    "1,025 tiles, the last one element": lambda t: [1024 * t + 1],
    "1,030 tiles of three tensors": lambda t: [1027 * t + 77, 1, 0, t - 1],
    "1,024 tensors": lambda t: [5] * 1024,
    "1,025 tensors of one element": lambda t: [1] * 1025,
    "2,003 tensors": lambda t: [1] * 1000 + [0, 7, 0] + [3] * 1002,
    "2,051 tiles": lambda t: [2049 * t + 4, 1],
}


@pytest.mark.parametrize("grad", [F.FR_BF16, F.FR_F32])
@pytest.mark.parametrize("case", LAUNCHES)
def test_norms_of_one_launch_and_of_two(case, grad):
    """Gradients are whole numbers up to 15, whose squares add up exactly in any order: sum_sq is the sum, and a tile
    left out or taken twice shows.  The second call finds the lines of arrivals as the first one left them; the third
    has other gradients, with a tensor's first element not finite in the fourth."""
    numel = LAUNCHES[case](F32_TILE if grad == F.FR_F32 else BF16_TILE)
    table, rows, arena_bytes, grad_bytes = F.fr_adamw_state_table(numel, 32, grad)
    plan = F.Plan(table, 4096, arena_bytes, arena_bytes)
    opt = F.AdamW(plan, rows, 1, grad_bytes)
    dtype, size = (torch.float32, 4) if grad == F.FR_F32 else (torch.bfloat16, 2)
    grads = torch.full((grad_bytes // size,), float("nan"), dtype=dtype, device="cuda")  # between the tensors too
    rng = np.random.default_rng(19)
    stats = opt.empty_stats()
    first = next(k for k, n in enumerate(numel) if n)
    for call in range(4):
        if call != 1:
            host = grads.cpu()
            x = rng.integers(-15, 16, sum(numel))
            at = 0
            for k, n in enumerate(numel):
                o = int(rows[k]["grad_offset"]) // size
                host[o:o + n] = torch.from_numpy(x[at:at + n].astype(np.float32)).to(dtype)
                at += n
            want = int((x * x).sum())
            if call == 3:
                host[int(rows[first]["grad_offset"]) // size] = float("inf")
            grads.copy_(host)
        stats.fill_(-1)
        opt.grad_norm(grads, 2.0, stats)
        f = stats.view(torch.float32).cpu().numpy()
        if call == 3:
            assert float(stats[0]) == np.inf and int(stats.view(torch.int64)[2]) == 1 and f[3] == 0
        else:
            assert float(stats[0]) == want, call
            norm = np.float32(np.sqrt(float(want)))
            assert f[2] == norm and f[3] == np.float32(2) / norm and int(stats.view(torch.int64)[2]) == 0


def test_norms_of_two_launches_in_a_graph():
    """Replays between eager calls on the same optimizer, each with new gradients."""
    numel = [1024 * F32_TILE + 5, 3]
    table, rows, arena_bytes, grad_bytes = F.fr_adamw_state_table(numel, 32, F.FR_F32)
    plan = F.Plan(table, 4096, arena_bytes, arena_bytes)
    opt = F.AdamW(plan, rows, 1, grad_bytes)
    grads = torch.zeros(grad_bytes // 4, device="cuda")
    stats, eager = opt.empty_stats(), opt.empty_stats()
    opt.grad_norm(grads, 1.0, stats)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opt.grad_norm(grads, 1.0, stats)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    for _ in range(4):
        grads.normal_(generator=gen)
        graph.replay()
        opt.grad_norm(grads, 1.0, eager)
        torch.cuda.synchronize()
        assert torch.equal(stats, eager) and float(stats[0]) > 4e6
