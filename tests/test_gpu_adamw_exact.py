"""Every root and every divisor of the step's short forms, and sums of long
chunks, on the GPU."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2509_03047_amd import flashrestore as F  # noqa: E402

from tests.gpu_util import log  # noqa: E402
from tests.test_gpu_adamw import _gpu, hyper_dev  # noqa: E402, F401


def hard_numerators(b, e):
    """For each odd b in [2^23, 2^24) the a with 2^25 a = e (mod b): where a < b, a / b lies e / (2 b) of a unit of its
    24th bit from a number between two of 24 bits, or from one of 24 bits (the nearest that a quotient comes to
    either); else what is left of 2^24 - 1."""
    x = np.full(b.size, e, np.int64) % b
    for _ in range(25):
        x = np.where(x & 1, x + b, x) >> 1
    return np.where((b & 1 == 1) & (x >= 1 << 23), x, (1 << 24) - 1 - (b & 0xFF))


@pytest.mark.parametrize("low", [0, -96, 58])
def test_every_root_and_every_divisor(low):
    """All 2^24 second moments of [2^low, 2^(low + 2)): both parities of a root's exponent, and so, as roots, every
    divisor's mantissa.  Numerators for each: 2^24 - 1 and 2^24 - 12,345 of them (quotients by the smaller divisors
    just below 2, which a root that is one unit off moves), the two whose quotients by it are hardest to round, and a
    random one.  Masters of 0 and gradients of 0, so that masters become minus the quotients; numpy's roots and
    quotients are correctly rounded."""
    n = 1 << 24
    table, rows, arena_bytes, grad_bytes = F.fr_adamw_state_table([n], 32)
    plan = F.Plan(table, 1 << 20, arena_bytes, arena_bytes)
    opt = F.AdamW(plan, rows, 1, grad_bytes)
    state = torch.zeros(arena_bytes, dtype=torch.uint8, device="cuda")
    grads = torch.zeros(grad_bytes, dtype=torch.uint8, device="cuda")
    master, m_at, v_at = (state[int(table[int(rows[0][k])]["src_offset"]):][: 4 * n].view(torch.float32)
                          for k in ("master", "m", "v"))
    h = F.adamw_hyper([dict(lr=1.0, betas=(1.0, 1.0), eps=0.0)], 1)
    h["bias1"] = h["bias2"] = 1.0
    hyper = hyper_dev(h)
    v = (np.arange(n, dtype=np.uint32) + np.uint32((low + 127) << 23)).view(np.float32)
    v_at.copy_(torch.from_numpy(v))
    root = np.sqrt(v)
    assert root.dtype == np.float32
    b = ((root.view(np.uint32) & 0x7FFFFF) | 0x800000).astype(np.int64)
    rng = np.random.default_rng(23)
    for a in ((1 << 24) - 1, (1 << 24) - 12345, hard_numerators(b, 1), hard_numerators(b, -1),
              rng.integers(1 << 23, 1 << 24, n)):
        m = np.ldexp(np.broadcast_to(np.asarray(a, np.int64), (n,)).astype(np.float32), -23).astype(np.float32)
        m_at.copy_(torch.from_numpy(m))
        master.zero_()
        opt.step(state, grads, hyper)
        got = master.cpu().numpy()
        want = np.float32(0) - m / root
        assert np.array_equal(got, want), np.flatnonzero(got != want)[:5]
        assert np.array_equal(m_at.cpu().numpy(), m)
    log("every root and divisor from 2 **", low)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("chunk", [1 << 22, 1 << 26, 1 << 30])
def test_sums_of_long_chunks(bits, chunk):
    """Chunks that up to 156,000 tiles feed, the last ones short, beside a tensor of five elements: the sums that a step
    writes are fr_checksum_state's."""
    numel = [40_000_003, 5, 3_000_000]
    table, rows, arena_bytes, grad_bytes = F.fr_adamw_state_table(numel, bits)
    plan = F.Plan(table, chunk, arena_bytes, arena_bytes)
    opt = F.AdamW(plan, rows, 1, grad_bytes)
    state = torch.zeros(arena_bytes, dtype=torch.uint8, device="cuda")
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    for k, n in enumerate(numel):
        o = int(table[int(rows[k]["master"])]["src_offset"])
        state[o:o + 4 * n].view(torch.float32).normal_(0.0, 0.02, generator=gen)
    grads = torch.empty(grad_bytes // 2, dtype=torch.bfloat16, device="cuda").normal_(0.0, 1e-3, generator=gen)
    hyper = hyper_dev(F.adamw_hyper([dict(lr=1e-3, weight_decay=0.1, seed=9)], 3))
    got, want = plan.empty_sums().fill_(-7), plan.empty_sums()
    for _ in range(2):
        opt.step(state, grads, hyper, None, got)
        plan.checksum_state(state, want)
        assert torch.equal(got, want)
