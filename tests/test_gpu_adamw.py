"""The optimizer step on the GPU: the kernels give the bits of the plain fp32
model (tests/adamw_ref.py), which is the header's definition, and agree with
AdamW in 64 bits within the rounding errors of its operations; norms agree
with sums in 64 bits; what must not change does not."""
import ctypes
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2509_03047_amd import flashrestore as F  # noqa: E402

from tests import adamw_ref as R  # noqa: E402
from tests.gpu_util import log, sums_host, to_dev, to_host  # noqa: E402

RAGGED = [1, 3, 4, 5, 255, 256, 257, 0, 1023, 1024, 1025, 2047, 2048, 2049, 4095, 8191, 12345, 7]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def hyper_dev(h):
    return torch.from_numpy(h.view(np.uint8).copy()).cuda()


def two_groups(step=7, seed=0):
    return F.adamw_hyper([dict(lr=3e-4, betas=(0.9, 0.95), weight_decay=0.1, seed=seed),
                          dict(lr=1e-3, betas=(0.85, 0.999), eps=1e-6, seed=seed + 1 if seed else 0)], step)


class Dev:
    """A host State on the GPU with its plan and optimizer."""

    def __init__(self, s, chunk=4096):
        self.s = s
        self.plan = F.Plan(s.table, chunk, s.arena_bytes, s.arena_bytes)
        self.opt = F.AdamW(self.plan, s.rows, s.groups, s.grad_bytes)
        self.state, self.grads = to_dev(s.arena), to_dev(s.grads)
        self.stats = self.opt.empty_stats().zero_()

    def set_scale(self, x):
        self.stats.zero_()
        self.stats.view(torch.float32)[3] = x

    def host(self):
        torch.cuda.synchronize()
        return to_host(self.state)


def first_difference(s, got, want):
    bad = np.nonzero(got != want)[0]
    if not bad.size:
        return None
    for k in range(len(s.numel)):
        for name in ("param", "master", "m", "v", "m_scale", "v_scale"):
            if s.entry(k, name) >= 0:
                o, nb = s.span(k, name)
                if o <= bad[0] < o + nb:
                    return f"{bad.size} bytes, the first in tensor {k} ({s.numel[k]}) {name} + {bad[0] - o}"
    return f"{bad.size} bytes, the first outside the entries at {bad[0]}"


def same_floats(s, got, want):
    """Equal bits, or a NaN on both sides (its sign and payload are not defined)."""
    if np.array_equal(got, want):
        return True
    got, want = got.copy(), want.copy()
    for k in range(len(s.numel)):
        for name in ("master", "m", "v", "m_scale", "v_scale"):
            if s.entry(k, name) >= 0 and not (s.bits[k] == 8 and name in "mv"):
                for a in (got, want):
                    x = s.raw(k, name, a).view(np.float32)
                    x[np.isnan(x)] = np.nan
        if s.entry(k, "param") >= 0:
            for a in (got, want):
                x = s.raw(k, "param", a).view(np.uint16)
                x[(x & 0x7FFF) > 0x7F80] = 0x7FC0
    return np.array_equal(got, want)


@pytest.mark.parametrize("bits", [32, 8, "both"])
@pytest.mark.parametrize("grad", [F.FR_BF16, F.FR_F32])
@pytest.mark.parametrize("scaled", [False, True])
@pytest.mark.parametrize("seed", [0, 77])
def test_steps_give_the_models_bits(bits, grad, scaled, seed):
    """Three steps of ragged tensors at shuffled offsets: every byte of the arena, gaps included."""
    b = [32, 8] * (len(RAGGED) // 2) if bits == "both" else bits
    s = R.State(RAGGED, b, grad, groups=2, seed=11, shuffle=True)
    d = Dev(s)
    for step in range(3):
        h = two_groups(step + 1, seed and seed + step)
        if scaled:
            d.set_scale(0.37)
        d.opt.step(d.state, d.grads, hyper_dev(h), d.stats if scaled else None)
        s.arena = s.stepped(h, 0.37 if scaled else None)
        assert first_difference(s, d.host(), s.arena) is None, step


@pytest.mark.parametrize("bits", [32, 8, "both"])
def test_gradients_of_both_types_in_one_step(bits):
    numel = RAGGED + [20_000, 70_001]
    s = R.State(numel, [32, 8] * (len(numel) // 2) if bits == "both" else bits, F.FR_F32, groups=2, seed=14, shuffle=True)
    for k in range(0, len(numel), 3):
        g = s.grad(k)
        s.rows["grad_dtype"][k] = F.FR_BF16
        s.set_grad(k, g)
    d, h = Dev(s), two_groups(seed=9)
    got, want = d.plan.empty_sums(), d.plan.empty_sums()
    d.opt.grad_norm(d.grads, 1e-3, d.stats)
    sq = math.fsum(float(x) * float(x) for k in range(len(numel)) for x in s.grad(k))
    assert abs(float(d.stats[0]) - sq) <= sum(numel) * 2.0 ** -52 * sq
    d.opt.step(d.state, d.grads, hyper_dev(h), d.stats, got)
    s.arena = s.stepped(h, d.stats.view(torch.float32)[3].item())
    assert first_difference(s, d.host(), s.arena) is None
    d.plan.checksum_state(d.state, want)
    assert np.array_equal(sums_host(got, d.plan.n_chunks), sums_host(want, d.plan.n_chunks))


def test_step_in_64_bits():
    """Against AdamW in 64 bits, by the bounds derived in tests/test_adamw_cpu.py."""
    u = 2.0 ** -24
    s = R.State([70001], 32, F.FR_F32, seed=5)
    d, h = Dev(s), two_groups()[:1]
    d.set_scale(0.37)
    d.opt.step(d.state, d.grads, hyper_dev(h), d.stats)
    m, v = s.moments(0)
    w64, m64, v64, aw, au, am = R.step64(s.get(0, "master"), m, v, s.grad(0), h[0], np.float32(0.37))
    got = d.host()
    assert np.all(np.abs(s.get(0, "m", got) - m64) <= 5 * u * am)
    assert np.all(np.abs(s.get(0, "v", got) - v64) <= 7 * u * v64)
    assert np.all(np.abs(s.get(0, "master", got) - w64) <= 4 * u * aw + 20 * u * au)
    assert np.array_equal(s.get(0, "param", got), R.rne_bf16(s.get(0, "master", got)))


@pytest.mark.parametrize("bits", [32, 8])
def test_special_values(bits):
    """NaN, infinities, denormals, the largest values and zeros, in gradients and state, without statistics to stop
    them; eps = 0 where a moment is 0 divides 0 by 0."""
    s = R.State([3000], bits, F.FR_F32, groups=1, seed=3)
    rng = np.random.default_rng(4)
    special = np.array([0.0, -0.0, 1e-45, -1e-45, 1e-38, 3e38, -3e38, np.inf, -np.inf, np.nan, 1e-20, 1e19, 2e19, 1.0],
                       np.float32)
    for start in (0, 600, 1200, 2400):  # some blocks without any
        for name in ("g", "w", "m"):
            at = start + rng.integers(0, 500, 12)
            x = special[rng.integers(0, len(special), 12)]
            if name == "g":
                g = s.grad(0)
                g[at] = x
                s.set_grad(0, g)
            elif name == "w":
                w = s.get(0, "master")
                w[at] = x
                s.put(0, "master", w)
            else:
                m, v = s.moments(0)
                m[at], v[at[::-1]] = x, np.abs(x)
                s.set_moments(0, m, v)
    g = s.grad(0)
    g[1790:2390] = 0
    s.set_grad(0, g)
    m, v = s.moments(0)
    m[1790:2390] = v[1790:2390] = 0
    s.set_moments(0, m, v)
    for eps in (1e-8, 0.0):
        d = Dev(s)
        h = F.adamw_hyper([dict(lr=3e-4, eps=eps, weight_decay=0.1)], 2)
        d.opt.step(d.state, d.grads, hyper_dev(h))
        assert same_floats(s, d.host(), s.stepped(h)), eps


def _quotients(m, v, h):
    """A step that leaves m and v as they are and takes m / (sqrt(v) / sqrt(bias2) + eps) * (lr / bias1) off masters
    of 0: (the kernel's masters, numpy's)."""
    n = m.size
    s = R.State([n], 32, F.FR_BF16)
    s.put(0, "master", np.zeros(n, np.float32))
    s.put(0, "m", m)
    s.put(0, "v", v)
    s.set_grad(0, np.zeros(n, np.float32))
    d = Dev(s)
    d.opt.step(d.state, d.grads, hyper_dev(h))
    got = d.host()
    assert np.array_equal(s.get(0, "m", got).view(np.uint32), m.view(np.uint32))
    with np.errstate(all="ignore"):
        one = np.float32(1)
        q = m / (np.sqrt(v) * (one / np.sqrt(h[0]["bias2"])) + h[0]["eps"]) * (h[0]["lr"] / h[0]["bias1"])
        want = np.zeros(n, np.float32) - q
    return s.get(0, "master", got), want


def _same(got, want):
    return bool(np.all((got.view(np.uint32) == want.view(np.uint32)) | (np.isnan(got) & np.isnan(want))))


@pytest.mark.parametrize("case", ["ordinary", "wide", "edges", "one odd value a wave"])
def test_roots_and_quotients_are_correctly_rounded(case):
    """4 million quotients of random mantissas against numpy's: operands well inside the range (which take the short
    form), over all of it (the general form), next to the ends of the short form's ranges, and one element in a wave
    outside them."""
    rng = np.random.default_rng(17)
    n = 1 << 22
    man = lambda: rng.integers(0, 1 << 23, n).astype(np.uint32)  # noqa: E731
    lo, hi = {"ordinary": (-40, 20), "wide": (-126, 127), "edges": (-2, 2), "one odd value a wave": (-40, 20)}[case]
    em, ev = rng.integers(lo, hi, n), rng.integers(lo, hi, n)
    if case == "edges":
        em, ev = em + rng.choice([-80, 60, 0], n), ev + rng.choice([-96, 60, 0], n)
    m = ((em + 127).astype(np.uint32) << 23 | man()).view(np.float32) * rng.choice([-1, 1], n).astype(np.float32)
    v = ((ev + 127).astype(np.uint32) << 23 | man()).view(np.float32)
    if case == "one odd value a wave":
        at = np.arange(0, n, 256) + rng.integers(0, 256, n // 256)
        m[at[::3]], v[at[1::3]], v[at[2::3]] = 0.0, 0.0, np.float32(1e-42)
    for bias2, eps in ((1.0, 0.0), (0.25, 1e-8), (1e-9, 1.0), (1.0, 1e13)):
        h = F.adamw_hyper([dict(lr=1.0, betas=(1.0, 1.0), eps=eps)], 1)
        h["bias1"], h["bias2"] = 1.0, bias2
        got, want = _quotients(m, v, h)
        assert _same(got, want), (bias2, eps)


@pytest.mark.parametrize("case", ["ordinary", "wide", "one odd value a wave"])
def test_roots_of_a_conversion_are_correctly_rounded(case):
    """Second moments with random mantissas to 8 bits: the codes of the model's correctly rounded roots."""
    rng = np.random.default_rng(18)
    n = 1 << 20
    lo, hi = (-126, 127) if case == "wide" else (-30, 2)
    v = ((rng.integers(lo, hi, n) + 127).astype(np.uint32) << 23 | rng.integers(0, 1 << 23, n).astype(np.uint32)).view(np.float32)
    # squares of the borders between codes, and their neighbours, where a root's last place decides
    c = rng.integers(0, 256, n).astype(np.uint32)
    border = ((c << 19) + (1 << 18)).astype(np.uint32).view(np.float32) * np.float32(2.0 ** 112)
    sq = (border.astype(np.float64) ** 2).astype(np.float32).view(np.uint32) + rng.integers(-1, 2, n).astype(np.uint32)
    pick = rng.random(n) < 0.5
    v = np.where(pick & (case != "wide"), sq.view(np.float32), v)
    if case == "one odd value a wave":
        v[np.arange(0, n, 256) + rng.integers(0, 256, n // 256)] = rng.choice(np.array([0.0, -0.0, 1e-44, 3e-39], np.float32), n // 256)
    a, b = R.State([n], 32, seed=1), R.State([n], 8, seed=2)
    a.put(0, "v", v)
    x, y = Dev(a), Dev(b)
    for seed in (0, 9):
        x.opt.convert(x.state, y.opt, y.state, seed)
        assert first_difference(b, y.host(), a.converted(b, seed)) is None


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [np.nan, np.inf])
def test_a_gradient_that_is_not_finite_stops_the_step(bits, bad):
    s = R.State(RAGGED, bits, F.FR_F32, groups=2, seed=6)
    g = s.grad(10)
    g[-1] = bad
    s.set_grad(10, g)
    d = Dev(s)
    want, got = d.plan.empty_sums(), d.plan.empty_sums().fill_(3)
    d.plan.checksum_state(d.state, want)
    d.opt.grad_norm(d.grads, 1.0, d.stats)
    d.opt.step(d.state, d.grads, hyper_dev(two_groups()), d.stats)
    d.opt.step(d.state, d.grads, hyper_dev(two_groups()), d.stats, got)
    assert first_difference(s, d.host(), s.arena) is None
    assert int(d.stats.view(torch.int64)[2]) == 1 and float(d.stats.view(torch.float32)[3]) == 0.0
    assert np.array_equal(sums_host(got, d.plan.n_chunks), sums_host(want, d.plan.n_chunks))


@pytest.mark.parametrize("bits", [32, 8, "both"])
@pytest.mark.parametrize("chunk", [4096, 8192, 1 << 16, 1 << 20])
def test_sums_are_those_of_the_new_state(bits, chunk):
    """The sums that a step writes equal fr_checksum_state's afterwards (and the step is the same); rows of chunks of
    entries that it does not write stay."""
    numel = RAGGED + [65536, 200_000, 65537, 300_001]
    b = [32, 8] * (len(numel) // 2) if bits == "both" else bits
    s = R.State(numel, b, F.FR_BF16, groups=2, seed=12, shuffle=True)
    s.rows["param"][5] = -1  # a tensor without a parameter image: its entry is not written
    s.rows[10]["flags"] = F.FR_GRAD_NOT_COUNTED
    d, h = Dev(s, chunk), two_groups(seed=5)
    got, want = d.plan.empty_sums().fill_(-7), d.plan.empty_sums()
    for _ in range(2):
        d.opt.step(d.state, d.grads, hyper_dev(h), None, got)
        s.arena = s.stepped(h)
        assert first_difference(s, d.host(), s.arena) is None
        d.plan.checksum_state(d.state, want)
        w = sums_host(want, d.plan.n_chunks).copy()
        _, first, count = d.plan.entry_layout(4 * 5 if bits == 32 else sum(4 if x == 32 else 6 for x in s.bits[:5]))
        assert count >= 1
        w.reshape(-1, 2)[first:first + count] = np.uint64(2 ** 64 - 7)
        assert np.array_equal(sums_host(got, d.plan.n_chunks), w)


@pytest.mark.parametrize("grad", [F.FR_BF16, F.FR_F32])
@pytest.mark.parametrize("numel", [[1], [5, 0, 300], RAGGED, [8192 * 3 + 5, 1 << 20, 7], []])
def test_norm(grad, numel):
    """sum_sq in 64 bits: n additions of squares exact to 2^-53 each, so within n 2^-53 of the exact sum; the norm is
    its root rounded to fp32 (half of that error and 2^-24), the scale one division more."""
    s = R.State(numel, 32, grad, seed=8)
    d = Dev(s)
    sq = math.fsum(float(x) * float(x) for k in range(len(numel)) for x in s.grad(k))
    n = max(sum(numel), 1)
    for max_norm in (1e-3, 1e6, math.inf):
        d.stats.fill_(-1)
        d.opt.grad_norm(d.grads, max_norm, d.stats)
        got, f = float(d.stats[0]), d.stats.view(torch.float32).cpu().numpy()
        assert abs(got - sq) <= n * 2.0 ** -52 * sq
        norm = np.float32(np.sqrt(got))
        assert f[2] == norm and int(d.stats.view(torch.int64)[2]) == 0
        assert f[3] == (np.float32(max_norm) / norm if norm > max_norm else 1.0)
        again = d.stats.clone()
        d.opt.grad_norm(d.grads, max_norm, d.stats)
        assert torch.equal(again, d.stats)


def test_norm_beyond_32_bits_and_uncounted_tensors():
    s = R.State([1000, 2000, 3000], 32, F.FR_F32, seed=9)
    for k, x in enumerate((1e30, 1e-30, 3e38)):
        s.set_grad(k, np.full(s.numel[k], x, np.float32))
    s.rows["flags"][2] = F.FR_GRAD_NOT_COUNTED
    d = Dev(s)
    d.opt.grad_norm(d.grads, 1.0, d.stats)
    want = 1000 * float(np.float32(1e30)) ** 2
    assert abs(float(d.stats[0]) - want) < 1e-12 * want and int(d.stats.view(torch.int64)[2]) == 0
    assert float(d.stats.view(torch.float32)[2]) == np.float32(math.sqrt(float(d.stats[0])))
    g = s.grad(2)
    g[5] = np.nan  # not counted either
    s.set_grad(2, g)
    d.grads.copy_(to_dev(s.grads))
    d.opt.grad_norm(d.grads, 1.0, d.stats)
    assert int(d.stats.view(torch.int64)[2]) == 0
    # parts of a model: their sums of squares added up
    d.stats[0] += 1.25e60
    d.opt.grad_scale(2.0, d.stats)
    f = d.stats.view(torch.float32).cpu().numpy()
    assert f[2] == np.float32(math.sqrt(float(d.stats[0]))) and f[3] == np.float32(2.0) / f[2]
    d.stats[0] = math.inf
    d.opt.grad_scale(2.0, d.stats)
    assert int(d.stats.view(torch.int64)[2]) == 1 and float(d.stats.view(torch.float32)[3]) == 0.0


@pytest.mark.parametrize("frm, to", [(32, 8), (8, 32), (32, 32), (8, 8), ("both", 8), (32, "both"), ("both", "htob")])
@pytest.mark.parametrize("seed", [0, 123])
def test_convert(frm, to, seed):
    half = {"both": [32, 8] * (len(RAGGED) // 2), "htob": [8, 32, 32, 8, 8, 32] * (len(RAGGED) // 6)}
    a = R.State(RAGGED, half.get(frm, frm), F.FR_F32, seed=21, shuffle=True)
    b = R.State(RAGGED, half.get(to, to), F.FR_BF16, seed=22, shuffle=True)
    x, y = Dev(a), Dev(b, 64)
    x.opt.convert(x.state, y.opt, y.state, seed)
    assert first_difference(b, y.host(), a.converted(b, seed)) is None
    assert first_difference(a, x.host(), a.arena) is None


def test_convert_of_special_values():
    a, b = R.State([2600], 32, seed=1), R.State([2600], 8, seed=2)
    m, v = a.moments(0)
    for at, x in ((0, np.nan), (300, np.inf), (600, 1e38), (900, 1e-45), (1200, 2.0 ** 120), (1500, 0.0)):
        m[at], v[at + 20] = x, abs(x)
    m[1792:2048], v[1792:2048] = 1e-40, 0.0
    v[2100] = -1.0  # no root
    a.put(0, "m", m)
    a.put(0, "v", v)
    x, y = Dev(a), Dev(b)
    x.opt.convert(x.state, y.opt, y.state)
    assert same_floats(b, y.host(), a.converted(b))
    y.opt.convert(y.state, x.opt, x.state)
    back = x.host()
    got, want = R.decode(*(b.get(0, k, y.host()) for k in ("m", "v", "m_scale", "v_scale"))), a.moments(0, back)
    assert np.array_equal(got[0], want[0], equal_nan=True) and np.array_equal(got[1], want[1], equal_nan=True)


def test_convert_inside_one_arena():
    """Both forms of the moments in one arena, over one plan; meeting ones are refused."""
    n = 5000
    t, r8, ab, gb = F.fr_adamw_state_table([n], 8)
    t = np.concatenate([t, np.array([(ab, ab, n, F.FR_F32, -1), (ab + 20000, ab + 20000, n, F.FR_F32, -1)], t.dtype)])
    r32 = r8.copy()
    r32["m"], r32["v"], r32["m_scale"], r32["v_scale"] = 6, 7, -1, -1
    plan = F.Plan(t, 4096, ab + 40000, ab + 40000)
    o8, o32 = F.AdamW(plan, r8, 1, gb), F.AdamW(plan, r32, 1, gb)
    a = R.State([n], 32, seed=1)
    m, v = a.moments(0)
    state = torch.zeros(ab + 40000, dtype=torch.uint8, device="cuda")
    state[ab:ab + 20000] = to_dev(m.view(np.uint8))
    state[ab + 20000:] = to_dev(v.view(np.uint8))
    o32.convert(state, o8, state)
    state[ab:] = 0
    o8.convert(state, o32, state)
    want = R.decode(*R.encode(m, np.sqrt(v), 0, 0))
    assert np.array_equal(to_host(state)[ab:].view(np.float32), np.concatenate(want))
    other = F.AdamW(plan, r32, 1, gb)
    for args in ((o32, state, other, state), (o32, state, o32, state)):
        with pytest.raises(F.FlashRestoreError):
            F.fr_adamw_convert(*args)
    wrong = F.fr_adamw_state_table([n + 1], 32)
    p2 = F.Plan(wrong[0], 4096, wrong[2], wrong[2])
    o2 = F.AdamW(p2, wrong[1], 1, wrong[3])
    with pytest.raises(F.FlashRestoreError) as ei:
        o8.convert(state, o2, torch.zeros(wrong[2], dtype=torch.uint8, device="cuda"))
    assert ei.value.status == -1


def test_tensors_past_32_bits():
    """One tensor of 2^32 + 777 elements: offsets and counters past 32 bits, compared at its start, around the 32-bit
    boundary and at its end (whole blocks; zeros elsewhere)."""
    n = (1 << 32) + 777
    s = F.fr_adamw_state_table([n], 8)
    plan = F.Plan(s[0], 1 << 20, s[2], s[2])
    opt = F.AdamW(plan, s[1], 1, s[3])
    state = torch.zeros(s[2], dtype=torch.uint8, device="cuda")
    grads = torch.zeros(s[3], dtype=torch.uint8, device="cuda")
    h = F.adamw_hyper([dict(lr=1e-3, weight_decay=0.1, seed=99)], 5)
    spans = [(0, 4096), ((1 << 32) - 4096, (1 << 32) + 512), ((1 << 32) + 512, n)]
    small = R.State([b - a for a, b in spans], 8, F.FR_BF16, seed=31)
    small.base = np.array([a for a, _ in spans])
    names = ("param", "master", "m", "v", "m_scale", "v_scale")
    size = dict(param=2, master=4, m=1, v=1, m_scale=4 / 256, v_scale=4 / 256)
    small2 = R.State(small.numel, 8, F.FR_BF16, seed=31)

    def where(k, name):
        o = int(s[0][int(s[1][0][name])]["src_offset"])
        return o + int(spans[k][0] * size[name])

    for k in range(len(spans)):
        for name in names:
            raw = small.raw(k, name)
            o = where(k, name)
            state[o:o + raw.size] = to_dev(raw)
        g = small.grads[int(small.rows[k]["grad_offset"]):][: 2 * small.numel[k]]
        grads[2 * spans[k][0]: 2 * spans[k][0] + g.size] = to_dev(g)
    assert small2.numel == small.numel
    sums, again = plan.empty_sums(), plan.empty_sums()
    opt.step(state, grads, hyper_dev(h), None, sums)
    plan.checksum_state(state, again)
    assert torch.equal(sums, again)
    want = small.stepped(h)
    for k in range(len(spans)):
        for name in names:
            raw = small.raw(k, name, want)
            o = where(k, name)
            assert np.array_equal(to_host(state[o:o + raw.size]), raw), (k, name)
    log("one step of", n, "elements")


def test_graph_capture():
    """Norm, step with sums and conversion in one graph: replays with new gradients and hyperparameters between them,
    eager work and synchronizations in between, each replay against the eager calls."""
    s = R.State(RAGGED, [32, 8] * (len(RAGGED) // 2), F.FR_BF16, groups=2, seed=41)
    t = R.State(RAGGED, 32, F.FR_BF16, groups=2, seed=42)
    d, e, wide, wide2 = Dev(s), Dev(s), Dev(t), Dev(t)
    hd = hyper_dev(two_groups(seed=3))
    sums, sums_e = d.plan.empty_sums(), e.plan.empty_sums()

    def calls(x, y, out):
        x.opt.grad_norm(x.grads, 0.5, x.stats)
        x.opt.step(x.state, x.grads, hd, x.stats, out)
        x.opt.convert(x.state, y.opt, y.state)

    calls(d, wide, sums)  # warm
    d.state.copy_(to_dev(s.arena))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(d, wide, sums)
    for i in range(4):
        hd.copy_(hyper_dev(two_groups(step=i + 1, seed=100 + i)))
        g = R.State(RAGGED, [32, 8] * (len(RAGGED) // 2), F.FR_BF16, groups=2, seed=50 + i).grads
        d.grads.copy_(to_dev(g))
        e.grads.copy_(to_dev(g))
        graph.replay()
        torch.cuda.synchronize()
        calls(e, wide2, sums_e)
        torch.cuda.synchronize()
        assert torch.equal(d.state, e.state) and torch.equal(d.stats, e.stats)
        assert torch.equal(sums, sums_e) and torch.equal(wide.state, wide2.state)


def test_another_stream():
    s = R.State(RAGGED + [300_000], 8, F.FR_BF16, groups=2, seed=61)
    d, h = Dev(s), two_groups(seed=9)
    hd = hyper_dev(h)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        d.opt.grad_norm(d.grads, 0.01, d.stats, stream=st)
        d.opt.step(d.state, d.grads, hd, d.stats, stream=st)
    st.synchronize()
    scale = float(d.stats.view(torch.float32)[3])
    for _ in range(3):
        s.arena = s.stepped(h, scale)
    assert first_difference(s, d.host(), s.arena) is None


def test_replicas_in_different_layouts_stay_identical():
    """The same tensors in two layouts and chunk sizes: equal values after steps with stochastic rounding."""
    a = R.State(RAGGED, 8, F.FR_F32, groups=2, seed=71)
    b = R.State(RAGGED, 8, F.FR_F32, groups=2, seed=71, shuffle=True)
    for k in range(len(RAGGED)):
        for name in ("param", "master", "m", "v", "m_scale", "v_scale"):
            b.raw(k, name)[:] = a.raw(k, name)
    b.grads[:] = a.grads
    x, y = Dev(a), Dev(b, 1 << 16)
    for i in range(3):
        h = hyper_dev(two_groups(i + 1, 7 * i + 1))
        for d in (x, y):
            d.opt.grad_norm(d.grads, 0.02, d.stats)
            d.opt.step(d.state, d.grads, h, d.stats, d.plan.empty_sums() if d is y else None)
    for k in range(len(RAGGED)):
        for name in ("param", "master", "m", "v", "m_scale", "v_scale"):
            assert np.array_equal(a.raw(k, name, x.host()), b.raw(k, name, y.host())), (k, name)


def test_refusals():
    s = R.State([5000, 77], [32, 8], F.FR_BF16, groups=2, seed=1)
    d = Dev(s)
    h, sums, lib, st = hyper_dev(two_groups()), d.plan.empty_sums(), F._lib, None
    o, p = d.opt.handle, (lambda x, k=0: x.data_ptr() + k)
    host = torch.zeros(1 << 16, dtype=torch.uint8)
    inf = ctypes.c_float(math.inf)
    before = d.host().copy()
    for call, code in [
        ((lib.fr_adamw_step, o, None, p(d.grads), p(h), None, None, st), -1),
        ((lib.fr_adamw_step, o, p(d.state), None, p(h), None, None, st), -1),
        ((lib.fr_adamw_step, o, p(d.state), p(d.grads), None, None, None, st), -1),
        ((lib.fr_adamw_step, o, p(d.state, 8), p(d.grads), p(h), None, None, st), -2),
        ((lib.fr_adamw_step, o, p(d.state), p(d.grads, 4), p(h), None, None, st), -2),
        ((lib.fr_adamw_step, o, p(d.state), p(d.grads), p(h, 4), None, None, st), -2),
        ((lib.fr_adamw_step, o, p(d.state), p(d.grads), p(h), p(d.stats, 4), None, st), -2),
        ((lib.fr_adamw_step, o, p(d.state), p(d.grads), p(h), None, p(sums, 8), st), -2),
        ((lib.fr_adamw_step, o, p(host), p(d.grads), p(h), None, None, st), -1),
        ((lib.fr_adamw_step, o, p(d.state), p(d.state), p(h), None, None, st), -4),
        ((lib.fr_adamw_step, o, p(d.state), p(d.grads), p(d.state, 32), None, None, st), -4),
        ((lib.fr_adamw_step, o, p(d.state), p(d.grads), p(h), None, p(d.state), st), -4),
        ((lib.fr_grad_norm, o, p(d.grads), 0.0, p(d.stats), st), -1),
        ((lib.fr_grad_norm, o, p(d.grads), math.nan, p(d.stats), st), -1),
        ((lib.fr_grad_norm, o, p(d.grads), -1.0, p(d.stats), st), -1),
        ((lib.fr_grad_norm, o, None, 1.0, p(d.stats), st), -1),
        ((lib.fr_grad_norm, o, p(d.grads), 1.0, None, st), -1),
        ((lib.fr_grad_norm, o, p(d.grads), 1.0, p(d.grads, 8), st), -4),
        ((lib.fr_grad_scale, o, inf, p(d.stats, 2), st), -2),
        ((lib.fr_grad_scale, o, 0.0, p(d.stats), st), -1),
        ((lib.fr_adamw_convert, o, p(d.state), None, p(d.state), 0, st), -1),
    ]:
        assert call[0](*call[1:]) == code, call
    big = F.AdamW(F.Plan(s.table, 4096, 1 << 40, 1 << 40), s.rows, 2, s.grad_bytes)
    assert lib.fr_adamw_step(big.handle, p(d.state), p(d.grads), p(h), None, None, st) == -3
    small = Dev(s, 1024)
    assert lib.fr_adamw_step(small.opt.handle, p(small.state), p(d.grads), p(h), None, p(sums), st) == -1
    with pytest.raises(ValueError):
        d.opt.step(d.state[:-16], d.grads, h)
    with pytest.raises(ValueError):
        d.opt.step(d.state, d.grads, h[:32])
    with pytest.raises(ValueError):
        d.opt.step(d.state, d.grads.cpu(), h)
    rows = s.rows.copy()
    rows["group"] = 2
    with pytest.raises(F.FlashRestoreError) as ei:
        F.AdamW(d.plan, rows, 2, s.grad_bytes)
    assert ei.value.status == -1
    assert np.array_equal(before, d.host())


def test_empty():
    plan = F.Plan([], 4096, 16, 16)
    opt = F.AdamW(plan, [], 0, 0)
    state, stats = torch.zeros(16, dtype=torch.uint8, device="cuda"), opt.empty_stats()
    opt.grad_norm(None, 1.0, stats)
    opt.step(state, None, None, stats)
    assert float(stats[0]) == 0.0 and float(stats.view(torch.float32)[3]) == 1.0
