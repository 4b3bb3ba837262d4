"""The step by orthogonalised momentum on the GPU: momenta, masters, parameters
and sums have the bits of the plain fp32 model (tests/muon_ref.py), updates
agree with the orthogonalisation in 64 bits, and a matrix's update does not
depend on what else is in the call."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2509_03047_amd import flashrestore as F  # noqa: E402

from tests import muon_ref as R  # noqa: E402
from tests.gpu_util import log, sums_host, to_dev, to_host  # noqa: E402

SHAPES = [(1, 1), (1, 300), (300, 1), (5, 7), (64, 64), (128, 128), (129, 127), (200, 700), (700, 200), (0, 5),
          (257, 1025), (31, 1024), (3, 2049), (384, 384)]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def tolerance(steps=5):
    """Of an update's 2-norm.  The last rounding is off by at most 2^-8 of each element.  In each step X, A and Q are
    rounded to fp16, 2^-11 of themselves at most and independently of each other, which moves singular values and
    vectors by about as much; the steps behind it bring all singular values together and pass on about as much."""
    return 2.0 ** -8 + steps * 2.0 ** -11


def hyper_dev(h):
    return torch.from_numpy(h.view(np.uint8).copy()).cuda()


class Dev:
    def __init__(self, s, chunk=4096, coeffs=None):
        self.s = s
        self.plan = F.Plan(s.table, chunk, s.arena_bytes, s.arena_bytes)
        self.opt = F.Muon(self.plan, s.rows, s.groups, s.grad_bytes, s.update_bytes, coeffs)
        self.state, self.grads = to_dev(s.arena), to_dev(s.grads)
        self.updates = self.opt.empty_updates().fill_(0xEE)
        self.stats = torch.zeros(3, dtype=torch.float64, device="cuda")

    def set_stats(self, scale, nonfinite=0):
        self.stats.zero_()
        self.stats.view(torch.float32)[3] = scale
        self.stats.view(torch.int64)[2] = nonfinite

    def orthogonalized(self, eps=1e-7):
        h = F.muon_hyper([dict(lr=0.0, eps=eps)] * self.s.groups)
        self.opt.orthogonalize(self.grads, hyper_dev(h), self.updates)
        torch.cuda.synchronize()
        return to_host(self.updates)


def off(got, want):
    return float(np.linalg.norm(got.astype(np.float64) - want) / max(np.linalg.norm(want), 1e-300))


def outside(s, updates, fill):
    """Whether the bytes of an update arena outside its matrices hold `fill`."""
    left = np.ones(len(updates), bool)
    for k, (a, b) in enumerate(s.shapes):
        o = int(s.rows[k]["update_offset"])
        left[o:o + 2 * a * b] = False
    return bool((updates[left] == fill).all())


@pytest.mark.parametrize("dtype", [F.FR_BF16, F.FR_F32])
def test_updates_of_all_shapes(dtype):
    s = R.Matrices(SHAPES, dtype, seed=1)
    d = Dev(s)
    u = d.orthogonalized()
    for k, shape in enumerate(s.shapes):
        if min(shape):
            e = off(s.update(k, u), R.orthogonalized(s.grad(k).reshape(shape)))
            log(shape, f"{e:.2e}")
            assert e <= tolerance(), shape
    assert outside(s, u, 0xEE)


@pytest.mark.parametrize("shape", [(1, 1), (5, 7), (129, 127), (700, 200)])
def test_an_update_depends_on_its_matrix_alone(shape):
    """Alone, among others, at another place of the arenas: the same bits."""
    s = R.Matrices([shape], F.FR_F32, seed=2)
    want = s.update(0, Dev(s).orthogonalized())
    t = R.Matrices([(333, 128), shape, (1, 9), (640, 640), shape], F.FR_F32, seed=3, shuffle=True)
    t.set_grad(1, s.grad(0))
    t.set_grad(4, s.grad(0))
    u = Dev(t).orthogonalized()
    assert np.array_equal(t.update(1, u), want) and np.array_equal(t.update(4, u), want)


def orthogonalized_on_gpu(g, eps=1e-7, coeffs=R.STEPS):
    """tests/muon_ref.py's, by fp64 products of the GPU."""
    x = torch.from_numpy(g).cuda().double()
    x = x / (torch.linalg.norm(x) + eps)
    tall = x.shape[0] > x.shape[1]
    x = x.t().contiguous() if tall else x
    for a, b, c in np.asarray(coeffs, np.float32).astype(np.float64).tolist():
        m = x @ x.t().contiguous()
        x = a * x + (b * m + c * (m @ m)) @ x
    return (x.t() if tall else x).cpu().numpy()


LARGE = [(2048, 2048), (300, 2100), (2500, 140), (7, 9), (129, 5000), (1, 4000), (1500, 3), (2048, 2300), (2200, 2048),
         (2048, 2048), (600, 700), (0, 3), (257, 2049)]


@pytest.mark.parametrize("dtype", [F.FR_BF16, F.FR_F32])
def test_large_tiles_and_two_steps_as_one(dtype):
    """A list that takes tiles of 256 x 256: updates agree with 64 bits and have the bits that each matrix alone has,
    whose products take tiles of 64 x 64; matrices whose first two steps are one are among them and others."""
    s = R.Matrices(LARGE, dtype, seed=21)
    tiles = sum(-(-a // 256) * -(-b // 256) for a, b in LARGE)
    assert tiles >= 256  # else these are small tiles
    u = Dev(s).orthogonalized()
    for k, shape in enumerate(LARGE):
        if not min(shape):
            continue
        want = orthogonalized_on_gpu(s.grad(k).reshape(shape))
        e = off(s.update(k, u), want)
        log(shape, f"{e:.2e}")
        assert e <= tolerance(), shape
        alone = R.Matrices([shape], dtype, seed=22)
        alone.set_grad(0, s.grad(k))
        assert np.array_equal(alone.update(0, Dev(alone).orthogonalized()), s.update(k, u)), shape
    assert outside(s, u, 0xEE)


@pytest.mark.parametrize("coeffs", [[(1.5, -0.5, 0.0)], [(1.5, -0.5, 0.0), (1.875, -1.25, 0.375)],
                                    [(2.0, -1.5, 0.5)] * 3, [(3.4445, -4.775, 2.0315), (2.0, -1.5, 0.5)] * 4,
                                    [(8.5, -34.0, 27.2), (8.8235, -12.2125, 3.3806)]])
def test_other_steps_of_matrices_with_two_as_one(coeffs):
    """Also of few steps, and where the first two may not be one (the last: their product's parts are too large)."""
    s = R.Matrices([(130, 2050), (2050, 130), (64, 512)], F.FR_F32, seed=24)
    u = Dev(s, coeffs=coeffs).orthogonalized()
    for k, shape in enumerate(s.shapes):
        want = R.orthogonalized(s.grad(k).reshape(shape), coeffs=coeffs)
        assert off(s.update(k, u), want) <= tolerance(len(coeffs)), (shape, coeffs)


@pytest.mark.parametrize("coeffs", [[(1.5, -0.5, 0.0)], [(1.5, -0.5, 0.0), (1.875, -1.25, 0.375)],
                                    [(2.0, -1.5, 0.5)] * 3, [(3.4445, -4.775, 2.0315), (2.0, -1.5, 0.5)] * 4,
                                    [(0.0, 0.0, 0.0)]])
def test_other_steps(coeffs):
    s = R.Matrices([(130, 260), (260, 130), (64, 512)], F.FR_F32, seed=4)
    u = Dev(s, coeffs=coeffs).orthogonalized()
    for k, shape in enumerate(s.shapes):
        want = R.orthogonalized(s.grad(k).reshape(shape), coeffs=coeffs)
        assert off(s.update(k, u), want) <= tolerance(len(coeffs)), (shape, coeffs)


def test_zeros_nan_and_infinity_stay_in_their_matrix():
    s = R.Matrices([(40, 50)] * 5, F.FR_F32, seed=5)
    g = s.grad(0)
    s.set_grad(1, np.zeros(2000))
    for k, bad in ((2, np.nan), (3, np.inf)):
        x = g.copy()
        x[1234] = bad
        s.set_grad(k, x)
    s.set_grad(4, g)
    for eps in (1e-7, 0.0):
        u = Dev(s).orthogonalized(eps)
        assert (s.update(1, u) == 0).all()
        assert np.isnan(s.update(2, u)).all() and np.isnan(s.update(3, u)).all()
        for k in (0, 4):
            assert off(s.update(k, u), R.orthogonalized(g.reshape(40, 50), eps)) <= tolerance()


@pytest.mark.parametrize("size", [1e-42, 1e-30, 1.0, 1e30])
def test_gradients_of_any_magnitude(size):
    """The norm is kept in 64 bits; with eps = 0 the update does not depend on it (denormals have few bits: 1e-42 is
    714 of their steps, so that elements are rounded by up to 0.5 / 714 / their size)."""
    s = R.Matrices([(48, 100)], F.FR_F32, seed=6)
    g = s.grad(0).astype(np.float64) * 1e3
    s.set_grad(0, (g * size).astype(np.float32))
    u = Dev(s).orthogonalized(0.0)
    want = R.orthogonalized(s.grad(0).reshape(48, 100).astype(np.float64), 0.0)
    assert off(s.update(0, u), want) <= tolerance()


def test_eps_counts():
    s = R.Matrices([(32, 32)], F.FR_F32, seed=7)
    norm = float(np.linalg.norm(s.grad(0).astype(np.float64)))
    u = Dev(s).orthogonalized(norm)
    assert off(s.update(0, u), R.orthogonalized(s.grad(0).reshape(32, 32), float(np.float32(norm)))) <= tolerance()


def test_rank_one_and_repeated_rows():
    rng = np.random.default_rng(8)
    s = R.Matrices([(100, 300), (300, 100), (64, 64)], F.FR_F32, seed=8)
    s.set_grad(0, np.outer(rng.standard_normal(100), rng.standard_normal(300)))
    s.set_grad(1, np.tile(rng.standard_normal(100), 300))
    s.set_grad(2, np.eye(64) * 5)
    u = Dev(s).orthogonalized()
    for k, shape in enumerate(s.shapes):
        assert off(s.update(k, u), R.orthogonalized(s.grad(k).reshape(shape))) <= tolerance(), shape


# --------------------------------------------------------- momentum and step


TWO = [dict(lr=2e-3, momentum=0.95, weight_decay=0.1), dict(lr=1e-2, momentum=0.8, nesterov=False, eps=1e-3)]


@pytest.mark.parametrize("dtype", [F.FR_BF16, F.FR_F32])
@pytest.mark.parametrize("scale", [None, 0.37])
@pytest.mark.parametrize("sums", [False, True])
def test_direction(dtype, scale, sums):
    s = R.Matrices(SHAPES, dtype, groups=2, seed=9, shuffle=True)
    d = Dev(s)
    h = F.muon_hyper(TWO)
    if scale:
        d.set_stats(scale)
    out = d.plan.empty_sums().fill_(-1)
    d.opt.direction(d.state, d.grads, hyper_dev(h), d.updates, d.stats if scale else None, out if sums else None)
    torch.cuda.synchronize()
    want, u = s.arena.copy(), to_host(d.updates)
    for k, shape in enumerate(s.shapes):
        row = h[int(s.rows[k]["group"])]
        m, direction = s.momentum(k, row, scale)
        s.put(k, "m", m, want)
        if min(shape):
            assert off(s.update(k, u), R.orthogonalized(direction.reshape(shape), float(row["eps"]))) <= tolerance()
    assert np.array_equal(to_host(d.state)[: len(want)], want)
    assert outside(s, u, 0xEE)
    if sums:
        check_sums(d, out, ("m",))


def check_sums(d, out, kinds):
    """The sums of these arrays' chunks are those of the state as it is, the others as they were (-1)."""
    all_sums = d.plan.empty_sums()
    d.plan.checksum_state(d.state, all_sums)
    torch.cuda.synchronize()
    want = np.full(2 * d.plan.n_chunks, (1 << 64) - 1, np.uint64).reshape(-1, 2)
    have = sums_host(all_sums, d.plan.n_chunks).reshape(-1, 2)
    _, _, base = F.fr_layout_query(d.s.table, d.plan.info["chunk_bytes"], d.s.arena_bytes, d.s.arena_bytes)
    for k in range(len(d.s.shapes)):
        for name in kinds:
            e = int(d.s.rows[k][name])
            if e >= 0:
                want[int(base[e]):int(base[e + 1])] = have[int(base[e]):int(base[e + 1])]
    assert np.array_equal(sums_host(out, d.plan.n_chunks).reshape(-1, 2), want)


@pytest.mark.parametrize("chunk", [4096, 1 << 14, 1 << 20])
@pytest.mark.parametrize("sums", [False, True])
def test_apply(chunk, sums):
    s = R.Matrices(SHAPES + [(900, 900)], groups=2, seed=10, shuffle=True)
    s.rows[4]["param"] = -1
    s.rows["scale"][5] = -1.5
    d = Dev(s, chunk)
    h = F.muon_hyper(TWO)
    rng = np.random.default_rng(11)
    u = R.rne_bf16(rng.standard_normal(s.update_bytes // 2).astype(np.float32)).view(np.uint8)
    out = d.plan.empty_sums().fill_(-1)
    d.opt.apply(d.state, to_dev(u), hyper_dev(h), None, out if sums else None)
    torch.cuda.synchronize()
    assert np.array_equal(to_host(d.state), s.applied(u, h))
    if sums:
        check_sums(d, out, ("param", "master"))


def test_nonfinite_gradients_change_nothing():
    s = R.Matrices([(70, 90), (300, 20)], seed=12)
    d = Dev(s)
    d.set_stats(0.0, 1)
    h = hyper_dev(F.muon_hyper(TWO[:1]))
    sums = d.plan.empty_sums().fill_(-1)
    d.opt.direction(d.state, d.grads, h, d.updates, d.stats, sums)
    check_sums(d, sums, ("m",))
    sums.fill_(-1)
    d.opt.apply(d.state, d.updates, h, d.stats, sums)
    check_sums(d, sums, ("param", "master"))
    assert np.array_equal(to_host(d.state), s.arena) and (to_host(d.updates) == 0xEE).all()


def test_values_that_are_not_finite_in_momentum_and_updates():
    """fp32 operations as they are: NaN and infinities go where the formulas bring them."""
    s = R.Matrices([(16, 128)], F.FR_F32, seed=13)
    g = s.grad(0)
    g[:4] = [np.nan, np.inf, -np.inf, 3e38]
    s.set_grad(0, g)
    d = Dev(s)
    h = F.muon_hyper(TWO[:1])
    d.set_stats(2.0)
    d.opt.direction(d.state, d.grads, hyper_dev(h), d.updates, d.stats)
    torch.cuda.synchronize()
    got = s.get(0, "m", to_host(d.state))
    want, _ = s.momentum(0, h[0], 2.0)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(got[~np.isnan(got)], want[~np.isnan(want)])
    assert np.isnan(s.update(0, to_host(d.updates))).all()


def test_no_matrices():
    s = R.Matrices([(0, 7), (3, 0)], seed=14)
    d = Dev(s)
    h = hyper_dev(F.muon_hyper(TWO[:1]))
    d.opt.direction(d.state, d.grads, h, d.updates)
    d.opt.orthogonalize(d.grads, h, d.updates)
    d.opt.apply(d.state, d.updates, h)
    torch.cuda.synchronize()
    assert (to_host(d.updates) == 0xEE).all()


@pytest.mark.parametrize("dtype", [F.FR_BF16, F.FR_F32])
@pytest.mark.parametrize("shapes", [SHAPES, [(0, 4)], [(3000, 3000)]])
def test_gradient_norm(dtype, shapes):
    """Squares are exact in 64 bits, and so many sums of them are off by less than 2^-52 of the whole each in any order."""
    s = R.Matrices(shapes, dtype, seed=18)
    d = Dev(s)
    want = sum(float((s.grad(k).astype(np.float64) ** 2).sum()) for k in range(len(shapes)))
    n = sum(a * b for a, b in shapes)
    for _ in range(2):
        d.stats.fill_(-1)
        d.opt.grad_norm(d.grads, 1e-2, d.stats)
        got, norm, scale = float(d.stats[0]), *(float(x) for x in d.stats.view(torch.float32)[2:4])
        assert abs(got - want) <= n * 2.0 ** -52 * want
        assert norm == np.float32(np.sqrt(got)) and int(d.stats.view(torch.int64)[2]) == 0
        assert scale == (np.float32(1e-2) / np.float32(norm) if norm > np.float32(1e-2) else 1.0)
    g = s.grad(0)
    if g.size:
        g[-1] = np.inf
        s.set_grad(0, g)
        d.opt.grad_norm(to_dev(s.grads), 1e-2, d.stats)
        assert int(d.stats.view(torch.int64)[2]) == 1 and float(d.stats.view(torch.float32)[3]) == 0.0


def test_gradient_norm_refusals():
    s = R.Matrices([(5, 7), (64, 64)], F.FR_F32)
    d = Dev(s)
    lib, o, st = F._lib, d.opt.handle, torch.cuda.current_stream().cuda_stream
    g, t = d.grads.data_ptr(), d.stats.data_ptr()
    for args, want in (((o, g, 0.0, t, st), -1), ((o, g, float("nan"), t, st), -1), ((o, g, 1.0, None, st), -1),
                       ((o, g + 8, 1.0, t, st), -2), ((o, g, 1.0, t + 4, st), -2)):
        assert lib.fr_muon_grad_norm(*args) == want, args
    assert lib.fr_muon_grad_norm(o, g, 1.0, g + 16, st) < 0  # the statistics lie in the gradients
    with pytest.raises(ValueError):
        d.opt.grad_norm(d.grads[:-16], 1.0, d.stats)
    torch.cuda.synchronize()
    assert np.array_equal(to_host(d.grads), s.grads)


# ---------------------------------------------------------- streams, graphs


def test_steps_in_a_graph_and_on_a_stream():
    """Replays of a captured step, eager steps between them on another stream: each has the eager step's bits."""
    s = R.Matrices([(200, 300), (300, 100), (17, 1000)], seed=15)
    a, b = Dev(s), Dev(s)
    h = hyper_dev(F.muon_hyper(TWO[:1]))
    sums = [x.plan.empty_sums().zero_() for x in (a, b)]

    def step(x, out):
        x.opt.direction(x.state, x.grads, h, x.updates, None, out)
        x.opt.apply(x.state, x.updates, h, None, out)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a, sums[0])
    side = torch.cuda.Stream()
    for i in range(4):
        g = torch.from_numpy(np.random.default_rng(i).integers(0, 0x3C00, s.grad_bytes // 2).astype(np.uint16)
                             .view(np.uint8)).cuda()
        for x in (a, b):
            x.grads[: s.grad_bytes].copy_(g)
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(side):
            step(b, sums[1])
        torch.cuda.synchronize()
        assert torch.equal(a.state, b.state) and torch.equal(a.updates, b.updates) and torch.equal(*sums), i
        b.opt.orthogonalize(b.grads, h, b.updates)
        torch.cuda.synchronize()


def test_two_optimizers_at_once():
    """Each has scratch of its own."""
    s = R.Matrices([(500, 700)], seed=16)
    one, two = Dev(s), Dev(s)
    want = one.orthogonalized()
    h = hyper_dev(F.muon_hyper([dict(lr=0.0)]))
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for x, st in zip((one, two), streams):
            x.opt.orthogonalize(x.grads, h, x.updates, stream=st)
    torch.cuda.synchronize()
    for x in (one, two):
        assert np.array_equal(to_host(x.updates), want)


def test_refusals_of_buffers():
    s = R.Matrices([(64, 64)], seed=17)
    d = Dev(s)
    h = hyper_dev(F.muon_hyper([dict(lr=0.0)]))
    with pytest.raises(F.FlashRestoreError):
        d.opt.orthogonalize(d.updates, h, d.updates)
    with pytest.raises(ValueError):
        d.opt.orthogonalize(d.grads[:64], h, d.updates)
    with pytest.raises(ValueError):
        d.opt.apply(d.state, d.updates.cpu(), h)
    with pytest.raises(F.FlashRestoreError):
        d.opt.orthogonalize(d.grads, h.data_ptr() + 4, d.updates)
    small = F.Plan(s.table, 64, s.arena_bytes, s.arena_bytes)
    opt = F.Muon(small, s.rows, 1, s.grad_bytes, s.update_bytes)
    with pytest.raises(F.FlashRestoreError):  # no sums of chunks below 4 KiB
        opt.apply(d.state, d.updates, h, None, small.empty_sums())
    opt.destroy()
    with pytest.raises(ValueError):
        opt.apply(d.state, d.updates, h)
