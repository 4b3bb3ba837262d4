"""The embedding on the GPU: lookups have the bits of the one product and
rounding that the header defines, gradients those of its order of sums
(tests/muon_ref.py), and agree with sums in 64 bits."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2509_03047_amd import flashrestore as F  # noqa: E402

from tests import muon_ref as R  # noqa: E402
from tests.gpu_util import to_dev  # noqa: E402

TYPES = {"bf16": (F.FR_BF16, torch.bfloat16), "f32": (F.FR_F32, torch.float32)}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


class Emb:
    def __init__(self, rows, cols, table="bf16", grad="bf16", tokens=64, first=0, seed=0):
        self.rows, self.cols, self.first = rows, cols, first
        fr, self.t = TYPES[table]
        frg, self.gt = TYPES[grad]
        es = 2 if table == "bf16" else 4
        at = 4096  # behind something else
        self.arena = at + -(-rows * cols * es // 16) * 16
        self.plan = F.Plan(F.as_table([(0, 0, 1000, F.FR_F32, -1), (at, at, rows * cols, fr, -1)]), 4096, self.arena,
                           self.arena)
        self.goff = 32
        self.gbytes = self.goff + rows * cols * (2 if grad == "bf16" else 4) + 48
        self.e = F.Embedding(self.plan, 1, rows, cols, max_tokens=tokens, first=first, grad_dtype=frg,
                             grad_arena_bytes=self.gbytes, grad_offset=self.goff)
        gen = torch.Generator().manual_seed(seed)
        self.w = torch.randn(rows, cols, generator=gen).to(self.t)
        self.state = torch.zeros(self.arena, dtype=torch.uint8)
        self.state[at: at + rows * cols * es].view(self.t).copy_(self.w.view(-1))
        self.state = self.state.cuda()
        self.grads = torch.full((self.gbytes,), 0xA5, dtype=torch.uint8, device="cuda")

    def grad(self):
        es = 2 if self.gt == torch.bfloat16 else 4
        return self.grads[self.goff: self.goff + self.rows * self.cols * es].view(self.gt).view(self.rows, self.cols)

    def around(self):
        es = 2 if self.gt == torch.bfloat16 else 4
        end = self.goff + self.rows * self.cols * es
        return bool((self.grads[: self.goff] == 0xA5).all()) and bool((self.grads[end:] == 0xA5).all())


def tokens(rng, kind, n, rows, first):
    if kind == "zipf":
        ids = np.exp(rng.random(n) * np.log(2 * rows + 1)).astype(np.int64) - 1  # the second half: no rows here
    elif kind == "one":
        ids = np.full(n, rows - 1)
    else:
        ids = rng.integers(-3, rows + 3, n)
    return ids + first


@pytest.mark.parametrize("table", ["bf16", "f32"])
@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols,n", [(1, 1, 1), (50, 7, 33), (300, 256, 100), (77, 1000, 5), (9, 515, 64)])
def test_lookup(table, out, rows, cols, n):
    rng = np.random.default_rng(rows)
    e = Emb(rows, cols, table, first=5)
    for dtype, scale in ((np.int32, 1.0), (np.int64, 1.7)):
        ids = tokens(rng, "any", n, rows, 5).astype(dtype)
        wide = torch.full((n, cols + 3), 9.0, dtype=TYPES[out][1], device="cuda")  # rows further apart than cols
        e.e.lookup(e.state, to_dev(ids), wide[:, :cols], scale=scale)
        i = torch.from_numpy(ids.astype(np.int64)) - 5
        here = (i >= 0) & (i < rows)
        want = torch.where(here[:, None], e.w[i.clamp(0, rows - 1)].float() * torch.tensor(scale, dtype=torch.float32),
                           torch.zeros(1)).to(TYPES[out][1])
        torch.cuda.synchronize()
        assert torch.equal(wide[:, :cols].cpu(), want)
        assert bool((wide[:, cols:] == 9.0).all())


def test_lookup_of_extreme_ids_and_values():
    e = Emb(8, 24, "bf16", first=1 << 40)
    e.w[:] = torch.tensor([float("nan"), float("inf"), -0.0, 3e38] * 6, dtype=torch.bfloat16)
    e.state[4096: 4096 + 8 * 24 * 2].view(torch.bfloat16).copy_(e.w.view(-1))
    ids = torch.tensor([-(1 << 63), (1 << 63) - 1, -1, 0, (1 << 40) - 1, 1 << 40, (1 << 40) + 7, (1 << 40) + 8],
                       device="cuda")
    out = torch.ones(2, 4, 24, device="cuda")
    e.e.lookup(e.state, ids.view(2, 4), out)
    torch.cuda.synchronize()
    got = out.view(8, 24).cpu()
    for k in (0, 1, 2, 3, 4, 7):
        assert bool((got[k] == 0).all())
    for k in (5, 6):
        assert torch.equal(got[k].nan_to_num(7.0), e.w[0].float().nan_to_num(7.0))


CASES = [  # rows, cols, tokens, their distribution
    (1, 1, 1, "any"), (1, 8, 200, "one"), (50, 7, 33, "any"), (300, 256, 1000, "zipf"), (3, 515, 700, "any"),
    (40, 100, 64, "one"), (40, 100, 65, "one"), (40, 72, 4200, "one"), (1000, 9, 20000, "zipf"), (70000, 8, 500, "any"),
    (2, 16, 8193, "any"), (600, 1040, 128, "zipf"),
]


@pytest.mark.parametrize("rows,cols,n,kind", CASES)
@pytest.mark.parametrize("dout,grad,add", [("bf16", "bf16", False), ("f32", "f32", False), ("bf16", "f32", True),
                                           ("f32", "bf16", True)])
def test_gradient(rows, cols, n, kind, dout, grad, add):
    rng = np.random.default_rng(n)
    e = Emb(rows, cols, grad=grad, tokens=n + 3, first=11)
    ids = tokens(rng, kind, n, rows, 11)
    x = torch.from_numpy(rng.standard_normal((n, cols)).astype(np.float32)).to(TYPES[dout][1])
    dev = torch.empty(n, cols + 5, dtype=x.dtype, device="cuda")
    dev[:, :cols].copy_(x)
    old = torch.from_numpy(rng.standard_normal((rows, cols)).astype(np.float32)).to(e.gt)
    sums, there = R.embedding_gradient(ids, x.float().numpy(), rows, 11, 0.3)
    want = torch.from_numpy(sums)
    if add:
        want = torch.where(torch.from_numpy(there)[:, None], old.float() + want, old.float())
    want = want.to(e.gt)
    for dtype in (np.int64, np.int32):
        e.grad().copy_(old)
        e.e.grad(to_dev(ids.astype(dtype)), dev[:, :cols], e.grads, scale=0.3, add=add)
        torch.cuda.synchronize()
        assert torch.equal(e.grad().cpu(), want)
        assert e.around()


@pytest.mark.parametrize("rows,cols,n,kind", [(16385, 515, 3000, "zipf"), (16384, 515, 3000, "zipf"),
                                              (10923, 1040, 700, "zipf"), (32769, 513, 200, "any"), (8200, 2055, 65, "one")])
@pytest.mark.parametrize("dout,grad,add", [("bf16", "f32", False), ("f32", "bf16", True)])
def test_gradient_of_many_rows(rows, cols, n, kind, dout, grad, add):
    """On both sides of what a unit takes of a row, with slices that its end cuts off."""
    test_gradient(rows, cols, n, kind, dout, grad, add)


def test_gradient_in_64_bits():
    """Sums of n terms of fp32 in runs: at most about 3 * 64 roundings of 2^-24 of the terms' sum of magnitudes, and a
    product's."""
    rng = np.random.default_rng(3)
    rows, cols, n = 500, 130, 30000
    e = Emb(rows, cols, grad="f32", tokens=n)
    ids = tokens(rng, "zipf", n, rows, 0)
    x = rng.standard_normal((n, cols)).astype(np.float32)
    e.e.grad(to_dev(ids), to_dev(x), e.grads, scale=0.7)
    want, size = np.zeros((rows, cols)), np.zeros((rows, cols))
    here = ids < rows
    np.add.at(want, ids[here], x[here].astype(np.float64) * float(np.float32(0.7)))
    np.add.at(size, ids[here], np.abs(x[here]).astype(np.float64))
    got = e.grad().cpu().numpy()
    assert (np.abs(got - want) <= (3 * 64 + 2) * 2.0 ** -24 * size + 1e-30).all()


def test_tokens_without_rows_and_none():
    e = Emb(30, 40, tokens=100)
    x = torch.full((100, 40), float("nan"), dtype=torch.bfloat16, device="cuda")  # read by nobody
    ids = torch.full((100,), -100, device="cuda")
    for add in (False, True):
        e.grad().fill_(3.0)
        e.e.grad(ids, x, e.grads, add=add)
        torch.cuda.synchronize()
        assert bool((e.grad() == (3.0 if add else 0.0)).all())
        e.grad().fill_(3.0)
        e.e.grad(ids[:0], x[:0], e.grads, add=add)
        torch.cuda.synchronize()
        assert bool((e.grad() == (3.0 if add else 0.0)).all())
    out = torch.empty(0, 40, device="cuda")
    e.e.lookup(e.state, ids[:0], out)
    assert e.around()


def test_a_nan_stays_in_its_row():
    e = Emb(100, 64, tokens=400)
    rng = np.random.default_rng(5)
    ids = rng.integers(0, 20, 400)
    x = rng.standard_normal((400, 64)).astype(np.float32)
    x[123] = np.nan
    e.e.grad(to_dev(ids), to_dev(x), e.grads)
    torch.cuda.synchronize()
    bad = torch.isnan(e.grad()).all(1).cpu().numpy()
    assert np.array_equal(np.nonzero(bad)[0], [ids[123]]) and not torch.isnan(e.grad()).any(1).cpu().numpy()[~bad].any()


def test_gradient_agrees_with_differences_of_the_lookup():
    """The gradient of f(W) = sum(lookup(W) * c) with respect to W in a direction D is sum(grad * D): f is linear, so its
    difference is exact but for fp32 roundings, 2^-24 of the sum of magnitudes for each of two products and the sums."""
    rng = np.random.default_rng(6)
    rows, cols, n = 60, 48, 300
    e = Emb(rows, cols, "f32", "f32", tokens=n)
    ids = to_dev(rng.integers(-5, rows + 5, n))
    c = torch.from_numpy(rng.standard_normal((n, cols)).astype(np.float32)).cuda()
    d = torch.from_numpy(rng.standard_normal((rows, cols)).astype(np.float32)).cuda()
    out = torch.empty(n, cols, device="cuda")

    def f(w):
        e.state[4096: 4096 + rows * cols * 4].view(torch.float32).copy_(w.view(-1))
        e.e.lookup(e.state, ids, out, scale=1.3)
        return float((out.double() * c.double()).sum()), float((out.double() * c.double()).abs().sum())

    (up, size), (zero, _) = f(d), f(torch.zeros_like(d))
    assert zero == 0.0
    e.e.grad(ids, c, e.grads, scale=1.3)
    got = float((e.grad().double() * d.double()).sum())
    assert abs(up - got) <= (64 + 4) * 2.0 ** -24 * size


def test_graph_and_streams():
    """Replays with new tokens and gradients, eager calls of another embedding between them."""
    rows, cols, n = 700, 96, 5000
    a, b = Emb(rows, cols, grad="f32", tokens=n), Emb(rows, cols, grad="f32", tokens=n)
    ids = torch.zeros(n, dtype=torch.int64, device="cuda")
    x = torch.zeros(n, cols, dtype=torch.bfloat16, device="cuda")
    outs = [torch.zeros(n, cols, device="cuda") for _ in range(2)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.e.lookup(a.state, ids, outs[0])
        a.e.grad(ids, x, a.grads)
    side = torch.cuda.Stream()
    for i in range(4):
        rng = np.random.default_rng(i)
        ids.copy_(to_dev(tokens(rng, "zipf" if i % 2 else "any", n, rows, 0)))
        x.normal_()
        torch.cuda.synchronize()
        graph.replay()
        b.e.lookup(b.state, ids, outs[1], stream=side)
        b.e.grad(ids, x, b.grads, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(a.grads, b.grads) and torch.equal(*outs), i


def test_refusals():
    e = Emb(20, 16, tokens=10)
    ids = torch.zeros(10, dtype=torch.int64, device="cuda")
    x = torch.zeros(10, 16, dtype=torch.bfloat16, device="cuda")
    for bad in (dict(ids=ids.to(torch.int16)), dict(ids=ids.cpu()), dict(x=x.half()), dict(x=x[:, :8]), dict(x=x[:9]),
                dict(x=x.t().contiguous().t()), dict(grads=e.grads[:64]), dict(x=x[:1].expand(10, 16)),
                dict(ids=torch.zeros(20, dtype=torch.int64, device="cuda")[::2])):
        with pytest.raises(ValueError):
            e.e.grad(bad.get("ids", ids), bad.get("x", x), bad.get("grads", e.grads))
    many = torch.zeros(11, dtype=torch.int64, device="cuda")
    with pytest.raises(F.FlashRestoreError):  # more than max_tokens
        e.e.grad(many, torch.zeros(11, 16, device="cuda"), e.grads)
    with pytest.raises(F.FlashRestoreError):  # NaN
        e.e.grad(ids, x, e.grads, scale=float("nan"))
    with pytest.raises(F.FlashRestoreError):  # into what is read
        e.e.lookup(e.state, ids, e.state[4096: 4096 + 320].view(torch.bfloat16).view(10, 16))
    none = F.Embedding(e.plan, 1, 20, 16)
    none.lookup(e.state, ids, x)
    with pytest.raises(F.FlashRestoreError):  # made for lookups only
        none.grad(ids, x, e.grads)
