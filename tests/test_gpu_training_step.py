"""Embedding, orthogonalised momentum and AdamW over one state, as a training
step uses them together: two replicas stay equal bit for bit, whether a step is
captured or not, and their sums find and repair what differs."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2509_03047_amd import flashrestore as F  # noqa: E402

from tests import muon_ref as R  # noqa: E402
from tests.gpu_util import to_host  # noqa: E402

VOCAB, D, HIDDEN, TOKENS, CHUNK = 997, 72, 200, 1500, 4096
SHAPES = [(D, HIDDEN), (HIDDEN, D)]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


class Model:
    """An embedding and a gain under AdamW, two matrices under Muon: one table, one plan."""

    def __init__(self):
        t, self.rows, ab, gb = F.fr_adamw_state_table([VOCAB * D, D])
        u, self.mats, self.arena_bytes, self.grad_bytes, self.update_bytes = F.fr_muon_state_table(
            SHAPES, first_entry=len(t), arena_bytes=ab, grad_bytes=gb)
        self.table = np.concatenate([t, u])
        self.plan = F.Plan(self.table, CHUNK, self.arena_bytes, self.arena_bytes)
        self.adamw = F.AdamW(self.plan, self.rows, 1, self.grad_bytes)
        self.muon = F.Muon(self.plan, self.mats, 1, self.grad_bytes, self.update_bytes)
        self.emb = F.Embedding(self.plan, int(self.rows[0]["param"]), VOCAB, D, max_tokens=TOKENS,
                               grad_arena_bytes=self.grad_bytes, grad_offset=int(self.rows[0]["grad_offset"]))


class Replica:
    def __init__(self, m, seed=1):
        self.m = m
        self.state = torch.zeros(m.arena_bytes, dtype=torch.uint8, device="cuda")
        self.grads = torch.zeros(m.grad_bytes, dtype=torch.uint8, device="cuda")
        self.updates, self.sums = m.muon.empty_updates().zero_(), m.plan.empty_sums().zero_()
        self.stats, self.mat_stats = (m.adamw.empty_stats().zero_() for _ in range(2))
        self.x = torch.zeros(TOKENS, D, dtype=torch.bfloat16, device="cuda")
        self.ids = torch.zeros(TOKENS, dtype=torch.int64, device="cuda")
        gen = torch.Generator().manual_seed(seed)
        for rows in (m.rows, m.mats):
            for r in rows:
                w = torch.randn(int(m.table[r["master"]]["numel"]), generator=gen) * 0.05
                self.array(r, "master").copy_(w)
                self.array(r, "param").copy_(self.array(r, "master"))

    def array(self, row, name):
        e = self.m.table[int(row[name])]
        size, dtype = (2, torch.bfloat16) if e["dtype"] == F.FR_BF16 else (4, torch.float32)
        o = int(e["src_offset"])
        return self.state[o: o + size * int(e["numel"])].view(dtype)

    def grad(self, row, numel):
        o = int(row["grad_offset"])
        return self.grads[o: o + 2 * numel].view(torch.bfloat16)

    def step(self, ids, hyper):
        """Forward and backward of |gain * (relu(x A) B)|^2 / 2 by torch, the embedding's and the steps by the library."""
        m = self.m
        self.ids.copy_(ids)
        m.emb.lookup(self.state, self.ids, self.x)
        x = self.x.float()
        gain = self.array(m.rows[1], "param").float()
        a, b = (self.array(r, "param").float().view(s) for r, s in zip(m.mats, SHAPES))
        h = (x @ a).relu()
        y = h @ b
        dy = y * gain * gain
        self.grad(m.rows[1], D).copy_((y * y * gain).sum(0))
        self.grad(m.mats[1], HIDDEN * D).copy_((h.t().contiguous() @ dy).view(-1))
        dh = (dy @ b.t().contiguous()) * (h > 0)
        self.grad(m.mats[0], D * HIDDEN).copy_((x.t().contiguous() @ dh).view(-1))
        dx = (dh @ a.t().contiguous()).to(torch.bfloat16)
        m.emb.grad(self.ids, dx, self.grads)
        m.adamw.grad_norm(self.grads, 1.0, self.stats)
        m.muon.grad_norm(self.grads, 1.0, self.mat_stats)
        self.stats[0] += self.mat_stats[0]  # over all tensors
        m.adamw.grad_scale(1.0, self.stats)
        m.muon.direction(self.state, self.grads, hyper[1], self.updates, self.stats, self.sums)
        m.muon.apply(self.state, self.updates, hyper[1], self.stats, self.sums)
        m.adamw.step(self.state, self.grads, hyper[0], self.stats, self.sums)
        return dx


def hypers(step):
    h = F.adamw_hyper([dict(lr=1e-3, weight_decay=0.01)], step), F.muon_hyper([dict(lr=2e-2, weight_decay=0.01)])
    return [torch.from_numpy(x.view(np.uint8).copy()).cuda() for x in h]


def batch(step):
    g = torch.Generator().manual_seed(step)
    return torch.randint(-2, VOCAB + 2, (TOKENS,), generator=g).cuda()


def test_replicas_stay_equal_and_repair():
    m = Model()
    a, b = Replica(m), Replica(m)
    diff, n = m.plan.empty_bitmap(), m.plan.empty_counter()
    check = m.plan.empty_sums()
    start = a.state.clone()
    for step in range(1, 5):
        for r in (a, b):
            dx = r.step(batch(step), hypers(step))
        m.plan.checksum_state(a.state, check)
        assert torch.equal(check, a.sums)  # the step's own sums are all of the state's
        assert len(m.plan.compare_sums(a.sums, b.sums, diff, n, sync=True)) == 0, step
        assert torch.equal(a.state, b.state) and torch.equal(a.grads, b.grads)
    want, _ = R.embedding_gradient(to_host(batch(4)), to_host(dx.float()), VOCAB, 0, 1.0)
    assert torch.equal(b.grad(m.rows[0], VOCAB * D).view(VOCAB, D).cpu(), torch.from_numpy(want).to(torch.bfloat16))
    for r in list(m.rows) + list(m.mats):  # everything has moved
        assert not torch.equal(a.array(r, "master"), start[int(m.table[int(r["master"])]["src_offset"]):][
            : 4 * int(m.table[int(r["master"])]["numel"])].view(torch.float32))
    # a bit of b's momentum flips: its own next step is another
    o = int(m.table[int(m.mats[0]["m"])]["src_offset"])
    b.state[o + 4 * 100 + 3] ^= 1
    for r in (a, b):
        r.step(batch(9), hypers(9))
    bad = m.plan.compare_sums(a.sums, b.sums, diff, n, sync=True)
    assert len(bad)
    payload, sums, flags, k = m.plan.empty_delta_payload(), m.plan.empty_sums(), m.plan.empty_bitmap(), m.plan.empty_counter()
    m.plan.pack_flagged(a.state, diff, payload, sums)
    m.plan.unpack_flagged(payload, sums, diff, b.state, flags, k)
    torch.cuda.synchronize()
    assert int(k) == 0 and torch.equal(a.state, b.state)


def test_captured_steps_are_the_eager_ones():
    """The library's part of a step, captured; torch's and another replica's eager work between the replays."""
    m, other = Model(), Model()
    a, b = Replica(m), Replica(other)
    h = hypers(1)
    ids, dx = batch(0), torch.zeros(TOKENS, D, dtype=torch.bfloat16, device="cuda")

    def part(r):
        r.m.emb.lookup(r.state, ids, r.x)
        r.m.emb.grad(ids, dx, r.grads)
        r.m.adamw.grad_norm(r.grads, 1.0, r.stats)
        r.m.muon.grad_norm(r.grads, 1.0, r.mat_stats)
        r.m.muon.direction(r.state, r.grads, h[1], r.updates, r.stats, r.sums)
        r.m.muon.apply(r.state, r.updates, h[1], r.stats, r.sums)
        r.m.adamw.step(r.state, r.grads, h[0], r.stats, r.sums)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        part(a)
    for step in range(1, 5):
        ids.copy_(batch(step))
        dx.normal_().mul_(1e-2)
        for r in (a, b):
            for row, shape in zip(r.m.mats, SHAPES):
                g = torch.randn(shape[0] * shape[1], generator=torch.Generator().manual_seed(step)) * 1e-2
                r.grad(row, shape[0] * shape[1]).copy_(g)
        for x, y in zip(h, hypers(step)):
            x.copy_(y)
        graph.replay()
        part(b)
        torch.cuda.synchronize()
        for x, y in ((a.state, b.state), (a.grads, b.grads), (a.updates, b.updates), (a.sums, b.sums), (a.x, b.x)):
            assert torch.equal(x, y), step
