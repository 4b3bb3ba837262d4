"""Two data-parallel replicas that train, watch each other and repair.

A small decoder's tensors are fitted to random targets (the gradient of half
the squared distance is the distance), by two replicas of its state on one
GPU.  Every step each takes the norm of its gradients, the clipped AdamW step
and, in the same pass, the chunk sums of its new state, which the replicas
compare: 16 bytes a chunk instead of the state.  Then

  * a bit of one replica flips: the next comparison names the chunks it has
    reached, and only those are sent again;
  * that replica is lost altogether and restored from the other;
  * both go over to moments in 8 bits and train on, still bit-identical,
    although their rounding is stochastic (the seed is the step's).

Run it with the repository's root as the working folder:
python examples/replica_training.py
"""
from __future__ import annotations

import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import numpy as np  # noqa: E402
import torch  # noqa: E402

from paper_2509_03047_amd import flashrestore as F  # noqa: E402
from paper_2509_03047_amd import workloads as W  # noqa: E402

CHUNK = 1 << 14


class Replica:
    """One replica's state arena and what its steps need."""

    def __init__(self, form: "Form"):
        self.form = form
        self.state = torch.zeros(form.arena_bytes, dtype=torch.uint8, device="cuda")
        self.grads = torch.zeros(form.grad_bytes, dtype=torch.uint8, device="cuda")
        self.stats = form.opt.empty_stats().zero_()
        self.sums = form.plan.empty_sums()

    def step(self, hyper, max_norm=1.0):
        opt = self.form.opt
        opt.grad_norm(self.grads, max_norm, self.stats)
        opt.step(self.state, self.grads, hyper, self.stats, self.sums)


class Form:
    """The layout of a state with moments of so many bits: its plan and optimizer, and views of its arrays."""

    def __init__(self, numel, bits):
        self.numel = numel
        self.table, rows, self.arena_bytes, self.grad_bytes = F.fr_adamw_state_table(numel, bits)
        rows["group"] = [n < 4096 for n in numel]  # norms do not decay
        self.rows = rows
        self.plan = F.Plan(self.table, CHUNK, self.arena_bytes, self.arena_bytes)
        self.opt = F.AdamW(self.plan, rows, 2, self.grad_bytes)

    def array(self, r: Replica, k: int, name: str):
        e = self.table[int(self.rows[k][name])]
        size, dtype = (2, torch.bfloat16) if e["dtype"] == F.FR_BF16 else (4, torch.float32)
        o = int(e["src_offset"])
        return r.state[o: o + size * int(e["numel"])].view(dtype)

    def grad(self, r: Replica, k: int):
        o = int(self.rows[k]["grad_offset"])
        return r.grads[o: o + 2 * self.numel[k]].view(torch.bfloat16)


def losses(r: Replica, targets):
    """Writes the gradients of half the squared distance to the targets; the mean of it."""
    total = 0.0
    for k, t in enumerate(targets):
        d = r.form.array(r, k, "param").float() - t
        r.form.grad(r, k).copy_(d)
        total += float(d.square().sum())
    return 0.5 * total / sum(r.form.numel)


def take_over(src: Replica, dst: Replica):
    """dst <- src, which has the other form: parameters and masters by a plan between the two layouts, moments
    converted (rounded to nearest)."""
    a, b = src.form, dst.form
    rows = []
    for x, y in zip(a.rows, b.rows):
        for name in ("param", "master"):
            e, f = a.table[x[name]], b.table[y[name]]
            rows.append((e["src_offset"], f["dst_offset"], e["numel"], e["dtype"], len(rows) + 1 if name == "param" else -1))
    plan = F.Plan(rows, CHUNK, a.arena_bytes, b.arena_bytes)
    payload, sums, bad, n_bad = plan.empty_payload(), plan.empty_sums(), plan.empty_bitmap(), plan.empty_counter()
    plan.pack(src.state, payload, sums)
    plan.unpack(payload, sums, dst.state, bad, n_bad)
    a.opt.convert(src.state, b.opt, dst.state)
    if int(n_bad):
        raise RuntimeError("the masters arrived damaged")


def restore(src: Replica, dst: Replica):
    """dst <- src, of the same form, as a recreated rank gets it."""
    plan = src.form.plan
    payload, sums, bad, n_bad = plan.empty_payload(), plan.empty_sums(), plan.empty_bitmap(), plan.empty_counter()
    plan.pack(src.state, payload, sums)
    plan.unpack(payload, sums, dst.state, bad, n_bad)
    return int(n_bad)


def repair(src: Replica, dst: Replica, diff):
    """Sends the chunks whose bits are set in `diff` again."""
    plan = src.form.plan
    payload, sums, bad, n_bad = plan.empty_delta_payload(), plan.empty_sums(), plan.empty_bitmap(), plan.empty_counter()
    plan.pack_flagged(src.state, diff, payload, sums)
    plan.unpack_flagged(payload, sums, diff, dst.state, bad, n_bad)
    return int(n_bad)


def main(steps: int = 20, log=print) -> dict:
    numel = [n for _, n in W.toy_decoder_tensors()]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    targets = [torch.empty(n, device="cuda").normal_(0.0, 0.05, generator=gen) for n in numel]
    form = Form(numel, 32)
    a, b = Replica(form), Replica(form)  # both start from zeros
    seen = dict(losses=[], flagged=[], differing_after_repair=None, restored_bad=None, form8_differs=0)

    def train(first, last):
        for i in range(first, last):
            f = a.form
            h = F.adamw_hyper([dict(lr=3e-3, betas=(0.9, 0.95), weight_decay=0.01, seed=i),
                               dict(lr=3e-3, betas=(0.9, 0.95), seed=i)], i)
            hyper = torch.from_numpy(h.view(np.uint8)).cuda()
            seen["losses"].append(losses(a, targets))
            losses(b, targets)
            a.step(hyper)
            b.step(hyper)
            diff, n = f.plan.empty_bitmap(), f.plan.empty_counter()
            flagged = f.plan.compare_sums(a.sums, b.sums, diff, n, sync=True)
            log(f"step {i}: loss {seen['losses'][-1]:.6f}, norm {float(a.stats.view(torch.float32)[2]):.4f}, "
                f"{len(flagged)} of {f.plan.n_chunks} chunks differ")
            seen["flagged"].append(len(flagged))
            if len(flagged):
                repair(a, b, diff)
                seen["differing_after_repair"] = len(f.plan.verify_replicas(a.state, b.state, diff, n, sync=True))
                log(f"  sent again; {seen['differing_after_repair']} chunks differ")

    train(1, steps // 2)
    at = int(form.table[form.rows[0]["v"]]["src_offset"]) + 4 * 12345
    b.state[at + 2] ^= 4
    log("a bit of replica b's second moments flips")
    train(steps // 2, steps + 1)

    b.state.fill_(0xEE)
    seen["restored_bad"] = restore(a, b)
    log(f"replica b is lost and restored: {seen['restored_bad']} bad chunks")
    train(steps + 1, steps + 3)

    form8 = Form(numel, 8)
    a8, b8 = Replica(form8), Replica(form8)
    take_over(a, a8)
    take_over(b, b8)
    log(f"moments in 8 bits: {form.arena_bytes} -> {form8.arena_bytes} bytes of state")
    a, b = a8, b8
    before = sum(seen["flagged"])
    train(steps + 3, 2 * steps)
    seen["form8_differs"] = sum(seen["flagged"]) - before
    seen["losses"].append(losses(a, targets))
    return seen


if __name__ == "__main__":
    main()
