"""Plain models of the step by orthogonalised momentum and of the embedding, from
the header's definitions: momenta, steps and gradients operation by operation
in fp32, orthogonalisation in 64 bits."""
from __future__ import annotations

import numpy as np

from paper_2509_03047_amd import flashrestore as F
from tests.adamw_ref import from_bf16, rne_bf16

f32 = np.float32
STEPS = ((3.4445, -4.7750, 2.0315),) * 5
RUN = 64


def orthogonalized(d, eps=1e-7, coeffs=STEPS):
    """The update of the matrix d in 64 bits."""
    x = np.asarray(d, np.float64)
    with np.errstate(all="ignore"):
        norm = np.sqrt((x * x).sum())
        if norm == 0:
            return np.zeros_like(x)
        if not np.isfinite(norm):
            return np.full_like(x, np.nan)
        x = x / (norm + eps)
        tall = x.shape[0] > x.shape[1]
        x = x.T if tall else x
        for a, b, c in np.asarray(coeffs, f32).astype(np.float64):
            g = x @ x.T
            x = a * x + (b * g + c * (g @ g)) @ x
    return x.T if tall else x


class Matrices:
    """A state laid out by fr_muon_state_table, with random values, on the host."""

    def __init__(self, shapes, grad_dtype=F.FR_BF16, groups=1, seed=0, shuffle=False):
        rng = np.random.default_rng(seed)
        self.shapes = [(int(a), int(b)) for a, b in shapes]
        self.table, self.rows, self.arena_bytes, self.grad_bytes, self.update_bytes = F.fr_muon_state_table(
            self.shapes, grad_dtype)
        self.rows["group"] = np.arange(len(self.shapes)) % groups
        if shuffle:  # the table's entries at other places of the arena, with gaps
            order, pos = rng.permutation(len(self.table)), 0
            for k in order:
                pos += 16 * int(rng.integers(0, 9))
                self.table[k]["src_offset"] = self.table[k]["dst_offset"] = pos
                pos += -(-int(self.table[k]["numel"]) * (2 if self.table[k]["dtype"] == F.FR_BF16 else 4) // 16) * 16
            self.arena_bytes = pos + 48
        self.groups = groups
        self.arena = np.full(max(self.arena_bytes, 16), 0xA5, np.uint8)
        self.grads = np.full(max(self.grad_bytes, 16), 0xFF, np.uint8)  # NaN between the matrices
        for k, (a, b) in enumerate(self.shapes):
            self.put(k, "master", (rng.standard_normal(a * b) * 0.02).astype(f32))
            if self.rows[k]["param"] >= 0:
                self.put(k, "param", rne_bf16(self.get(k, "master")))
            self.put(k, "m", (rng.standard_normal(a * b) * 1e-2).astype(f32))
            r = min(4, a, b)
            g = rng.standard_normal((a, b)) + rng.standard_normal((a, r)) @ rng.standard_normal((r, b))
            self.set_grad(k, (1e-3 * g).astype(f32))

    def span(self, k, name):
        e = self.table[int(self.rows[k][name])]
        return int(e["src_offset"]), int(e["numel"]) * (2 if e["dtype"] == F.FR_BF16 else 4)

    def raw(self, k, name, arena=None):
        o, nb = self.span(k, name)
        return (self.arena if arena is None else arena)[o:o + nb]

    def get(self, k, name, arena=None):
        return self.raw(k, name, arena).view(np.uint16 if name == "param" else f32).copy()

    def put(self, k, name, x, arena=None):
        self.raw(k, name, arena)[:] = np.ascontiguousarray(x).view(np.uint8)

    def set_grad(self, k, g):
        o = int(self.rows[k]["grad_offset"])
        g = np.ascontiguousarray(g, f32).reshape(-1)
        b = (rne_bf16(g) if self.rows[k]["grad_dtype"] == F.FR_BF16 else g).view(np.uint8)
        self.grads[o:o + b.size] = b

    def grad(self, k):
        o, n = int(self.rows[k]["grad_offset"]), self.shapes[k][0] * self.shapes[k][1]
        if self.rows[k]["grad_dtype"] == F.FR_BF16:
            return from_bf16(self.grads[o:o + 2 * n].view(np.uint16))
        return self.grads[o:o + 4 * n].view(f32).copy()

    def update(self, k, updates):
        """A matrix of an update arena (bytes), as floats."""
        o, (a, b) = int(self.rows[k]["update_offset"]), self.shapes[k]
        return from_bf16(np.ascontiguousarray(updates[o:o + 2 * a * b]).view(np.uint16)).reshape(a, b)

    def momentum(self, k, h, scale=None):
        """(next momentum, direction), operation by operation."""
        with np.errstate(all="ignore"):
            x = self.grad(k) * f32(1.0 if scale is None else scale)
            m = self.get(k, "m") * h["momentum"] + x
            return m, x + h["momentum"] * m if h["nesterov"] else m

    def applied(self, updates, hyper):
        """The arena after a step along these updates (bytes)."""
        out = self.arena.copy()
        for k in range(len(self.shapes)):
            h = hyper[int(self.rows[k]["group"])]
            with np.errstate(all="ignore"):
                keep, step = f32(1) - h["lr"] * h["weight_decay"], h["lr"] * self.rows[k]["scale"]
                w = self.get(k, "master") * keep - self.update(k, updates).reshape(-1) * step
            self.put(k, "master", w, out)
            if self.rows[k]["param"] >= 0:
                self.put(k, "param", rne_bf16(w), out)
        return out


def _in_turn(x):
    """The sum of x's rows, one after another, in fp32."""
    s = np.zeros(x.shape[1:], f32)
    for r in x:
        s = s + r
    return s


def embedding_gradient(ids, dout, rows, first, scale):
    """(sums times scale, rows with tokens), in the header's order."""
    g = np.zeros((rows, dout.shape[1]), f32)
    where = {}
    for t, i in enumerate(np.asarray(ids).reshape(-1).tolist()):
        if 0 <= i - first < rows:
            where.setdefault(i - first, []).append(t)
    for v, ts in where.items():
        x = dout[ts].astype(f32)
        if len(ts) > RUN:
            x = np.stack([_in_turn(x[i:i + RUN]) for i in range(0, len(x), RUN)])
            x = np.stack([_in_turn(x[i:i + RUN]) for i in range(0, len(x), RUN)])
        g[v] = _in_turn(x)
    there = np.zeros(rows, bool)
    there[list(where)] = True
    return g * f32(scale), there
