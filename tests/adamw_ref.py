"""Plain models of the optimizer step, in numpy: `step32` and the codec follow
the header's definitions operation by operation in fp32 (numpy rounds each one
to nearest even, denormals kept), so the library has to give their bits;
`step64` is AdamW in 64 bits."""
from __future__ import annotations

import numpy as np

from paper_2509_03047_amd import flashrestore as F

BLOCK, SPAN = F.FR_ADAMW_BLOCK, F.FR_ADAMW_SPAN
f32, u32 = np.float32, np.uint32


def rne_bf16(x):
    """bf16 patterns (uint16) of an fp32 array, as the header's RNE."""
    u = np.ascontiguousarray(x, f32).view(u32).astype(np.uint64)
    r = (u + 0x7FFF + ((u >> 16) & 1)) >> 16
    return np.where((u & 0x7FFFFFFF) > 0x7F800000, (u >> 16) | 0x40, r).astype(np.uint16)


def from_bf16(h):
    return (np.ascontiguousarray(h, np.uint16).astype(u32) << 16).view(f32)


def step32(w, m, v, g, h, scale=None):
    """(w', m', v', sqrt(v')) of fp32 arrays; h a HYPER_DTYPE row."""
    with np.errstate(all="ignore"):
        one = f32(1)
        g = g * (one if scale is None else f32(scale))
        m = m * h["beta1"] + g * (one - h["beta1"])
        v = v * h["beta2"] + (g * g) * (one - h["beta2"])
        r = np.sqrt(v)
        d = r * (one / np.sqrt(h["bias2"])) + h["eps"]
        w = w * (one - h["lr"] * h["weight_decay"]) - (m / d) * (h["lr"] / h["bias1"])
    for x in (w, m, v, r):
        assert x.dtype == f32
    return w, m, v, r


def step64(w, m, v, g, h, scale=1.0):
    """AdamW in 64 bits, and the sum of the magnitudes that each result is made of (what its rounding errors scale by)."""
    w, m, v, g = (np.asarray(x, np.float64) for x in (w, m, v, g))
    lr, b1, b2, eps, wd, c1, c2 = (float(h[k]) for k in ("lr", "beta1", "beta2", "eps", "weight_decay", "bias1", "bias2"))
    g = g * float(scale)
    sm = np.abs(b1 * m) + np.abs((1 - b1) * g)
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    d = np.sqrt(v / c2) + eps
    return w * (1 - lr * wd) - lr * (m / c1) / d, m, v, np.abs(w), lr / c1 * sm / d, sm


# ------------------------------------------------------------------- codec


def counter_hash(counter, seed):
    c = np.asarray(counter, np.uint64)
    M = np.uint64(0xFFFFFFFF)
    h = ((c & M) ^ (((c >> np.uint64(32)) * np.uint64(0x85157AF5)) & M))
    h = (h * np.uint64(0x9E3779B9) + np.uint64(seed)) & M
    h ^= h >> np.uint64(16)
    h = (h * np.uint64(0xB504F333)) & M
    h ^= h >> np.uint64(15)
    h = (h * np.uint64(0x93CD3A2D)) & M
    return (h ^ (h >> np.uint64(16))).astype(u32)


def _blocks(x):
    pad = -x.size % BLOCK
    return np.concatenate([x, np.zeros(pad, x.dtype)]).reshape(-1, BLOCK)


def _codes(mag, drop, rnd):
    """(codes, scales) of fp32 magnitudes."""
    n = mag.size
    b = _blocks(mag)
    r = _blocks(np.broadcast_to(np.asarray(rnd, np.int64), (n,)).copy())
    top = b.view(u32).max(1).astype(np.int64) if n else np.zeros(0, np.int64)
    e = ((top - 1) >> 23) + 1  # of the smallest power of two not below any
    none, bad = e < 28, e >= 254
    ok = ~(none | bad)
    inv = (np.where(ok, 254 - e, 127).astype(u32) << 23).view(f32)
    scale = (np.where(ok, e, 0).astype(u32) << 23).view(f32)
    scale = np.where(bad, f32(np.nan), scale).astype(f32)
    with np.errstate(all="ignore"):
        y = (b * inv[:, None]) * f32(2.0 ** -112)
    c = (y.view(u32).astype(np.int64) + r) >> drop
    return np.where(ok[:, None], c, 0).reshape(-1)[:n], scale


def encode(m, r, base, seed):
    """Codes and scales of first moments m and roots r of second ones: (uint8, uint8, scales, scales)."""
    if seed:
        h = counter_hash(np.arange(m.size, dtype=np.uint64) + np.uint64(base), seed).astype(np.int64)
        rm, rr = h >> 12, h & 0x7FFFF
    else:
        rm, rr = 1 << 19, 1 << 18
    cm, sm = _codes(np.abs(m), 20, rm)
    cr, sr = _codes(np.abs(r), 19, rr)
    sign = (np.ascontiguousarray(m).view(u32) >> 24) & 128
    # a block kept as zeros, or that stands for NaN, has the signs alone
    return (cm | sign).astype(np.uint8), cr.astype(np.uint8), sm, sr


def decode(cm, cr, sm, sr):
    """The moments that codes stand for, as fp32."""
    n = cm.size
    with np.errstate(all="ignore"):
        def values(pattern, scale):
            return (_blocks((pattern.astype(u32).view(f32) * f32(2.0 ** 112))) * scale[:, None]).reshape(-1)[:n]
        c = cm.astype(u32)
        m = values(((c & 127) << 20) | ((c & 128) << 24), sm)
        r = values(cr.astype(u32) << 19, sr)
        return m, r * r


# ------------------------------------------------------------------- state


class State:
    """A state laid out by fr_adamw_state_table, with random values, on the host."""

    def __init__(self, numel, bits=32, grad_dtype=F.FR_BF16, groups=1, seed=0, shuffle=False):
        rng = np.random.default_rng(seed)
        self.numel = [int(n) for n in numel]
        self.bits = [int(b) for b in np.broadcast_to(np.asarray(bits), len(self.numel))]
        self.table, self.rows, self.arena_bytes, self.grad_bytes = F.fr_adamw_state_table(self.numel, self.bits, grad_dtype)
        self.rows["group"] = np.arange(len(self.numel)) % groups
        if shuffle:  # the table's entries at other places of the arena, with gaps
            order, pos = rng.permutation(len(self.table)), 0
            for k in order:
                pos += 16 * int(rng.integers(0, 9))
                self.table[k]["src_offset"] = self.table[k]["dst_offset"] = pos
                pos += -(-int(self.table[k]["numel"]) * (2 if self.table[k]["dtype"] == F.FR_BF16 else 4) // 16) * 16
            self.arena_bytes = pos + 48
        self.groups = groups
        self.base = np.concatenate([[0], np.cumsum([-(-n // SPAN) * SPAN for n in self.numel])])
        self.arena = np.full(max(self.arena_bytes, 1), 0xA5, np.uint8)
        self.grads = np.full(max(self.grad_bytes, 1), 0xFF, np.uint8)  # bf16 and fp32 NaN between the tensors
        for k, n in enumerate(self.numel):
            size = np.exp(rng.standard_normal(n)) * 1e-3
            self.put(k, "master", (rng.standard_normal(n) * 0.02).astype(f32))
            self.put(k, "param", rne_bf16(self.get(k, "master")))
            self.set_moments(k, (0.3 * size * rng.standard_normal(n)).astype(f32),
                             (size * size * np.abs(1 + 0.2 * rng.standard_normal(n))).astype(f32))
            self.set_grad(k, (size * rng.standard_normal(n)).astype(f32))

    def entry(self, k, name):
        return int(self.rows[k][name])

    def span(self, k, name):
        e = self.table[self.entry(k, name)]
        return int(e["src_offset"]), int(e["numel"]) * (2 if e["dtype"] == F.FR_BF16 else 4)

    def raw(self, k, name, arena=None):
        o, nb = self.span(k, name)
        return (self.arena if arena is None else arena)[o:o + nb]

    def get(self, k, name, arena=None):
        raw = self.raw(k, name, arena)
        if name == "param":
            return raw.view(np.uint16).copy()
        if name in ("m", "v") and self.bits[k] == 8:
            return raw[: self.numel[k]].copy()
        return raw.view(f32).copy()

    def put(self, k, name, x, arena=None):
        raw = self.raw(k, name, arena)
        b = np.ascontiguousarray(x).view(np.uint8)
        raw[: b.size] = b
        raw[b.size:] = 0  # the rest of the last word of codes

    def set_moments(self, k, m, v, seed=0, arena=None, root=None):
        if self.bits[k] == 32:
            self.put(k, "m", m, arena)
            self.put(k, "v", v, arena)
        else:
            with np.errstate(all="ignore"):
                cm, cr, sm, sr = encode(m, np.sqrt(v) if root is None else root, self.base[k], seed)
            for name, x in (("m", cm), ("v", cr), ("m_scale", sm), ("v_scale", sr)):
                self.put(k, name, x, arena)

    def moments(self, k, arena=None):
        if self.bits[k] == 32:
            return self.get(k, "m", arena), self.get(k, "v", arena)
        return decode(*(self.get(k, name, arena) for name in ("m", "v", "m_scale", "v_scale")))

    def set_grad(self, k, g):
        o = int(self.rows[k]["grad_offset"])
        b = (rne_bf16(g) if self.rows[k]["grad_dtype"] == F.FR_BF16 else np.ascontiguousarray(g, f32)).view(np.uint8)
        self.grads[o:o + b.size] = b

    def grad(self, k):
        o, n = int(self.rows[k]["grad_offset"]), self.numel[k]
        if self.rows[k]["grad_dtype"] == F.FR_BF16:
            return from_bf16(self.grads[o:o + 2 * n].view(np.uint16))
        return self.grads[o:o + 4 * n].view(f32).copy()

    def stepped(self, hyper, scale=None):
        """The arena after a step."""
        out = self.arena.copy()
        for k in range(len(self.numel)):
            h = hyper[int(self.rows[k]["group"])]
            m, v = self.moments(k)
            w, m, v, r = step32(self.get(k, "master"), m, v, self.grad(k), h, scale)
            self.put(k, "master", w, out)
            if self.entry(k, "param") >= 0:
                self.put(k, "param", rne_bf16(w), out)
            self.set_moments(k, m, v, int(h["seed"]), out, r)
        return out

    def converted(self, other, seed=0):
        """other's arena after it has got these moments."""
        out = other.arena.copy()
        for k in range(len(self.numel)):
            if self.bits[k] == other.bits[k]:
                for name in ("m", "v") + (("m_scale", "v_scale") if self.bits[k] == 8 else ()):
                    other.put(k, name, self.raw(k, name), out)
            else:
                other.set_moments(k, *self.moments(k), seed, out)
        return out
