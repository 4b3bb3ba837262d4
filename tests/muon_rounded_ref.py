"""The orthogonalisation with the operands' roundings that the library states, in
64 bits otherwise: X in fp16 with a rest of eight bits while three or more steps
are to come, A and its polynomials in fp16 with what that leaves of their
diagonals, two first steps as one where matrices are long.  Sums run in another
order than the kernels', so that bits differ, but not what the errors come to."""
from __future__ import annotations

import numpy as np

from tests.adamw_ref import from_bf16, rne_bf16
from tests.muon_ref import STEPS, orthogonalized

f32 = np.float32
A_LIFT = 256.0


def f16(x):
    return np.asarray(x, f32).astype(np.float16).astype(np.float64)


def rest8(v, h, bits=8):
    """What v is more than its fp16 number h, in `bits` bits of its last place."""
    more = (v.astype(f32).view(np.int32) - h.astype(f32).view(np.int32) + (1 << (12 - bits))) >> (13 - bits)
    more = np.clip(more, -(1 << (bits - 1)), (1 << (bits - 1)) - 1) << (13 - bits)
    return (h.astype(f32).view(np.int32) + more).view(f32).astype(np.float64) - h


def two_as_one(m, n):
    return m >= 128 and n >= 2048 and n >= 2 * m


def rounded(d, coeffs=STEPS, eps=1e-7, diagonals=True, bits=8):
    """The update of the matrix d, in bf16 as floats.  diagonals False, or other bits of a rest (0: none): mistakes that
    tests have to notice."""
    x = np.asarray(d, np.float64)
    tall = x.shape[0] > x.shape[1]
    x = x.T if tall else x
    m, n = x.shape
    lift = 2.0 ** round(0.5 * np.log2(n))
    x = (x * (lift / (np.sqrt((x * x).sum()) + eps))).astype(f32)
    steps = np.asarray(coeffs, f32).astype(np.float64)

    def kept(a):  # an fp16 matrix, and what its diagonal is more
        h = f16(a)
        return h, (np.diag(a) - np.diag(h) if diagonals else np.zeros(m))

    def of(p):
        return p[0] + np.diag(p[1])

    def times(p, q):
        return (p[0] @ q[0] + p[1][:, None] * q[0] + p[0] * q[1][None, :]) / A_LIFT

    k = 0
    while k < len(steps):
        a, b, c = steps[k]
        h = f16(x)
        carried = h + rest8(x, h, bits) if bits and (k == 0 or k + 2 < len(steps)) else h
        g = kept(h @ h.T * (A_LIFT / lift ** 2))
        q = kept(b * of(g) + c * times(g, g))
        if k == 0 and len(steps) > 1 and two_as_one(m, n):
            a2, b2, c2 = steps[1]
            t = kept(a * of(g) + times(q, g))
            g2 = kept(a * of(t) + times(t, q))
            q2 = kept(b2 * of(g2) + c2 * times(g2, g2))
            q = kept(a * of(q2) + a2 * of(q) + times(q2, q))
            a, k = a * a2, k + 1
        x = ((a + q[1][:, None] / A_LIFT) * carried + q[0] @ h / A_LIFT).astype(f32)
        k += 1
    u = from_bf16(rne_bf16((x / f32(lift)).reshape(-1))).reshape(m, n)
    return u.T if tall else u


def off(got, want):
    return float(np.linalg.norm(got.astype(np.float64) - want) / np.linalg.norm(want))


def beyond_rounding(got, want):
    """What an update's error has more than the rounding of the exact one to bf16 makes, as these add up: in squares."""
    last = off(from_bf16(rne_bf16(want.astype(f32).reshape(-1))).reshape(want.shape), want)
    return np.sqrt(max(off(got, want) ** 2 - last ** 2, 0.0))


def allowed(d, want, coeffs=STEPS):
    """Of beyond_rounding: the model's own, and four deviations more.  Where a sum in another order tips a rounding, the
    error is as large but another one; its square is a mean over the smaller side's singular directions, and so varies by
    sqrt(2 / m) of itself."""
    m = min(d.shape)
    return beyond_rounding(rounded(d, coeffs), want) * np.sqrt(1 + 4 * np.sqrt(2 / m))


def matrices():
    """(name, matrix) whose updates show the diagonals or the rests."""
    rng = np.random.default_rng(31)

    def noise(m, n):
        return rng.standard_normal((m, n))

    def low(m, n, r):
        x = noise(m, r) @ noise(r, n)
        return x / np.linalg.norm(x)

    def orthogonal(m, n):
        return np.linalg.qr(noise(n, m))[0].T

    yield "noise 128 x 2048", noise(128, 2048)
    yield "noise 2100 x 300", noise(2100, 300)
    yield "orthogonal 64 x 64", orthogonal(64, 64)
    yield "orthogonal 100 x 260", orthogonal(100, 260)
    yield "orthogonal 300 x 2100", orthogonal(300, 2100)
    yield "rank 1, 100 x 300", low(100, 300, 1)
    yield "rank 1, 300 x 2100", low(300, 2100, 1)
    yield "rank 1 in noise, 257 x 129", low(257, 129, 1) + 1e-4 * noise(257, 129) / np.sqrt(257 * 129)
    yield "rank 1 of one large element, 64 x 4100", low(64, 4100, 1) + np.eye(64, 4100) * (np.arange(64) == 3)[:, None] * 9
    yield "rank 4, 128 x 128", low(128, 128, 4)


MATRICES = list(matrices())


def kinds():
    """(kind, the most that its updates are off by as the library's header states it, matrices)."""
    rng = np.random.default_rng(32)

    def noise(m, n):
        return rng.standard_normal((m, n))

    def unit(x):
        return x / np.linalg.norm(x)

    large = [(64, 64), (128, 128), (300, 70), (256, 256), (128, 2048), (300, 2100), (64, 4100), (300, 500)]
    yield "spread", 2.5e-3, [noise(m, n) for m, n in large] + [rng.standard_t(1.5, (m, n)) for m, n in large] + [
        np.linalg.qr(noise(max(s), min(s)))[0] for s in large]
    yield "low rank", 3.5e-3, [noise(m, r) @ noise(r, n) for r in (1, 2, 3, 8, 16) for m, n in large] + [
        unit(noise(m, 1) @ noise(1, n)) + e * unit(noise(m, n)) for e in (1e-5, 1e-4, 1e-3, 1e-2) for m, n in large]
    yield "few elements", 5e-3, [noise(m, n) for m in (1, 2, 3, 5, 7, 16) for n in (1, 2, 5, 9, 31, 300)]
    yield "equal magnitudes", 1.5e-2, [np.ones(s) for s in ((5, 7), (64, 1000), (128, 700), (150, 2100), (300, 2100))] + [
        np.kron(np.eye(4), np.ones(s)) for s in ((5, 33), (25, 16), (25, 70), (25, 512))] + [
        np.eye(m, n) for m, n in ((33, 66), (300, 300), (400, 2100))] + [
        np.outer(np.sign(noise(m, 1)), np.sign(noise(n, 1))) for m, n in large]


KINDS = {name: (most, [np.asarray(d, np.float32) for d in ds]) for name, most, ds in kinds()}
EXACT = {}


def exact(name, d, coeffs=STEPS):
    key = name, tuple(map(tuple, coeffs))
    if key not in EXACT:
        EXACT[key] = orthogonalized(d.astype(f32), coeffs=coeffs)
    return EXACT[key]
