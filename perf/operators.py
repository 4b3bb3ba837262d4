"""The optimizer step of a training state, and what goes with it, as cases to measure.

A case is one pass of an operator over all tensors of a state at once: the
global norm of the gradients with its clip scale ("norm"); a clipped AdamW
step with moments in 32 bits ("step"); the step of a rank whose replicas are
compared after every step, which also writes the chunk sums of the new state
("step_sums"); the step with moments in 8 bits ("step8"); moments brought from
32 to 8 bits ("narrow") and back ("widen").

Values held in 8 bits are returned as what they stand for, so "step8" and
"narrow" end with the widening of the moments that they wrote.

All tensors of a kind (parameters, masters, moments, gradients) lie behind one
another, each from a multiple of 1,024 elements on, as flat optimizer buffers
do.  The tensors come from decoders ("decoder"), from one rank's shard of a
flattened decoder ("zero": one long tensor), or have log-uniform sizes
("scatter").
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

BLOCK = 256   # elements that share a scale in 8 bits
SPAN = 1024   # a tensor starts at a multiple of it in the flat buffers
GROUPS = 2    # with weight decay, and without
_M, _V = 20, 19  # dropped bits of a code of a first moment, of a root of a second


# ------------------------------------------------------------------- cases


def listed():
    return [
        # the norm of a small model's gradients: two launches' worth of latency
        dict(name="toy-norm", op="norm", layout="decoder", model="toy", grad="bf16"),
        # one optimizer shard of odd size, gradients in 32 bits
        dict(name="zero-norm", op="norm", layout="zero", layers=12, hidden=1500, ffn=4001, vocab=32003, shard=3,
             grad="f32"),
        # one rank's share of an 8B model
        dict(name="8b-norm", op="norm", layout="decoder", model="llama3-8b-tp8", grad="bf16"),
        # adapters, norms, biases: many small tensors of odd sizes, launches count
        dict(name="tiny-step", op="step", layout="scatter", entries=48, lo=16, hi=4096, table_seed=5, grad="f32"),
        dict(name="zero-step", op="step", layout="zero", layers=12, hidden=1500, ffn=4001, vocab=32003, shard=3,
             grad="f32"),
        dict(name="8b-step", op="step", layout="decoder", model="llama3-8b-tp8", grad="bf16"),
        # replicas compared after every step, on a small model and on the 8B share
        dict(name="toy-step-sums", op="step_sums", layout="decoder", model="toy", grad="bf16", chunk=1 << 14),
        dict(name="8b-step-sums", op="step_sums", layout="decoder", model="llama3-8b-tp8", grad="bf16",
             chunk=1 << 16),
        # moments in 8 bits: ragged tensors rounded to nearest, the 8B share stochastically
        dict(name="scatter-step8", op="step8", layout="scatter", entries=2000, lo=64, hi=1 << 17, table_seed=2,
             grad="f32", stochastic=False),
        dict(name="8b-step8", op="step8", layout="decoder", model="llama3-8b-tp8", grad="bf16", stochastic=True),
        # a rank goes over to 8 bits; a rank in 32 bits takes over the moments of one in 8
        dict(name="8b-narrow", op="narrow", layout="decoder", model="llama3-8b-tp8", grad="bf16", stochastic=False),
        dict(name="zero-widen", op="widen", layout="zero", layers=12, hidden=1500, ffn=4001, vocab=32003, shard=3,
             grad="f32", stochastic=False),
    ]


def _log(rng, lo, hi):
    """A whole number, spread evenly over the logarithm of [lo, hi]."""
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    while True:
        c = dict(op=rng.choice(["norm", "step", "step_sums", "step8", "narrow", "widen"]),
                 layout=rng.choice(["decoder", "zero", "scatter"]), grad=rng.choice(["bf16", "f32"]))
        if c["op"] == "step_sums":
            c["chunk"] = 1 << rng.randint(12, 20)
        if c["op"] in ("step8", "narrow", "widen"):
            c["stochastic"] = rng.random() < 0.5
        if c["layout"] == "scatter":
            lo = _log(rng, 1, 4096)
            c.update(entries=_log(rng, 2, 4000), lo=lo, hi=lo * _log(rng, 4, 8192), table_seed=rng.randrange(1 << 20))
        else:
            hidden = _log(rng, 32, 8192)
            c.update(layers=_log(rng, 1, 40), hidden=hidden, ffn=int(hidden * rng.uniform(0.4, 4)),
                     vocab=_log(rng, 100, 130000))
            if c["layout"] == "zero":
                c["shard"] = rng.randint(2, 8)
        n = sum(_numels(c))
        if 2000 <= n <= 700_000_000:
            return c


# ----------------------------------------------------------------- tensors


def _decoder(case):
    """A decoder's tensors: sizes, and whether weights decay."""
    if case.get("model") == "toy":
        layers, d, qkv, o, ff1, ff2, vocab, head = 2, 256, 3 * 256, 256, 1024, 1024, 8192, False
    elif case.get("model") == "llama3-8b-tp8":
        layers, d, qkv, o, ff1, ff2, vocab, head = 32, 4096, 768, 512, 3584, 1792, 16032, True
    else:
        d, f = case["hidden"], case["ffn"]
        layers, qkv, o, ff1, ff2, vocab, head = case["layers"], 3 * d, d, 2 * f, f, case["vocab"], False
    t = [(vocab * d, True)]
    for _ in range(layers):
        t += [(d, False), (qkv * d, True), (o * d, True), (d, False), (ff1 * d, True), (ff2 * d, True)]
    t.append((d, False))
    return t + [(vocab * d, True)] if head else t


def _tensors(case):
    """(sizes of the tensors that decay, sizes of the others), the order in which they lie."""
    if case["layout"] == "scatter":
        rng = np.random.Generator(np.random.PCG64(case["table_seed"]))
        n = np.floor(case["lo"] * (case["hi"] / case["lo"]) ** rng.random(case["entries"])).astype(np.int64).tolist()
        at = (2 * len(n) + 2) // 3
        return n[:at], n[at:]
    t = _decoder(case)
    if case["layout"] == "zero":  # one rank's share of all of it
        n = sum(n for n, _ in t)
        return [-(-n // (8 * case["shard"])) * 8], []
    return [n for n, d in t if d], [n for n, d in t if not d]


def _numels(case):
    a, b = _tensors(case)
    return a + b


def _starts(numels):
    """Where each tensor starts in the flat buffers, and their length."""
    ends = np.cumsum(-(-np.asarray(numels, dtype=np.int64) // SPAN) * SPAN)
    return np.concatenate([[0], ends[:-1]]), int(ends[-1])


# ------------------------------------------------------------------ inputs


def _hyper(stochastic, seed):
    """lr, beta1, beta2, eps, weight decay, 1 - beta1^t, 1 - beta2^t and the seed's bits, for both groups."""
    t = 1000 + seed % 1000
    row = [3e-4, 0.9, 0.95, 1e-8, 0.1, 1 - 0.9 ** t, 1 - 0.95 ** t, 0.0]
    h = np.array([row, row], dtype=np.float32)
    h[1, 4] = 0.0
    if stochastic:
        h.view(np.uint32)[:, 7] = [(seed * 40503 + k) % (1 << 32) | 1 for k in range(GROUPS)]
    return h


def _arena(s, numels, kinds):
    """One arena that holds flat buffers of these (name, type, elements for one) behind one another."""
    s["starts"], s["flat"] = _starts(numels)
    at, where = 0, {}
    for name, dtype, per in kinds:
        where[name] = at
        at += s["flat"] // per * torch.empty(0, dtype=dtype).element_size()
    s["state"], s["where"] = torch.zeros(at, dtype=torch.uint8, device="cuda"), where
    for name, dtype, per in kinds:
        n = s["flat"] // per * torch.empty(0, dtype=dtype).element_size()
        s[name] = s["state"][where[name]: where[name] + n].view(dtype)


def prepare(case, seed):
    numels = _numels(case)
    first = len(_tensors(case)[0])
    op, dev = case["op"], torch.device("cuda")
    s = dict(op=op)
    if op == "norm":  # the state is not read
        s["starts"], s["flat"] = _starts(numels)
    else:
        kinds = [("param", torch.bfloat16, 1)] + [(x, torch.float32, 1) for x in ("master", "m", "v")]
        if op in ("step8", "narrow", "widen"):
            kinds += [("m8", torch.uint8, 1), ("v8", torch.uint8, 1), ("ms", torch.float32, BLOCK),
                      ("vs", torch.float32, BLOCK)]
        if op == "narrow":
            kinds += [("m_back", torch.float32, 1), ("v_back", torch.float32, 1)]
        _arena(s, numels, kinds)
    n, starts = s["flat"], s["starts"]
    s["split"] = int(starts[first]) if first < len(numels) else n
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)

    def normal(sd):
        return torch.empty(n, dtype=torch.float32, device=dev).normal_(0.0, sd, generator=gen)

    # 1 where a tensor has an element, 0 in the rest of its last 1,024
    edge = torch.zeros(n + 1, dtype=torch.int8, device=dev)
    full = torch.from_numpy(starts).to(dev)
    edge.index_add_(0, full, torch.ones(len(numels), dtype=torch.int8, device=dev))
    edge.index_add_(0, full + torch.tensor(numels, device=dev), -torch.ones(len(numels), dtype=torch.int8, device=dev))
    there = torch.cumsum(edge[:n], 0, dtype=torch.int8)
    del edge

    # each element's gradients have a size of their own, over a few powers of ten
    size = normal(1.0).exp_().mul_(1e-3)
    if op in ("norm", "step", "step_sums", "step8"):
        s["grad"] = (normal(1.0) * size * there).to(torch.bfloat16 if case["grad"] == "bf16" else torch.float32)
    if op != "norm":
        m, v = normal(0.3) * size * there, (size * size * normal(0.2).add_(1.0).abs_()) * there
        s["m"].copy_(m)
        s["v"].copy_(v)
        del m, v
    del size
    if op in ("step8", "widen"):
        rnd = (1 << (_M - 1), 1 << (_V - 1))
        _keep(s, s["m"], s["v"].sqrt(), rnd)
        s["m"].zero_()
        s["v"].zero_()
    if op != "norm":
        s["master"].copy_(normal(0.02) * there)
        s["param"].copy_(s["master"])
    del there
    h = _hyper(case.get("stochastic", False), seed)
    s["seeds"] = h.view(np.uint32)[:, 7].tolist()
    s["hyper"] = torch.from_numpy(h).to(dev)
    s["max_norm"] = 1e-3 * math.sqrt(n)
    s["scale"] = torch.tensor(0.25 + (seed % 64) / 128, dtype=torch.float32, device=dev)
    if op == "step_sums":
        _chunks(s, numels, case["chunk"])
        s["sums"] = torch.zeros(s["n_chunks"], 2, dtype=torch.int64, device=dev)
    if own:
        _handles(s, case, numels, first)
    return s


def _chunks(s, numels, chunk):
    """The chunks of [parameter, master, m, v] of every tensor in turn: for each kind, each chunk's first and last word
    in the flat buffer, and its number."""
    nb = np.asarray(numels, dtype=np.int64)[:, None] * np.array([2, 4, 4, 4])
    count = -(-nb // chunk)
    base = np.concatenate([[0], np.cumsum(count.reshape(-1))])
    s["n_chunks"] = int(base[-1])
    s["chunks"] = {}
    for j, kind in enumerate(("param", "master", "m", "v")):
        k = np.repeat(np.arange(len(numels)), count[:, j])
        i = np.arange(len(k)) - np.repeat(np.cumsum(count[:, j]) - count[:, j], count[:, j])
        first = s["starts"][k] * (2 if j == 0 else 4) // 4 + i * (chunk // 4)
        last = first + np.minimum(chunk, nb[k, j] - i * chunk + 3) // 4
        s["chunks"][kind] = tuple(torch.from_numpy(x).cuda() for x in (first, last, base[:-1].reshape(-1, 4)[k, j] + i))


def _handles(s, case, numels, first):
    """The plan over the state's tensors and the optimizer over its entries, as a user's program keeps them."""
    from paper_2509_03047_amd import flashrestore as F

    op, gsize = s["op"], 2 if case["grad"] == "bf16" else 4
    ns, st = np.asarray(numels, dtype=np.int64), s["starts"]
    gtype = F.FR_BF16 if gsize == 2 else F.FR_F32
    where = s.get("where") or {k: j * s["flat"] for k, j in (("param", 0), ("master", 2), ("m", 6), ("v", 10))}
    arena = s["state"].numel() if "state" in s else 14 * s["flat"]
    form = [("param", F.FR_BF16, 2, ns)] + [(k, F.FR_F32, 4, ns) for k in ("master", "m", "v")]
    if "m8" in where:
        form += [("m8", F.FR_F32, 1, -(-ns // 4)), ("v8", F.FR_F32, 1, -(-ns // 4)),
                 ("ms", F.FR_F32, 4 / BLOCK, -(-ns // BLOCK)), ("vs", F.FR_F32, 4 / BLOCK, -(-ns // BLOCK))]
    if "m_back" in where:
        form += [("m_back", F.FR_F32, 4, ns), ("v_back", F.FR_F32, 4, ns)]
    names, w = [f[0] for f in form], len(form)
    table = np.zeros((len(numels), w), dtype=F.DESC_DTYPE)
    for j, (name, dtype, per, count) in enumerate(form):
        at = where[name] + (st * per).astype(np.int64)
        table[:, j]["src_offset"] = table[:, j]["dst_offset"] = at
        table[:, j]["numel"], table[:, j]["dtype"], table[:, j]["derive_from"] = count, dtype, -1
    table[:, 0]["derive_from"] = np.arange(len(numels)) * w + 1
    plan = s["plan"] = F.Plan(table.reshape(-1), case.get("chunk", 1 << 16), arena, arena)

    def rows(m, v, ms, vs):
        r = np.zeros(len(numels), dtype=F.ADAMW_DTYPE)
        e = np.arange(len(numels)) * w
        r["grad_offset"], r["grad_dtype"], r["group"] = st * gsize, gtype, np.arange(len(numels)) >= first
        for field, name in (("param", "param"), ("master", "master"), ("m", m), ("v", v), ("m_scale", ms),
                            ("v_scale", vs)):
            r[field] = e + names.index(name) if name in names else -1
        return r

    grad_bytes = s["flat"] * gsize
    s["opt"] = F.AdamW(plan, rows("m", "v", "", ""), GROUPS, grad_bytes)
    if "m8" in where:
        s["opt8"] = F.AdamW(plan, rows("m8", "v8", "ms", "vs"), GROUPS, grad_bytes)
    if "m_back" in where:
        s["opt_back"] = F.AdamW(plan, rows("m_back", "v_back", "", ""), GROUPS, grad_bytes)
    s["stats"] = s["opt"].empty_stats().zero_()
    if op in ("step_sums", "step8"):  # what the norm over all ranks has left
        s["stats"].view(torch.float32)[3] = s["scale"]


# ------------------------------------------------------------- plain forms


def _noise(s, seeds):
    """Each element's two random numbers: a hash of its place and its group's seed; one half without a seed."""
    out = []
    for lo, hi, seed in ((0, s["split"], seeds[0]), (s["split"], s["flat"], seeds[1])):
        if not seed:
            return 1 << (_M - 1), 1 << (_V - 1)
        x = torch.arange(lo, hi, device="cuda").mul_(0x9E3779B9).add_(seed).bitwise_and_(0xFFFFFFFF)
        x.bitwise_xor_(x >> 16).mul_(0xB504F333).bitwise_and_(0xFFFFFFFF)
        x.bitwise_xor_(x >> 15).mul_(0x93CD3A2D).bitwise_and_(0xFFFFFFFF)
        out.append(x.bitwise_xor_(x >> 16))
    x = torch.cat(out)
    return (x >> 12).to(torch.int32), (x & 0x7FFFF).to(torch.int32)


def _codes(x, drop, rnd):
    """Codes of magnitudes and each block's scale."""
    x = x.view(-1, BLOCK)
    e = (x.view(torch.int32).amax(1, keepdim=True) - 1 >> 23) + 1  # of the power of two not below any
    y = (x * ((254 - e) << 23).view(torch.float32) * 2.0 ** -112).view(torch.int32)
    y = (y + (rnd.view(-1, BLOCK) if torch.is_tensor(rnd) else rnd)) >> drop
    none, bad = e < 28, e >= 254
    scale = (e << 23).view(torch.float32).masked_fill(none, 0.0).masked_fill(bad, math.nan)
    return y.masked_fill(none | bad, 0).view(-1), scale.view(-1)


def _keep(s, m, r, rnd):
    """The moments m and r * r, kept in 8 bits."""
    c, scale = _codes(m.abs(), _M, rnd[0])
    s["m8"].copy_(c | ((m.view(torch.int32) >> 24) & 128))
    s["ms"].copy_(scale)
    c, scale = _codes(r, _V, rnd[1])
    s["v8"].copy_(c)
    s["vs"].copy_(scale)


def _kept(s):
    """The moments that the codes stand for."""
    c = s["m8"].to(torch.int32)
    m = ((c & 127) << _M).view(torch.float32) * 2.0 ** 112
    m = ((m * torch.where(c > 127, -1.0, 1.0)).view(-1, BLOCK) * s["ms"].view(-1, 1)).view(-1)
    r = (s["v8"].to(torch.int32) << _V).view(torch.float32) * 2.0 ** 112
    r = (r.view(-1, BLOCK) * s["vs"].view(-1, 1)).view(-1)
    return m, r * r


def _norm(s):
    g = s["grad"].float()
    norm = (g * g).sum().sqrt()
    return norm, torch.where(norm > s["max_norm"], s["max_norm"] / norm, 1.0)


def _step(s, m, v, scale):
    """New masters, moments and roots of second moments; both groups in one pass over halves of the buffers."""
    a, b = slice(0, s["split"]), slice(s["split"], s["flat"])
    return [torch.cat(x) for x in zip(_step_of(s["master"][a], m[a], v[a], s["grad"][a], scale, s["hyper"][0]),
                                      _step_of(s["master"][b], m[b], v[b], s["grad"][b], scale, s["hyper"][1]))]


def _step_of(p, m, v, g, scale, h):
    lr, b1, b2, eps, wd, c1, c2, _ = h.unbind()
    g = g.float() * scale
    m = m * b1 + g * (1 - b1)
    v = v * b2 + (g * g) * (1 - b2)
    r = v.sqrt()
    d = r * (1 / c2.sqrt()) + eps
    return p * (1 - lr * wd) - (m / d) * (lr / c1), m, v, r


def _frsum(s):
    """(sum of w_i, sum of (i + 1) w_i) of the 32-bit words of each chunk, in 64 bits that wrap."""
    for kind, (first, last, at) in s["chunks"].items():
        w = s[kind].view(torch.int32).to(torch.int64) & 0xFFFFFFFF
        i = torch.arange(1, w.numel() + 1, device=w.device)
        one, many = _behind(w), _behind(w * i)
        total = one[last] - one[first]
        s["sums"][at, 0] = total
        s["sums"][at, 1] = many[last] - many[first] - first * total


def _behind(w):
    """Sums of the words in front of each place, and of all."""
    return torch.cat([w.new_zeros(1), torch.cumsum(w, 0)])


# ------------------------------------------------------------------ passes


def run(s):
    if own:
        return _run_own(s)
    op = s["op"]
    if op == "norm":
        norm, scale = _norm(s)
        return {"norm": norm, "scale": scale}
    if op == "widen":
        m, v = _kept(s)
        return {"m": s["m"].copy_(m), "v": s["v"].copy_(v)}
    if op == "narrow":
        _keep(s, s["m"], s["v"].sqrt(), _noise(s, s["seeds"][:1] * 2))
        m, v = _kept(s)
        return {"m": s["m_back"].copy_(m), "v": s["v_back"].copy_(v)}
    out = {}
    scale = s["scale"]
    if op == "step":
        out["norm"], scale = _norm(s)
        out["scale"] = scale
    m, v = _kept(s) if op == "step8" else (s["m"], s["v"])
    p, m, v, r = _step(s, m, v, scale)
    if op == "step8":
        _keep(s, m, r, _noise(s, s["seeds"]))
        m, v = _kept(s)
    out["m"], out["v"] = s["m"].copy_(m), s["v"].copy_(v)
    out["master"] = s["master"].copy_(p)
    out["param"] = s["param"].copy_(p)
    if op == "step_sums":
        _frsum(s)
        out["sums"] = s["sums"]
    return out


def _run_own(s):
    op, opt, state, stats = s["op"], s["opt"], s.get("state"), s["stats"]
    parts = stats.view(torch.float32)
    if op == "norm":
        opt.grad_norm(s["grad"], s["max_norm"], stats)
        return {"norm": parts[2], "scale": parts[3]}
    if op == "widen":
        s["opt8"].convert(state, opt, state)
        return {"m": s["m"], "v": s["v"]}
    if op == "narrow":
        opt.convert(state, s["opt8"], state, s["seeds"][0])
        s["opt8"].convert(state, s["opt_back"], state)
        return {"m": s["m_back"], "v": s["v_back"]}
    out = {}
    if op == "step":
        opt.grad_norm(s["grad"], s["max_norm"], stats)
        out["norm"], out["scale"] = parts[2], parts[3]
    if op == "step8":
        s["opt8"].step(state, s["grad"], s["hyper"], stats)
        s["opt8"].convert(state, opt, state)
    else:
        opt.step(state, s["grad"], s["hyper"], stats, s.get("sums"))
    out.update(m=s["m"], v=s["v"], master=s["master"], param=s["param"])
    if op == "step_sums":
        out["sums"] = s["sums"]
    return out


def work(case):
    n, g = sum(_numels(case)), 2 if case["grad"] == "bf16" else 4
    b, f = {"norm": (g, 2), "step": (26 + g, 20), "step_sums": (26 + g, 34), "step8": (14 + 8 / BLOCK * 2 + g + 8, 50),
            "narrow": (8 + 2 + 8, 20), "widen": (2 + 8, 6)}[case["op"]]
    b = b * n
    if case["op"] == "step_sums":
        b += 16 * sum(-(-2 * k // case["chunk"]) + 3 * -(-4 * k // case["chunk"]) for k in _numels(case))
    return {"bytes": float(b), "flops": float(f * n)}


# ------------------------------------------------------------ in 64 bits


def _shares(s, seed):
    """Each element's two thresholds in [0, 1) by which its magnitude is rounded up."""
    if not any(seed):
        return 0.5, 0.5
    m, v = _noise(s, seed)
    return m.double() / 2 ** _M, v.double() / 2 ** _V


def _rounded(x, bits, up):
    """x with every block's magnitudes rounded to `bits` bits behind the leading one, down to 2^-14 of the scale."""
    b = x.abs().view(-1, BLOCK)
    top = b.amax(1, keepdim=True)
    mantissa, exponent = torch.frexp(top)
    scale = torch.ldexp(torch.ones_like(top), exponent - (mantissa == 0.5).to(exponent.dtype))
    y = b / scale
    lsb = torch.ldexp(torch.ones_like(y), torch.clamp(torch.frexp(y).exponent - 1, min=-14) - bits)
    y = torch.floor(y / lsb + (up.view(-1, BLOCK) if torch.is_tensor(up) else up)) * lsb * scale
    y = torch.where(top <= 2.0 ** -100, 0.0, torch.where(top <= 2.0 ** 126, y, math.nan))
    return torch.copysign(y.view(-1), x)


def _meant(s):
    """The moments that the codes stand for."""
    c, d = s["m8"].double(), s["v8"].double()
    m, r = [torch.where(q < 2 ** b, q / 2 ** b * 2.0 ** -14,
                        (1 + q % 2 ** b / 2 ** b) * torch.exp2((q / 2 ** b).floor() - 15))
            for q, b in ((c % 128, 3), (d, 4))]
    m = (torch.where(c >= 128, -m, m).view(-1, BLOCK) * s["ms"].double().view(-1, 1)).view(-1)
    r = (r.view(-1, BLOCK) * s["vs"].double().view(-1, 1)).view(-1)
    return m, r * r


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "widen":
        m, v = _meant(s)
        return {"m": m, "v": v}
    if op == "narrow":
        um, uv = _shares(s, s["seeds"][:1] * 2)
        return {"m": _rounded(s["m"].double(), 3, um), "v": _rounded(s["v"].double().sqrt(), 4, uv).square()}
    out, scale = {}, s["scale"].double()
    if op in ("norm", "step"):
        norm = s["grad"].double().square().sum().sqrt()
        scale = torch.clamp(s["max_norm"] / norm, max=1.0)
        out = {"norm": norm, "scale": scale}
        if op == "norm":
            return out
    m0, v0 = _meant(s) if op == "step8" else (s["m"], s["v"])
    new = []
    for at, h in ((slice(0, s["split"]), s["hyper"][0]), (slice(s["split"], s["flat"]), s["hyper"][1])):
        lr, b1, b2, eps, wd, c1, c2 = h[:7].double().tolist()
        g = s["grad"][at].double() * scale
        m = torch.lerp(g, m0[at].double(), b1)
        v = torch.lerp(g.square_(), v0[at].double(), b2)
        p = s["master"][at].double() * (1 - lr * wd) - lr * (m / c1) / ((v / c2).sqrt() + eps)
        new.append((p, m, v))
    p, m, v = [torch.cat(x) for x in zip(*new)]
    if op == "step8":
        um, uv = _shares(s, s["seeds"])
        m, v = _rounded(m, 3, um), _rounded(v.sqrt(), 4, uv).square()
    out.update(m=m, v=v, master=p, param=p.to(torch.bfloat16))
    if op == "step_sums":
        out["sums"] = None
    return out
