"""Orthogonalised updates of a training state's matrices and its embedding, as cases to measure.

A case is one pass of an operator: the Newton-Schulz orthogonalisation of all
matrices of a gradient arena at once ("orthogonalize"); the same behind the
momentum that a state keeps ("direction"); the step that writes masters and
bf16 parameters from such updates, with the chunk sums that replicas exchange
where the case has a chunk size ("apply"); the embedding's rows for a batch of
tokens ("lookup") and the gradient that they leave in its place of the gradient
arena ("embed_grad").

Matrices of a kind (parameters, masters, momenta, gradients, updates) lie
behind one another, each from a multiple of 1,024 elements on.  They are those
of the toy decoder ("toy"), of layers of one tensor-parallel rank's share of an
8B model ("8b"), or have log-uniform sides ("ragged").
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

SPAN = 1024  # a matrix starts at a multiple of it in the flat buffers
STEPS = ((3.4445, -4.7750, 2.0315),) * 5  # x -> a x + b x^3 + c x^5 on singular values
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}


# ------------------------------------------------------------------- cases


def listed():
    return [
        # a small model's eight matrices: launches count
        dict(name="toy-orthogonalize", op="orthogonalize", layout="toy", layers=2, grad="bf16"),
        # odd sides, tall and wide, rows, columns, a matrix of zeros
        dict(name="odd-orthogonalize", op="orthogonalize", layout="ragged", count=12, lo=1, hi=1300, table_seed=3,
             grad="f32", zeros=True),
        # a rank's gradients of four layers, as pipeline stages and sharded optimizers hand them over
        dict(name="8b-orthogonalize", op="orthogonalize", layout="8b", layers=4, grad="bf16", zeros=False),
        # momentum in front of it: the small model, with gradients in 32 bits; the whole of a rank's share
        dict(name="toy-direction", op="direction", layout="toy", layers=2, grad="f32", nesterov=True, chunk=1 << 14),
        dict(name="8b-direction", op="direction", layout="8b", layers=32, grad="bf16", nesterov=True, chunk=0),
        # the step itself: small, over the whole share, and there with the sums that replicas compare
        dict(name="toy-apply", op="apply", layout="toy", layers=2, grad="bf16", chunk=1 << 14),
        dict(name="8b-apply", op="apply", layout="8b", layers=32, grad="bf16", chunk=0),
        dict(name="8b-apply-sums", op="apply", layout="8b", layers=32, grad="bf16", chunk=1 << 16),
        # a small decoder's batch; the first rank's share of a vocabulary, which has the frequent tokens
        dict(name="toy-lookup", op="lookup", vocab=8192, first=0, rows=8192, cols=256, tokens=2048, table="bf16",
             act="bf16", ids="i64", scaled=True),
        dict(name="8b-lookup", op="lookup", vocab=128256, first=0, rows=16032, cols=4096, tokens=16384, table="bf16",
             act="bf16", ids="i64", scaled=False),
        # their gradients: all rows of the toy's table; the share's, on top of what the tied head has left
        dict(name="toy-embed-grad", op="embed_grad", vocab=8192, first=0, rows=8192, cols=256, tokens=2048,
             table="bf16", act="bf16", ids="i64", scaled=True, grad="f32", add=False),
        dict(name="8b-embed-grad", op="embed_grad", vocab=128256, first=0, rows=16032, cols=4096, tokens=16384,
             table="bf16", act="bf16", ids="i64", scaled=False, grad="bf16", add=True),
    ]


def _log(rng, lo, hi):
    """A whole number, spread evenly over the logarithm of [lo, hi]."""
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    while True:
        op = rng.choice(["orthogonalize", "direction", "apply", "lookup", "embed_grad"])
        c = dict(op=op)
        if op in ("lookup", "embed_grad"):
            vocab = _log(rng, 200, 250000)
            rows = vocab if rng.random() < 0.5 else -(-vocab // rng.choice([2, 4, 8]))
            c.update(vocab=vocab, rows=rows, first=rng.choice([0, vocab - rows]), cols=_log(rng, 16, 8192),
                     tokens=_log(rng, 1, 65536), table=rng.choice(["bf16", "f32"]), act=rng.choice(["bf16", "f32"]),
                     ids=rng.choice(["i32", "i64"]), scaled=rng.random() < 0.5)
            if op == "embed_grad":
                c.update(grad=rng.choice(["bf16", "f32"]), add=rng.random() < 0.5)
            if c["cols"] * max(c["tokens"], c["rows"]) <= 1 << 28:
                return c
            continue
        c["grad"] = rng.choice(["bf16", "f32"])
        kind = rng.choice(["toy", "8b", "ragged", "ragged"])
        c.update(layout=kind)
        if kind == "ragged":
            c.update(count=_log(rng, 1, 40), lo=_log(rng, 1, 512), table_seed=rng.randrange(1 << 20))
            c["hi"] = c["lo"] * _log(rng, 1, 16)
        else:
            c["layers"] = _log(rng, 1, 24)
        if op == "orthogonalize":
            c["zeros"] = rng.random() < 0.3
        if op == "direction":
            c["nesterov"] = rng.random() < 0.7
        if op in ("direction", "apply"):
            c["chunk"] = rng.choice([0, 1 << rng.randint(12, 20)])
        if _multiplications(c) <= _multiplications(dict(layout="8b", layers=32)):
            return c


# ------------------------------------------------------------------ shapes


def _shapes(case):
    """(rows, columns) of the matrices in their order."""
    if case["layout"] == "toy":
        return [(256, 768), (256, 256), (256, 1024), (1024, 256)] * case["layers"]
    if case["layout"] == "8b":
        layer = [(512, 4096), (128, 4096), (128, 4096), (4096, 512), (1792, 4096), (1792, 4096), (4096, 1792)]
        return layer * case["layers"]
    rng = np.random.Generator(np.random.PCG64(case["table_seed"]))
    sides = np.floor(case["lo"] * (case["hi"] / case["lo"]) ** rng.random((case["count"], 2))).astype(np.int64)
    return [(int(a), int(b)) for a, b in sides]


def _starts(shapes):
    """Where each matrix starts in the flat buffers, and their length."""
    ends = np.cumsum([-(-a * b // SPAN) * SPAN for a, b in shapes])
    return np.concatenate([[0], ends[:-1]]).astype(np.int64), int(ends[-1])


def _multiplications(case):
    """Of one orthogonalisation of all matrices: half of those of X X^T and of its square, which are symmetric."""
    total = 0
    for a, b in _shapes(case):
        m, n = min(a, b), max(a, b)
        total += len(STEPS) * (m * m * n / 2 + m ** 3 / 2 + m * m * n)
    return total


def work(case):
    op = case["op"]
    if op in ("lookup", "embed_grad"):
        return _embedding_work(case)
    n, g, f = sum(a * b for a, b in _shapes(case)), SIZE[case["grad"]], 2 * _multiplications(case)
    if op == "orthogonalize":
        return {"bytes": float(n * (g + 2)), "flops": float(f + 2 * n)}
    if op == "direction":
        return {"bytes": float(n * (g + 4 + 4 + 2)), "flops": float(f + 6 * n)}
    return {"bytes": float(n * (4 + 2 + 4 + 2)), "flops": float(n * (3 + (6 if case["chunk"] else 0)))}


def _embedding_work(case):
    D, lo, hi = case["cols"], case["first"] + 1, case["first"] + case["rows"] + 1
    here = case["tokens"] * math.log(hi / lo) / math.log(case["vocab"] + 1)  # tokens of the rank's rows
    ids = np.arange(lo, hi)
    p = np.log1p(1.0 / ids) / math.log(case["vocab"] + 1)
    rows = float(np.sum(-np.expm1(case["tokens"] * np.log1p(-p))))  # of which so many differ
    idb, a = {"i32": 4, "i64": 8}[case["ids"]], SIZE[case["act"]]
    if case["op"] == "lookup":
        return {"bytes": idb * case["tokens"] + D * (rows * SIZE[case["table"]] + case["tokens"] * a),
                "flops": D * here}
    g = SIZE[case["grad"]]
    written = 2 * rows if case["add"] else case["rows"]
    return {"bytes": idb * case["tokens"] + D * (here * a + written * g), "flops": D * (here + rows)}


# ------------------------------------------------------------------ inputs


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    if case["op"] in ("lookup", "embed_grad"):
        return _prepare_embedding(case, gen)
    shapes = _shapes(case)
    starts, flat = _starts(shapes)
    op = case["op"]
    s = dict(op=op, shapes=shapes, starts=starts, flat=flat, chunk=case.get("chunk", 0))

    def normal(sd, dtype):
        x = torch.zeros(flat, dtype=dtype, device="cuda")
        for (a, b), at in zip(shapes, starts.tolist()):
            x[at: at + a * b].normal_(0.0, sd, generator=gen)
        return x

    def gradients(dtype):
        """Rows and columns of sizes of their own, a few directions above the noise of a batch, as gradients have."""
        x = torch.zeros(flat, dtype=dtype, device="cuda")
        for (a, b), at in zip(shapes, starts.tolist()):
            r = min(8, a, b)
            u, v = (torch.randn(k, generator=gen, device="cuda") for k in ((a, r), (r, b)))
            g = torch.randn((a, b), generator=gen, device="cuda") + 0.5 * (u @ v)
            g *= torch.exp(0.3 * torch.randn((a, 1), generator=gen, device="cuda"))
            x[at: at + a * b] = (1e-3 * g).reshape(-1).to(dtype)
        return x

    s["updates"] = torch.zeros(flat, dtype=torch.bfloat16, device="cuda")
    if op == "apply":
        s["updates"].copy_(normal(1.0 / math.sqrt(max(max(x) for x in shapes)), torch.float32))
    else:
        s["grad"] = gradients(TORCH[case["grad"]])
        if case.get("zeros"):
            k = len(shapes) // 2
            s["grad"][int(starts[k]): int(starts[k]) + shapes[k][0] * shapes[k][1]] = 0
    if op != "orthogonalize":
        s["state"] = torch.zeros(10 * flat, dtype=torch.uint8, device="cuda")
        for name, dtype, lo, hi in (("param", torch.bfloat16, 0, 2), ("master", torch.float32, 2, 6),
                                    ("m", torch.float32, 6, 10)):
            s[name] = s["state"][lo * flat: hi * flat].view(dtype)
        s["master"].copy_(normal(0.02, torch.float32))
        s["param"].copy_(s["master"])
        if op == "direction":
            s["m"].copy_(gradients(torch.float32)).mul_(5.0)
    # learning rate, momentum, eps, weight decay; the clip scale of a step
    s["hyper"] = (2e-3, 0.95, 1e-7, 0.1)
    s["nesterov"] = bool(case.get("nesterov", True))
    s["scales"] = [0.2 * math.sqrt(max(x)) for x in shapes]
    s["clip"] = torch.tensor(0.5 + (seed % 64) / 128, dtype=torch.float32, device="cuda")
    if s["chunk"]:
        _chunks(s)
        s["sums"] = torch.zeros(s["n_chunks"], 2, dtype=torch.int64, device="cuda")
    if own:
        _handles(s, case)
    return s


def _prepare_embedding(case, gen):
    V, D, T, dev = case["rows"], case["cols"], case["tokens"], "cuda"
    s = dict(op=case["op"], V=V, D=D, first=case["first"], scale=math.sqrt(D) if case["scaled"] else 1.0)
    # tokens of a text: the k-th most frequent one comes about 1 / k as often as the first
    u = torch.rand(T, generator=gen, device=dev, dtype=torch.float64)
    ids = (torch.exp(u * math.log(case["vocab"] + 1)).long() - 1).clamp_(0, case["vocab"] - 1)
    s["ids"] = ids.to({"i32": torch.int32, "i64": torch.int64}[case["ids"]])
    if case["op"] == "lookup":
        dtype = TORCH[case["table"]]
        s["table"] = torch.empty(V * D, dtype=dtype, device=dev).normal_(0.0, 0.02, generator=gen).view(V, D)
        s["out"] = torch.zeros(T, D, dtype=TORCH[case["act"]], device=dev)
    else:
        s["dout"] = torch.empty(T, D, dtype=TORCH[case["act"]], device=dev).normal_(0.0, 1e-3, generator=gen)
        s["add"] = case["add"]
        s["grad"] = torch.empty(V, D, dtype=TORCH[case["grad"]], device=dev).normal_(0.0, 1e-3, generator=gen)
    if own:
        from paper_2509_03047_amd import flashrestore as F

        lookup = case["op"] == "lookup"
        es = SIZE[case["table"]]
        arena = -(-V * D * es // 16) * 16
        types = {"bf16": F.FR_BF16, "f32": F.FR_F32}
        s["plan"] = F.Plan(F.as_table([(0, 0, V * D, types[case["table"]], -1)]), 1 << 16, arena, arena)
        s["emb"] = F.Embedding(s["plan"], 0, V, D, max_tokens=T, first=case["first"],
                               grad_dtype=types[case.get("grad", "bf16")],
                               grad_arena_bytes=V * D * SIZE[case.get("grad", "bf16")])
        if lookup:
            s["state"] = torch.zeros(arena, dtype=torch.uint8, device=dev)
            s["state"][: V * D * es].view(s["table"].dtype).copy_(s["table"].view(-1))
    return s


def _chunks(s):
    """The chunks of [parameter, master, momentum] of every matrix in turn: for each kind, each chunk's first and last
    word in the flat buffer, and its number."""
    nb = np.array([a * b for a, b in s["shapes"]], dtype=np.int64)[:, None] * np.array([2, 4, 4])
    count = -(-nb // s["chunk"])
    base = np.concatenate([[0], np.cumsum(count.reshape(-1))])
    s["n_chunks"], s["chunks"] = int(base[-1]), {}
    for j, kind in enumerate(("param", "master", "m")):
        k = np.repeat(np.arange(len(nb)), count[:, j])
        i = np.arange(len(k)) - np.repeat(np.cumsum(count[:, j]) - count[:, j], count[:, j])
        first = s["starts"][k] * (2 if j == 0 else 4) // 4 + i * (s["chunk"] // 4)
        last = first + np.minimum(s["chunk"], nb[k, j] - i * s["chunk"] + 3) // 4
        s["chunks"][kind] = tuple(torch.from_numpy(x).cuda() for x in (first, last, base[:-1].reshape(-1, 3)[k, j] + i))


def _handles(s, case):
    """The plan over the state's tensors and the optimizer over its matrices, as a user's program keeps them."""
    from paper_2509_03047_amd import flashrestore as F

    flat, st, n = s["flat"], s["starts"], len(s["shapes"])
    numel = np.array([a * b for a, b in s["shapes"]], dtype=np.int64)
    table = np.zeros((n, 3), dtype=F.DESC_DTYPE)
    for j, (at, size, dtype) in enumerate(((0, 2, F.FR_BF16), (2 * flat, 4, F.FR_F32), (6 * flat, 4, F.FR_F32))):
        table[:, j]["src_offset"] = table[:, j]["dst_offset"] = at + st * size
        table[:, j]["numel"], table[:, j]["dtype"], table[:, j]["derive_from"] = numel, dtype, -1
    e = 3 * np.arange(n)
    table[:, 0]["derive_from"] = e + 1
    s["plan"] = F.Plan(table.reshape(-1), s["chunk"] or 1 << 16, 10 * flat, 10 * flat)
    gsize = SIZE[case["grad"]]
    r = np.zeros(n, dtype=F.MUON_DTYPE)
    r["grad_offset"], r["grad_dtype"] = st * gsize, F.FR_BF16 if gsize == 2 else F.FR_F32
    r["update_offset"] = st * 2
    r["rows"], r["cols"] = np.array(s["shapes"]).T
    r["param"], r["master"], r["m"] = e, e + 1, e + 2
    r["scale"] = s["scales"]
    s["opt"] = F.Muon(s["plan"], r, 1, flat * gsize, flat * 2, STEPS)
    lr, momentum, eps, decay = s["hyper"]
    h = F.muon_hyper([dict(lr=lr, momentum=momentum, eps=eps, weight_decay=decay, nesterov=s["nesterov"])])
    s["rows"] = torch.from_numpy(h.view(np.uint8)).cuda()
    s["stats"] = torch.zeros(3, dtype=torch.float64, device="cuda")
    s["stats"].view(torch.float32)[3] = s["clip"]  # what the norm over all ranks has left


# ------------------------------------------------------------- plain forms


def _orthogonalised(s, x):
    """bf16 updates of the matrices in the flat buffer x: all of one shape in batches."""
    alike = {}
    for k, shape in enumerate(s["shapes"]):
        alike.setdefault(shape, []).append(k)
    for (a, b), which in alike.items():
        at = torch.from_numpy(s["starts"][which]).cuda()[:, None] + torch.arange(a * b, device="cuda")
        X = x[at].view(len(which), a, b)
        if a > b:
            X = X.mT.contiguous()
        norm = X.double().square().sum((1, 2), keepdim=True).sqrt()
        X = X / (norm + s["hyper"][2]).float()
        for ca, cb, cc in STEPS:
            A = X @ X.mT.contiguous()
            X = ca * X + (cb * A + cc * (A @ A)) @ X
        if a > b:
            X = X.mT
        s["updates"][at] = X.reshape(len(which), a * b).to(torch.bfloat16)


def _frsum(s, kinds):
    """(sum of w_i, sum of (i + 1) w_i) of the 32-bit words of each chunk, in 64 bits that wrap."""
    for kind in kinds:
        first, last, at = s["chunks"][kind]
        w = s[kind].view(torch.int32).to(torch.int64) & 0xFFFFFFFF
        i = torch.arange(1, w.numel() + 1, device=w.device)
        one, many = _behind(w), _behind(w * i)
        total = one[last] - one[first]
        s["sums"][at, 0] = total
        s["sums"][at, 1] = many[last] - many[first] - first * total


def _behind(w):
    """Sums of the words in front of each place, and of all."""
    return torch.cat([w.new_zeros(1), torch.cumsum(w, 0)])


def _matrix_factors(s):
    """lr times each element's matrix's scale, over the flat buffers."""
    lengths = np.diff(np.append(s["starts"], s["flat"]))
    lr = torch.tensor(s["hyper"][0], dtype=torch.float32, device="cuda")
    per = lr * torch.tensor(s["scales"], dtype=torch.float32, device="cuda")
    return torch.repeat_interleave(per, torch.from_numpy(lengths).cuda())


def _rows_of(s):
    """Each token's row of the table, one past the end for another rank's; and whether it is here."""
    i = s["ids"].long() - s["first"]
    here = (i >= 0) & (i < s["V"])
    return torch.where(here, i, s["V"]), here


def run(s):
    if own:
        return _run_own(s)
    op = s["op"]
    if op == "lookup":
        i, here = _rows_of(s)
        x = s["table"][i.clamp(max=s["V"] - 1)].float() * s["scale"]
        return {"out": s["out"].copy_(torch.where(here[:, None], x, 0.0))}
    if op == "embed_grad":
        i, _ = _rows_of(s)
        g = torch.zeros(s["V"] + 1, s["D"], dtype=torch.float32, device="cuda")
        g.index_add_(0, i, s["dout"].float())
        g = g[:-1] * s["scale"]
        return {"grad": s["grad"].copy_(s["grad"].float() + g if s["add"] else g)}
    f32 = torch.float32
    lr, mu, _, wd = (torch.tensor(v, dtype=f32, device="cuda") for v in s["hyper"])
    if op == "orthogonalize":
        _orthogonalised(s, s["grad"].float())
        return {"updates": s["updates"]}
    if op == "direction":
        x = s["grad"].float() * s["clip"]
        s["m"].mul_(mu).add_(x)
        _orthogonalised(s, x + s["m"] * mu if s["nesterov"] else s["m"])
        out = {"m": s["m"], "updates": s["updates"]}
        kinds = ("m",)
    else:
        p = s["master"] * (1 - lr * wd) - s["updates"].float() * _matrix_factors(s)
        out = {"master": s["master"].copy_(p), "param": s["param"].copy_(p)}
        kinds = ("param", "master")
    if s["chunk"]:
        _frsum(s, kinds)
        out["sums"] = s["sums"]
    return out


def _run_own(s):
    op = s["op"]
    if op == "lookup":
        s["emb"].lookup(s["state"], s["ids"], s["out"], scale=s["scale"])
        return {"out": s["out"]}
    if op == "embed_grad":
        s["emb"].grad(s["ids"], s["dout"], s["grad"], scale=s["scale"], add=s["add"])
        return {"grad": s["grad"]}
    if op == "orthogonalize":
        s["opt"].orthogonalize(s["grad"], s["rows"], s["updates"])
        return {"updates": s["updates"]}
    if op == "direction":
        s["opt"].direction(s["state"], s["grad"], s["rows"], s["updates"], s["stats"], s.get("sums"))
        out = {"m": s["m"], "updates": s["updates"]}
    else:
        s["opt"].apply(s["state"], s["updates"], s["rows"], s["stats"], s.get("sums"))
        out = {"master": s["master"], "param": s["param"]}
    if s["chunk"]:
        out["sums"] = s["sums"]
    return out


# ------------------------------------------------------------ in 64 bits


def _polar(x, rows, cols, eps):
    """One matrix's update: the polynomials of x^T x or x x^T, whichever is smaller, applied to x."""
    X = x.double().view(rows, cols)
    X = X / (torch.linalg.norm(X) + eps)
    for a, b, c in STEPS:
        if rows > cols:
            G = torch.mm(X.t().contiguous(), X)
            Y = torch.mm(X, G)
            X = a * X + b * Y + c * torch.mm(Y, G)
        else:
            G = torch.mm(X, X.t().contiguous())
            Y = torch.mm(G, X)
            X = a * X + b * Y + c * torch.mm(G, Y)
    return X.reshape(-1)


def _all_polar(s, x):
    out = torch.zeros(s["flat"], dtype=torch.float64, device="cuda")
    for (a, b), at in zip(s["shapes"], s["starts"].tolist()):
        out[at: at + a * b] = _polar(x[at: at + a * b], a, b, s["hyper"][2])
    return out


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "lookup":
        out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
        i = s["ids"].long()
        (t,) = torch.nonzero((i >= s["first"]) & (i < s["first"] + s["V"]), as_tuple=True)
        out[t] = s["table"].double()[i[t] - s["first"]] * s["scale"]
        return {"out": out}
    if op == "embed_grad":
        # differences of running sums over the tokens in their rows' order
        i, order = torch.sort(s["ids"].long() - s["first"])
        ends = torch.searchsorted(i, torch.arange(s["V"] + 1, device="cuda"))
        grad = torch.empty(s["V"], s["D"], dtype=torch.float64, device="cuda")
        for c in range(0, s["D"], 256):
            run = torch.cumsum(s["dout"][:, c: c + 256][order].double(), 0)
            run = torch.cat([run.new_zeros(1, run.shape[1]), run])
            grad[:, c: c + 256] = (run[ends[1:]] - run[ends[:-1]]) * s["scale"]
        return {"grad": grad + s["grad"].double() if case["add"] else grad}
    lr, mu, _, wd = s["hyper"]
    if op == "orthogonalize":
        return {"updates": _all_polar(s, s["grad"])}
    sums = {"sums": None} if case["chunk"] else {}
    if op == "direction":
        x = s["grad"].double() * float(s["clip"])
        m = s["m"].double() * mu + x
        return {"m": m, "updates": _all_polar(s, x + mu * m if s["nesterov"] else m), **sums}
    step = torch.zeros(s["flat"], dtype=torch.float64, device="cuda")
    for (a, b), at, scale in zip(s["shapes"], s["starts"].tolist(), s["scales"]):
        step[at: at + a * b] = lr * scale
    p = s["master"].double() * (1 - lr * wd) - step * s["updates"].double()
    return {"master": p, "param": p, **sums}
