"""The step by orthogonalised momentum and the embedding on the CPU: what they
refuse, the layout of a state, and properties of the plain models that the GPU
tests hold the kernels to."""
import numpy as np
import pytest

from paper_2509_03047_amd import flashrestore as F

from tests import muon_ref as R

INVAL, ALIGN, RANGE, OVERLAP = -1, -2, -3, -4


def _valid():
    return F.fr_muon_state_table([(20, 30), (7, 5), (0, 9)], F.FR_BF16)


def _status(t, r, ab, gb, ub, groups=1, C=4096, coeffs=None):
    try:
        F.fr_muon_query(t, C, ab, r, groups, gb, ub, coeffs)
        return 0
    except F.FlashRestoreError as e:
        return e.status


def test_state_table():
    shapes = [(20, 30), (7, 5), (0, 9), (1, 1), (128, 1024)]
    t, r, ab, gb, ub = F.fr_muon_state_table(shapes, F.FR_F32)
    numel = [a * b for a, b in shapes]
    i = F.fr_muon_query(t, 4096, ab, r, 1, gb, ub)
    assert i["n_tensors"] == 5 and i["n_steps"] == 5 and i["device"] == -1 and i["device_bytes"] == 0
    assert i["n_elements"] == sum(numel) and i["arena_bytes"] == ab
    assert i["grad_arena_bytes"] == gb == sum(-(-4 * n // 16) * 16 for n in numel)
    assert i["update_arena_bytes"] == ub == sum(-(-2 * n // 16) * 16 for n in numel)
    info, _, base = F.fr_layout_query(t, 4096, ab, ab)
    assert i["sums_chunks"] == info["n_chunks"] == int(base[-1])
    for k, n in enumerate(numel):
        assert [int(t[r[k][f]]["numel"]) for f in ("param", "master", "m")] == [n] * 3
        assert int(t[r[k]["param"]]["derive_from"]) == int(r[k]["master"])
        assert r[k]["scale"] == np.float32(0.2 * np.sqrt(max(shapes[k])))
    assert F.fr_muon_query(t, 64, ab, r, 1, gb, ub)["sums_chunks"] == 0
    assert len(F.fr_muon_state_table([])[0]) == 0


def test_state_table_behind_another():
    """The embedding and the norms under AdamW, the matrices behind them: one table, one plan."""
    t, r, ab, gb = F.fr_adamw_state_table([8000, 77])
    u, q, ab2, gb2, ub = F.fr_muon_state_table([(20, 30), (7, 5)], first_entry=len(t), arena_bytes=ab, grad_bytes=gb)
    both = np.concatenate([t, u])
    info, _, _ = F.fr_layout_query(both, 4096, ab2, ab2)
    assert info["n_entries"] == len(t) + 6
    assert F.fr_adamw_query(both, 4096, ab2, r, 1, gb2)["n_elements"] == 8077
    assert F.fr_muon_query(both, 4096, ab2, q, 1, gb2, ub)["n_elements"] == 635
    assert int(q["grad_offset"].min()) >= gb and int(u["src_offset"].min()) >= ab


def test_valid_baseline():
    assert _status(*_valid()) == 0
    t, r, ab, gb, ub = _valid()
    r["param"] = -1
    assert _status(t, r, ab, gb, ub) == 0
    r["grad_offset"] = 0  # gradients may overlap
    assert _status(t, r, ab, gb, ub) == 0
    assert _status(t, r[:0], ab, 0, 0) == 0


@pytest.mark.parametrize("field,value,status", [
    ("rows", 21, INVAL), ("cols", 29, INVAL), ("group", 1, INVAL), ("flags", 1, INVAL), ("reserved", 1, INVAL),
    ("grad_dtype", 3, INVAL), ("grad_dtype", 0, INVAL), ("param", -2, INVAL), ("param", 1, INVAL), ("param", 9, INVAL),
    ("master", -1, INVAL), ("master", 0, INVAL), ("master", 4, INVAL), ("m", -1, INVAL), ("m", 5, INVAL),
    ("m", 1, OVERLAP), ("scale", np.nan, INVAL), ("scale", np.inf, INVAL), ("grad_offset", 8, ALIGN),
    ("update_offset", 8, ALIGN), ("grad_offset", 1 << 40, RANGE), ("update_offset", 1 << 40, RANGE),
    ("update_offset", (1 << 64) - 16, RANGE), ("update_offset", 1200, OVERLAP), ("rows", 1 << 31, RANGE),
    ("cols", (1 << 20) + 1, RANGE),
])
def test_refusals(field, value, status):
    t, r, ab, gb, ub = _valid()
    r[field][0] = value
    assert _status(t, r, ab, gb + 4096, ub + 4096) == status


def test_refusals_of_arenas_and_tables():
    t, r, ab, gb, ub = _valid()
    assert _status(t, r, ab, gb - 32, ub) == RANGE
    assert _status(t, r, ab, gb, ub - 32) == RANGE
    t2 = t.copy()
    t2["derive_from"][0], t2["derive_from"][3] = -1, -1  # not derived at all: fine
    assert _status(t2, r, ab, gb, ub) == 0
    t2["src_offset"][2] = t2["src_offset"][1]  # momentum over the master
    assert _status(t2, r, ab, gb, ub) == OVERLAP
    twice = np.concatenate([r, r[:1]])
    twice["update_offset"][-1] = 1 << 13
    assert _status(t, twice, ab, gb, 1 << 14) == OVERLAP


@pytest.mark.parametrize("coeffs", [
    [], [(1.0, 0.0, 0.0)] * 17, [(np.nan, 0, 0)], [(1, np.inf, 0)], [(1, 0, -np.inf)], [(5.0, 0.0, 0.0)],
    [(2.0, 0.0, 0.0)] * 3, [(1.0, 70.0, -70.0)], [(1.0, 0.0, 0.0), (3.0, 1.5, 0.0)]])
def test_refusals_of_coefficients(coeffs):
    c = np.array(coeffs, np.float32).reshape(-1, 3)
    assert _status(*_valid(), coeffs=c) == INVAL
    assert _status(*_valid(), coeffs=[(1.5, -0.5, 0.0)] * 16) == 0


@pytest.mark.parametrize("shape,ok", [((1 << 20, 1), True), ((1, 1 << 20), True), (((1 << 20) + 1, 1), False),
                                      ((1 << 15, 1 << 15), True), ((1 << 15, 1 << 16), False),
                                      (((1 << 15) + 1, (1 << 15) + 1), False), ((46341, 46341), False)])
def test_limits_of_shapes(shape, ok):
    if ok:
        t, r, ab, gb, ub = F.fr_muon_state_table([shape])
        assert F.fr_muon_query(t, 1 << 20, ab, r, 1, gb, ub)["n_elements"] == shape[0] * shape[1]
    else:
        with pytest.raises(F.FlashRestoreError) as e:
            F.fr_muon_state_table([shape])
        assert e.value.status == RANGE


def test_too_many_elements():
    t, r, ab, gb, ub = F.fr_muon_state_table([(1 << 15, 1 << 15)] * 16)
    assert _status(t, r, ab, gb, ub, C=1 << 20) == RANGE


def test_null_pointers():
    L = F._lib
    assert L.fr_muon_create(None, None, 0, 0, 0, 0, None, 0, None) == INVAL
    assert L.fr_muon_get_info(None, None) == INVAL and L.fr_muon_destroy(None) == 0
    assert L.fr_muon_query(None, 0, 4096, 0, None, 0, 0, 0, 0, None, 0, None) == INVAL
    assert L.fr_muon_direction(None, None, None, None, None, None, None, None) == INVAL
    assert L.fr_muon_grad_norm(None, None, 1.0, None, None) == INVAL
    assert L.fr_muon_orthogonalize(None, None, None, None, None) == INVAL
    assert L.fr_muon_apply(None, None, None, None, None, None, None) == INVAL
    assert L.fr_embed_create(None, None, 0, None) == INVAL
    assert L.fr_embed_get_info(None, None) == INVAL and L.fr_embed_destroy(None) == 0
    assert L.fr_embed_lookup(None, None, None, 8, 0, 1.0, None, 1, 1, None) == INVAL
    assert L.fr_embed_grad(None, None, 8, 0, None, 1, 1, 1.0, None, 0, None) == INVAL


def test_hyperparameters():
    h = F.muon_hyper([dict(lr=0.1), dict(lr=0.2, momentum=0.5, nesterov=False, eps=0.0, weight_decay=0.3)])
    assert h.dtype.itemsize == 32 and h["nesterov"].tolist() == [1, 0] and h["momentum"][0] == np.float32(0.95)
    with pytest.raises(ValueError):
        F.muon_hyper([dict(lr=0.1, betas=(0.9, 0.95))])
    with pytest.raises(ValueError):
        F.fr_muon_state_table([(1, 2, 3)])
    with pytest.raises(ValueError):
        F.fr_muon_state_table([(-1, 2)])
    with pytest.raises(ValueError):
        F.fr_muon_query(*_query_of(_valid()), coeffs=[1.0, 2.0, 3.0])


def _query_of(v):
    t, r, ab, gb, ub = v
    return t, 4096, ab, r, 1, gb, ub


# ------------------------------------------------------------------ embedding


TABLE = F.as_table([(0, 0, 600, F.FR_BF16, 1), (2048, 2048, 600, F.FR_F32, -1)])


def _embed(**more):
    a = dict(entry=0, rows=20, cols=30, max_tokens=100, grad_arena_bytes=2400)
    a.update(more)
    try:
        return F.fr_embed_query(TABLE, 8192, **a)
    except F.FlashRestoreError as e:
        return e.status


def test_embedding_info():
    i = _embed(first=-5, grad_dtype=F.FR_F32)
    assert i["rows"] == 20 and i["cols"] == 30 and i["first"] == -5 and i["dtype"] == F.FR_BF16 and i["device"] == -1
    assert _embed(entry=1)["dtype"] == F.FR_F32
    assert _embed(max_tokens=0, grad_arena_bytes=0)["max_tokens"] == 0  # lookups only


@pytest.mark.parametrize("more,status", [
    (dict(entry=2), INVAL), (dict(entry=-1), INVAL), (dict(rows=19), INVAL), (dict(cols=31), INVAL),
    (dict(rows=0), INVAL), (dict(cols=0), INVAL), (dict(grad_dtype=3), INVAL), (dict(grad_offset=8), ALIGN),
    (dict(grad_arena_bytes=1199), RANGE), (dict(grad_offset=1216), RANGE), (dict(max_tokens=1 << 30), RANGE),
    (dict(grad_offset=(1 << 64) - 16), RANGE), (dict(first=(1 << 63) - 20), RANGE),
])
def test_embedding_refusals(more, status):
    assert _embed(**more) == status


def test_embedding_limits():
    big = F.as_table([(0, 0, 1 << 30, F.FR_BF16, -1)])
    ok = F.fr_embed_query(big, 1 << 31, 0, 1 << 20, 1 << 10, max_tokens=10,
                          grad_arena_bytes=1 << 31)
    assert ok["rows"] == 1 << 20
    for rows, tokens in ((1 << 26, 10), (1 << 20, (1 << 30) - 1)):
        with pytest.raises(F.FlashRestoreError) as e:
            F.fr_embed_query(big, 1 << 31, 0, rows, (1 << 30) // rows, max_tokens=tokens, grad_arena_bytes=1 << 31)
        assert e.value.status == RANGE


# --------------------------------------------------------------- plain models


def test_plain_orthogonalisation_is_the_polynomial_of_singular_values():
    rng = np.random.default_rng(0)
    for shape in ((6, 9), (9, 6), (5, 5)):
        g = rng.standard_normal(shape)
        u, s, v = np.linalg.svd(g, full_matrices=False)
        s = s / (np.linalg.norm(g) + 1e-7)
        for a, b, c in np.asarray(R.STEPS, np.float32).astype(np.float64):
            s = a * s + b * s ** 3 + c * s ** 5
        assert np.allclose(R.orthogonalized(g), (u * s) @ v, atol=1e-12)


def test_plain_gradient_sums_all_tokens():
    rng = np.random.default_rng(1)
    ids = rng.integers(-2, 5, 9000)
    x = rng.integers(-8, 9, (9000, 3)).astype(np.float32)  # exact in any order
    g, there = R.embedding_gradient(ids, x, 5, 0, 0.5)
    for v in range(5):
        assert np.array_equal(g[v], 0.5 * x[ids == v].sum(0))
    assert there.all()
