"""The optimizer step on the CPU: what an optimizer refuses, the layout of its
states, and the properties that the definition of 8-bit moments promises (of
the plain model, which the GPU tests hold the kernels to bit for bit)."""
import numpy as np
import pytest

from paper_2509_03047_amd import flashrestore as F

from tests import adamw_ref as R


def _valid():
    t, r, ab, gb = F.fr_adamw_state_table([1000, 77], [32, 8], F.FR_BF16)
    return t, r, ab, gb


def _status(t, r, ab, gb, groups=1, C=4096):
    try:
        F.fr_adamw_query(t, C, ab, r, groups, gb)
        return 0
    except F.FlashRestoreError as e:
        return e.status


def test_state_table():
    numel, bits = [1000, 0, 77, 1, 256, 257], [32, 8, 8, 32, 8, 8]
    t, r, ab, gb = F.fr_adamw_state_table(numel, bits, F.FR_F32)
    i = F.fr_adamw_query(t, 4096, ab, r, 1, gb)
    assert i["n_tensors"] == 6 and i["n_groups"] == 1 and i["device"] == -1
    assert i["n_elements"] == sum(numel) and i["n_elements_8bit"] == 0 + 77 + 256 + 257
    assert i["n_counters"] == 4 * 1024 + 1024 and i["arena_bytes"] == ab and i["grad_arena_bytes"] == gb
    info, _, base = F.fr_layout_query(t, 4096, ab, ab)  # a valid table of a plan, and contiguous
    assert i["sums_chunks"] == info["n_chunks"] == int(base[-1])
    end = 0
    for e in t:
        assert int(e["src_offset"]) == int(e["dst_offset"]) == end
        end += -(-int(e["numel"]) * (2 if e["dtype"] == F.FR_BF16 else 4) // 16) * 16
    assert end == ab
    for k, n in enumerate(numel):
        words = -(-n // 4) if bits[k] == 8 else n
        assert [int(t[r[k][f]]["numel"]) for f in ("param", "master", "m", "v")] == [n, n, words, words]
        assert int(t[r[k]["param"]]["derive_from"]) == int(r[k]["master"])
        if bits[k] == 8:
            assert [int(t[r[k][f]]["numel"]) for f in ("m_scale", "v_scale")] == [-(-n // 256)] * 2
        else:
            assert int(r[k]["m_scale"]) == int(r[k]["v_scale"]) == -1
    assert F.fr_adamw_query(t, 64, ab, r, 1, gb)["sums_chunks"] == 0
    with pytest.raises(F.FlashRestoreError):
        F.fr_adamw_state_table([5], [16])
    with pytest.raises(F.FlashRestoreError):
        F.fr_adamw_state_table([5], grad_dtype=3)
    assert len(F.fr_adamw_state_table([])[0]) == 0


def test_valid_baseline():
    assert _status(*_valid()) == 0
    t, r, ab, gb = _valid()
    r["param"] = -1  # masters alone
    assert _status(t, r, ab, gb) == 0
    r["grad_offset"] = 0  # gradients may overlap
    assert _status(t, r, ab, gb) == 0
    r["flags"] = F.FR_GRAD_NOT_COUNTED
    assert _status(t, r, ab, gb) == 0
    assert _status(t, r[:0], ab, gb) == 0


@pytest.mark.parametrize("field, value, code", [
    ("grad_dtype", 3, -1), ("group", 1, -1), ("flags", 2, -1), ("reserved", 1, -1),
    ("param", 99, -1), ("param", -2, -1), ("param", 1, -1),           # past the table; not -1; an fp32 entry
    ("master", -1, -1), ("master", 99, -1), ("master", 0, -1),        # none; past the table; a bf16 entry
    ("m", -1, -1), ("m", 6, -1), ("v", 99, -1),                       # none; another numel; past the table
    ("m_scale", 7, -1),                                               # one scale alone
    ("grad_offset", 8, -2), ("grad_offset", 1 << 40, -3), ("grad_offset", 160, 0), ("grad_offset", 176, -3),
    ("v", 2, -4),                                                     # m's entry again
])
def test_refusals(field, value, code):
    t, r, ab, gb = _valid()
    r[0][field] = value
    assert _status(t, r, ab, gb) == code


def test_refusals_of_overlaps_and_scales():
    t, r, ab, gb = _valid()
    r[1]["m_scale"], r[1]["v_scale"] = -1, -1  # codes are not values
    assert _status(t, r, ab, gb) == -1
    t, r, ab, gb = _valid()
    t[2]["src_offset"] = t[1]["src_offset"]  # sender ranges of a table may overlap, written ones may not
    assert F.fr_layout_query(t, 4096, ab, ab) and _status(t, r, ab, gb) == -4
    t, r, ab, gb = _valid()
    assert _status(t, np.concatenate([r, r[:1]]), ab, gb) == -4
    assert _status(t, r, ab - 16, gb) == -3 and _status(t, r, ab, gb, C=24) == -1
    assert _status(t, r, ab, gb, groups=0) == -1


@pytest.mark.parametrize("bits", [32, 8])
def test_refusal_of_more_threads_than_a_launch_has(bits):
    counters = (1 << 34) - 2048 - 1024  # with the tensor's own 2,048 just below 2^34
    for numel, code in ((counters, 0), (counters + 1, -3)):
        t, r, ab, gb = F.fr_adamw_state_table([numel], bits)
        assert _status(t, r, ab, gb, C=1 << 20) == code
    t, r, ab, gb = F.fr_adamw_state_table([1 << 33, 1 << 32], bits)
    assert _status(t, r, ab, gb, C=1 << 20) == 0


def test_create_without_a_plan_or_output():
    assert F._lib.fr_adamw_create(None, None, 0, 0, 0, None) == -1
    assert F._lib.fr_adamw_get_info(None, None) == -1 and F._lib.fr_adamw_destroy(None) == 0
    assert F._lib.fr_grad_norm(None, None, 1.0, None, None) == -1
    assert F._lib.fr_grad_scale(None, 1.0, None, None) == -1
    assert F._lib.fr_adamw_step(None, None, None, None, None, None, None) == -1
    assert F._lib.fr_adamw_convert(None, None, None, None, 0, None) == -1


def test_hyper_rows():
    h = F.adamw_hyper([dict(lr=1e-3), dict(lr=2e-3, betas=(0.8, 0.9), eps=1e-6, weight_decay=0.1, seed=7)], 3)
    assert h.nbytes == 64
    assert h[0]["bias1"] == np.float32(1 - 0.9 ** 3) and h[1]["bias2"] == np.float32(1 - 0.9 ** 3)
    assert h[1]["seed"] == 7 and h[0]["eps"] == np.float32(1e-8) and h[0]["weight_decay"] == 0
    with pytest.raises(ValueError):
        F.adamw_hyper([dict(lr=1e-3, beta=0.9)], 1)


# ------------------------------------------------- the definition's promises


def test_codes_stand_for_what_they_say():
    """Every code of a block with scale 1: a first moment's is sign, e4, m3 (denormal below 2^-14), a root's e4, m4."""
    one = np.array([1.0], np.float32)
    c = np.arange(256)
    m, v = R.decode(c.astype(np.uint8), c.astype(np.uint8), one, one)
    e, f = c % 128 // 8, c % 8
    want = np.where(e == 0, f / 8 * 2.0 ** -14, (1 + f / 8) * 2.0 ** (e - 15.0)) * np.where(c >= 128, -1, 1)
    assert np.array_equal(m.astype(np.float64), want)
    e, f = c // 16, c % 16
    want = np.where(e == 0, f / 16 * 2.0 ** -14, (1 + f / 16) * 2.0 ** (e - 15.0))
    assert np.array_equal(v.astype(np.float64), want * want)


@pytest.mark.parametrize("seed", [0, 5])
def test_a_kept_value_keeps_its_code(seed):
    """Encoding what codes stand for gives the same values, whatever the rounding (the scale is a power of two)."""
    rng = np.random.default_rng(1)
    m = (rng.standard_normal(5000) * np.exp(3 * rng.standard_normal(5000))).astype(np.float32)
    r = np.abs(m[::-1]).copy()
    a = R.decode(*R.encode(m, r, 0, 0))
    b = R.decode(*R.encode(a[0], np.sqrt(a[1]), 0, seed))
    assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])


def test_rounding_to_nearest_is_within_half_a_code():
    """Half a code: 2^-4 of a first moment, 2^-5 of a root, and below 2^-14 of the scale 2^-18 and 2^-19 of it."""
    rng = np.random.default_rng(2)
    m = (rng.standard_normal(1 << 16) * np.exp(4 * rng.standard_normal(1 << 16))).astype(np.float32)
    cm, cr, sm, sr = R.encode(m, np.abs(m), 0, 0)
    dm, dv = R.decode(cm, cr, sm, sr)
    s = np.repeat(sm, 256).astype(np.float64)
    assert np.all(np.abs(m).reshape(-1, 256).max(1) <= sm) and np.all(np.abs(m).reshape(-1, 256).max(1) * 2 > sm)
    x = m.astype(np.float64)
    assert np.all(np.abs(dm - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -18 * s) * (1 + 1e-6))
    assert np.all(np.abs(np.sqrt(dv.astype(np.float64)) - np.abs(x)) <= np.maximum(2.0 ** -5 * np.abs(x), 2.0 ** -19 * s) * (1 + 1e-6))


def test_stochastic_rounding_has_the_right_mean():
    """2^14 seeds of one block: the mean of a value lies within 5 standard errors, of at most half a code each."""
    rng = np.random.default_rng(3)
    m = (rng.standard_normal(256) * np.exp(2 * rng.standard_normal(256))).astype(np.float32)
    n = 1 << 14
    total = np.zeros((2, 256))
    for seed in range(1, n + 1):
        a, b = R.decode(*R.encode(m, np.abs(m), 4096, seed * 2654435 + 1))
        total += np.stack([a.astype(np.float64), np.sqrt(b.astype(np.float64))])
    top = 2.0 ** np.ceil(np.log2(np.abs(m).max()))
    x = np.abs(m).astype(np.float64)
    exponent = np.maximum(2.0 ** np.floor(np.log2(x)), 2.0 ** -14 * top)
    for mean, want, bits in ((total[0] / n, m.astype(np.float64), 3), (total[1] / n, x, 4)):
        assert np.all(np.abs(mean - want) <= 5 * 0.5 * exponent * 2.0 ** -bits / np.sqrt(n))


@pytest.mark.parametrize("seed", [1, 12345, 0xFFFFFFFF])
def test_hash_is_even_and_its_two_shares_independent(seed):
    """2^18 consecutive counters: top 6 bits of each share, alone, together and with the next counter's, against the
    uniform distribution (chi-square within 6 standard deviations), also across a carry into the high word."""
    for start in (0, (1 << 32) - (1 << 17)):
        h = R.counter_hash(np.arange(1 << 18, dtype=np.uint64) + np.uint64(start), seed).astype(np.int64)
        a, b = h >> 26, (h & 0x7FFFF) >> 13
        for x, k in ((a, 64), (b, 64), (a * 64 + b, 4096), (a[:-1] * 64 + a[1:], 4096), (b[:-1] * 64 + b[1:], 4096)):
            count = np.bincount(x, minlength=k)
            chi = float(((count - x.size / k) ** 2).sum() / (x.size / k))
            assert abs(chi - (k - 1)) < 6 * np.sqrt(2 * (k - 1)), (start, k, chi)


def test_special_blocks():
    z = np.zeros(256, np.float32)
    for x, scale in ((np.nan, np.nan), (np.inf, np.nan), (2.0 ** 126.5, np.nan), (2.0 ** 126, 2.0 ** 126),
                     (2.0 ** 125, 2.0 ** 125), (2.0 ** -99, 2.0 ** -99), (2.0 ** -100, 0.0), (1e-45, 0.0), (0.0, 0.0)):
        m = z.copy()
        m[7], m[9] = x, 1e-3 if not np.isfinite(x) else 0.0
        cm, cr, sm, sr = R.encode(m, m, 0, 0)
        assert np.array_equal(sm, np.array([scale], np.float32), equal_nan=True) and np.array_equal(sm, sr, equal_nan=True)
        dm, dv = R.decode(cm, cr, sm, sr)
        if np.isnan(scale):
            assert np.isnan(dm).all() and np.isnan(dv).all()
        else:
            assert dm[7] == (x if scale else 0.0) and np.count_nonzero(dm) == (1 if scale else 0)


def test_step_in_32_bits_is_the_step_in_64():
    """The definition against AdamW in 64 bits.  With u = 2^-24: m' sums two products of a rounded gradient, 5 u of
    their magnitudes; v' 7 u; in the update d carries half of v's and 5 u more, m' its 5 u, and three further
    roundings, under 20 u; w' three roundings of w and the update's."""
    u = 2.0 ** -24
    s = R.State([4099], 32, F.FR_F32, seed=4)
    h = F.adamw_hyper([dict(lr=3e-4, betas=(0.9, 0.95), weight_decay=0.1)], 10)[0]
    m, v = s.moments(0)
    w32, m32, v32, _ = R.step32(s.get(0, "master"), m, v, s.grad(0), h, 0.37)
    w64, m64, v64, aw, au, am = R.step64(s.get(0, "master"), m, v, s.grad(0), h, np.float32(0.37))
    assert np.all(np.abs(m32 - m64) <= 5 * u * am)
    assert np.all(np.abs(v32 - v64) <= 7 * u * v64)
    assert np.all(np.abs(w32 - w64) <= 4 * u * aw + 20 * u * au)


@pytest.mark.slow
def test_host_code_under_sanitizers(tmp_path):
    """tests/host/adamw_fuzz.cpp with the optimizer's and the plan's host code, the kernel launchers (never reached)
    left out."""
    import os
    import shutil
    import subprocess

    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    csrc, rocm = os.path.join(root, "paper_2509_03047_amd", "csrc"), os.environ.get("ROCM_PATH", "/opt/rocm")
    if shutil.which("g++") is None or not os.path.isdir(os.path.join(rocm, "include", "hip")):
        pytest.skip("needs g++ and the HIP headers")
    exe = str(tmp_path / "adamw_fuzz")
    b = subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                        "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(root, "include"), "-I", csrc,
                        "-I", os.path.join(rocm, "include"), os.path.join(root, "tests", "host", "adamw_fuzz.cpp"),
                        os.path.join(csrc, "adamw.cpp"), os.path.join(csrc, "plan.cpp"),
                        "-L", os.path.join(rocm, "lib"), "-lamdhip64", "-Wl,-rpath," + os.path.join(rocm, "lib"),
                        "-Wl,--unresolved-symbols=ignore-all", "-o", exe], capture_output=True, text=True, timeout=600)
    assert b.returncode == 0, b.stderr[-3000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, (r.stdout + r.stderr)[-3000:]
    assert " 0 wrong" in r.stdout
