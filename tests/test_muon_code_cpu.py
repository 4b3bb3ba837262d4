"""What the compiler makes of the orthogonalisation's and the embedding's
kernels: properties of the gfx950 assembly that no test of their results shows
reliably (CPU; hipcc cross-compiles)."""
import re

import pytest

from tests.test_kernel_code_cpu import assembly, stale_conditions


@pytest.fixture(scope="module")
def muon_code(tmp_path_factory):
    return assembly("muon.hip", tmp_path_factory.mktemp("asm") / "muon.s")


def kernels(lines, name):
    """The bodies of the kernels whose names hold `name`."""
    found, body = {}, None
    for line in lines:
        m = re.match(r"(_Z\w+):", line)
        if m:
            body = found.setdefault(m.group(1), []) if name in m.group(1) else None
        elif line.startswith(".Lfunc_end"):
            body = None
        elif body is not None:
            body.append(line.split(";")[0].strip())
    return {k: [x for x in v if x] for k, v in found.items()}


def test_m0_is_the_loads_own(muon_code):
    """Loads into LDS set m0 in an asm block that the compiler does not know to change it: it must not use m0 itself."""
    found = kernels(muon_code, "k_muon_product")
    assert len(found) == 8  # four products, two shapes
    for name, body in found.items():
        loads = [i for i, x in enumerate(body) if x.startswith("global_load_lds")]
        assert loads, name
        for i in loads:
            assert body[i - 1].startswith("s_nop") and re.match(r"s_mov_b32 m0, s\d+", body[i - 2]), (name, body[i - 3:i + 1])
        others = [x for i, x in enumerate(body) if re.search(r"\bm0\b", x) and i + 2 not in loads]
        assert not others, (name, others)


def test_the_products_loop_spills_nothing(muon_code):
    """Between two barriers of a product's main loop (blocks with matrix instructions and loads into LDS) no register goes
    to memory: its loads and stores would be waited for with those into LDS."""
    for name, body in kernels(muon_code, "k_muon_product").items():
        block, blocks = [], []
        for x in body:
            if x.endswith(":") or x.startswith(("s_cbranch", "s_branch")):
                blocks.append(block)
                block = []
            else:
                block.append(x)
        loops = [b for b in blocks if sum(x.startswith("v_mfma") for x in b) >= 8 and any("global_load_lds" in x for x in b)]
        if "Lj256" in name:
            assert loops, name
        for b in loops:
            assert not any(x.startswith("scratch_") for x in b), name


@pytest.mark.slow
@pytest.mark.parametrize("source", ["muon.hip", "embed.hip"])
def test_no_kernel_uses_a_stale_condition(source, muon_code, tmp_path):
    code = muon_code if source == "muon.hip" else assembly(source, tmp_path / "code.s")
    assert sum(1 for x in code if x.strip().startswith("s_endpgm")) >= 2
    assert stale_conditions(code) == []


@pytest.mark.slow
def test_any_alignment_is_loaded_whole(tmp_path):
    """Rows of the embedding start at any element's address, and are loaded by 16 bytes a lane all the same."""
    code = assembly("embed.hip", tmp_path / "code.s")
    for name, body in kernels(code, "k_embed_lookup").items():
        if name.find("Lb0EEEvNS") > 0:  # not of fewer than 8 columns
            loads = [x.split()[0] for x in body if x.startswith("global_load")]
            assert "global_load_dwordx4" in loads and "global_load_ushort" not in loads, (name, loads)
