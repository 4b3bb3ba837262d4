"""More of what the compiler makes of the orthogonalisation's and the embedding's
kernels (CPU; hipcc cross-compiles): over whole kernels, each of which has to
be found."""
import re

import pytest

from tests.test_kernel_code_cpu import assembly
from tests.test_muon_code_cpu import kernels


@pytest.mark.slow
def test_few_registers_leave_a_product(tmp_path):
    """Over whole kernels: small tiles spill nothing, large ones a few registers once a tile, in front of and behind
    their loops (a quarter of the kernel's sums is 32 registers)."""
    found = kernels(assembly("muon.hip", tmp_path / "muon.s"), "k_muon_product")
    assert len(found) == 8
    assert sum("ShapeILj256E" in k for k in found) == sum("ShapeILj64E" in k for k in found) == 4
    for name, body in found.items():
        words = {"": 1, "x2": 2, "x3": 3, "x4": 4}
        spilled = sum(words[re.fullmatch(r"scratch_store_dword(|x2|x3|x4)", x.split()[0]).group(1)]
                      for x in body if x.startswith("scratch_store"))
        assert spilled <= (8 if "ShapeILj256E" in name else 0), (name, spilled)


def wide(code, name, arguments, expected):
    """The forms of a kernel for rows of at least 8 columns, with the loads of each."""
    found = {k: b for k, b in kernels(code, name).items() if re.search(f"{name}I{arguments}ELb0EEEv", k)}
    assert len(found) == expected, sorted(found)
    return {k: [x.split()[0] for x in b if x.startswith(("global_load", "flat_load"))] for k, b in found.items()}


@pytest.mark.slow
def test_rows_at_any_alignment_are_loaded_whole(tmp_path):
    """Rows of a table, of gradients and of sums start at any element's address: 16 bytes a load all the same, and no
    more single words than ids and places are."""
    code = assembly("embed.hip", tmp_path / "embed.s")
    for name, loads in wide(code, "k_embed_lookup", "Lb[01]ELb[01]", 4).items():
        assert loads.count("global_load_dwordx4") == (2 if "lookupILb1" in name else 1), name
        assert loads.count("global_load_dword") <= 1 and "global_load_ushort" not in loads, name
    for name, loads in wide(code, "k_embed_rows", "Lb[01]ELb[01]ELj[12]", 8).items():
        tokens = 16 + 8  # runs', and rows' (of two slices: half as many, twice each)
        assert loads.count("global_load_dwordx4") >= tokens * (2 if "rowsILb1" in name else 1), name
        assert loads.count("global_load_dword") <= tokens + 4 and "global_load_ushort" not in loads, name
    for name, loads in wide(code, "k_embed_long", "Lb[01]", 2).items():
        assert loads.count("global_load_dwordx4") >= 2 * 8, name
        assert loads.count("global_load_dword") <= 4 and "global_load_ushort" not in loads, name
