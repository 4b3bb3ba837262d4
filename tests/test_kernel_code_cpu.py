"""What the compiler makes of the kernels: properties of the gfx950 assembly
that no test of their results shows reliably (CPU; hipcc cross-compiles)."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2509_03047_amd import build as B


def assembly(source, out):
    """The device assembly of one source, compiled as the library is."""
    if shutil.which(os.path.join(B.ROCM, "bin", "hipcc")) is None:
        pytest.skip("needs hipcc")
    cmd = [a for a in B.hipcc_command(str(out), sources=[source]) if a != "-shared" and not a.startswith("-Wl,")]
    subprocess.run(cmd + ["-S", "--cuda-device-only"], check=True, capture_output=True, timeout=600)
    return out.read_text().splitlines()


@pytest.fixture(scope="module")
def adamw_code(tmp_path_factory):
    return assembly("adamw.hip", tmp_path_factory.mktemp("asm") / "adamw.s")


def test_parts_of_a_norm_are_left_by_exchanges_that_return(adamw_code):
    """A workgroup adds its arrival once the exchange that leaves its part has returned.  An exchange without a
    result is compiled to the form that returns nothing to wait for."""
    swaps = [x.split(";")[0].split() for x in adamw_code if re.match(r"\s*global_atomic_swap_x2", x)]
    assert len(swaps) == 2  # k_norm of one launch, k_norm_fold
    assert all(s[-1] == "sc0" for s in swaps), swaps


# Scalar instructions that leave the condition code alone; all others may set it.
KEEP = re.compile(r"s_(mov|cmov|mul|bfm|brev|ff[01]|flbit|sext|pack|bitset|bitreplicate|cselect|load|store|buffer|scratch|"
                  r"dcache|branch|cbranch|setpc|getpc|swappc|call|waitcnt|nop|sleep|barrier|endpgm|sendmsg|setprio|set|get|mem|"
                  r"trap|icache|ttrace|inst|code_end)")
USE = re.compile(r"s_(cselect|cmov|cbranch_scc|addc|subb)")


def stale_conditions(lines):
    """Instructions that use the scalar condition code in a block that has not set it."""
    known, found = False, []
    for at, line in enumerate(lines, 1):
        if re.match(r"(\.LBB\w+|_Z\w+):|; %bb", line):  # a block starts, by a label or after a branch
            known = False
            continue
        op = line.split(";")[0].split()
        if not op or not op[0].startswith("s_"):
            continue
        if USE.match(op[0]) and not known:
            found.append((at, line.strip()))
        known = known or not KEEP.match(op[0])
    return found


def test_a_stale_condition_is_found():
    """What clang 22 of ROCm 7.2.0 made of `n = left < 512 ? uint32_t(left) : 512` for 64-bit scalars in k_adamw, behind
    a branch on the same comparison: the comparison is a vector one, the select takes the carry of an earlier sum."""
    lines = ["_ZN1f:", "\ts_addc_u32 s29, s7, s1", "\tv_cmp_lt_u64_e32 vcc, s[2:3], v[2:3]", "\ts_cbranch_vccz .LBB6_156",
             "; %bb.1:", "\ts_cselect_b32 s70, s2, 0x200"]
    assert [x for x, _ in stale_conditions(lines)] == [2, 6]
    lines[1:2] = ["\ts_add_u32 s28, s6, s0", "\ts_addc_u32 s29, s7, s1"]
    lines[-1:-1] = ["\ts_and_b64 s[4:5], vcc, exec"]
    assert stale_conditions(lines) == []


@pytest.mark.slow
@pytest.mark.parametrize("source", ["adamw.hip", "kernels.hip", "ceilings.hip"])
def test_no_kernel_uses_a_stale_condition(source, adamw_code, tmp_path):
    code = adamw_code if source == "adamw.hip" else assembly(source, tmp_path / "code.s")
    assert sum(1 for x in code if x.strip().startswith("s_endpgm")) >= 2
    assert stale_conditions(code) == []
