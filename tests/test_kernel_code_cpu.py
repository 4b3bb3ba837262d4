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
