"""The short division of the optimizer step on a CPU's correctly rounded
operations: right for the quotients that are hardest to round."""
import os
import shutil
import subprocess

import pytest


@pytest.mark.slow
def test_short_division_is_correctly_rounded(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("needs gcc")
    src = os.path.join(os.path.dirname(os.path.abspath(__file__)), "host", "quotients.c")
    exe = str(tmp_path / "quotients")
    subprocess.run(["gcc", "-std=c11", "-O3", "-march=native", "-ffp-contract=off", "-fopenmp", "-Wall", "-Wextra", src,
                    "-lm", "-o", exe], check=True, timeout=120)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=900)
    assert r.returncode == 0 and " 0 wrong" in r.stdout, r.stdout
