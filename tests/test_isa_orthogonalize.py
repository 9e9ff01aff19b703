"""The loads through inline asm in the compiled products of the orthogonalised updates: the rules of test_isa_asm_loads, which their unit keeps
too (no GPU needed)."""
import os
import shutil
import subprocess

import pytest

from test_isa_asm_loads import find_odd_loads, find_other_uses_of_m0, find_young_scalars


def test_no_hazard_around_the_loads(tmp_path):
    from paper_2605_19945_amd import build as moe_build
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("no hipcc")
    path = tmp_path / "orth.s"
    r = subprocess.run([hipcc, *moe_build.FLAGS, "-S", "--cuda-device-only", "-o", str(path), os.path.join(moe_build.CSRC, "moe_orth.hip")],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    lines = path.read_text().splitlines()
    n, young = find_young_scalars(lines)
    assert n > 50 and not young, "\n".join(young[:10])
    odd = find_odd_loads(lines)
    assert not odd, "\n".join(odd[:10])
    others = find_other_uses_of_m0(lines)
    assert not others, "\n".join(others[:10])
